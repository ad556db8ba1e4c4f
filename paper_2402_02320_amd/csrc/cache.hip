// Upkeep of the paged cache of shares (spin_cache_append, _copy, _compact): pure HBM streams, 16 bytes a lane.
#include "generation.hpp"

namespace spin {
namespace {

constexpr int kBlock = 256;

// Prompts and runs of pages are read and written once: non-temporal accesses from 16 MB on, as in elementwise.hip.
constexpr size_t kStreamingBytes = (size_t)16 << 20;
template <class F> inline void for_streaming(size_t bytes, F &&fn)
{
    if (bytes >= kStreamingBytes) fn(std::true_type());
    else fn(std::false_type());
}
template <class T> union Vec {         // 16 bytes
    u32x4 all;
    T e[16 / sizeof(T)];
};
template <bool NT, class T> __device__ inline Vec<T> ld(const T *p)
{
    Vec<T> v;
    v.all = NT ? __builtin_nontemporal_load((const u32x4 *)p) : *(const u32x4 *)p;
    return v;
}
template <bool NT, class T> __device__ inline void st(T *p, Vec<T> v)
{
    if (NT) __builtin_nontemporal_store(v.all, (u32x4 *)p);
    else *(u32x4 *)p = v.all;
}

// One thread: 16 bytes of one new row, all slots.  F = sum (x_i - b_i) stays in registers; a row moves 2n words an element in and n + 1
// out, each once: HBM bounds it (two parties' 4 x 8 heads x 2048 x 128, ragged: 151 us, 5.3 TB/s; 161 with ordinary accesses).
// blockIdx.y = sequence and head, blockIdx.z = K or V.
template <int NP, class T, bool NT> __global__ __launch_bounds__(kBlock) void append_kernel(AppendArgs<T> a)
{
    constexpr int VEC = 16 / sizeof(T);
    const unsigned per_row = a.c.dim / VEC;
    const unsigned u = blockIdx.x * kBlock + threadIdx.x, row = u / per_row;
    const int b = blockIdx.y / a.c.heads, g = blockIdx.y % a.c.heads;
    const int rows = a.count ? min(a.count[b], a.rows) : a.rows;
    if ((int)row >= rows) return;
    const long pos = (long)a.start[b] + row;
    const int page = page_of(a.c, b, pos);
    if (page < 0) return;
    const int at = (u - row * per_row) * VEC;
    const size_t party = (size_t)a.batch * a.c.heads * a.rows * a.c.dim;
    const size_t from = ((size_t)blockIdx.y * a.rows + row) * a.c.dim + at;
    const T *x = a.x[blockIdx.z], *m = a.b[blockIdx.z];
    Vec<T> xv[NP], mv[NP], f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        xv[i] = ld<NT>(x + i * party + from);
        mv[i] = ld<NT>(m + i * party + from);
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        f.e[k] = 0;
#pragma unroll
        for (int i = 0; i < NP; ++i) f.e[k] += xv[i].e[k] - mv[i].e[k];
        mv[0].e[k] += f.e[k];
    }
    T *to = a.pool[blockIdx.z] + row_at(a.c, 0, page, g, pos) + at;
    const size_t slot = ((size_t)a.c.pages * a.c.heads << a.c.shift) * a.c.dim;
    st<NT>(to, f);
#pragma unroll
    for (int i = 0; i < NP; ++i) st<NT>(to + (i + 1) * slot, mv[i]);
}

// A page of one slot is contiguous over its heads; a thread moves 16 bytes (48 pages of three parties, 2 x 4 MB each: 71 us, 5.7 TB/s; with four or eight
// a thread 74 and 77, with ordinary accesses 80).  blockIdx.y = pair, blockIdx.z = slot and pool.
template <class T, bool NT>
__global__ __launch_bounds__(kBlock) void copy_kernel(CacheView c, const int32_t *src, const int32_t *dst, T *K, T *V)
{
    const int from = src[blockIdx.y], to = dst[blockIdx.y];
    if ((unsigned)from >= (unsigned)c.pages || (unsigned)to >= (unsigned)c.pages) return;
    constexpr int W = 16 / sizeof(T);
    const size_t words = ((size_t)c.heads << c.shift) * c.dim, vecs = words / W;
    T *pool = (blockIdx.z & 1 ? V : K) + (blockIdx.z >> 1) * words * c.pages;
    const T *in = pool + from * words;
    T *out = pool + to * words;
    const size_t v = (size_t)blockIdx.x * kBlock + threadIdx.x;
    if (v < vecs) st<NT>(out + v * W, ld<NT>(in + v * W));
}

// One thread: 16 bytes of one head and slot of all kept rows, kAhead rows read before the first of them is written.  kept ascends, so a row
// is written only where no later row is read from: j <= kept[j] < kept[j + 1].  blockIdx.y = sequence, blockIdx.z = slot and pool.
constexpr int kAhead = 8;
template <class T>
__global__ __launch_bounds__(kBlock) void compact_kernel(CacheView c, int nodes, const int32_t *context, const int32_t *kept, const int32_t *kept_count, T *K, T *V)
{
    constexpr int VEC = 16 / sizeof(T);
    const unsigned per_row = c.dim / VEC, u = blockIdx.x * kBlock + threadIdx.x;
    const int g = u / per_row, at = (u - g * per_row) * VEC, b = blockIdx.y, slot = blockIdx.z >> 1;
    const int first = context[b], count = min(kept_count[b], nodes);
    if (g >= c.heads || first < 0) return;
    T *pool = blockIdx.z & 1 ? V : K;
    for (int j = 0; j < count; j += kAhead) {
        u32x4 v[kAhead];
        int page[kAhead];                                  // to write to
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int node = j + k < count ? kept[(size_t)b * nodes + j + k] : -1;
            const int from = node >= 0 && node < nodes ? page_of(c, b, (long)first + node) : -1;
            page[k] = from >= 0 ? page_of(c, b, (long)first + j + k) : -1;
            v[k] = *(const u32x4 *)(pool + row_at(c, slot, max(from, 0), g, from >= 0 ? (long)first + node : 0) + at);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (page[k] >= 0) *(u32x4 *)(pool + row_at(c, slot, page[k], g, (long)first + j + k) + at) = v[k];
    }
}

}  // namespace

template <class T> spin_status launch_cache_append(const AppendArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_CACHE, s);
    const size_t vecs = (size_t)a.rows * a.c.dim / (16 / sizeof(T));
    const dim3 grid((unsigned)((vecs + kBlock - 1) / kBlock), a.batch * a.c.heads, 2);
    for_party_count(a.n, [&](auto np) {
        for_streaming((size_t)a.n * a.batch * a.c.heads * a.rows * a.c.dim * sizeof(T),
                      [&](auto nt) { append_kernel<decltype(np)::value, T, decltype(nt)::value><<<grid, kBlock, 0, s>>>(a); });
    });
    return check_launch("spin_cache_append");
}

template <class T> spin_status launch_cache_copy(const CacheView &c, int n, int pairs, const int32_t *src, const int32_t *dst, T *K, T *V, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_CACHE, s);
    const size_t vecs = ((size_t)c.heads << c.shift) * c.dim / (16 / sizeof(T));
    const dim3 grid((unsigned)((vecs + kBlock - 1) / kBlock), pairs, 2 * (n + 1));
    for_streaming(vecs * 32 * (n + 1) * pairs, [&](auto nt) { copy_kernel<T, decltype(nt)::value><<<grid, kBlock, 0, s>>>(c, src, dst, K, V); });
    return check_launch("spin_cache_copy");
}

template <class T>
spin_status launch_cache_compact(const CacheView &c, int n, int batch, int nodes, const int32_t *context, const int32_t *kept, const int32_t *kept_count,
                                 T *K, T *V, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_CACHE, s);
    const size_t vecs = (size_t)c.heads * c.dim / (16 / sizeof(T));
    const dim3 grid((unsigned)((vecs + kBlock - 1) / kBlock), batch, 2 * (n + 1));
    compact_kernel<T><<<grid, kBlock, 0, s>>>(c, nodes, context, kept, kept_count, K, V);
    return check_launch("spin_cache_compact");
}

#define INSTANTIATE(T)                                                                                                                             \
    template spin_status launch_cache_append<T>(const AppendArgs<T> &, hipStream_t);                                                               \
    template spin_status launch_cache_copy<T>(const CacheView &, int, int, const int32_t *, const int32_t *, T *, T *, hipStream_t);               \
    template spin_status launch_cache_compact<T>(const CacheView &, int, int, int, const int32_t *, const int32_t *, const int32_t *, T *, T *, hipStream_t)
INSTANTIATE(u64);
INSTANTIATE(u32);
#undef INSTANTIATE

}  // namespace spin
