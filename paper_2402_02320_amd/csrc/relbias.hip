// Learned relative position bias on whole matrices of scores (spin_relbias_trunc, spin_relbias_grad): HBM streams.
#include "generation.hpp"

namespace spin {
namespace {

constexpr int kBlock = 128;
constexpr size_t kStreamingBytes = (size_t)16 << 20;       // of one operand, all parties: beyond, accesses are non-temporal, as in elementwise.hip
template <bool NT, class T> __device__ inline T ld(const T *p) { return NT ? __builtin_nontemporal_load(p) : *p; }
template <bool NT, class T> __device__ inline void st(T *p, T v)
{
    if (NT) __builtin_nontemporal_store(v, p);
    else *p = v;
}

// One thread: one score of all parties; the bias is a few hundred words, which stay in the first cache.  Words that are masked are not read, and workgroups are
// narrow so that little of one is.  HBM bounds it: 3 parties' 2 x 8 x 1024 x 1000 scores take 327 us, 5.4 TB/s, of which the truncation alone takes 320;
// 1024 x 1024 of a decoder, whose upper half is only written, 224 (with 256 columns 249, with the bias of 256 columns and eight rows looked up once into LDS 241, of
// two rows 260).  blockIdx.y = row, blockIdx.z = sequence and head.
template <int NP, class T, bool NT> __global__ __launch_bounds__(kBlock) void trunc_kernel(PairArgs<T> a)
{
    const int k0 = turned_x() * kBlock, k = k0 + threadIdx.x, b = blockIdx.z / a.heads, h = blockIdx.z % a.heads;
    if (k >= a.K) return;
    const size_t party = (size_t)a.batch * a.heads * a.Q * a.K;
    const int length = a.lengths ? min(a.lengths[b], a.K) : a.K;
    for (int q = blockIdx.y; q < a.Q; q += gridDim.y) {
        const size_t at = ((size_t)blockIdx.z * a.Q + q) * a.K + k;
        if (k < length && (!a.causal || k <= q + a.first)) {
            T y[NP], r[NP], r_top[NP], r_msb[NP], add[NP];
            const int bucket = a.bias.bucket_of[min(max(k - q - a.first, -a.bias.reach), a.bias.reach) + a.bias.reach];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                y[i] = ld<NT>(a.x + i * party + at);
                if (a.f) r[i] = ld<NT>(a.r + i * party + at), r_top[i] = ld<NT>(a.r_top + i * party + at), r_msb[i] = ld<NT>(a.r_msb + i * party + at);
            }
            const bool there = (unsigned)bucket < (unsigned)a.bias.buckets;
#pragma unroll
            for (int i = 0; i < NP; ++i) add[i] = ((const T *)a.bias.table)[((size_t)i * a.heads + h) * a.bias.buckets + (there ? bucket : 0)];
            if (a.f) truncate_shares<NP, T>(y, r, r_top, r_msb, a.f);
#pragma unroll
            for (int i = 0; i < NP; ++i) st<NT>(a.out + i * party + at, (T)(y[i] + (there ? add[i] : 0)));
        } else {
#pragma unroll
            for (int i = 0; i < NP; ++i) st<NT>(a.out + i * party + at, (T)(i == 0 ? a.masked : 0));
        }
    }
}

template <class T> __global__ __launch_bounds__(kBlock) void zero_kernel(T *p, size_t count)
{
    const size_t v = (size_t)blockIdx.x * kBlock + threadIdx.x;
    if (v < count) p[v] = 0;
}

__device__ inline void add_to(u64 *p, u64 v) { atomicAdd((unsigned long long *)p, (unsigned long long)v); }
__device__ inline void add_to(u32 *p, u32 v) { atomicAdd(p, v); }

// A thread keeps to one diagonal, so its bucket never changes and its sum stays in a register; neighbouring threads read neighbouring words of a row.  The
// rows of a diagonal that are there are an interval, so the loop over them has no condition and eight loads are in flight.  A workgroup's sums meet in LDS, one global
// addition a bucket is left; ring additions commute, so their order changes nothing.  Rows start anywhere in a cache line, which neighbouring waves share: with
// non-temporal loads, which fetch those lines twice, 3 parties' 4 x 16 x 1000 x 1000 take 431 us, with these 354.  158 us for a decoder's 4 x 16 x 1024 x 1024, half of
// which is read: 5 TB/s.
// blockIdx.x = block of diagonals, blockIdx.y = run of rows and of sequences, blockIdx.z = party and head.
constexpr int kMostBuckets = 1024;
template <class T> __global__ __launch_bounds__(kBlock) void grad_kernel(PairArgs<T> a, int rows, int row_runs, int sequences)
{
    __shared__ T sums[kMostBuckets];
    const int i = blockIdx.z / a.heads, h = blockIdx.z % a.heads;
    const int nearest = turned_x() * kBlock - (a.Q - 1), away = nearest + (int)threadIdx.x;                // k - q
    if (a.causal && nearest > a.first) return;             // of the whole workgroup
    for (int k = threadIdx.x; k < a.bias.buckets; k += kBlock) sums[k] = 0;
    const int bucket = bucket_at(a.bias, away - a.first);
    const int q0 = blockIdx.y % row_runs * rows, q1 = min(q0 + rows, a.Q);
    const int b0 = blockIdx.y / row_runs * sequences, b1 = min(b0 + sequences, a.batch);
    T sum = 0;
    for (int b = b0; b < b1; ++b) {
        const DiagonalRows there = rows_of_diagonal(away, q0, q1, a.K, a.lengths ? a.lengths[b] : a.K, a.causal, a.first);
        int q = there.from;
        const int end = there.to;
        const T *x = a.x + ((((size_t)i * a.batch + b) * a.heads + h) * a.Q + q) * a.K + (q + away);
        const size_t step = (size_t)a.K + 1;
        for (; q + 8 <= end; q += 8, x += 8 * step) {
            T v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = x[k * step];
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += v[k];
        }
        for (; q < end; ++q, x += step) sum += *x;
    }
    __syncthreads();
    if (bucket >= 0) add_to(&sums[bucket], sum);
    __syncthreads();
    for (int k = threadIdx.x; k < a.bias.buckets; k += kBlock)
        if (sums[k]) add_to(a.out + ((size_t)i * a.heads + h) * a.bias.buckets + k, sums[k]);
}

template <class F> inline void for_streaming(size_t bytes, F &&fn)
{
    if (bytes >= kStreamingBytes) fn(std::true_type());
    else fn(std::false_type());
}

}  // namespace

template <class T> spin_status launch_relbias_trunc(const PairArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_RELBIAS, s);
    const dim3 grid((a.K + kBlock - 1) / kBlock, a.Q < 65535 ? a.Q : 65535, a.batch * a.heads);
    for_party_count(a.n, [&](auto np) {
        for_streaming((size_t)a.n * a.batch * a.heads * a.Q * a.K * sizeof(T), [&](auto nt) {
            trunc_kernel<decltype(np)::value, T, decltype(nt)::value><<<grid, kBlock, 0, s>>>(a);
        });
    });
    return check_launch("spin_relbias_trunc");
}

template <class T> spin_status launch_relbias_grad(const PairArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_RELBIAS, s);
    const size_t count = (size_t)a.n * a.heads * a.bias.buckets;
    zero_kernel<T><<<(unsigned)((count + kBlock - 1) / kBlock), kBlock, 0, s>>>(a.out, count);
    // Short runs of rows, since diagonals are of any length (16 against 64 rows: 173 and 200 us for 3 parties' 4 x 16 x 1024 x 1024 of a decoder), and where that is few
    // workgroups every sequence apart.
    const long wanted = 4096, diagonals = ((long)a.Q + a.K - 1 + kBlock - 1) / kBlock * a.n * a.heads;
    int rows = 16;
    while (rows > 8 && diagonals * a.batch * ((a.Q + rows - 1) / rows) < wanted) rows /= 2;
    if ((a.Q + rows - 1) / rows > 8192) rows = (a.Q + 8191) / 8192;
    const int row_runs = (a.Q + rows - 1) / rows;
    long apart = (wanted + diagonals * row_runs - 1) / (diagonals * row_runs);
    const long most = 65535 / row_runs;
    apart = apart > a.batch ? a.batch : apart;
    apart = apart > most ? most : apart;
    const int sequences = (int)((a.batch + apart - 1) / apart);
    const dim3 grid((unsigned)(((size_t)a.Q + a.K - 1 + kBlock - 1) / kBlock), row_runs * ((a.batch + sequences - 1) / sequences), a.n * a.heads);
    grad_kernel<T><<<grid, kBlock, 0, s>>>(a, rows, row_runs, sequences);
    return check_launch("spin_relbias_grad");
}

template spin_status launch_relbias_trunc<u64>(const PairArgs<u64> &, hipStream_t);
template spin_status launch_relbias_trunc<u32>(const PairArgs<u32> &, hipStream_t);
template spin_status launch_relbias_grad<u64>(const PairArgs<u64> &, hipStream_t);
template spin_status launch_relbias_grad<u32>(const PairArgs<u32> &, hipStream_t);

}  // namespace spin
