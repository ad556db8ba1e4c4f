// Products of new tokens with the paged cache of shares (spin_cache_scores, spin_cache_values).
#include "generation.hpp"

namespace spin {
namespace {

constexpr int kBlock = 256;

// One thread: one score of all parties.  blockIdx.y = head and node, blockIdx.z = sequence.
template <int NP, class T> __global__ __launch_bounds__(kBlock) void scores_kernel(AttentionArgs<T> a)
{
    const int t = blockIdx.x * kBlock + threadIdx.x, b = blockIdx.z, h = blockIdx.y / a.d.nodes, m = blockIdx.y % a.d.nodes;
    if (t >= a.d.columns) return;
    const size_t rows = (size_t)a.batch * a.heads * a.d.nodes, row = (size_t)b * a.heads * a.d.nodes + blockIdx.y;
    const int context = a.d.context[b], page = page_of(a.c, b, t);
    const bool seen = page >= 0 && sees(tree_row(a.d, b, m), a.d.nodes, context, t);
    T z[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) z[i] = 0;
    if (seen) {
        const size_t slot = ((size_t)a.c.pages * a.c.heads << a.c.shift) * a.c.dim;
        const T *key = a.pool + row_at(a.c, 0, page, h / (a.heads / a.c.heads), t);
        for (int d = 0; d < a.c.dim; ++d) {
            T e = 0, mask[NP];
            const T f = key[d];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                mask[i] = a.A[(i * rows + row) * a.c.dim + d];
                e += a.x[(i * rows + row) * a.c.dim + d] - mask[i];
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) z[i] += e * key[(i + 1) * slot + d] + mask[i] * f;
        }
        T r[NP], r_top[NP], r_msb[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const size_t at = (i * rows + row) * a.d.columns + t;
            z[i] += a.C[at];
            if (a.f) r[i] = a.r[at], r_top[i] = a.r_top[at], r_msb[i] = a.r_msb[at];
        }
        if (a.f) truncate_shares<NP, T>(z, r, r_top, r_msb, a.f);
        if (a.bias.table) {
            auto place = [&](int node) { return a.depth ? a.depth[(size_t)b * a.d.nodes + node] : node; };
            const long key_at = t < context ? (long)t - context : place(t - context);
            const long away = key_at - place(m);
            const int bucket = bucket_at(a.bias, (int)min(max(away, -(long)a.bias.reach), (long)a.bias.reach));
#pragma unroll
            for (int i = 0; i < NP; ++i)
                if (bucket >= 0) z[i] += ((const T *)a.bias.table)[((size_t)i * a.heads + h) * a.bias.buckets + bucket];
        }
    } else {
        z[0] = a.masked;
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) a.out[(i * rows + row) * a.d.columns + t] = z[i];
}

// One thread: one element of the sum of all parties.  blockIdx.y = head and node, blockIdx.z = sequence.
template <int NP, class T> __global__ __launch_bounds__(kBlock) void values_kernel(AttentionArgs<T> a)
{
    const int d = blockIdx.x * kBlock + threadIdx.x, b = blockIdx.z, h = blockIdx.y / a.d.nodes, m = blockIdx.y % a.d.nodes;
    if (d >= a.c.dim) return;
    const size_t rows = (size_t)a.batch * a.heads * a.d.nodes, row = (size_t)b * a.heads * a.d.nodes + blockIdx.y;
    const int context = a.d.context[b];
    const u64 tree = tree_row(a.d, b, m);
    const size_t slot = ((size_t)a.c.pages * a.c.heads << a.c.shift) * a.c.dim;
    T z[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) z[i] = a.C[(i * rows + row) * a.c.dim + d];
    for (long t = 0; t < a.d.columns && t < (long)context + a.d.nodes; ++t) {
        const int page = page_of(a.c, b, t);
        if (page < 0 || !sees(tree, a.d.nodes, context, (int)t)) continue;
        const T *value = a.pool + row_at(a.c, 0, page, h / (a.heads / a.c.heads), t) + d;
        T e = 0, mask[NP];
        const T f = value[0];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            mask[i] = a.A[(i * rows + row) * a.d.columns + t];
            e += a.x[(i * rows + row) * a.d.columns + t] - mask[i];
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) z[i] += e * value[(i + 1) * slot] + mask[i] * f;
    }
    if (a.f) {
        T r[NP], r_top[NP], r_msb[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const size_t at = (i * rows + row) * a.c.dim + d;
            r[i] = a.r[at], r_top[i] = a.r_top[at], r_msb[i] = a.r_msb[at];
        }
        truncate_shares<NP, T>(z, r, r_top, r_msb, a.f);
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) a.out[(i * rows + row) * a.c.dim + d] = z[i];
}

}  // namespace

size_t cache_values_workspace(int, int, int, int, int, int, int, int) { return 256; }

template <class T> spin_status launch_cache_scores(const AttentionArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_ATTENTION, s);
    const dim3 grid((a.d.columns + kBlock - 1) / kBlock, a.heads * a.d.nodes, a.batch);
    for_party_count(a.n, [&](auto np) { scores_kernel<decltype(np)::value, T><<<grid, kBlock, 0, s>>>(a); });
    return check_launch("spin_cache_scores");
}

template <class T> spin_status launch_cache_values(const AttentionArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_ATTENTION, s);
    const dim3 grid((a.c.dim + kBlock - 1) / kBlock, a.heads * a.d.nodes, a.batch);
    for_party_count(a.n, [&](auto np) { values_kernel<decltype(np)::value, T><<<grid, kBlock, 0, s>>>(a); });
    return check_launch("spin_cache_values");
}

template spin_status launch_cache_scores<u64>(const AttentionArgs<u64> &, hipStream_t);
template spin_status launch_cache_scores<u32>(const AttentionArgs<u32> &, hipStream_t);
template spin_status launch_cache_values<u64>(const AttentionArgs<u64> &, hipStream_t);
template spin_status launch_cache_values<u32>(const AttentionArgs<u32> &, hipStream_t);

}  // namespace spin
