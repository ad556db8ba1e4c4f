// Learned relative position bias on whole matrices of scores (spin_relbias_trunc, spin_relbias_grad): HBM streams.
#include "generation.hpp"

namespace spin {
namespace {

constexpr int kBlock = 256;

template <class T> __device__ inline bool is_there(const PairArgs<T> &a, int length, int q, int k) { return k < length && (!a.causal || k <= q + a.first); }

// One thread: one score of all parties.  blockIdx.y = row, blockIdx.z = sequence and head.
template <int NP, class T> __global__ __launch_bounds__(kBlock) void trunc_kernel(PairArgs<T> a)
{
    const int k = blockIdx.x * kBlock + threadIdx.x, b = blockIdx.z / a.heads, h = blockIdx.z % a.heads;
    if (k >= a.K) return;
    const size_t party = (size_t)a.batch * a.heads * a.Q * a.K;
    for (int q = blockIdx.y; q < a.Q; q += gridDim.y) {
        const size_t at = ((size_t)blockIdx.z * a.Q + q) * a.K + k;
        T y[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) y[i] = 0;
        if (is_there(a, a.lengths ? a.lengths[b] : a.K, q, k)) {
            T r[NP], r_top[NP], r_msb[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                y[i] = a.x[i * party + at];
                if (a.f) r[i] = a.r[i * party + at], r_top[i] = a.r_top[i * party + at], r_msb[i] = a.r_msb[i * party + at];
            }
            if (a.f) truncate_shares<NP, T>(y, r, r_top, r_msb, a.f);
            const int bucket = bucket_at(a.bias, k - (q + a.first));
#pragma unroll
            for (int i = 0; i < NP; ++i)
                if (bucket >= 0) y[i] += ((const T *)a.bias.table)[((size_t)i * a.heads + h) * a.bias.buckets + bucket];
        } else {
            y[0] = a.masked;
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) a.out[i * party + at] = y[i];
    }
}

template <class T> __global__ __launch_bounds__(kBlock) void zero_kernel(T *p, size_t count)
{
    const size_t v = (size_t)blockIdx.x * kBlock + threadIdx.x;
    if (v < count) p[v] = 0;
}

__device__ inline void add_to(u64 *p, u64 v) { atomicAdd((unsigned long long *)p, (unsigned long long)v); }
__device__ inline void add_to(u32 *p, u32 v) { atomicAdd(p, v); }

// A thread keeps to one diagonal, so its bucket never changes and its sum stays in a register; neighbouring threads read neighbouring words of a
// row.  Ring additions commute, so the order of the atomic ones changes nothing.  blockIdx.x = block of diagonals, blockIdx.y = run of rows, blockIdx.z = party and head.
template <class T> __global__ __launch_bounds__(kBlock) void grad_kernel(PairArgs<T> a, int rows)
{
    const int i = blockIdx.z / a.heads, h = blockIdx.z % a.heads;
    const int away = (int)(blockIdx.x * kBlock + threadIdx.x) - (a.Q - 1);       // k - q
    const int bucket = bucket_at(a.bias, away - a.first);
    T sum = 0;
    for (int b = 0; b < a.batch; ++b) {
        const int length = a.lengths ? min(a.lengths[b], a.K) : a.K;
        const T *x = a.x + (((size_t)i * a.batch + b) * a.heads + h) * a.Q * a.K;
        for (int q = blockIdx.y * rows; q < min((int)(blockIdx.y + 1) * rows, a.Q); ++q) {
            const int k = q + away;
            if (k >= 0 && is_there(a, length, q, k)) sum += x[(size_t)q * a.K + k];
        }
    }
    if (bucket >= 0) add_to(a.out + ((size_t)i * a.heads + h) * a.bias.buckets + bucket, sum);
}

}  // namespace

template <class T> spin_status launch_relbias_trunc(const PairArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_RELBIAS, s);
    const dim3 grid((a.K + kBlock - 1) / kBlock, a.Q < 65535 ? a.Q : 65535, a.batch * a.heads);
    for_party_count(a.n, [&](auto np) { trunc_kernel<decltype(np)::value, T><<<grid, kBlock, 0, s>>>(a); });
    return check_launch("spin_relbias_trunc");
}

template <class T> spin_status launch_relbias_grad(const PairArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_RELBIAS, s);
    const size_t count = (size_t)a.n * a.heads * a.bias.buckets;
    zero_kernel<T><<<(unsigned)((count + kBlock - 1) / kBlock), kBlock, 0, s>>>(a.out, count);
    const int rows = a.Q > 64 * 65535 ? (a.Q + 65534) / 65535 : 64;
    const dim3 grid((unsigned)(((size_t)a.Q + a.K - 1 + kBlock - 1) / kBlock), (a.Q + rows - 1) / rows, a.n * a.heads);
    grad_kernel<T><<<grid, kBlock, 0, s>>>(a, rows);
    return check_launch("spin_relbias_grad");
}

template spin_status launch_relbias_trunc<u64>(const PairArgs<u64> &, hipStream_t);
template spin_status launch_relbias_trunc<u32>(const PairArgs<u32> &, hipStream_t);
template spin_status launch_relbias_grad<u64>(const PairArgs<u64> &, hipStream_t);
template spin_status launch_relbias_grad<u32>(const PairArgs<u32> &, hipStream_t);

}  // namespace spin
