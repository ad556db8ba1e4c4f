// Layer norm of shares, forward and backward (spin_layernorm, spin_layernorm_grad): HBM streams with a short chain of truncations in the middle of each row.
#include "linear.hpp"
#include "limb_common.hpp"

namespace spin {
namespace {

constexpr int kBlock = 256, kWaves = kBlock / 64;

template <class T> __device__ inline T wave_sum(T v)
{
#pragma unroll
    for (int by = 32; by; by /= 2) v += __shfl_xor(v, by);
    return v;
}
// Sums over the workgroup, for all of its threads.  `room`: COUNT x waves words, free again at the next barrier.
template <int COUNT, class T> __device__ inline void block_sums(T (&v)[COUNT], T *room)
{
#pragma unroll
    for (int k = 0; k < COUNT; ++k) {
        v[k] = wave_sum(v[k]);
        if (threadIdx.x % 64 == 0) room[k * kWaves + threadIdx.x / 64] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < COUNT; ++k) {
        v[k] = 0;
        for (int w = 0; w < kWaves; ++w) v[k] += room[k * kWaves + w];
    }
}

// What belongs to whole rows (or columns): word k of all parties, and truncation with words k, k + 1 and k + 2.
template <int NP, class T> struct Words {
    const T *words;
    size_t party, each;                // words of a party, and from one word to the next
    __device__ T at(int i, int k) const { return words[i * party + k * each]; }
    // sum: of the shares, which nobody needs one by one, and what is public
    __device__ void truncate(T sum, int k, int f, T (&y)[NP]) const
    {
        Opened<T> c{f};
        c.add(sum);
        T top[NP], msb[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) c.add(at(i, k)), top[i] = at(i, k + 1), msb[i] = at(i, k + 2);
#pragma unroll
        for (int i = 0; i < NP; ++i) y[i] = c.truncated(i, top[i], msb[i]);
    }
    __device__ T open(const T (&y)[NP], int k) const
    {
        T e = 0;
#pragma unroll
        for (int i = 0; i < NP; ++i) e += y[i] - at(i, k);
        return e;
    }
    // The parties' sum of dealt word c + x . y, opened against words a and b
    __device__ T product(int c, T e, int a, T f, int b) const
    {
        T z = e * f;
#pragma unroll
        for (int i = 0; i < NP; ++i) z += at(i, c) + e * at(i, b) + at(i, a) * f;
        return z;
    }
};
template <int NP, class T> __device__ inline T sum_of(const T (&y)[NP])
{
    T s = 0;
#pragma unroll
    for (int i = 0; i < NP; ++i) s += y[i];
    return s;
}

// From the sum of inv x to the means, and from the sum of (x - mu)^2 to 1 / sqrt(variance).
template <int NP, class T> __device__ inline void rstd_of(const NormArgs<T> &a, const Words<NP, T> &w, T square, T (&y)[NP])
{
    T v[NP], u[NP], h[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) square += w.at(i, 3);
    w.truncate(square, 4, a.f, v);
    w.truncate(a.inv * sum_of<NP>(v), 7, a.shift, v);
    v[0] += a.eps;
    w.truncate((a.offset << a.f) - a.slope * sum_of<NP>(v), 10, a.f, y);
    const T fv = w.open(v, 13);
    for (int k = 14; k < 14 + kNormWords * a.iterations; k += kNormWords) {
        const T e = w.open(y, k);
        w.truncate(w.product(k + 1, e, k, e, k), k + 2, a.f, u);
        w.truncate(w.product(k + 6, w.open(u, k + 5), k + 5, fv, 13), k + 7, a.f, h);
#pragma unroll
        for (int i = 0; i < NP; ++i) h[i] = (i == 0 ? (T)3 << a.f : 0) - h[i];
        w.truncate(w.product(k + 11, e, k, w.open(h, k + 10), k + 10), k + 12, a.f + 1, y);
    }
}

template <int NP, class T> __global__ __launch_bounds__(kBlock) void norm_kernel(NormArgs<T> a)
{
    extern __shared__ __align__(16) char lds[];
    __shared__ T room[(NP + 1) * kWaves];
    T *const opened = (T *)lds;
    const size_t party = (size_t)a.rows * a.dim;
    for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const size_t first = (size_t)row * a.dim;
        const int last = 14 + kNormWords * a.iterations;
        const Words<NP, T> w{a.row_words + row, (size_t)kNormWords * (a.iterations + 1) * a.rows, (size_t)a.rows};
        T s[1] = {0}, mu[NP], y[NP];
        for (int d = threadIdx.x; d < a.dim; d += kBlock)
#pragma unroll
            for (int i = 0; i < NP; ++i) s[0] += a.x[i * party + first + d];
        __syncthreads();
        block_sums(s, room);
        w.truncate(a.inv * s[0], 0, a.shift, mu);
        const T mean = sum_of<NP>(mu);
        s[0] = 0;
        for (int d = threadIdx.x; d < a.dim; d += kBlock) {
            T e = 0 - mean, mask[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                mask[i] = a.mask_x[i * party + first + d];
                e += a.x[i * party + first + d] - mask[i];
            }
            opened[d] = e;
#pragma unroll
            for (int i = 0; i < NP; ++i) s[0] += e * (2 * mask[i] + (i == 0 ? e : 0));
        }
        __syncthreads();
        block_sums(s, room);
        rstd_of<NP, T>(a, w, s[0], y);
        const T fr = w.open(y, last);
        if (a.rstd && threadIdx.x == 0)
#pragma unroll
            for (int i = 0; i < NP; ++i) a.rstd[(size_t)i * a.rows + row] = y[i];
        T b[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) b[i] = w.at(i, last) + (i == 0 ? fr : 0);
        for (int d = threadIdx.x; d < a.dim; d += kBlock) {
            const size_t at = first + d;
            const T e = opened[d];
            T z = 0, top[NP], msb[NP], xhat[NP], mask[NP], g = 0, e2 = 0;
            Opened<T> c{a.f}, c2{a.f};
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                c.add(a.C1[i * party + at] + e * b[i] + a.mask_x[i * party + at] * fr + a.t1.r[i * party + at]);
                top[i] = a.t1.r_top[i * party + at], msb[i] = a.t1.r_msb[i * party + at];
                mask[i] = a.mask_xhat[i * party + at];
                g += a.gamma.x[(size_t)i * a.dim + d] - a.gamma.a[(size_t)i * a.dim + d];
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                xhat[i] = c.truncated(i, top[i], msb[i]);
                e2 += xhat[i] - mask[i];
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                z += a.C2[i * party + at] + e2 * a.gamma.a[(size_t)i * a.dim + d] + mask[i] * g + a.t2.r[i * party + at];
                top[i] = a.t2.r_top[i * party + at], msb[i] = a.t2.r_msb[i * party + at];
            }
            c2.add(z + e2 * g);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                if (a.xhat) a.xhat[i * party + at] = xhat[i];
                a.out[i * party + at] = c2.truncated(i, top[i], msb[i]) + a.beta[(size_t)i * a.dim + d];
            }
        }
    }
}

template <int NP, class T> __global__ __launch_bounds__(kBlock) void norm_grad_kernel(NormGradArgs<T> a)
{
    extern __shared__ __align__(16) char lds[];
    __shared__ T room[2 * kWaves];
    T *const open_g = (T *)lds, *const open_x = open_g + a.dim;
    const size_t party = (size_t)a.rows * a.dim;
    for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const size_t first = (size_t)row * a.dim;
        const Words<NP, T> w{a.row_words + row, (size_t)kNormGradWords * a.rows, (size_t)a.rows};
        T s[2] = {0, 0};
        for (int d = threadIdx.x; d < a.dim; d += kBlock) {
            const size_t at = first + d;
            T e1 = 0, e2 = 0, e3 = 0, fg = 0, top[NP], msb[NP], z = 0;
            Opened<T> c{a.f};
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                e1 += a.dy.x[i * party + at] - a.dy.a[i * party + at];
                e2 += a.xhat.x[i * party + at] - a.xhat.a[i * party + at];
                fg += a.gamma.x[(size_t)i * a.dim + d] - a.gamma.a[(size_t)i * a.dim + d];
            }
            c.add(e1 * fg);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                c.add(a.C1[i * party + at] + e1 * a.gamma.a[(size_t)i * a.dim + d] + a.dy.a[i * party + at] * fg + a.t1.r[i * party + at]);
                top[i] = a.t1.r_top[i * party + at], msb[i] = a.t1.r_msb[i * party + at];
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const T g = c.truncated(i, top[i], msb[i]), mask = a.mask_g[i * party + at];
                e3 += g - mask;
                s[0] += g;
                z += mask * e2;
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) z += e3 * a.xhat.a[i * party + at];
            s[1] += z + e3 * e2;
            open_g[d] = e3;
            open_x[d] = e2;
        }
        __syncthreads();
        block_sums(s, room);
        T m[NP], k1[NP], k2[NP], r[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            s[1] += w.at(i, 3);
            r[i] = a.rstd[(size_t)i * a.rows + row];
        }
        const T fr = w.open(r, 10);
        w.truncate(a.inv * s[0], 0, a.shift, m);
        w.truncate(w.product(12, w.open(m, 11), 11, fr, 10), 13, a.f, k1);
        w.truncate(s[1], 4, a.f, m);
        w.truncate(a.inv * sum_of<NP>(m), 7, a.shift, m);
        w.truncate(w.product(17, w.open(m, 16), 16, fr, 10), 18, a.f, k2);
        const T ek = w.open(k2, 21);
        for (int d = threadIdx.x; d < a.dim; d += kBlock) {
            const size_t at = first + d;
            const T e3 = open_g[d], e2 = open_x[d];
            T top[NP], msb[NP];
            Opened<T> c{a.f};
            c.add(e3 * fr - e2 * ek);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                c.add(a.C2[i * party + at] + a.t2.r[i * party + at] + e3 * w.at(i, 10) + a.mask_g[i * party + at] * fr);
                c.add(0 - (e2 * w.at(i, 21) + a.xhat.a[i * party + at] * ek));
                top[i] = a.t2.r_top[i * party + at], msb[i] = a.t2.r_msb[i * party + at];
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) a.dx[i * party + at] = c.truncated(i, top[i], msb[i]) - k1[i];
        }
        __syncthreads();
    }
}

// Sums over the rows, a thread a column.
template <int NP, class T> __global__ __launch_bounds__(64) void columns_kernel(NormGradArgs<T> a)
{
    const int d = blockIdx.x * 64 + threadIdx.x;
    if (d >= a.dim) return;
    const size_t party = (size_t)a.rows * a.dim;
    T beta[NP] = {}, z = 0, y[NP];
    for (int row = 0; row < a.rows; ++row) {
        const size_t at = (size_t)row * a.dim + d;
        T e1 = 0, e2 = 0;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const T dy = a.dy.x[i * party + at];
            beta[i] += dy;
            e1 += dy - a.dy.a[i * party + at];
            e2 += a.xhat.x[i * party + at] - a.xhat.a[i * party + at];
        }
        z += e1 * e2;
#pragma unroll
        for (int i = 0; i < NP; ++i) z += e1 * a.xhat.a[i * party + at] + a.dy.a[i * party + at] * e2;
    }
    const Words<NP, T> w{a.column_words + d, (size_t)4 * a.dim, (size_t)a.dim};
#pragma unroll
    for (int i = 0; i < NP; ++i) z += w.at(i, 0);
    w.truncate(z, 1, a.f, y);
#pragma unroll
    for (int i = 0; i < NP; ++i) a.dgamma[(size_t)i * a.dim + d] = y[i], a.dbeta[(size_t)i * a.dim + d] = beta[i];
}

}  // namespace

size_t layernorm_workspace(int, int, int, int) { return 256; }
size_t layernorm_grad_workspace(int, int, int, int) { return 256; }

template <class T> spin_status launch_layernorm(const NormArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_LAYERNORM, s);
    spin_status st = SPIN_OK;
    for_party_count(a.n, [&](auto np) {
        static OncePerDevice lds_flags;
        st = allow_dynamic_lds((const void *)norm_kernel<decltype(np)::value, T>, kMostDim * sizeof(T), lds_flags);
        if (st == SPIN_OK) norm_kernel<decltype(np)::value, T><<<a.rows, kBlock, a.dim * sizeof(T), s>>>(a);
    });
    return st != SPIN_OK ? st : check_launch("spin_layernorm");
}

template <class T> spin_status launch_layernorm_grad(const NormGradArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_LAYERNORM, s);
    spin_status st = SPIN_OK;
    for_party_count(a.n, [&](auto np) {
        static OncePerDevice lds_flags;
        st = allow_dynamic_lds((const void *)norm_grad_kernel<decltype(np)::value, T>, 2 * kMostDim * sizeof(T), lds_flags);
        if (st != SPIN_OK) return;
        norm_grad_kernel<decltype(np)::value, T><<<a.rows, kBlock, 2 * a.dim * sizeof(T), s>>>(a);
        columns_kernel<decltype(np)::value, T><<<(a.dim + 63) / 64, 64, 0, s>>>(a);
    });
    return st != SPIN_OK ? st : check_launch("spin_layernorm_grad");
}

template spin_status launch_layernorm<u64>(const NormArgs<u64> &, hipStream_t);
template spin_status launch_layernorm<u32>(const NormArgs<u32> &, hipStream_t);
template spin_status launch_layernorm_grad<u64>(const NormGradArgs<u64> &, hipStream_t);
template spin_status launch_layernorm_grad<u32>(const NormGradArgs<u32> &, hipStream_t);

}  // namespace spin
