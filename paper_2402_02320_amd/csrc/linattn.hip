// Linear attention with a decay over chunks of shares (spin_linattn_*).
#include "linear.hpp"

namespace spin {
namespace {

constexpr int kBlock = 256;

// An operand of a product at one place: what is opened, and every party's mask.
template <int NP, class T> struct Factor {
    T open = 0, mask[NP];
};
template <int NP, class T> __device__ inline Factor<NP, T> factor(const Masked<T> &m, size_t party, size_t at)
{
    Factor<NP, T> f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        f.mask[i] = m.a[i * party + at];
        f.open += m.x[i * party + at] - f.mask[i];
    }
    return f;
}
// The sum over the parties of their parts of a product, each from its own mask.
template <int NP, class T> __device__ inline T product(const Factor<NP, T> &x, const Factor<NP, T> &y)
{
    T z = 0;
#pragma unroll
    for (int i = 0; i < NP; ++i) z += x.open * (i == 0 ? y.mask[i] + y.open : y.mask[i]) + x.mask[i] * y.open;
    return z;
}
template <class T> __device__ inline T weight(const T *decay, int head, int chunk, int j) { return decay ? decay[(size_t)head * (chunk + 1) + j] : 1; }

// One element of a result whose parties' products sum to z.
template <int NP, class T> __device__ inline void finish(T z, const T *C, const Tuple<T> &t, int f, size_t party, size_t at, T *out)
{
    Opened<T> c{f};
    c.add(z);
    T top[NP], msb[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        c.add(C[i * party + at] + t.r[i * party + at]);
        top[i] = t.r_top[i * party + at];
        msb[i] = t.r_msb[i * party + at];
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) out[i * party + at] = c.truncated(i, top[i], msb[i]);
}

template <int NP, class T> __global__ __launch_bounds__(kBlock) void scores_kernel(ScoresArgs<T> a)
{
    const int C = a.c.chunk, u = blockIdx.x * kBlock + threadIdx.x, chunk = u / (C * C), i = u / C % C, j = u % C, b = blockIdx.y / a.c.heads, h = blockIdx.y % a.c.heads;
    if (chunk >= a.c.chunks) return;
    const size_t rows = (size_t)a.c.batch * a.c.heads, each = rows * a.c.chunks * C * C, at = ((size_t)blockIdx.y * a.c.chunks + chunk) * C * C + i * C + j;
    if (j > i || i >= tokens_in(a.c, b, chunk)) {
        for (int k = 0; k < NP; ++k) a.out[k * each + at] = 0;
        return;
    }
    const size_t party = rows * a.c.tokens * a.dim, first = ((size_t)blockIdx.y * a.c.tokens + chunk * C) * a.dim;
    T z = 0;
    for (int k = 0; k < a.dim; ++k) z += product(factor<NP>(a.x, party, first + i * a.dim + k), factor<NP>(a.y, party, first + j * a.dim + k));
    finish<NP>(weight(a.decay, h, C, i - j) * z, a.C, a.t, a.c.f + a.c.g, each, at, a.out);
}

// What is opened of a chunk's own part of the next state.
template <int NP, class T> __global__ __launch_bounds__(kBlock) void sums_kernel(StatesArgs<T> a)
{
    const int state = a.rows * a.columns, C = a.c.chunk, b = blockIdx.z / a.c.heads, h = blockIdx.z % a.c.heads, chunk = blockIdx.x, u = blockIdx.y * kBlock + threadIdx.x;
    const int L = tokens_in(a.c, b, chunk);
    if (L == 0 || u >= state) return;
    const int r = u / a.columns, d = u % a.columns;
    const size_t heads = (size_t)a.c.batch * a.c.heads, each = heads * a.c.chunks * state, at = ((size_t)blockIdx.z * a.c.chunks + chunk) * state + u;
    const size_t token = (size_t)blockIdx.z * a.c.tokens + chunk * C;
    T z = 0;
    for (int j = 0; j < L; ++j)
        z += weight(a.decay, h, C, a.reverse ? j + 1 : L - 1 - j) * product(factor<NP>(a.x, heads * a.c.tokens * a.rows, (token + j) * a.rows + r),
                                                                            factor<NP>(a.y, heads * a.c.tokens * a.columns, (token + j) * a.columns + d));
    for (int i = 0; i < NP; ++i) z += a.C[i * each + at] + a.t.r[i * each + at];
    a.opened[at] = z;
}

// From chunk to chunk, a thread an element of the state.
template <int NP, class T> __global__ __launch_bounds__(kBlock) void scan_kernel(StatesArgs<T> a)
{
    const int state = a.rows * a.columns, b = blockIdx.y / a.c.heads, h = blockIdx.y % a.c.heads, u = blockIdx.x * kBlock + threadIdx.x;
    if (u >= state) return;
    const size_t heads = (size_t)a.c.batch * a.c.heads, each = heads * a.c.chunks * state, one = heads * state;
    T S[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) S[i] = a.first ? a.first[i * one + (size_t)blockIdx.y * state + u] : 0;
    for (int k = 0; k < a.c.chunks; ++k) {
        const int chunk = a.reverse ? a.c.chunks - 1 - k : k, L = tokens_in(a.c, b, chunk);
        const size_t at = ((size_t)blockIdx.y * a.c.chunks + chunk) * state + u;
        T top[NP], msb[NP], old[NP];
        Opened<T> c{a.c.f + a.c.g};
        if (L) {
            const T w = weight(a.decay, h, a.c.chunk, L) << a.c.f;
            c.add(a.opened[at]);
#pragma unroll
            for (int i = 0; i < NP; ++i) c.add(w * S[i]), top[i] = a.t.r_top[i * each + at], msb[i] = a.t.r_msb[i * each + at];
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            old[i] = S[i];
            if (L) S[i] = c.truncated(i, top[i], msb[i]);
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) a.states[i * each + at] = old[i];
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) a.last[i * one + (size_t)blockIdx.y * state + u] = S[i];
}

template <int NP, class T> __global__ __launch_bounds__(kBlock) void outputs_kernel(OutputsArgs<T> a)
{
    const int C = a.c.chunk, b = blockIdx.y / a.c.heads, h = blockIdx.y % a.c.heads;
    const size_t u = (size_t)blockIdx.x * kBlock + threadIdx.x;
    if (u >= (size_t)a.c.tokens * a.columns) return;
    const int token = u / a.columns, d = u % a.columns, chunk = token / C, i = token % C, L = tokens_in(a.c, b, chunk);
    const size_t heads = (size_t)a.c.batch * a.c.heads, each = heads * a.c.tokens * a.columns, at = ((size_t)blockIdx.y * a.c.tokens + token) * a.columns + d;
    if (i >= L) {
        for (int k = 0; k < NP; ++k) a.out[k * each + at] = 0;
        return;
    }
    const size_t pairs = ((size_t)blockIdx.y * a.c.chunks + chunk) * C * C, first = (size_t)blockIdx.y * a.c.tokens + chunk * C;
    const size_t state = ((size_t)blockIdx.y * a.c.chunks + chunk) * a.rows * a.columns;
    T z = 0, s = 0;
    for (int j = a.reverse ? i : 0; j < (a.reverse ? L : i + 1); ++j)
        z += product(factor<NP>(a.P, heads * a.c.chunks * C * C, pairs + (a.reverse ? j * C + i : i * C + j)), factor<NP>(a.y, each, (first + j) * a.columns + d));
    for (int k = 0; k < a.rows; ++k)
        s += product(factor<NP>(a.x, heads * a.c.tokens * a.rows, (first + i) * a.rows + k),
                     factor<NP>(a.S, heads * a.c.chunks * a.rows * a.columns, state + (a.transposed ? d * a.rows + k : k * a.columns + d)));
    finish<NP>((z << a.c.g) + weight(a.decay, h, C, a.reverse ? L - 1 - i : i + 1) * s, a.C, a.t, a.c.f + a.c.g, each, at, a.out);
}

// blockIdx.x: 64 columns, of which a thread has one of every fourth row.
template <int NP, class T> __global__ __launch_bounds__(kBlock) void step_kernel(StepArgs<T> a)
{
    __shared__ T sums[kBlock];
    const int d = blockIdx.x * 64 + threadIdx.x % 64, part = threadIdx.x / 64, b = blockIdx.y / a.heads, h = blockIdx.y % a.heads;
    const size_t heads = (size_t)a.batch * a.heads, one = heads * a.rows * a.columns;
    const bool live = !a.active || a.active[b] > 0, mine = d < a.columns;
    T sum = 0;
    if (mine) {
        const T w0 = weight(a.decay, h, 1, 0), w1 = weight(a.decay, h, 1, 1) << a.f;
        const Factor<NP, T> v = factor<NP>(a.v, heads * a.columns, (size_t)blockIdx.y * a.columns + d);
        for (int r = part; r < a.rows; r += kBlock / 64) {
            const size_t at = ((size_t)blockIdx.y * a.rows + r) * a.columns + d;
            T S[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) S[i] = a.S[i * one + at];
            if (live) {
                Opened<T> c{a.f + a.g};
                Factor<NP, T> s;
                T top[NP], msb[NP];
                c.add(w0 * product(factor<NP>(a.k, heads * a.rows, (size_t)blockIdx.y * a.rows + r), v));
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    c.add(w1 * S[i] + a.CS[i * one + at] + a.tS.r[i * one + at]);
                    top[i] = a.tS.r_top[i * one + at], msb[i] = a.tS.r_msb[i * one + at];
                    s.mask[i] = a.S_mask[i * one + at];
                }
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    S[i] = c.truncated(i, top[i], msb[i]);
                    s.open += S[i] - s.mask[i];
                }
                sum += product(factor<NP>(a.q, heads * a.rows, (size_t)blockIdx.y * a.rows + r), s);
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) a.S_out[i * one + at] = S[i];
        }
    }
    sums[threadIdx.x] = sum;
    __syncthreads();
    if (part || !mine) return;
    for (int k = 1; k < kBlock / 64; ++k) sum += sums[threadIdx.x + 64 * k];
    const size_t each = heads * a.columns, at = (size_t)blockIdx.y * a.columns + d;
    if (live) {
        finish<NP>(sum, a.CO, a.tO, a.f, each, at, a.out);
    } else {
        for (int i = 0; i < NP; ++i) a.out[i * each + at] = 0;
    }
}

}  // namespace

template <class T> spin_status launch_linattn_scores(const ScoresArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_LINATTN, s);
    const size_t count = (size_t)a.c.chunks * a.c.chunk * a.c.chunk;
    for_party_count(a.c.n, [&](auto np) {
        scores_kernel<decltype(np)::value, T><<<dim3((unsigned)(count / kBlock), a.c.batch * a.c.heads), kBlock, 0, s>>>(a);
    });
    return check_launch("spin_linattn_scores");
}

template <class T> spin_status launch_linattn_states(const StatesArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_LINATTN, s);
    const unsigned blocks = (a.rows * a.columns + kBlock - 1) / kBlock;
    for_party_count(a.c.n, [&](auto np) {
        sums_kernel<decltype(np)::value, T><<<dim3(a.c.chunks, blocks, a.c.batch * a.c.heads), kBlock, 0, s>>>(a);
        scan_kernel<decltype(np)::value, T><<<dim3(blocks, a.c.batch * a.c.heads), kBlock, 0, s>>>(a);
    });
    return check_launch("spin_linattn_states");
}

template <class T> spin_status launch_linattn_outputs(const OutputsArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_LINATTN, s);
    const size_t count = (size_t)a.c.tokens * a.columns;
    for_party_count(a.c.n, [&](auto np) {
        outputs_kernel<decltype(np)::value, T><<<dim3((unsigned)((count + kBlock - 1) / kBlock), a.c.batch * a.c.heads), kBlock, 0, s>>>(a);
    });
    return check_launch("spin_linattn_outputs");
}

template <class T> spin_status launch_linattn_step(const StepArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_LINATTN, s);
    for_party_count(a.n, [&](auto np) {
        step_kernel<decltype(np)::value, T><<<dim3((a.columns + 63) / 64, a.batch * a.heads), kBlock, 0, s>>>(a);
    });
    return check_launch("spin_linattn_step");
}

template spin_status launch_linattn_scores<u64>(const ScoresArgs<u64> &, hipStream_t);
template spin_status launch_linattn_scores<u32>(const ScoresArgs<u32> &, hipStream_t);
template spin_status launch_linattn_states<u64>(const StatesArgs<u64> &, hipStream_t);
template spin_status launch_linattn_states<u32>(const StatesArgs<u32> &, hipStream_t);
template spin_status launch_linattn_outputs<u64>(const OutputsArgs<u64> &, hipStream_t);
template spin_status launch_linattn_outputs<u32>(const OutputsArgs<u32> &, hipStream_t);
template spin_status launch_linattn_step<u64>(const StepArgs<u64> &, hipStream_t);
template spin_status launch_linattn_step<u32>(const StepArgs<u32> &, hipStream_t);

}  // namespace spin
