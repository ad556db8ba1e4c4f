// Layer norm of shares (spin_layernorm).  A stream of 13 words an element and party with the chain in the middle: 3 parties, 4096 rows of 1024 286 us, 4.6 TB/s, bound by trips to
// memory one after another: a column's words of the first phase are waited for before the next column's are asked for, and of 64-bit words the last phase's come in several batches (below).
// Few rows are bound by the chain, some seventy dependent steps: 2 rows of 1024 12.2 us.
#include "layernorm.hpp"

namespace spin {
namespace {

// From sum (x - mu)^2 to this lane's share of 1 / sqrt(variance).
template <int NP, class T> __device__ inline T rstd_of(const NormArgs<T> &a, const Chain<NP, T> &w, T square)
{
    T v = w.truncate(w.public_word(square) + w.at(3), 4, a.f);
    v = w.truncate(a.inv * v, 7, a.shift) + w.public_word(a.eps);
    T y = w.truncate(w.public_word(a.offset << a.f) - a.slope * v, 10, a.f);
    const T fv = w.open(v, 13);
#pragma unroll 1
    for (int k = 14; k < 14 + kNormWords * a.iterations; k += kNormWords) {
        const T e = w.open(y, k), u = w.truncate(w.product(k + 1, e, k, e, k), k + 2, a.f);
        const T h = w.public_word((T)3 << a.f) - w.truncate(w.product(k + 6, w.open(u, k + 5), k + 5, fv, 13), k + 7, a.f);
        y = w.truncate(w.product(k + 11, e, k, w.open(h, k + 10), k + 10), k + 12, a.f + 1);
    }
    return y;
}

template <int NP, class T, int WAVES, int EACH>
__global__ __launch_bounds__(kNormBlock<WAVES>, WAVES > 4 ? 4 : 1) void norm_kernel(NormArgs<T> a, bool streamed)
{
    constexpr int ROWS = kRowsAtOnce<WAVES>, THREADS = 64 * WAVES;
    constexpr bool KEEP = NP * EACH * sizeof(T) <= (WAVES > 4 ? 112 : 128);    // the masks stay in registers
    extern __shared__ __align__(16) char lds[];
    __shared__ T partial[ROWS][2][WAVES], shared[ROWS][NP + 2];
    const int slot = WAVES == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : 0, wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int t = threadIdx.x % THREADS, count = kNormWords * (a.iterations + 1);
    const long row = xcd_contiguous_id(blockIdx.x, gridDim.x) * ROWS + slot;
    if (WAVES == 1 && row >= a.rows) return;               // of a whole wave, which meets no barrier
    const size_t party = (size_t)a.rows * a.dim, first = (size_t)row * a.dim;
    T *const words = (T *)lds + (size_t)slot * count * NP;
    const Chain<NP, T> chain{words};
    const bool mine = wave == row % WAVES;                 // this wave runs the chain: another one from row to row, and so on another SIMD
    T open[EACH], mask[EACH][KEEP ? NP : 1], s = 0;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        if (j * THREADS >= a.dim) break;
        const int d = min(j * THREADS + t, a.dim - 1);
        const bool there = j * THREADS + t < a.dim;
        T x[NP], m[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) x[i] = a.x[i * party + first + d], m[i] = a.mask_x[i * party + first + d];
        open[j] = 0;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            open[j] += x[i] - m[i];
            s += there ? x[i] : 0;
            if (KEEP) mask[j][KEEP ? i : 0] = m[i];
        }
        if (NP * EACH > 12) __builtin_amdgcn_sched_barrier(0);
    }
    // One load a turn, waited for before the next: one wave a row takes five turns for three parties and six steps.
    for (int k = t; k < count * NP; k += THREADS) words[k] = a.row_words[((size_t)(k % NP) * count + k / NP) * a.rows + row];
    s = wave_sum(s);
    if (t % 64 == 0) partial[slot][0][wave] = s;
    row_barrier<WAVES>();
    if (mine) {
        s = 0;
        for (int w = 0; w < WAVES; ++w) s += partial[slot][0][w];
        const T mean = chain.sum(chain.truncate(chain.public_word(a.inv * s), 0, a.shift));
        if (t % 64 == 0) shared[slot][0] = mean;
    }
    row_barrier<WAVES>();
    const T mean = shared[slot][0];
    s = 0;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        if (j * THREADS >= a.dim) break;
        const int d = min(j * THREADS + t, a.dim - 1);
        const T e = open[j] -= mean;
        T z = 0;
#pragma unroll
        for (int i = 0; i < NP; ++i) z += e * (2 * (KEEP ? mask[j][KEEP ? i : 0] : a.mask_x[i * party + first + d]) + (i == 0 ? e : 0));
        s += j * THREADS + t < a.dim ? z : 0;
    }
    s = wave_sum(s);
    if (t % 64 == 0) partial[slot][1][wave] = s;
    row_barrier<WAVES>();
    if (mine) {
        s = 0;
        for (int w = 0; w < WAVES; ++w) s += partial[slot][1][w];
        const T y = rstd_of<NP, T>(a, chain, s), fr = chain.open(y, count - 1);
        if (t % 64 < NP) {
            if (a.rstd) a.rstd[(size_t)(t % 64) * a.rows + row] = y;
            shared[slot][1 + t % 64] = chain.at(count - 1) + chain.public_word(fr);
        }
        if (t % 64 == 0) shared[slot][NP + 1] = fr;
    }
    row_barrier<WAVES>();
    const T fr = shared[slot][NP + 1];
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        if (j * THREADS >= a.dim) break;
        u32 d = (u32)min(j * THREADS + t, a.dim - 1);
        const bool there = j * THREADS + t < a.dim;
        auto word = [&](const T *array, int i) __attribute__((always_inline)) { return (array + (i * party + first))[d]; };
        auto dealt = [&](const T *array, int i) __attribute__((always_inline)) { return once(array + (i * party + first) + d); };
        auto column = [&](const T *array, int i) __attribute__((always_inline)) { return (array + (size_t)i * a.dim)[d]; };
        const T e = open[j];
        T top[NP], msb[NP], xhat[NP], g = 0, e2 = 0;
        Opened<T> c{a.f}, c2{a.f};
        if (!KEEP) make_new(d);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            c.add(dealt(a.C1, i) + dealt(a.t1.r, i));
            c.add(e * shared[slot][1 + i] + (KEEP ? mask[j][KEEP ? i : 0] : word(a.mask_x, i)) * fr);
            top[i] = dealt(a.t1.r_top, i), msb[i] = dealt(a.t1.r_msb, i);
        }
        // Where a thread has registers for them all its words can be asked for at once; otherwise the second truncation's behind the first's.  As built, 32-bit words of two parties are (22
        // in one batch); of 64-bit words, three parties, four words a thread, the last column's, while the first three wait six to twelve times each.
        auto first_part = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                xhat[i] = c.truncated(i, top[i], msb[i]);
                e2 += xhat[i] - word(a.mask_xhat, i);
            }
        };
        if (!KEEP) {
            first_part();
            if (a.xhat && there)
#pragma unroll
                for (int i = 0; i < NP; ++i) put(streamed, a.xhat + (i * party + first) + d, xhat[i]);
            make_new(d);
        }
        T top2[NP], msb2[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            g += column(a.gamma.x, i) - column(a.gamma.a, i);
            c2.add(dealt(a.C2, i) + dealt(a.t2.r, i));
            top2[i] = dealt(a.t2.r_top, i), msb2[i] = dealt(a.t2.r_msb, i);
        }
        if (KEEP) first_part();
#pragma unroll
        for (int i = 0; i < NP; ++i) c2.add(e2 * (column(a.gamma.a, i) + (i == 0 ? g : 0)) + word(a.mask_xhat, i) * g);
        if (!there) continue;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if (KEEP && a.xhat) put(streamed, a.xhat + (i * party + first) + d, xhat[i]);
            put(streamed, a.out + (i * party + first) + d, c2.truncated(i, top2[i], msb2[i]) + column(a.beta, i));
        }
        __builtin_amdgcn_sched_barrier(0);                 // a column's words at a time
    }
}

}  // namespace

template <class T> spin_status launch_layernorm(const NormArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_LAYERNORM, s);
    const bool streamed = (size_t)a.n * a.rows * a.dim * sizeof(T) >= kStreamingBytes;
    spin_status st = SPIN_OK;
    for_party_count(a.n, [&](auto np) {
        for_dim(a.rows, a.dim, [&](auto waves, auto each) {
            constexpr int NP = decltype(np)::value, WAVES = decltype(waves)::value, ROWS = kRowsAtOnce<WAVES>;
            constexpr auto kernel = norm_kernel<NP, T, WAVES, decltype(each)::value>;
            constexpr int row_bytes = kNormWords * NP * (int)sizeof(T) * ROWS;
            static OncePerDevice lds_flags;
            st = allow_dynamic_lds((const void *)kernel, row_bytes * (SPIN_MAX_NORM_ITERATIONS + 1), lds_flags);
            if (st == SPIN_OK) kernel<<<(a.rows + ROWS - 1) / ROWS, kNormBlock<WAVES>, row_bytes * (a.iterations + 1), s>>>(a, streamed);
        });
    });
    return st != SPIN_OK ? st : check_launch("spin_layernorm");
}

template spin_status launch_layernorm<u64>(const NormArgs<u64> &, hipStream_t);
template spin_status launch_layernorm<u32>(const NormArgs<u32> &, hipStream_t);

}  // namespace spin
