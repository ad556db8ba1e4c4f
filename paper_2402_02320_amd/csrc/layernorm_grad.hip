// The gradients of layer norm on shares (spin_layernorm_grad).  A stream of 14 words an element and party with the chain in the middle: 3 parties, 2048 rows of 2048 308 us, 4.6 TB/s, of
// which the sums' join is 6; 5 parties, 1568 rows of 256 52 us.  Bound by trips to memory one after another: as built a column of the former waits about twelve times before the sums
// and four times behind them, with one workgroup a CU to go on meanwhile.
#include "layernorm.hpp"

namespace spin {
namespace {

__device__ inline void add_to(u64 *p, u64 v) { atomicAdd((unsigned long long *)p, (unsigned long long)v); }
__device__ inline void add_to(u32 *p, u32 v) { atomicAdd(p, v); }

// A wave's or workgroup's rows are `run` successive ones; its sums over them (of dgamma one word a column, since that is truncated, of dbeta a party's) stay in registers and are
// added by a second kernel.
// Where registers for those sums are not left (more parties, or words a thread: LEAN) columns_kernel makes them from memory, and no party's words are kept from one use to the next.
template <int NP, class T, int WAVES, int EACH> constexpr bool kLean = EACH > 4 || NP * sizeof(T) * EACH > (WAVES > 4 ? 96 : 160);
template <int NP, class T, int WAVES, int EACH>
__global__ __launch_bounds__(kNormBlock<WAVES>, WAVES > 4 ? 4 : 1) void norm_grad_kernel(NormGradArgs<T> a, int run, T *sums, bool streamed)
{
    constexpr int ROWS = kRowsAtOnce<WAVES>, THREADS = 64 * WAVES;
    constexpr bool LEAN = kLean<NP, T, WAVES, EACH>, KEEP = !LEAN && 2 * NP * EACH * sizeof(T) <= (WAVES > 4 ? 96 : 128);
    __shared__ T partial[ROWS][2][WAVES], shared[ROWS][3 * NP + 2], words_of[ROWS][(kNormGradWords + 1) * NP];
    const int slot = WAVES == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : 0, wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int t = threadIdx.x % THREADS;
    const long group = (long)blockIdx.x * ROWS + slot;     // of rows: a wave's or workgroup's
    const long row0 = group * run, row1 = min(row0 + run, (long)a.rows);
    const size_t party = (size_t)a.rows * a.dim;
    T *const words = words_of[slot];
    const Chain<NP, T> chain{words};
    T gamma_sum[LEAN ? 1 : EACH] = {}, beta_sum[LEAN ? 1 : EACH][NP] = {};
    for (long row = row0; row < row1; ++row) {
        const size_t first = (size_t)row * a.dim;
        const bool mine = wave == row % WAVES;
        T open_g[EACH], open_x[EACH], mask_g[EACH][KEEP ? NP : 1], mask_x[EACH][KEEP ? NP : 1], s[2] = {0, 0};
        for (int k = t; k < kNormGradWords * NP; k += THREADS) words[k] = a.row_words[((size_t)(k % NP) * kNormGradWords + k / NP) * a.rows + row];
        if (t < NP) words[kNormGradWords * NP + t] = a.rstd[(size_t)t * a.rows + row];
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            if (j * THREADS >= a.dim) break;
            u32 d = (u32)min(j * THREADS + t, a.dim - 1);
            make_new(d);
            const bool there = j * THREADS + t < a.dim;
            auto word = [&](const T *array, int i) __attribute__((always_inline)) { return (array + (i * party + first))[d]; };
            auto dealt = [&](const T *array, int i) __attribute__((always_inline)) { return once(array + (i * party + first) + d); };
            auto column = [&](const T *array, int i) __attribute__((always_inline)) { return (array + (size_t)i * a.dim)[d]; };
            T fg = 0, e1 = 0, e2 = 0, e3 = 0, z = 0;
            Opened<T> c{a.f};
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                e1 += word(a.dy.x, i) - word(a.dy.a, i);
                e2 += word(a.xhat.x, i) - word(a.xhat.a, i);
                fg += column(a.gamma.x, i) - column(a.gamma.a, i);
                if (!LEAN) beta_sum[LEAN ? 0 : j][i] += word(a.dy.x, i);
            }
            if (LEAN) make_new(d);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                c.add(dealt(a.C1, i) + dealt(a.t1.r, i));
                c.add(e1 * (column(a.gamma.a, i) + (i == 0 ? fg : 0)) + word(a.dy.a, i) * fg);
                if (!LEAN) gamma_sum[LEAN ? 0 : j] += e1 * (word(a.xhat.a, i) + (i == 0 ? e2 : 0)) + word(a.dy.a, i) * e2;
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const T g = c.truncated(i, dealt(a.t1.r_top, i), dealt(a.t1.r_msb, i));
                e3 += g - word(a.mask_g, i);
                s[0] += there ? g : 0;
            }
            if (LEAN) make_new(d);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                z += e3 * (word(a.xhat.a, i) + (i == 0 ? e2 : 0)) + word(a.mask_g, i) * e2;
                if (KEEP) mask_g[j][KEEP ? i : 0] = word(a.mask_g, i), mask_x[j][KEEP ? i : 0] = word(a.xhat.a, i);
            }
            s[1] += there ? z : 0;
            open_g[j] = e3;
            open_x[j] = e2;
            // Computed here: left alone sums are put off, and the words they are made of stay in registers.
            if (!LEAN) {
                computed_here(gamma_sum[LEAN ? 0 : j]);
#pragma unroll
                for (int i = 0; i < NP; ++i) computed_here(beta_sum[LEAN ? 0 : j][i]);
            }
            computed_here(s[0]);
            computed_here(s[1]);
            computed_here(open_g[j]);
            computed_here(open_x[j]);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            s[k] = wave_sum(s[k]);
            if (t % 64 == 0) partial[slot][k][wave] = s[k];
        }
        row_barrier<WAVES>();
        if (mine) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                s[k] = 0;
                for (int w = 0; w < WAVES; ++w) s[k] += partial[slot][k][w];
            }
            const T fr = chain.open(chain.at(kNormGradWords), 10);
            T m = chain.truncate(chain.public_word(a.inv * s[0]), 0, a.shift);
            const T k1 = chain.truncate(chain.product(12, chain.open(m, 11), 11, fr, 10), 13, a.f);
            m = chain.truncate(a.inv * chain.truncate(chain.public_word(s[1]) + chain.at(3), 4, a.f), 7, a.shift);
            const T k2 = chain.truncate(chain.product(17, chain.open(m, 16), 16, fr, 10), 18, a.f), ek = chain.open(k2, 21);
            if (t % 64 < NP) {
                shared[slot][2 + t % 64] = chain.at(10) + chain.public_word(fr);
                shared[slot][2 + NP + t % 64] = chain.at(21) + chain.public_word(ek);
                shared[slot][2 + 2 * NP + t % 64] = k1;
            }
            if (t % 64 == 0) shared[slot][0] = fr, shared[slot][1] = ek;
        }
        row_barrier<WAVES>();
        const T fr = shared[slot][0], ek = shared[slot][1];
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            if (j * THREADS >= a.dim) break;
            u32 d = (u32)min(j * THREADS + t, a.dim - 1);
            make_new(d);
            auto word = [&](const T *array, int i) __attribute__((always_inline)) { return (array + (i * party + first))[d]; };
            auto dealt = [&](const T *array, int i) __attribute__((always_inline)) { return once(array + (i * party + first) + d); };
            const T e3 = open_g[j], e2 = open_x[j];
            T top[NP], msb[NP];
            Opened<T> c{a.f};
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                c.add(dealt(a.C2, i) + dealt(a.t2.r, i));
                c.add(e3 * shared[slot][2 + i] + (KEEP ? mask_g[j][KEEP ? i : 0] : word(a.mask_g, i)) * fr);
                c.add(0 - (e2 * shared[slot][2 + NP + i] + (KEEP ? mask_x[j][KEEP ? i : 0] : word(a.xhat.a, i)) * ek));
                top[i] = dealt(a.t2.r_top, i), msb[i] = dealt(a.t2.r_msb, i);
            }
            if (j * THREADS + t >= a.dim) continue;
#pragma unroll
            for (int i = 0; i < NP; ++i) put(streamed, a.dx + (i * party + first) + d, c.truncated(i, top[i], msb[i]) - shared[slot][2 + 2 * NP + i]);
            __builtin_amdgcn_sched_barrier(0);
        }
        row_barrier<WAVES>();
    }
    if constexpr (!LEAN) {
        T *const to = sums + (size_t)blockIdx.x * (NP + 1) * a.dim;
        if constexpr (WAVES == 1) {                        // four waves' sums first meet in LDS
            __shared__ T room[(NP + 1) * THREADS * EACH];
            for (int k = threadIdx.x; k < (NP + 1) * a.dim; k += kNormBlock<WAVES>) room[k] = 0;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const int d = j * THREADS + t;
                if (d >= a.dim) break;
                add_to(&room[d], gamma_sum[j]);
#pragma unroll
                for (int i = 0; i < NP; ++i) add_to(&room[(1 + i) * a.dim + d], beta_sum[j][i]);
            }
            __syncthreads();
            for (int k = threadIdx.x; k < (NP + 1) * a.dim; k += kNormBlock<WAVES>) to[k] = room[k];
        } else {
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const int d = j * THREADS + t;
                if (d >= a.dim) break;
                to[d] = gamma_sum[j];
#pragma unroll
                for (int i = 0; i < NP; ++i) to[(size_t)(1 + i) * a.dim + d] = beta_sum[j][i];
            }
        }
    }
}

// The same sums, of the rows of a group, from memory.  blockIdx.x = 64 columns, blockIdx.y = group.
constexpr int kColumnRows = 4;
template <int NP, class T> __global__ __launch_bounds__(64 * kColumnRows) void columns_kernel(NormGradArgs<T> a, int run, T *sums)
{
    __shared__ T room[kColumnRows][NP + 1][64];
    const int lane = threadIdx.x % 64, part = threadIdx.x / 64, d = blockIdx.x * 64 + lane, at = min(d, a.dim - 1);
    const size_t party = (size_t)a.rows * a.dim;
    const long row0 = (long)blockIdx.y * run, row1 = min(row0 + run, (long)a.rows);
    T beta[NP] = {}, z = 0;
    for (long row = row0 + part; row < row1; row += kColumnRows) {
        const size_t first = (size_t)row * a.dim + at;
        T e1 = 0, e2 = 0, m1[NP], m2[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const T dy = a.dy.x[i * party + first];
            m1[i] = a.dy.a[i * party + first], m2[i] = a.xhat.a[i * party + first];
            beta[i] += dy;
            e1 += dy - m1[i];
            e2 += a.xhat.x[i * party + first] - m2[i];
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) z += e1 * (m2[i] + (i == 0 ? e2 : 0)) + m1[i] * e2;
    }
    room[part][0][lane] = z;
#pragma unroll
    for (int i = 0; i < NP; ++i) room[part][1 + i][lane] = beta[i];
    __syncthreads();
    if (d >= a.dim) return;
    for (int k = part; k < NP + 1; k += kColumnRows) {
        T sum = 0;
        for (int p = 0; p < kColumnRows; ++p) sum += room[p][k][lane];
        sums[((size_t)blockIdx.y * (NP + 1) + k) * a.dim + d] = sum;
    }
}

// Adds them: kJoinRows threads a column, each every kJoinRows-th group.  blockIdx.y: 0 dgamma, 1 + i party i's dbeta.
constexpr int kJoinBlock = 256, kJoinColumns = 32, kJoinRows = kJoinBlock / kJoinColumns;
template <int NP, class T> __global__ __launch_bounds__(kJoinBlock) void join_kernel(NormGradArgs<T> a, long groups, const T *sums)
{
    __shared__ T room[kJoinRows][kJoinColumns];
    const int d = blockIdx.x * kJoinColumns + threadIdx.x % kJoinColumns, part = threadIdx.x / kJoinColumns;
    T z = 0;
    if (d < a.dim) {
#pragma unroll 8
        for (long k = part; k < groups; k += kJoinRows) z += sums[(k * (NP + 1) + blockIdx.y) * a.dim + d];
    }
    room[part][threadIdx.x % kJoinColumns] = z;
    __syncthreads();
    if (part || d >= a.dim) return;
#pragma unroll
    for (int k = 1; k < kJoinRows; ++k) z += room[k][threadIdx.x];
    if (blockIdx.y) {
        a.dbeta[(size_t)(blockIdx.y - 1) * a.dim + d] = z;
        return;
    }
    Opened<T> c{a.f};
    c.add(z);
    T top[NP], msb[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const T *w = a.column_words + (size_t)4 * i * a.dim + d;
        c.add(w[0] + w[a.dim]);
        top[i] = w[2 * (size_t)a.dim], msb[i] = w[3 * (size_t)a.dim];
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) a.dgamma[(size_t)i * a.dim + d] = c.truncated(i, top[i], msb[i]);
}

}  // namespace

size_t layernorm_grad_workspace(int n, int rows, int dim, int word_bytes) { return (size_t)norm_most_groups(rows, dim) * (n + 1) * dim * word_bytes; }

template <class T> spin_status launch_layernorm_grad(const NormGradArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_LAYERNORM, s);
    const NormRuns r = norm_runs(a.rows, a.dim);
    const bool streamed = (size_t)a.n * a.rows * a.dim * sizeof(T) >= kStreamingBytes;
    T *const sums = (T *)a.workspace;
    for_party_count(a.n, [&](auto np) {
        constexpr int NP = decltype(np)::value;
        for_dim(a.rows, a.dim, [&](auto waves, auto each) {
            constexpr int WAVES = decltype(waves)::value, ROWS = kRowsAtOnce<WAVES>;
            norm_grad_kernel<NP, T, WAVES, decltype(each)::value><<<r.groups, kNormBlock<WAVES>, 0, s>>>(a, r.run, sums, streamed);
            if constexpr (kLean<NP, T, WAVES, decltype(each)::value>)
                columns_kernel<NP, T><<<dim3((a.dim + 63) / 64, r.groups), 64 * kColumnRows, 0, s>>>(a, r.run * ROWS, sums);
        });
        join_kernel<NP, T><<<dim3((a.dim + kJoinColumns - 1) / kJoinColumns, NP + 1), kJoinBlock, 0, s>>>(a, r.groups, sums);
    });
    return check_launch("spin_layernorm_grad");
}

template spin_status launch_layernorm_grad<u64>(const NormGradArgs<u64> &, hipStream_t);
template spin_status launch_layernorm_grad<u32>(const NormGradArgs<u32> &, hipStream_t);

}  // namespace spin
