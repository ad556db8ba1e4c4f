// Products of new tokens with the paged cache of shares (spin_cache_scores, spin_cache_values), on int8 MFMA.
//
// A ring word is rewritten as ND balanced digits of eight bits (limb_common.hpp); a product of words is the sum over digit pairs i + j < ND on
// v_mfma_i32_16x16x64_i8, pairs of one diagonal sharing an accumulator: 36 int8 products a multiply-add of 64-bit words, 10 of 32-bit ones.
// The cache stays in ring words, read once from HBM straight into the registers of the wave that multiplies them and split there: a lane's 16 k of a
// fragment may be any 16 as long as both factors take the same, so they are those that its 16-byte loads bring,
//     k(j, h, e) = 4 W j + W h + e       (W words in 16 bytes, h = lane / 16, e < W),
// which makes the four lanes of a row read 64 bytes side by side.  The new tokens' factor (E and every A_i, 16 rows) is split once a workgroup
// into LDS, in fragment order.  All parties' products stay in the registers of one wave, so the truncation needs no second pass.
#include "generation.hpp"
#include "limb_common.hpp"

namespace spin {
namespace {

constexpr int kTile = 16;              // query rows, and cached rows (scores) or columns (values), of one MFMA
constexpr int kDepth = 64;             // k of one MFMA

template <class T> struct Lane {
    static constexpr int ND = sizeof(T), W = 16 / sizeof(T), loads = 16 / W;
};

// 16 words -> ND fragments of 16 bytes: byte q of fragment d is digit d of word q.
template <class T> __device__ inline void split(const T (&w)[16], v4i (&p)[sizeof(T)])
{
#pragma unroll
    for (int half = 0; half < (int)sizeof(T) / 4; ++half)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            u32 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = (u32)(to_digits<T>(w[4 * q + k]) >> (32 * half));
            const u32 t0 = __builtin_amdgcn_perm(v[1], v[0], 0x05010400u), t1 = __builtin_amdgcn_perm(v[1], v[0], 0x07030602u);
            const u32 t2 = __builtin_amdgcn_perm(v[3], v[2], 0x05010400u), t3 = __builtin_amdgcn_perm(v[3], v[2], 0x07030602u);
            p[4 * half + 0][q] = (int)__builtin_amdgcn_perm(t2, t0, 0x05040100u);
            p[4 * half + 1][q] = (int)__builtin_amdgcn_perm(t2, t0, 0x07060302u);
            p[4 * half + 2][q] = (int)__builtin_amdgcn_perm(t3, t1, 0x05040100u);
            p[4 * half + 3][q] = (int)__builtin_amdgcn_perm(t3, t1, 0x07060302u);
        }
}

// The digits of W words, the e-th of them at byte q + e of lane `lane`, into the ND fragments at `frag`.
__device__ inline void put_digits(char *frag, int lane, int q, const u64 (&w)[2])
{
    const u64 a = to_digits<u64>(w[0]), b = to_digits<u64>(w[1]);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const u32 lo = (u32)(a >> (32 * half)), hi = (u32)(b >> (32 * half));
        const u32 p = __builtin_amdgcn_perm(hi, lo, 0x05010400u), r = __builtin_amdgcn_perm(hi, lo, 0x07030602u);
        char *at = frag + 4 * half * kFrag + lane * 16 + q;
        *(uint16_t *)(at) = (uint16_t)p;
        *(uint16_t *)(at + kFrag) = (uint16_t)(p >> 16);
        *(uint16_t *)(at + 2 * kFrag) = (uint16_t)r;
        *(uint16_t *)(at + 3 * kFrag) = (uint16_t)(r >> 16);
    }
}
__device__ inline void put_digits(char *frag, int lane, int q, const u32 (&w)[4])
{
    u32 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = to_digits<u32>(w[k]);
    const u32 t0 = __builtin_amdgcn_perm(v[1], v[0], 0x05010400u), t1 = __builtin_amdgcn_perm(v[1], v[0], 0x07030602u);
    const u32 t2 = __builtin_amdgcn_perm(v[3], v[2], 0x05010400u), t3 = __builtin_amdgcn_perm(v[3], v[2], 0x07030602u);
    char *at = frag + lane * 16 + q;
    *(u32 *)(at) = __builtin_amdgcn_perm(t2, t0, 0x05040100u);
    *(u32 *)(at + kFrag) = __builtin_amdgcn_perm(t2, t0, 0x07060302u);
    *(u32 *)(at + 2 * kFrag) = __builtin_amdgcn_perm(t3, t1, 0x05040100u);
    *(u32 *)(at + 3 * kFrag) = __builtin_amdgcn_perm(t3, t1, 0x07060302u);
}

// acc += left . right over all digit pairs that count; left: ND fragments in LDS, this lane's 16 bytes of the first at `left`.
template <class T> __device__ inline void multiply(v4i (&acc)[sizeof(T)], const char *left, const v4i (&right)[sizeof(T)])
{
#pragma unroll
    for (int j = 0; j < (int)sizeof(T); ++j) {
        const v4i a = *(const v4i *)(left + j * kFrag);
#pragma unroll
        for (int i = 0; i + j < (int)sizeof(T); ++i) acc[i + j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, right[i], acc[i + j], 0, 0, 0);
    }
}

// The word whose diagonals are acc[..][r].
template <class T> __device__ inline T recombine(const v4i (&acc)[sizeof(T)], int r)
{
    T v = 0;
#pragma unroll
    for (int d = (int)sizeof(T) - 1; d >= 0; --d) v = (v << 8) + (T)(std::make_signed_t<T>)acc[d][r];
    return v;
}

// ---- scores -----------------------------------------------------------------------------------------------------
// A workgroup: 16 rows (query heads of one cached head, times nodes) against runs of 64 cached tokens, 16 a wave.  One k-tile of 64 elements after another;
// `held` k-tiles of the rows' digits are in LDS: all of them, or (heads so long and parties so many that they do not fit) the one at hand.
constexpr int kScoreWaves = 4, kScoreBlock = 64 * kScoreWaves;

template <int NP, class T>
__global__ __launch_bounds__(kScoreBlock, NP * (int)sizeof(T) <= 40 ? 2 : 1) void scores_kernel(AttentionArgs<T> a, int runs, int held)
{
    using L = Lane<T>;
    constexpr int ND = L::ND, W = L::W;
    typedef T vec __attribute__((ext_vector_type(L::W)));
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane / 16;
    const int b = blockIdx.z, share = a.heads / a.c.heads, R = share * a.d.nodes, row_tiles = (R + kTile - 1) / kTile;
    const int g = blockIdx.y / row_tiles, row0 = blockIdx.y % row_tiles * kTile;
    const size_t rows = (size_t)a.batch * a.heads * a.d.nodes, first_row = ((size_t)b * a.heads + (size_t)g * share) * a.d.nodes + row0;
    const int context = a.d.context[b], dim = a.c.dim;
    const int limit = context < 0 ? 0 : (int)min((long)a.d.columns, (long)context + a.d.nodes);
    const int k_tiles = (dim + kDepth - 1) / kDepth;

    auto stage = [&](int kt0, int count) __attribute__((always_inline)) {                // digits of E and A_i of k-tiles kt0 .. kt0 + count - 1
        const int per_row = count * (kDepth / W);
        for (int c = threadIdx.x; c < kTile * per_row; c += kScoreBlock) {
            const int row = c / per_row, part = c % per_row, at = (kt0 * (kDepth / W) + part) * W;
            const bool there = row0 + row < R && at < dim;
            const size_t from = there ? (first_row + row) * dim + at : 0;
            vec q[NP], m[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                q[i] = *(const vec *)(a.x + i * rows * dim + from);
                m[i] = *(const vec *)(a.A + i * rows * dim + from);
            }
            const int p = part % (kDepth / W), to = (p % 4) * 16 + row, byte = p / 4 * W;
            char *frag = lds + (part / (kDepth / W)) * (ND * kFrag);
            T e[W];
#pragma unroll
            for (int k = 0; k < W; ++k) {
                e[k] = 0;
#pragma unroll
                for (int i = 0; i < NP; ++i) e[k] += there ? q[i][k] - m[i][k] : 0;
            }
            put_digits(frag, to, byte, e);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                T w[W];
#pragma unroll
                for (int k = 0; k < W; ++k) w[k] = there ? m[i][k] : 0;
                put_digits(frag + (i + 1) * held * (ND * kFrag), to, byte, w);
            }
        }
    };
    const bool whole = held >= k_tiles;
    if (whole && blockIdx.x * (runs * kDepth) < (unsigned)limit) {
        stage(0, k_tiles);
        __syncthreads();
    }
    const size_t slot = ((size_t)a.c.pages * a.c.heads << a.c.shift) * dim;
    for (int run = 0; run < runs; ++run) {
        const int first = (blockIdx.x * runs + run) * (kScoreWaves * kTile);
        if (first >= a.d.columns) break;                   // of the whole workgroup
        const int t0 = first + wave * kTile, t = t0 + lane % 16;
        const int page = page_of(a.c, b, t);
        T z[NP][4];
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) z[i][r] = 0;
        if (first < limit) {                               // of the whole workgroup
            const T *key = a.pool + row_at(a.c, 0, max(page, 0), g, page < 0 ? 0 : t) + h * W;
            for (int kt = 0; kt < k_tiles; ++kt) {
                if (!whole) {
                    __syncthreads();
                    stage(kt, 1);
                    __syncthreads();
                }
                const char *left = lds + (whole ? kt : 0) * (ND * kFrag) + lane * 16;
                const bool full = (kt + 1) * kDepth <= dim;
                vec raw[L::loads];
                auto load = [&](int s) __attribute__((always_inline)) {
                    const T *from = key + (s * slot + kt * kDepth);
                    if (full) {
#pragma unroll
                        for (int j = 0; j < L::loads; ++j) raw[j] = *(const vec *)(from + j * (4 * W));
                    } else {                               // past the row's end the rows' digits are zero, whatever is read
#pragma unroll
                        for (int j = 0; j < L::loads; ++j) raw[j] = *(const vec *)(kt * kDepth + j * (4 * W) + h * W < dim ? from + j * (4 * W) : key + s * slot);
                    }
                };
                // A slot's words are split into fragments before its products, which leaves their registers to the next slot's loads.
                auto take = [&](v4i (&p)[ND]) __attribute__((always_inline)) {
                    T w[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) w[j] = raw[j / W][j % W];
                    split<T>(w, p);
                };
                v4i f[ND];
                load(0);
                take(f);
                load(1);
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    v4i right[ND], acc[ND];
#pragma unroll
                    for (int d = 0; d < ND; ++d) acc[d] = v4i{0, 0, 0, 0};
                    take(right);
                    __builtin_amdgcn_sched_barrier(0);
                    if (i + 1 < NP) load(i + 2);
                    __builtin_amdgcn_sched_barrier(0);
                    multiply<T>(acc, left, right);
                    multiply<T>(acc, left + (i + 1) * held * (ND * kFrag), f);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        z[i][r] += recombine<T>(acc, r);
                        computed_here(z[i][r]);            // not at the end, with all parties' diagonals kept until then
                    }
                }
            }
        }
        // row 4 h + r, token t
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            __builtin_amdgcn_sched_barrier(0);
            const int row = row0 + 4 * h + r, m = row % a.d.nodes;
            if (row >= R || t >= a.d.columns) continue;
            const size_t at = (first_row + 4 * h + r) * a.d.columns + t, party = rows * a.d.columns;
            if (page < 0 || !sees(tree_row(a.d, b, m), a.d.nodes, context, t)) {
#pragma unroll
                for (int i = 0; i < NP; ++i) a.out[i * party + at] = i == 0 ? a.masked : 0;
                continue;
            }
            int bucket = -1;
            const T *bias = (const T *)a.bias.table + (size_t)(g * share + row / a.d.nodes) * a.bias.buckets;
            if (a.bias.table) {
                auto place = [&](int node) { return a.depth ? a.depth[(size_t)b * a.d.nodes + node] : node; };
                const long away = (t < context ? (long)t - context : place(t - context)) - (long)place(m);
                bucket = bucket_at(a.bias, (int)min(max(away, -(long)a.bias.reach), (long)a.bias.reach));
            }
            Opened<T> c{a.f};
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                z[i][r] += a.C[i * party + at];
                if (a.f) c.add(z[i][r] + a.r[i * party + at]);
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                T y = a.f ? c.truncated(i, a.r_top[i * party + at], a.r_msb[i * party + at]) : z[i][r];
                if (bucket >= 0) y += bias[(size_t)i * a.heads * a.bias.buckets + bucket];
                a.out[i * party + at] = y;
            }
        }
    }
}

// ---- values -----------------------------------------------------------------------------------------------------
// A workgroup: 16 rows and a few tiles of 16 columns over a range of cached tokens, 64 at a time.  A wave has one column tile and up to three
// parties (64-bit words), whose diagonals stay in its registers: 4 ND a party of the 256 that two waves a SIMD leave each.  The rows' digits of the next 64
// tokens are split into the other half of LDS while the matrix cores work on these.  int32 diagonals hold eight pairs and two products of at
// most 2^14 a token, so a range is at most kMostTokens long (16 x 4096 x 2^14 = 2^30).
constexpr int kMostTokens = 4096;
constexpr int kValueWaves = 8, kValueBlock = 64 * kValueWaves;
constexpr int value_groups(int n, int word_bytes) { return word_bytes == 4 || n <= 3 ? 1 : n <= 6 ? 2 : 4; }      // of parties
template <int NP, class T> struct ValueShape {
    static constexpr int groups = value_groups(NP, sizeof(T)), parties = (NP + groups - 1) / groups, tiles = kValueWaves / groups;
    static constexpr int lds = 2 * (NP + 1) * (int)sizeof(T) * kFrag;
};

template <int NP, class T>
__global__ __launch_bounds__(kValueBlock) void values_kernel(AttentionArgs<T> a, int range, T *partial)
{
    using L = Lane<T>;
    using S = ValueShape<NP, T>;
    constexpr int ND = L::ND, W = L::W, kStage = (NP + 1) * ND * kFrag;
    constexpr bool kEarly = NP <= 4;                                    // their loads (8 registers a party) wait in registers during a turn's products
    typedef T vec __attribute__((ext_vector_type(L::W), aligned(sizeof(T))));
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane / 16;
    const int share = a.heads / a.c.heads, R = share * a.d.nodes, row_tiles = (R + kTile - 1) / kTile, dim = a.c.dim;
    const int column_blocks = (dim + S::tiles * kTile - 1) / (S::tiles * kTile);
    int rest = blockIdx.y;
    const int row0 = rest % row_tiles * kTile;
    rest /= row_tiles;
    const int col0 = (rest % column_blocks * S::tiles + wave % S::tiles) * kTile, party0 = wave / S::tiles * S::parties;
    const int g = rest / column_blocks, b = blockIdx.z;
    const size_t rows = (size_t)a.batch * a.heads * a.d.nodes, first_row = ((size_t)b * a.heads + (size_t)g * share) * a.d.nodes + row0;
    const int context = a.d.context[b];
    const int limit = context < 0 ? 0 : (int)min((long)a.d.columns, (long)context + a.d.nodes);
    const int begin = blockIdx.x * range, end = min(begin + range, limit);

    vec x[NP], m[NP];
    const int my_row = threadIdx.x / (kDepth / W), my_part = threadIdx.x % (kDepth / W);       // this thread's W tokens of the rows' 64
    const bool my_there = my_row < kTile && row0 + my_row < R;
    const u64 my_tree = my_there ? tree_row(a.d, b, (row0 + my_row) % a.d.nodes) : 0;
    auto fetch = [&](int t0) __attribute__((always_inline)) {                                  // P and A
        const int t = t0 + my_part * W;
        const size_t from = (first_row + my_row) * a.d.columns + t;
        if (my_there && t + W <= a.d.columns) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                x[i] = *(const vec *)(a.x + i * rows * a.d.columns + from);
                m[i] = *(const vec *)(a.A + i * rows * a.d.columns + from);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    const bool one = my_there && t + e < a.d.columns;
                    x[i][e] = one ? a.x[i * rows * a.d.columns + from + e] : 0;
                    m[i][e] = one ? a.A[i * rows * a.d.columns + from + e] : 0;
                }
        }
    };
    auto stage = [&](int t0, char *to) __attribute__((always_inline)) {                        // their digits, zero where nothing is seen
        if (my_row >= kTile) return;
        const int t = t0 + my_part * W, page = page_of(a.c, b, t);                             // a page holds a multiple of W tokens
        T w[W];
        bool seen[W];
#pragma unroll
        for (int e = 0; e < W; ++e) {
            seen[e] = my_there && page >= 0 && t + e < end && sees(my_tree, a.d.nodes, context, t + e);
            w[e] = 0;
#pragma unroll
            for (int i = 0; i < NP; ++i) w[e] += x[i][e] - m[i][e];
            w[e] = seen[e] ? w[e] : 0;
        }
        put_digits(to, (my_part % 4) * 16 + my_row, my_part / 4 * W, w);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
#pragma unroll
            for (int e = 0; e < W; ++e) w[e] = seen[e] ? m[i][e] : 0;
            put_digits(to + (i + 1) * (ND * kFrag), (my_part % 4) * 16 + my_row, my_part / 4 * W, w);
        }
    };
    static_assert(kTile * kDepth / W <= kValueBlock, "one piece a thread");
    v4i acc[S::parties][ND];
#pragma unroll
    for (int i = 0; i < S::parties; ++i)
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[i][d] = v4i{0, 0, 0, 0};
    const u32 column = min(col0 + lane % 16, dim - 1);     // a column past the row's end reads the last one; it is not stored
    const size_t slot = ((size_t)a.c.pages * a.c.heads << a.c.shift) * dim;
    if (begin < end) {
        fetch(begin);
        stage(begin, lds);
    }
    __syncthreads();
    for (int t0 = begin, turn = 0; t0 < end; t0 += kDepth, turn ^= 1) {
        if (kEarly && t0 + kDepth < end) fetch(t0 + kDepth);
        if (col0 < dim) {
            const T *base[L::loads];                       // of 4 W tokens, which are on one page
#pragma unroll
            for (int j = 0; j < L::loads; ++j) {
                const int page = __builtin_amdgcn_readfirstlane(page_of(a.c, b, t0 + j * 4 * W));
                base[j] = a.pool + row_at(a.c, 0, max(page, 0), g, page < 0 ? 0 : t0 + j * 4 * W);
            }
            T w[16];
            auto load = [&](int s) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 16; ++j) w[j] = (base[j / W] + s * slot)[(u32)((h * W + j % W) * dim) + column];
            };
            const char *left = lds + turn * kStage + lane * 16;
            v4i f[ND];
            load(0);
            split<T>(w, f);
            load(party0 + 1);
#pragma unroll
            for (int i = 0; i < S::parties; ++i) {         // a wave whose parties end before has its last one twice, and stores it once
                v4i right[ND];
                split<T>(w, right);
                __builtin_amdgcn_sched_barrier(0);         // its words' registers are the next slot's loads'
                if (i + 1 < S::parties) load(min(party0 + i + 2, NP));
                __builtin_amdgcn_sched_barrier(0);
                multiply<T>(acc[i], left, right);
                multiply<T>(acc[i], left + min(party0 + i + 1, NP) * (ND * kFrag), f);
            }
        }
        if (t0 + kDepth < end) {
            if (!kEarly) fetch(t0 + kDepth);
            stage(t0 + kDepth, lds + (turn ^ 1) * kStage);
        }
        __syncthreads();
    }
    const int col = col0 + lane % 16;
    if (col >= dim) return;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (row0 + 4 * h + r >= R) continue;
        const size_t at = (first_row + 4 * h + r) * dim + col, party = rows * dim;
        T y[S::parties];
#pragma unroll
        for (int i = 0; i < S::parties; ++i) y[i] = recombine<T>(acc[i], r);
        if (S::groups > 1 || partial) {
#pragma unroll
            for (int i = 0; i < S::parties; ++i)
                if (party0 + i < NP) partial[((size_t)blockIdx.x * NP + party0 + i) * party + at] = y[i];
            continue;
        }
        if constexpr (S::groups == 1) {
            T tr[NP], t_top[NP], t_msb[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                y[i] += a.C[i * party + at];
                if (a.f) tr[i] = a.r[i * party + at], t_top[i] = a.r_top[i * party + at], t_msb[i] = a.r_msb[i * party + at];
            }
            if (a.f) truncate_shares<NP, T>(y, tr, t_top, t_msb, a.f);
#pragma unroll
            for (int i = 0; i < NP; ++i) a.out[i * party + at] = y[i];
        }
    }
}

// Adds the ranges' parts onto C and truncates.
constexpr int kJoinBlock = 256;
template <int NP, class T> __global__ __launch_bounds__(kJoinBlock) void join_kernel(AttentionArgs<T> a, int ranges, const T *partial)
{
    const size_t party = (size_t)a.batch * a.heads * a.d.nodes * a.c.dim, at = (size_t)blockIdx.x * kJoinBlock + threadIdx.x;
    if (at >= party) return;
    T y[NP], tr[NP], t_top[NP], t_msb[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        y[i] = a.C[i * party + at];
        if (a.f) tr[i] = a.r[i * party + at], t_top[i] = a.r_top[i * party + at], t_msb[i] = a.r_msb[i * party + at];
    }
    for (int p = 0; p < ranges; ++p)
#pragma unroll
        for (int i = 0; i < NP; ++i) y[i] += partial[((size_t)p * NP + i) * party + at];
    if (a.f) truncate_shares<NP, T>(y, tr, t_top, t_msb, a.f);
#pragma unroll
    for (int i = 0; i < NP; ++i) a.out[i * party + at] = y[i];
}

int value_range(int n, int batch, int heads, int cached_heads, int nodes, int columns, int dim, int word_bytes)
{
    const int width = kValueWaves / value_groups(n, word_bytes) * kTile;
    const long groups = (long)batch * cached_heads * ((heads / cached_heads * nodes + kTile - 1) / kTile) * ((dim + width - 1) / width);
    const long wanted = 1024;                              // workgroups
    const long ranges = (wanted + groups - 1) / groups;
    const long range = ((columns + ranges - 1) / ranges + kDepth - 1) / kDepth * kDepth;
    return (int)(range > kMostTokens ? kMostTokens : range);
}
inline bool value_parts(int n, int ranges, int word_bytes) { return ranges > 1 || value_groups(n, word_bytes) > 1; }

}  // namespace

size_t cache_values_workspace(int n, int batch, int heads, int cached_heads, int nodes, int columns, int dim, int word_bytes)
{
    const int range = value_range(n, batch, heads, cached_heads, nodes, columns, dim, word_bytes);
    const size_t ranges = ((size_t)columns + range - 1) / range;
    return 256 + (value_parts(n, (int)ranges, word_bytes) ? ranges * n * batch * heads * nodes * dim * word_bytes : 0);
}

template <class T> spin_status launch_cache_scores(const AttentionArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_ATTENTION, s);
    constexpr int kMostLds = 160 << 10;
    const int R = a.heads / a.c.heads * a.d.nodes, row_tiles = (R + kTile - 1) / kTile, k_tiles = (a.c.dim + kDepth - 1) / kDepth;
    spin_status st = SPIN_OK;
    for_party_count(a.n, [&](auto np) {
        constexpr int NP = decltype(np)::value, kSlots = (NP + 1) * (int)sizeof(T) * kFrag;
        const int held = k_tiles * kSlots <= kMostLds ? k_tiles : 1;
        const long blocks = ((long)a.d.columns + kDepth - 1) / kDepth, groups = (long)row_tiles * a.c.heads * a.batch;
        long runs = blocks * groups / 1024;
        runs = runs < 1 ? 1 : runs > 16 ? 16 : runs;
        static OncePerDevice lds_flags;
        st = allow_dynamic_lds((const void *)scores_kernel<NP, T>, kMostLds, lds_flags);
        if (st != SPIN_OK) return;
        const dim3 grid((unsigned)((blocks + runs - 1) / runs), row_tiles * a.c.heads, a.batch);
        scores_kernel<NP, T><<<grid, kScoreBlock, held * kSlots, s>>>(a, (int)runs, held);
    });
    return st != SPIN_OK ? st : check_launch("spin_cache_scores");
}

template <class T> spin_status launch_cache_values(const AttentionArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_ATTENTION, s);
    const int R = a.heads / a.c.heads * a.d.nodes, row_tiles = (R + kTile - 1) / kTile;
    const int range = value_range(a.n, a.batch, a.heads, a.c.heads, a.d.nodes, a.d.columns, a.c.dim, sizeof(T));
    const int ranges = (a.d.columns - 1) / range + 1;
    T *partial = value_parts(a.n, ranges, sizeof(T)) ? (T *)a.workspace : nullptr;
    spin_status st = SPIN_OK;
    for_party_count(a.n, [&](auto np) {
        constexpr int NP = decltype(np)::value;
        using S = ValueShape<NP, T>;
        static OncePerDevice lds_flags;
        st = allow_dynamic_lds((const void *)values_kernel<NP, T>, S::lds, lds_flags);
        if (st != SPIN_OK) return;
        const dim3 grid(ranges, row_tiles * ((a.c.dim + S::tiles * kTile - 1) / (S::tiles * kTile)) * a.c.heads, a.batch);
        values_kernel<NP, T><<<grid, kValueBlock, S::lds, s>>>(a, range, partial);
        if (!partial) return;
        const size_t party = (size_t)a.batch * a.heads * a.d.nodes * a.c.dim;
        join_kernel<NP, T><<<(unsigned)((party + kJoinBlock - 1) / kJoinBlock), kJoinBlock, 0, s>>>(a, ranges, partial);
    });
    return st != SPIN_OK ? st : check_launch("spin_cache_values");
}

template spin_status launch_cache_scores<u64>(const AttentionArgs<u64> &, hipStream_t);
template spin_status launch_cache_scores<u32>(const AttentionArgs<u32> &, hipStream_t);
template spin_status launch_cache_values<u64>(const AttentionArgs<u64> &, hipStream_t);
template spin_status launch_cache_values<u32>(const AttentionArgs<u32> &, hipStream_t);

}  // namespace spin
