// Linear attention with a decay over chunks of shares (spin_linattn_*).
#include "limb_common.hpp"
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
template <class T> __device__ inline T weight(const T *decay, int head, int chunk, int j) { return decay ? decay[(size_t)head * (chunk + 1) + j] : 1; }

// One element of a result whose parties' products sum to z.
template <int NP, class T> __device__ inline void finish(T z, const T *C, const Tuple<T> &t, int f, size_t party, size_t at, T *out)
{
    Opened<T> c{f};
    c.add(z);
    T top[NP], msb[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        c.add(once(C + i * party + at) + once(t.r + i * party + at));
        top[i] = once(t.r_top + i * party + at);
        msb[i] = once(t.r_msb + i * party + at);
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) out[i * party + at] = c.truncated(i, top[i], msb[i]);
}

// ---- products within chunks ---------------------------------------------------------------------------------
// Scores, a chunk's part of the next state and the outputs are products of two secrets within a chunk, [64 rows] x [64 columns] a workgroup: for every party
// E . b_i + a_i . F (+ E . F, party 0), all in one sum, which is all that the parties open.  Words are rewritten as ND balanced digits of eight bits
// (limb_common.hpp) and multiplied on v_mfma_i32_32x32x32_i8, digit pairs of one diagonal sharing an accumulator (at most 8 pairs x 2 products x 8 parties x
// 384 k x 2^14 = 2^30 in one).
//
// 32 k at a time: the first four waves open and split the left factor, the others the right one, into LDS as MFMA fragments, E and F and up to kGroup
// parties' masks at a time (a_0 of the right with F added, which folds E . F in); then waves 0 to 3 multiply E . b_i, a 32 x 32 quarter each, and 4 to 7 a_i . F, as F^T . a_i^T so
// that both keep their one factor's digits in registers.  More parties than kGroup read the others' masks a second time.
// A factor is stored along its rows or along k; only the left one is cleared where it does not count, and weighed: by row, by k, or by 2^g.
constexpr int kProductWaves = 8, kProductBlock = 64 * kProductWaves, kTile = 64, kStep = 32, kWords = kTile * kStep / (kProductBlock / 2);
constexpr int kPitch = kTile + 1;      // of a workgroup's sums in LDS
template <class T> constexpr int kSlot = 2 * (int)sizeof(T) * kFrag;               // one factor's digits of 64 x 32
template <int NP, class T> constexpr int kGroup = sizeof(T) == 4 ? NP : NP < 3 ? NP : 3;
template <int NP, class T> constexpr int product_lds = 2 * (kGroup<NP, T> + 1) * kSlot<T>;

template <class T> struct Side {       // of a product: rows of the left factor, columns of the right one
    const T *x, *a;                    // of the workgroup's first row and k
    size_t party;
    u32 pitch;                         // words from row to row, or from k to k
    bool along;                        // k is contiguous
    int rows, ks;                      // how many may be read
};
template <class T> __device__ inline Side<T> either(bool second, const Side<T> &a, const Side<T> &b)       // field by field: in registers
{
    return {second ? b.x : a.x, second ? b.a : a.a, second ? b.party : a.party, second ? b.pitch : a.pitch, second ? b.along : a.along, second ? b.rows : a.rows,
            second ? b.ks : a.ks};
}
template <class T> struct Range {      // of k
    int begin, end;                    // whole steps but for the end
    int below, above;                  // row i counts for i + above <= k <= i + below only
    const T *w;                        // the weight of row 0, or of k = 0; null: all `same`
    int stride;                        // from weight to weight: 1 or -1
    T same;
};
template <class T> __device__ inline Range<T> either(bool second, const Range<T> &a, const Range<T> &b)
{
    return {second ? b.begin : a.begin, second ? b.end : a.end, second ? b.below : a.below, second ? b.above : a.above, second ? b.w : a.w, second ? b.stride : a.stride,
            second ? b.same : a.same};
}
template <class T> struct Segment {
    Side<T> left, right;
    Range<T> k;
};
enum Weight { kNone, kByRow, kByK };

// The digits of four words: byte e of digit d is digit d of word e.
template <class T> __device__ inline void digits_of(const T *w, u32 (&d)[sizeof(T)])
{
#pragma unroll
    for (int half = 0; half < (int)sizeof(T) / 4; ++half) {
        u32 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (u32)(to_digits<T>(w[k]) >> (32 * half));
        const u32 t0 = __builtin_amdgcn_perm(v[1], v[0], 0x05010400u), t1 = __builtin_amdgcn_perm(v[1], v[0], 0x07030602u);
        const u32 t2 = __builtin_amdgcn_perm(v[3], v[2], 0x05010400u), t3 = __builtin_amdgcn_perm(v[3], v[2], 0x07030602u);
        d[4 * half + 0] = __builtin_amdgcn_perm(t2, t0, 0x05040100u);
        d[4 * half + 1] = __builtin_amdgcn_perm(t2, t0, 0x07060302u);
        d[4 * half + 2] = __builtin_amdgcn_perm(t3, t1, 0x05040100u);
        d[4 * half + 3] = __builtin_amdgcn_perm(t3, t1, 0x07060302u);
    }
}
// Where a fragment has 16 k of a row: the second 16 eight rows further, off the first one's banks.
__device__ inline int place(int row, int half) { return (half * 32 + (row + 8 * half) % 32) * 16; }

// The sums of a 64 x 64 tile over two ranges of k, in LDS as [64][kPitch] words when it returns (all waves have passed a barrier).
template <int NP, class T, Weight WEIGH> __device__ inline void product_tile(const Segment<T> &one, const Segment<T> &two, char *lds)
{
    constexpr int ND = sizeof(T), GROUP = kGroup<NP, T>, kRowsAtOnce = kTile / 2;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const bool right = wave >= kProductWaves / 2;
    const int quarter = wave % 4;
    char *const mine = lds + (right ? (GROUP + 1) * kSlot<T> : 0);
    const Side<T> side0 = either(right, one.left, one.right), side1 = either(right, two.left, two.right);
    auto steps = [](const Range<T> &k) { return k.end > k.begin ? (k.end - k.begin + kStep - 1) / kStep : 0; };
    const int steps0 = steps(one.k), total = steps0 + steps(two.k);
    // This thread's words of a step: along k four of rows u / 8 and 32 further, along the rows eight k of one row.
    const int thread = threadIdx.x % (kProductBlock / 2);
    auto load = [&](T (&w)[kWords], const Side<T> &s, const T *from, int k0) __attribute__((always_inline)) {
        int u = thread;
        asm volatile("" : "+v"(u));                        // what follows from the thread's place is made anew, not kept over the products
        if (s.along) {
            typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
            constexpr int W = 16 / sizeof(T);
            const int k = min(k0 + u % 8 * 4, s.ks - 4);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const T *p = from + ((u32)min(half * kRowsAtOnce + u / 8, s.rows - 1) * s.pitch + (u32)k);
#pragma unroll
                for (int e = 0; e < 4; e += W) {
                    const vec v = *(const vec *)(p + e);
#pragma unroll
                    for (int q = 0; q < W; ++q) w[half * 4 + e + q] = v[q];
                }
            }
        } else {
            const u32 row = (u32)min(u % 64, s.rows - 1);
#pragma unroll
            for (int e = 0; e < kWords; ++e) w[e] = (from + (u32)min(k0 + quarter * kWords + e, s.ks - 1) * s.pitch)[row];
        }
    };
    auto stage = [&](const T (&w)[kWords], int slot, bool along) __attribute__((always_inline)) {
        int u = thread;
        asm volatile("" : "+v"(u));
        u32 d[2][ND];
        digits_of<T>(w, d[0]);
        digits_of<T>(w + 4, d[1]);
        char *const to = mine + slot * kSlot<T>;
        if (along) {
            char *const at = to + place(u / 8, u % 8 / 4) + u % 4 * 4;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int k = 0; k < ND; ++k) *(u32 *)(at + (half * ND + k) * kFrag) = d[half][k];
        } else {
            char *const at = to + u % 64 / 32 * (ND * kFrag) + place(u % 32, quarter / 2) + quarter % 2 * 8;
#pragma unroll
            for (int k = 0; k < ND; ++k) *(u32x2 *)(at + k * kFrag) = u32x2{d[0][k], d[1][k]};
        }
    };
    v16i acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] = 0;
    const int wm = quarter / 2, wn = quarter % 2, lane_at = place(lane % 32, lane / 32);
    const char *const own = right ? lds + (GROUP + 1) * kSlot<T> + wn * (ND * kFrag) + lane_at : lds + wm * (ND * kFrag) + lane_at;
    const char *const other = right ? lds + wm * (ND * kFrag) + lane_at : lds + (GROUP + 1) * kSlot<T> + wn * (ND * kFrag) + lane_at;
    auto multiply = [&](int parties) __attribute__((always_inline)) {
        asm volatile("" : "+s"(parties));                  // a loop for one party, too: unrolled, its products take a second set of sums
        v4i kept[ND];
#pragma unroll
        for (int d = 0; d < ND; ++d) kept[d] = *(const v4i *)(own + d * kFrag);
#pragma unroll 1
        for (int i = 1; i <= parties; ++i) {
            const char *const at = other + i * kSlot<T>;
            v4i ahead = *(const v4i *)at;
#pragma unroll
            for (int p = 0; p < ND; ++p) {                 // one fragment is read ahead: left alone the compiler reads all of them first
                const v4i b = ahead;
                if (p + 1 < ND) ahead = *(const v4i *)(at + (p + 1) * kFrag);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int d = 0; d + p < ND; ++d) acc[d + p] = __builtin_amdgcn_mfma_i32_32x32x32_i8(kept[d], b, acc[d + p], 0, 0, 0);
            }
        }
    };
    T x[2][kWords], a[2][kWords];
    auto load_party = [&](int to, int t, int i) __attribute__((always_inline)) {
        const bool second = t >= steps0;
        const Side<T> s = either(second, side0, side1);
        const int k0 = second ? two.k.begin + (t - steps0) * kStep : one.k.begin + t * kStep;
        load(x[to], s, s.x + i * s.party, k0);
        load(a[to], s, s.a + i * s.party, k0);
    };
    T by_row[2] = {1, 1};
    // The words of the next step's first party are under way during the products; registers for that are left where there is one group.
    if (NP <= GROUP && total) load_party((NP - 1) % 2, 0, NP - 1);
    for (int t = 0; t < total; ++t) {
        const bool second = t >= steps0;
        const Range<T> g = either(second, one.k, two.k);
        const Side<T> s = either(second, side0, side1);
        const int k0 = g.begin + (second ? t - steps0 : t) * kStep;
        if (WEIGH == kByRow && !right && (t == 0 || t == steps0))              // the right factor's rows have no weights: none are looked up for them
#pragma unroll
            for (int half = 0; half < 2; ++half) by_row[half] = g.w ? g.w[min(s.along ? half * kRowsAtOnce + thread / 8 : lane, s.rows - 1) * g.stride] : g.same;
        // What the words of the left factor count.
        auto weigh = [&](T (&w)[kWords]) __attribute__((always_inline)) {
            if (right) return;
            int u = thread;
            asm volatile("" : "+v"(u));
#pragma unroll
            for (int e = 0; e < kWords; ++e) {
                const int row = s.along ? e / 4 * kRowsAtOnce + u / 8 : u % 64, k = s.along ? k0 + u % 8 * 4 + e % 4 : k0 + quarter * kWords + e;
                if (WEIGH == kByRow) w[e] *= by_row[e / 4];
                if (WEIGH == kByK && g.w) w[e] *= ((const __attribute__((address_space(4))) T *)(uintptr_t)g.w)[min(k0 + quarter * kWords + e, s.ks - 1) * g.stride];
                w[e] = k < g.end && k <= row + g.below && k >= row + g.above ? w[e] : 0;
            }
        };
        T open[kWords];
#pragma unroll
        for (int e = 0; e < kWords; ++e) open[e] = 0;
        __syncthreads();                                   // the last step's digits have been read
        auto take = [&](const T (&value)[kWords], const T (&mask)[kWords], int i) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < kWords; ++e) open[e] += value[e] - mask[e];
            if (i < GROUP) {
                T w[kWords];
#pragma unroll
                for (int e = 0; e < kWords; ++e) w[e] = mask[e] + (i == 0 && right ? open[e] : 0);
                weigh(w);
                stage(w, 1 + i, s.along);
            }
#pragma unroll
            for (int e = 0; e < kWords; ++e) computed_here(open[e]);
        };
        if constexpr (NP <= GROUP) {
#pragma unroll
            for (int i = NP - 1; i >= 0; --i) {
                if (i) load_party((i - 1) % 2, t, i - 1);
                __builtin_amdgcn_sched_barrier(0);         // one party's words under way, not all of them
                take(x[i % 2], a[i % 2], i);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
#pragma unroll 1
            for (int i = NP - 1; i >= 0; --i) {
                load_party(0, t, i);
                take(x[0], a[0], i);
            }
        }
        weigh(open);
        stage(open, 0, s.along);
        __builtin_amdgcn_sched_barrier(0);
        if (NP <= GROUP && t + 1 < total) load_party((NP - 1) % 2, t + 1, NP - 1);
#pragma unroll 1
        for (int first = 0;;) {
            __syncthreads();
            multiply(min(GROUP, NP - first));
            first += GROUP;
            if (first >= NP) break;
            __syncthreads();
#pragma unroll 1
            for (int i = 0; i < min(GROUP, NP - first); ++i) {
                T w[kWords];
                load(w, s, s.a + (first + i) * s.party, k0);
                weigh(w);
                stage(w, 1 + i, s.along);
            }
        }
    }
    // The two halves' sums meet in LDS.
    T *const sums = (T *)lds;
    auto word = [&](int r) __attribute__((always_inline)) {
        T v = 0;
#pragma unroll
        for (int d = ND - 1; d >= 0; --d) v = (v << 8) + (T)(std::make_signed_t<T>)acc[d][r];
        return v;
    };
    __syncthreads();
    if (!right) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sums[(wm * 32 + 8 * (r / 4) + 4 * (lane / 32) + r % 4) * kPitch + wn * 32 + lane % 32] = word(r);
    }
    __syncthreads();
    if (right) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sums[(wm * 32 + lane % 32) * kPitch + wn * 32 + 8 * (r / 4) + 4 * (lane / 32) + r % 4] += word(r);
    }
    __syncthreads();
}

// Which tile of which chunk (sequence and head before chunk) a workgroup has.  The tiles of a chunk read the same words: they are eight workgroup ids apart, on
// one XCD, next to each other in time.
struct TileOf { size_t unit; int tile; };
__device__ inline TileOf tile_of_workgroup(int tiles)
{
    const size_t id = blockIdx.x + (size_t)blockIdx.y * gridDim.x, strip = id / (kXcds * tiles);
    const int within = (int)(id % (kXcds * tiles));
    return {strip * kXcds + within % kXcds, within / kXcds};
}
inline size_t workgroups(const ChunkView &c, int tiles)
{
    const size_t units = (size_t)c.batch * c.heads * c.chunks;
    return (units + kXcds - 1) / kXcds * kXcds * tiles;
}
struct Unit { int b, h, chunk, L; size_t head; };          // head: of all sequences'
__device__ inline Unit unit_of(const ChunkView &c, size_t unit)
{
    Unit u;
    u.head = unit / c.chunks;
    u.chunk = (int)(unit % c.chunks);
    u.b = (int)(u.head / c.heads);
    u.h = (int)(u.head % c.heads);
    u.L = tokens_in(c, u.b, u.chunk);
    return u;
}
constexpr int kEverywhere = 1 << 20;   // beyond all rows and k of a chunk
template <class T> __device__ inline Segment<T> nothing_after(Segment<T> s)
{
    s.k.begin = s.k.end;
    return s;
}

template <int NP, class T> __global__ __launch_bounds__(kProductBlock, 2) void scores_kernel(ScoresArgs<T> a)
{
    extern __shared__ __align__(16) char lds[];
    const int C = a.c.chunk, across = (C + kTile - 1) / kTile;
    const TileOf at = tile_of_workgroup(across * across);
    const size_t heads = (size_t)a.c.batch * a.c.heads;
    if (at.unit >= heads * a.c.chunks) return;
    const Unit u = unit_of(a.c, at.unit);
    const int i0 = at.tile / across * kTile, j0 = at.tile % across * kTile;
    const size_t each = heads * a.c.chunks * C * C, first = at.unit * C * C;
    const bool any = j0 <= i0 && i0 < u.L;
    if (any) {
        const size_t party = heads * a.c.tokens * a.dim, token = u.head * a.c.tokens + (size_t)u.chunk * C;
        const Segment<T> s{{a.x.x + (token + i0) * a.dim, a.x.a + (token + i0) * a.dim, party, (u32)a.dim, true, u.L - i0, a.dim},
                           {a.y.x + (token + j0) * a.dim, a.y.a + (token + j0) * a.dim, party, (u32)a.dim, true, u.L - j0, a.dim},
                           {0, a.dim, kEverywhere, -kEverywhere, nullptr, 0, 1}};
        product_tile<NP, T, kNone>(s, nothing_after(s), lds);
    }
    for (int e = threadIdx.x; e < kTile * kTile; e += kProductBlock) {
        const int r = e / kTile, d = e % kTile, i = i0 + r, j = j0 + d;
        if (i >= C || j >= C) continue;
        const size_t to = first + (size_t)i * C + j;
        if (any && j <= i && i < u.L) {
            finish<NP>(weight(a.decay, u.h, C, i - j) * ((const T *)lds)[r * kPitch + d], a.C, a.t, a.c.f + a.c.g, each, to, a.out);
        } else {
#pragma unroll
            for (int k = 0; k < NP; ++k) a.out[k * each + to] = 0;
        }
    }
}

// What is opened of a chunk's own part of the next state.
template <int NP, class T> __global__ __launch_bounds__(kProductBlock, 2) void sums_kernel(StatesArgs<T> a)
{
    extern __shared__ __align__(16) char lds[];
    const int C = a.c.chunk, across = (a.columns + kTile - 1) / kTile;
    const TileOf at = tile_of_workgroup((a.rows + kTile - 1) / kTile * across);
    const size_t heads = (size_t)a.c.batch * a.c.heads, state = (size_t)a.rows * a.columns, each = heads * a.c.chunks * state;
    if (at.unit >= heads * a.c.chunks) return;
    const Unit u = unit_of(a.c, at.unit);
    if (u.L == 0) return;
    const int r0 = at.tile / across * kTile, d0 = at.tile % across * kTile;
    const size_t token = u.head * a.c.tokens + (size_t)u.chunk * C;
    const T *const w = a.decay ? a.decay + (size_t)u.h * (C + 1) + (a.reverse ? 1 : u.L - 1) : nullptr;
    const Segment<T> s{{a.x.x + token * a.rows + r0, a.x.a + token * a.rows + r0, heads * a.c.tokens * a.rows, (u32)a.rows, false, a.rows - r0, u.L},
                       {a.y.x + token * a.columns + d0, a.y.a + token * a.columns + d0, heads * a.c.tokens * a.columns, (u32)a.columns, false, a.columns - d0, u.L},
                       {0, u.L, kEverywhere, -kEverywhere, w, a.reverse ? 1 : -1, 1}};
    product_tile<NP, T, kByK>(s, nothing_after(s), lds);
    for (int e = threadIdx.x; e < kTile * kTile; e += kProductBlock) {
        const int r = e / kTile, d = e % kTile;
        if (r0 + r >= a.rows || d0 + d >= a.columns) continue;
        const size_t to = at.unit * state + (size_t)(r0 + r) * a.columns + d0 + d;
        T z = ((const T *)lds)[r * kPitch + d];
#pragma unroll
        for (int i = 0; i < NP; ++i) z += once(a.C + i * each + to) + once(a.t.r + i * each + to);
        a.opened[to] = z;
    }
}

template <int NP, class T> __global__ __launch_bounds__(kProductBlock, 2) void outputs_kernel(OutputsArgs<T> a)
{
    extern __shared__ __align__(16) char lds[];
    const int C = a.c.chunk, across = (a.columns + kTile - 1) / kTile;
    const TileOf at = tile_of_workgroup((C + kTile - 1) / kTile * across);
    const size_t heads = (size_t)a.c.batch * a.c.heads, each = heads * a.c.tokens * a.columns;
    if (at.unit >= heads * a.c.chunks) return;
    const Unit u = unit_of(a.c, at.unit);
    const int i0 = at.tile / across * kTile, d0 = at.tile % across * kTile, there = min(C, a.c.tokens - u.chunk * C);
    const size_t token = u.head * a.c.tokens + (size_t)u.chunk * C;
    if (i0 < u.L) {
        const size_t pairs = at.unit * C * C + (a.reverse ? i0 : (size_t)i0 * C), state = at.unit * a.rows * a.columns + (a.transposed ? (size_t)d0 * a.rows : d0);
        const T *const w = a.decay ? a.decay + (size_t)u.h * (C + 1) + (a.reverse ? u.L - 1 - i0 : i0 + 1) : nullptr;
        const Segment<T> own{{a.P.x + pairs, a.P.a + pairs, heads * a.c.chunks * C * C, (u32)C, !a.reverse, C - i0, C},
                             {a.y.x + token * a.columns + d0, a.y.a + token * a.columns + d0, each, (u32)a.columns, false, a.columns - d0, u.L},
                             {a.reverse ? i0 : 0, a.reverse ? u.L : min(u.L, i0 + kTile), a.reverse ? kEverywhere : i0, a.reverse ? i0 : -kEverywhere, nullptr, 0,
                              (T)1 << a.c.g}};
        const Segment<T> before{{a.x.x + (token + i0) * a.rows, a.x.a + (token + i0) * a.rows, heads * a.c.tokens * a.rows, (u32)a.rows, true, u.L - i0, a.rows},
                                {a.S.x + state, a.S.a + state, heads * a.c.chunks * a.rows * a.columns, (u32)(a.transposed ? a.rows : a.columns), a.transposed,
                                 a.columns - d0, a.rows},
                                {0, a.rows, kEverywhere, -kEverywhere, w, a.reverse ? -1 : 1, 1}};
        product_tile<NP, T, kByRow>(own, before, lds);
    }
#pragma unroll 1
    for (int e = threadIdx.x; e < kTile * kTile; e += kProductBlock) {
        const int r = e / kTile, d = e % kTile, i = i0 + r;
        if (i >= there || d0 + d >= a.columns) continue;
        const size_t to = (token + i) * a.columns + d0 + d;
        if (i < u.L) {
            finish<NP>(((const T *)lds)[r * kPitch + d], a.C, a.t, a.c.f + a.c.g, each, to, a.out);
        } else {
#pragma unroll
            for (int k = 0; k < NP; ++k) a.out[k * each + to] = 0;
        }
    }
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

// ---- a single token -----------------------------------------------------------------------------------------
// A workgroup has `wide` columns of one head's state (a power of two), a thread one of them and every (kStepBlock / wide)-th row: all words of a state element are read and
// written once, 7 a party, and what q . S' takes of them is added in registers, then in LDS.
constexpr int kStepBlock = 256;
template <int NP, class T> __global__ __launch_bounds__(kStepBlock) void step_kernel(StepArgs<T> a, int wide, bool streamed)
{
    constexpr int kMostRows = 256;
    __shared__ T keys[kMostRows][NP + 1], queries[kMostRows][NP + 1], sums[kStepBlock];
    const int lane = threadIdx.x % wide, part = threadIdx.x / wide, parts = kStepBlock / wide, d = blockIdx.x * wide + lane, b = blockIdx.y / a.heads, h = blockIdx.y % a.heads;
    const size_t heads = (size_t)a.batch * a.heads, one = heads * a.rows * a.columns;
    const bool live = !a.active || a.active[b] > 0, mine = d < a.columns;
    const size_t first = (size_t)blockIdx.y * a.rows * a.columns + min(d, a.columns - 1);
    if (!live) {                                           // of a whole workgroup
        if (!mine) return;
        if (a.S_out != a.S)
            for (int r = part; r < a.rows; r += parts)
#pragma unroll
                for (int i = 0; i < NP; ++i) a.S_out[i * one + first + (size_t)r * a.columns] = a.S[i * one + first + (size_t)r * a.columns];
        if (part == 0)
#pragma unroll
            for (int i = 0; i < NP; ++i) a.out[i * heads * a.columns + (size_t)blockIdx.y * a.columns + d] = 0;
        return;
    }
    for (int k = threadIdx.x; k < 2 * a.rows; k += kStepBlock) {
        const int r = k % a.rows;
        const Factor<NP, T> f = factor<NP>(k < a.rows ? a.k : a.q, heads * a.rows, (size_t)blockIdx.y * a.rows + r);
        T *const to = k < a.rows ? keys[r] : queries[r];
        to[NP] = f.open;
#pragma unroll
        for (int i = 0; i < NP; ++i) to[i] = f.mask[i];
    }
    const T w0 = weight(a.decay, h, 1, 0), w1 = weight(a.decay, h, 1, 1) << a.f;
    const Factor<NP, T> v = factor<NP>(a.v, heads * a.columns, (size_t)blockIdx.y * a.columns + min(d, a.columns - 1));
    __syncthreads();
    T sum = 0;
    for (int r = mine ? part : a.rows; r < a.rows; r += parts) {
        const size_t at = first + (size_t)r * a.columns;
        T S[NP], top[NP], msb[NP], mask[NP], dealt[NP];
        Opened<T> c{a.f + a.g};
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            S[i] = a.S[i * one + at];
            dealt[i] = once(a.CS + i * one + at) + once(a.tS.r + i * one + at);
            top[i] = once(a.tS.r_top + i * one + at), msb[i] = once(a.tS.r_msb + i * one + at);
            mask[i] = once(a.S_mask + i * one + at);
        }
        T z = 0, open = 0;
        const T ek = keys[r][NP], eq = queries[r][NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            z += ek * (v.mask[i] + (i == 0 ? v.open : 0)) + keys[r][i] * v.open;
            c.add(w1 * S[i] + dealt[i]);
        }
        c.add(w0 * z);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            S[i] = c.truncated(i, top[i], msb[i]);
            open += S[i] - mask[i];
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            sum += eq * (mask[i] + (i == 0 ? open : 0)) + queries[r][i] * open;
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) put(streamed, a.S_out + i * one + at, S[i]);
    }
    sums[threadIdx.x] = sum;
    __syncthreads();
    if (part || !mine) return;
    for (int k = 1; k < parts; ++k) sum += sums[threadIdx.x + wide * k];
    finish<NP>(sum, a.CO, a.tO, a.f, heads * a.columns, (size_t)blockIdx.y * a.columns + d, a.out);
}

// Launches one of the kernels above on all tiles of all chunks.
template <int NP, class T, class Kernel, class Args> inline spin_status launch_products(Kernel kernel, const Args &a, int tiles, OncePerDevice &lds_flags, hipStream_t s)
{
    const spin_status st = allow_dynamic_lds((const void *)kernel, product_lds<NP, T>, lds_flags);
    if (st == SPIN_OK) kernel<<<grid_of(workgroups(a.c, tiles)), kProductBlock, product_lds<NP, T>, s>>>(a);
    return st;
}
inline int tiles_of(int rows, int columns) { return ((rows + kTile - 1) / kTile) * ((columns + kTile - 1) / kTile); }

}  // namespace

template <class T> spin_status launch_linattn_scores(const ScoresArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_LINATTN, s);
    spin_status st = SPIN_OK;
    for_party_count(a.c.n, [&](auto np) {
        constexpr int NP = decltype(np)::value;
        static OncePerDevice lds_flags;
        st = launch_products<NP, T>(scores_kernel<NP, T>, a, tiles_of(a.c.chunk, a.c.chunk), lds_flags, s);
    });
    return st != SPIN_OK ? st : check_launch("spin_linattn_scores");
}

template <class T> spin_status launch_linattn_states(const StatesArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_LINATTN, s);
    const unsigned blocks = (a.rows * a.columns + kBlock - 1) / kBlock;
    spin_status st = SPIN_OK;
    for_party_count(a.c.n, [&](auto np) {
        constexpr int NP = decltype(np)::value;
        static OncePerDevice lds_flags;
        st = launch_products<NP, T>(sums_kernel<NP, T>, a, tiles_of(a.rows, a.columns), lds_flags, s);
        if (st == SPIN_OK) scan_kernel<NP, T><<<dim3(blocks, a.c.batch * a.c.heads), kBlock, 0, s>>>(a);
    });
    return st != SPIN_OK ? st : check_launch("spin_linattn_states");
}

template <class T> spin_status launch_linattn_outputs(const OutputsArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_LINATTN, s);
    spin_status st = SPIN_OK;
    for_party_count(a.c.n, [&](auto np) {
        constexpr int NP = decltype(np)::value;
        static OncePerDevice lds_flags;
        st = launch_products<NP, T>(outputs_kernel<NP, T>, a, tiles_of(a.c.chunk, a.columns), lds_flags, s);
    });
    return st != SPIN_OK ? st : check_launch("spin_linattn_outputs");
}

template <class T> spin_status launch_linattn_step(const StepArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_LINATTN, s);
    const bool streamed = (size_t)a.n * a.batch * a.heads * a.rows * a.columns * sizeof(T) >= kStreamingBytes;
    int wide = 64;
    while (wide > 8 && (long)a.batch * a.heads * ((a.columns + wide - 1) / wide) < 1024) wide /= 2;
    for_party_count(a.n, [&](auto np) {
        step_kernel<decltype(np)::value, T><<<dim3((a.columns + wide - 1) / wide, a.batch * a.heads), kStepBlock, 0, s>>>(a, wide, streamed);
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
