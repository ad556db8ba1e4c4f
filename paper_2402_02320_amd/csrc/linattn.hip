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
// Scores, a chunk's part of the next state and the outputs are products of two secrets within a chunk, [TILE rows] x [TILE columns] a workgroup: for every party
// E . b_i + a_i . F (+ E . F, party 0), all in one sum, which is all that the parties open.  Words are rewritten as ND balanced digits of eight bits
// (limb_common.hpp) and multiplied on v_mfma_i32_32x32x32_i8, digit pairs of one diagonal sharing an accumulator (at most 8 pairs x 2 products x 8 parties x
// 384 k x 2^14 = 2^30 in one).
//
// 32 k at a time: half of the waves open and split the left factor, half the right one, into LDS as MFMA fragments, E and F and the masks of up to GROUP parties (a_0 of the right
// with F added, which folds E . F in); then the first half multiplies E . b_i, the others a_i . F, as F^T . a_i^T so that both keep their one factor's digits in registers.
// Tiles of 64: eight waves, of either product one has a 32 x 32 quarter; more parties than GROUP read the others' masks a second time.  Tiles of 32: four waves, of either product
// one has every second party; for few chunks, where the larger ones leave CUs idle.
// A factor is stored along its rows or along k; only the left one is cleared where it does not count, and weighed.
//
// Bound by the way of the factors' words to a CU and by what does not overlap with it: 3 parties, 2 x 16 heads of 128, 4096 and 2730 tokens, chunks of 128: scores 0.67 ms (their 2.4 GB
// take HBM 0.39 at the 6.2 TB/s of streams that mostly read), outputs 1.19 (4.1 GB, 0.66), a chunk's part of the next state 0.60 (2.1 GB, 0.34).  Of the 15,000 cycles of a step
// (2 parties, tiles of 64) the words' opening and splitting take 3,000, requests for the next ones 4,700, the products 5,000: registers (128 of sums, 64 of words under way) and LDS
// (96 to 128 KB) let one workgroup of eight waves on a CU.
constexpr int kStep = 32;              // k
template <int TILE> constexpr int kProductBlock = 8 * TILE;
template <class T, int TILE> constexpr int kSlot = TILE / 32 * (int)sizeof(T) * kFrag;             // one factor's digits of TILE x 32
template <int NP, class T, int TILE> constexpr int kGroup = TILE == 32 || NP < 3 ? NP : 3;
enum Weight { kNone, kByRow, kByK };
template <int NP, class T, int TILE, Weight W> constexpr int kAhead = NP == 1 || NP > 3 || (TILE == 32 ? sizeof(T) == 4 : NP == 3 && W == kByK) ? 1 : 2;
template <int NP, class T, int TILE> constexpr int product_lds = 2 * (kGroup<NP, T, TILE> + 1) * kSlot<T, TILE>;
template <int NP, class T, int TILE> constexpr int kProductOccupancy = sizeof(T) == 4 && NP > 1 ? 4 : 2;          // waves a SIMD

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
    const T *w;                        // the weight of row 0, or of k = 0; null: 1
    int stride;                        // from weight to weight: 1 or -1
    int shift;                         // and all by 2^shift
};
template <class T> __device__ inline Range<T> either(bool second, const Range<T> &a, const Range<T> &b)
{
    return {second ? b.begin : a.begin, second ? b.end : a.end, second ? b.below : a.below, second ? b.above : a.above, second ? b.w : a.w, second ? b.stride : a.stride,
            second ? b.shift : a.shift};
}
template <class T> struct Segment {
    Side<T> left, right;
    Range<T> k;
};

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
// Where a fragment has half of a row's k: every second row, the others, and either of the second half, all off each other's banks.
__device__ inline int place(int row, int half) { return (half * 32 + row % 2 * 16 + (row / 2 + row % 2 * 8 + half * 4) % 16) * 16; }

// The sums of a tile over two ranges of k, in LDS as words when it returns (all waves have passed a barrier): sum_at().
// `then` is called before they meet, when every wave's digits are words and their registers free: what it loads is under way meanwhile.
template <int NP, class T, int TILE, Weight WEIGH, class Then> __device__ inline void product_tile(const Segment<T> &one, const Segment<T> &two, char *lds, Then &&then)
{
    constexpr int ND = sizeof(T), GROUP = kGroup<NP, T, TILE>, WAVES = TILE / 8, SIDE = 4 * TILE, HALF = TILE / 2, kBlock = ND * kFrag;
    constexpr int kPitch = TILE + 1;
    const u32 lane = threadIdx.x % 64;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const bool right = wave >= WAVES / 2;
    u32 u = threadIdx.x % SIDE;        // among the threads of a side
    char *const rights = lds + (GROUP + 1) * kSlot<T, TILE>, *const mine = right ? rights : lds;
    const Side<T> side0 = either(right, one.left, one.right), side1 = either(right, two.left, two.right);
    auto steps = [](const Range<T> &k) { return k.end > k.begin ? (k.end - k.begin + kStep - 1) / kStep : 0; };
    const int steps0 = steps(one.k), total = steps0 + steps(two.k);
    // This thread's words of a step: of two rows those at k = 16 (e / 2) + 2 q + e % 2, e < 4; along k the rows u / 8 and HALF further, q = u % 8, along the rows neighbours, q = u /
    // HALF.  So either way a load has two words, and in a fragment, where k stands in place 4 (k % 16 / 2) + 2 (k / 16) + k % 2, a row's four are neighbours.  No load is
    // behind a branch: where branches met its words would be copied, and a copy waits for them.
    typedef T pair __attribute__((ext_vector_type(2)));
    auto q_of = [&](bool along) __attribute__((always_inline)) { return along ? u % 8 : u / HALF; };
    auto row_of = [&](bool along, int half) __attribute__((always_inline)) { return along ? u / 8 + half * HALF : u % HALF * 2 + half; };
    auto k_of = [&](bool along, int e) __attribute__((always_inline)) { return 16 * (e / 2) + e % 2 + 2 * (int)q_of(along); };
    constexpr int AHEAD = kAhead<NP, T, TILE, WEIGH>;
    pair x[AHEAD][4], a[AHEAD][4];     // of the parties at hand
    auto load = [&](const Side<T> &s, int k0, int i, bool masks_only, pair (&value)[4], pair (&mask)[4]) __attribute__((always_inline)) {
        const T *const px = s.x + i * s.party, *const pa = s.a + i * s.party;
        const int q = q_of(s.along);
        const u32 near = s.along ? __umul24(min((int)row_of(true, 0), s.rows - 1), s.pitch) : min((int)row_of(false, 0), s.rows - 2);
        const u32 far = s.along ? __umul24(min((int)row_of(true, 1), s.rows - 1), s.pitch) : near;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int k = min(k0 + 16 * (s.along ? v % 2 : v / 2) + (s.along ? 0 : v % 2) + 2 * q, s.ks - (s.along ? 2 : 1));
            const u32 at = (v < 2 ? near : far) + __umul24(k, s.along ? 1 : s.pitch);
            if (!masks_only) value[v] = *(const pair *)(px + at);
            mask[v] = *(const pair *)(pa + at);
        }
    };
    auto word_of = [](const pair (&v)[4], bool along, int half, int e) __attribute__((always_inline)) { return along ? v[2 * half + e / 2][e % 2] : v[e][half]; };
    auto stage = [&](const T (&w)[4], int half, int slot, bool along) __attribute__((always_inline)) {
        u32 d[ND];
        digits_of<T>(w, d);
        const int row = row_of(along, half), q = q_of(along);
        char *const to = mine + slot * kSlot<T, TILE> + (row / 32 * kBlock + place(row % 32, q / 4) + q % 4 * 4);
#pragma unroll
        for (int k = 0; k < ND; ++k) *(u32 *)(to + k * kFrag) = d[k];
    };
    v16i acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] = 0;
    const int wm = TILE == 64 ? wave % 4 / 2 : 0, wn = TILE == 64 ? wave % 2 : 0;
    const u32 lane_at = place(lane % 32, lane / 32);
    const char *const own = (right ? rights + wn * kBlock : lds + wm * kBlock) + lane_at, *const other = (right ? lds + wm * kBlock : rights + wn * kBlock) + lane_at;
    // Tiles of 32: the workgroups of a CU begin with different parties, so that where the parties are odd their SIMDs have the same work.  Four digits of the own factor at a time: all
    // eight take registers that the next words need.
    const int begin = TILE == 64 ? 1 : 1 + (wave + blockIdx.x / kXcds) % 2, by = TILE == 64 ? 1 : 2;
    auto multiply = [&](int parties, auto &&between) __attribute__((always_inline)) {
        asm volatile("" : "+s"(parties));                  // a loop for one party, too: unrolled, its products take a second set of sums
#pragma unroll
        for (int d0 = 0; d0 < ND; d0 += 4) {
            if (d0) {
                __builtin_amdgcn_sched_barrier(0);
                between();
                __builtin_amdgcn_sched_barrier(0);
            }
            v4i kept[4];
#pragma unroll
            for (int d = 0; d < 4; ++d) kept[d] = *(const v4i *)(own + (d0 + d) * kFrag);
#pragma unroll 1
            for (int i = begin; i <= parties; i += by) {
                const char *const at = other + i * kSlot<T, TILE>;
                v4i ahead = *(const v4i *)at;
#pragma unroll
                for (int p = 0; p < ND - d0; ++p) {        // one fragment is read ahead: left alone the compiler reads all of them first
                    const v4i b = ahead;
                    if (p + 1 < ND - d0) ahead = *(const v4i *)(at + (p + 1) * kFrag);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int d = 0; d < 4 && d0 + d + p < ND; ++d)
                        acc[d0 + d + p] = __builtin_amdgcn_mfma_i32_32x32x32_i8(kept[d], b, acc[d0 + d + p], 0, 0, 0);
                }
            }
        }
    };
    // The upper four digits' sums only have 32 bits to give.
    auto word = [&](int r) __attribute__((always_inline)) {
        u32 high = 0;
#pragma unroll
        for (int d = ND - 4; d < ND; ++d) high += (u32)acc[d][r] << (8 * (d - ND + 4));
        if constexpr (ND == 4) return (T)high;
        int64_t v = acc[0][r];
#pragma unroll
        for (int d = 1; d < 4; ++d) v += (int64_t)acc[d][r] * (1 << (8 * d));
        return (T)v + ((T)high << (8 * sizeof(T) - 32));
    };
    auto load_party = [&](int to, int t, int i) __attribute__((always_inline)) {
        const bool second = t >= steps0;
        load(either(second, side0, side1), second ? two.k.begin + (t - steps0) * kStep : one.k.begin + t * kStep, i, false, x[to], a[to]);
    };
    // The words of AHEAD parties are under way, the next step's during the products: one party's asked for before the first half of the digits, one's before the second.  All at
    // once, their requests wait for one another and the products for them.
    constexpr int BETWEEN = AHEAD > 1 && ND > 4 ? 1 : 0;
    auto load_ahead = [&](int t, int begin, int end) __attribute__((always_inline)) {
#pragma unroll
        for (int i = NP - 1 - begin; i >= NP - end; --i) load_party(i % AHEAD, t, i);
    };
    __shared__ T by_row[TILE];
    if (total) load_ahead(0, 0, AHEAD);
#pragma unroll 1
    for (int t = 0; t < total; ++t) {
        const bool second = t >= steps0;
        const Range<T> g = either(second, one.k, two.k);
        const Side<T> s = either(second, side0, side1);
        const int k0 = g.begin + (second ? t - steps0 : t) * kStep;
        if (WEIGH == kByRow && threadIdx.x < TILE && (t == 0 || t == steps0))                  // (of a left wave)
            by_row[threadIdx.x] = (g.w ? g.w[min((int)threadIdx.x, s.rows - 1) * g.stride] : 1) << g.shift;
        const bool whole = k0 + kStep <= g.end && k0 + kStep - 1 <= g.below && k0 >= TILE - 1 + g.above;       // every word of the left factor counts
        // What four words of the left factor count.
        auto weigh = [&](T (&w)[4], int half) __attribute__((always_inline)) {
            if (right) return;
            if (WEIGH == kByRow)
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] *= by_row[row_of(s.along, half)];
            if (whole) return;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = row_of(s.along, half), k = k0 + k_of(s.along, e);
                w[e] = k < g.end && k <= row + g.below && k >= row + g.above ? w[e] : 0;
            }
        };
        // Weights by k are asked for before the parties' words are dealt with, where those leave registers.
        constexpr bool EARLY = WEIGH == kByK && AHEAD == 1;
        T by_k[EARLY ? 4 : 1];
        auto weight_of = [&](int e) __attribute__((always_inline)) { return g.w ? g.w[min(k0 + k_of(s.along, e), s.ks - 1) * g.stride] : 1; };
        if (EARLY)
#pragma unroll
            for (int e = 0; e < 4; ++e) by_k[EARLY ? e : 0] = weight_of(e);
        pair open[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) open[v] = pair{0, 0};
        __syncthreads();                                   // the last step's digits have been read
        // A party's words: its masks' digits, four words at a time.
        auto take = [&](const pair (&value)[4], const pair (&mask)[4], int i) __attribute__((always_inline)) {
            if (AHEAD > 1) computed_here(u);  // places are made of it again: kept, they take registers that words need
#pragma unroll
            for (int v = 0; v < 4; ++v) open[v] += value[v] - mask[v];
            if (i >= GROUP) return;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                T w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = word_of(mask, s.along, half, e);
                if (i == 0 && right)
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] += word_of(open, s.along, half, e);
                weigh(w, half);
                stage(w, half, 1 + i, s.along);
            }
        };
        if constexpr (AHEAD > 1) {
#pragma unroll
            for (int i = NP - 1; i >= 0; --i) {
                take(x[i % AHEAD], a[i % AHEAD], i);
                __builtin_amdgcn_sched_barrier(0);         // these registers are another party's from here on
                if (i >= AHEAD) load_party(i % AHEAD, t, i - AHEAD);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {                                           // a loop: the code is what short calls wait for first
#pragma unroll 1
            for (int i = NP - 1; i >= 0; --i) {
                take(x[0], a[0], i);
                load_party(0, i ? t : min(t + 1, total - 1), i ? i - 1 : NP - 1);
            }
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {             // by k both opened factors are weighed, one in each product; the masks are not
            T w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = word_of(open, s.along, half, e);
            if (WEIGH == kByK && g.w)
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] *= EARLY ? by_k[EARLY ? e : 0] : weight_of(e);
            weigh(w, half);
            stage(w, half, 0, s.along);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (AHEAD > 1 && t + 1 < total) load_ahead(t + 1, 0, AHEAD - BETWEEN);
#pragma unroll 1
        for (int first = 0;;) {
            __syncthreads();
            multiply(min(GROUP, NP - first), [&] {
                if (BETWEEN && t + 1 < total) load_ahead(t + 1, AHEAD - BETWEEN, AHEAD);
            });
            first += GROUP;
            if (first >= NP) break;
            __syncthreads();
#pragma unroll 1
            for (int i = 0; i < min(GROUP, NP - first); ++i) {
                pair w[4];
                load(s, k0, first + i, true, w, w);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    T four[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) four[e] = word_of(w, s.along, half, e);
                    weigh(four, half);
                    stage(four, half, 1 + i, s.along);
                }
            }
        }
    }
    // The waves' sums meet in LDS: of tiles of 64 those of one product in front of the other's, of tiles of 32 one product's in a part of its own.
    T sums[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        sums[r] = word(r);
        computed_here(sums[r]);
    }
    __builtin_amdgcn_sched_barrier(0);
    then();
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    constexpr int PARTS = TILE == 64 ? 1 : 2;
    T *const to = (T *)lds + (right ? (PARTS - 1) * TILE * kPitch + (wm * 32 + lane % 32) * kPitch + wn * 32 + 4 * (lane / 32)
                                    : (wm * 32 + 4 * (lane / 32)) * kPitch + wn * 32 + lane % 32);
    const int stride = right ? 1 : kPitch, turn = TILE == 64 ? (right ? 1 : 0) : wave % 2;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if (turn == half) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                T &sum = to[(8 * (r / 4) + r % 4) * stride];
                sum = (half ? sum : 0) + sums[r];
            }
        }
        __syncthreads();
    }
}
// One of them.
template <class T, int TILE> __device__ inline T sum_at(const char *lds, int row, int column)
{
    const T *s = (const T *)lds + row * (TILE + 1) + column;
    return TILE == 64 ? s[0] : s[0] + s[TILE * (TILE + 1)];
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
    u.L = tokens_in(c, c.lengths ? c.lengths[u.b] : c.tokens, u.chunk);
    return u;
}
constexpr int kEverywhere = 1 << 20;   // beyond all rows and k of a chunk

// What is done with a tile's sums: a thread has one column of every eighth row.  The dealt words of kAtOnce rows are asked for together: one row after another
// waits for memory every time.
template <int NP, class T, int TILE, bool TUPLE> struct Rows {
    static constexpr int kEach = TILE / 8, kWordsEach = TUPLE ? 4 * NP : 2 * NP, kMost = (sizeof(T) == 8 ? 96 : 32) / ((int)sizeof(T) / 4 * kWordsEach);
    static constexpr int kAtOnce = kMost >= 4 ? 4 : kMost >= 2 ? 2 : 1, kRounds = kEach / kAtOnce;
    const T *C;
    Tuple<T> t;
    size_t party, corner;              // words of a party, and where the tile starts
    u32 pitch;
    int rows, columns;                 // of the tile that there are
    int below;                         // row i has columns up to i + below only: behind them its last word is read again
    T c[kAtOnce][NP], r[kAtOnce][NP], top[kAtOnce][TUPLE ? NP : 1], msb[kAtOnce][TUPLE ? NP : 1];
    static __device__ int column() { return threadIdx.x % TILE; }
    static __device__ int row(int round, int k) { return (round * kAtOnce + k) * 8 + threadIdx.x / TILE; }
    __device__ u32 offset(int row) const { return (u32)min(row, rows - 1) * pitch + (u32)min(min(column(), columns - 1), max(row + below, 0)); }
    __device__ void load(int round)
    {
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const u32 at = offset(row(round, k));
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const size_t from = i * party + corner;
                c[k][i] = once(C + from + at), r[k][i] = once(t.r + from + at);
                if (TUPLE) top[k][TUPLE ? i : 0] = once(t.r_top + from + at), msb[k][TUPLE ? i : 0] = once(t.r_msb + from + at);
            }
        }
    }
    __device__ T masked(int k, T z) const                  // what is opened of a result
    {
#pragma unroll
        for (int i = 0; i < NP; ++i) z += c[k][i] + r[k][i];
        return z;
    }
};
template <class T> __device__ inline Segment<T> nothing_after(Segment<T> s)
{
    s.k.begin = s.k.end;
    return s;
}

template <int NP, class T, int TILE> __global__ __launch_bounds__(kProductBlock<TILE>, (kProductOccupancy<NP, T, TILE>)) void scores_kernel(ScoresArgs<T> a)
{
    extern __shared__ __align__(16) char lds[];
    const int C = a.c.chunk, across = (C + TILE - 1) / TILE;
    const TileOf at = tile_of_workgroup(across * across);
    const size_t heads = (size_t)a.c.batch * a.c.heads;
    if (at.unit >= heads * a.c.chunks) return;
    const Unit u = unit_of(a.c, at.unit);
    const int i0 = at.tile / across * TILE, j0 = at.tile % across * TILE;
    const size_t each = heads * a.c.chunks * C * C, first = at.unit * C * C;
    if (j0 > i0 || i0 >= u.L) {                            // nothing of the tile is there
        for (int e = threadIdx.x; e < TILE * TILE; e += kProductBlock<TILE>)
            if (i0 + e / TILE < C && j0 + e % TILE < C)
#pragma unroll
                for (int k = 0; k < NP; ++k) a.out[k * each + first + (size_t)(i0 + e / TILE) * C + j0 + e % TILE] = 0;
        return;
    }
    const size_t party = heads * a.c.tokens * a.dim, token = u.head * a.c.tokens + (size_t)u.chunk * C;
    const Segment<T> s{{a.x.x + (token + i0) * a.dim, a.x.a + (token + i0) * a.dim, party, (u32)a.dim, true, u.L - i0, a.dim},
                       {a.y.x + (token + j0) * a.dim, a.y.a + (token + j0) * a.dim, party, (u32)a.dim, true, u.L - j0, a.dim},
                       {0, a.dim, kEverywhere, -kEverywhere, nullptr, 0, 0}};
    Rows<NP, T, TILE, true> rows{a.C, a.t, each, first + (size_t)i0 * C + j0, (u32)C, min(u.L, C) - i0, C - j0, i0 - j0};
    product_tile<NP, T, TILE, kNone>(s, nothing_after(s), lds, [&] { rows.load(0); });
    const int d = rows.column(), j = j0 + d;
#pragma unroll 1
    for (int round = 0; round < rows.kRounds; ++round) {
#pragma unroll
        for (int k = 0; k < rows.kAtOnce; ++k) {
            const int r = rows.row(round, k), i = i0 + r;
            if (i >= C || j >= C) continue;
            T *const to = a.out + rows.corner + (size_t)r * C + d;
            const bool there = j <= i && i < u.L;
            Opened<T> c{a.c.f + a.c.g};
            // The weight is asked for behind the dealt words and waited for with them, row by row: up to four trips to memory in a round.
            if (there) c.add(rows.masked(k, weight(a.decay, u.h, C, i - j) * sum_at<T, TILE>(lds, r, d)));
#pragma unroll
            for (int p = 0; p < NP; ++p) to[p * each] = there ? c.truncated(p, rows.top[k][p], rows.msb[k][p]) : 0;
        }
        if (round + 1 < rows.kRounds) rows.load(round + 1);
    }
}

// What is opened of a chunk's own part of the next state.
template <int NP, class T, int TILE> __global__ __launch_bounds__(kProductBlock<TILE>, (kProductOccupancy<NP, T, TILE>)) void sums_kernel(StatesArgs<T> a)
{
    extern __shared__ __align__(16) char lds[];
    const int C = a.c.chunk, across = (a.columns + TILE - 1) / TILE;
    const TileOf at = tile_of_workgroup((a.rows + TILE - 1) / TILE * across);
    const size_t heads = (size_t)a.c.batch * a.c.heads, state = (size_t)a.rows * a.columns, each = heads * a.c.chunks * state;
    if (at.unit >= heads * a.c.chunks) return;
    const Unit u = unit_of(a.c, at.unit);
    if (u.L == 0) return;
    const int r0 = at.tile / across * TILE, d0 = at.tile % across * TILE;
    const size_t token = u.head * a.c.tokens + (size_t)u.chunk * C;
    const T *const w = a.decay ? a.decay + (size_t)u.h * (C + 1) + (a.reverse ? 1 : u.L - 1) : nullptr;
    const Segment<T> s{{a.x.x + token * a.rows + r0, a.x.a + token * a.rows + r0, heads * a.c.tokens * a.rows, (u32)a.rows, false, a.rows - r0, u.L},
                       {a.y.x + token * a.columns + d0, a.y.a + token * a.columns + d0, heads * a.c.tokens * a.columns, (u32)a.columns, false, a.columns - d0, u.L},
                       {0, u.L, kEverywhere, -kEverywhere, w, a.reverse ? 1 : -1, 0}};
    Rows<NP, T, TILE, false> rows{a.C, a.t, each, at.unit * state + (size_t)r0 * a.columns + d0, (u32)a.columns, min(TILE, a.rows - r0), min(TILE, a.columns - d0), kEverywhere};
    product_tile<NP, T, TILE, kByK>(s, nothing_after(s), lds, [&] { rows.load(0); });
#pragma unroll 1
    for (int round = 0; round < rows.kRounds; ++round) {
#pragma unroll
        for (int k = 0; k < rows.kAtOnce; ++k) {
            const int r = rows.row(round, k), d = rows.column();
            if (r < rows.rows && d < rows.columns) a.opened[rows.corner + (size_t)r * a.columns + d] = rows.masked(k, sum_at<T, TILE>(lds, r, d));
        }
        if (round + 1 < rows.kRounds) rows.load(round + 1);
    }
}

template <int NP, class T, int TILE> __global__ __launch_bounds__(kProductBlock<TILE>, (kProductOccupancy<NP, T, TILE>)) void outputs_kernel(OutputsArgs<T> a)
{
    extern __shared__ __align__(16) char lds[];
    const int C = a.c.chunk, across = (a.columns + TILE - 1) / TILE;
    const TileOf at = tile_of_workgroup((C + TILE - 1) / TILE * across);
    const size_t heads = (size_t)a.c.batch * a.c.heads, each = heads * a.c.tokens * a.columns;
    if (at.unit >= heads * a.c.chunks) return;
    const Unit u = unit_of(a.c, at.unit);
    const int i0 = at.tile / across * TILE, d0 = at.tile % across * TILE, there = min(C, a.c.tokens - u.chunk * C);
    const size_t token = u.head * a.c.tokens + (size_t)u.chunk * C;
    if (i0 >= u.L) {
        for (int e = threadIdx.x; e < TILE * TILE; e += kProductBlock<TILE>)
            if (i0 + e / TILE < there && d0 + e % TILE < a.columns)
#pragma unroll
                for (int k = 0; k < NP; ++k) a.out[k * each + (token + i0 + e / TILE) * a.columns + d0 + e % TILE] = 0;
        return;
    }
    const size_t pairs = at.unit * C * C + (a.reverse ? i0 : (size_t)i0 * C), state = at.unit * a.rows * a.columns + (a.transposed ? (size_t)d0 * a.rows : d0);
    const T *const w = a.decay ? a.decay + (size_t)u.h * (C + 1) + (a.reverse ? u.L - 1 - i0 : i0 + 1) : nullptr;
    const Segment<T> own{{a.P.x + pairs, a.P.a + pairs, heads * a.c.chunks * C * C, (u32)C, !a.reverse, C - i0, C},
                         {a.y.x + token * a.columns + d0, a.y.a + token * a.columns + d0, each, (u32)a.columns, false, a.columns - d0, u.L},
                         {a.reverse ? i0 : 0, a.reverse ? u.L : min(u.L, i0 + TILE), a.reverse ? kEverywhere : i0, a.reverse ? i0 : -kEverywhere, nullptr, 0, a.c.g}};
    const Segment<T> before{{a.x.x + (token + i0) * a.rows, a.x.a + (token + i0) * a.rows, heads * a.c.tokens * a.rows, (u32)a.rows, true, u.L - i0, a.rows},
                            {a.S.x + state, a.S.a + state, heads * a.c.chunks * a.rows * a.columns, (u32)(a.transposed ? a.rows : a.columns), a.transposed, a.columns - d0,
                             a.rows},
                            {0, a.rows, kEverywhere, -kEverywhere, w, a.reverse ? -1 : 1, 0}};
    Rows<NP, T, TILE, true> rows{a.C, a.t, each, (token + i0) * a.columns + d0, (u32)a.columns, min(u.L, there) - i0, min(TILE, a.columns - d0), kEverywhere};
    product_tile<NP, T, TILE, kByRow>(own, before, lds, [&] { rows.load(0); });
    const int d = rows.column();
#pragma unroll 1
    for (int round = 0; round < rows.kRounds; ++round) {
#pragma unroll
        for (int k = 0; k < rows.kAtOnce; ++k) {
            const int r = rows.row(round, k), i = i0 + r;
            if (i >= there || d >= rows.columns) continue;
            T *const to = a.out + rows.corner + (size_t)r * a.columns + d;
            Opened<T> c{a.c.f + a.c.g};
            c.add(rows.masked(k, sum_at<T, TILE>(lds, r, d)));
#pragma unroll
            for (int p = 0; p < NP; ++p) to[p * each] = i < u.L ? c.truncated(p, rows.top[k][p], rows.msb[k][p]) : 0;
        }
        if (round + 1 < rows.kRounds) rows.load(round + 1);
    }
}

// From chunk to chunk, a thread an element of the state: a stream of 3 NP + 1 words an element, those of kScanAtOnce chunks under way together: 3 parties, 32 heads of 128 x 128, 32
// chunks 227 us, 5.9 TB/s.  Where a chunk has no tokens its
// part of `opened` was not written: what is read of it is not used.
template <int NP> constexpr int kScanAtOnce = NP <= 3 ? 4 : NP <= 6 ? 2 : 1;
template <int NP, class T> __global__ __launch_bounds__(kBlock) void scan_kernel(StatesArgs<T> a)
{
    constexpr int AT_ONCE = kScanAtOnce<NP>;
    const int state = a.rows * a.columns, b = blockIdx.y / a.c.heads, h = blockIdx.y % a.c.heads, u = blockIdx.x * kBlock + threadIdx.x;
    if (u >= state) return;
    const size_t heads = (size_t)a.c.batch * a.c.heads, each = heads * a.c.chunks * state, one = heads * state;
    const int length = a.c.lengths ? a.c.lengths[b] : a.c.tokens;
    T S[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) S[i] = a.first ? a.first[i * one + (size_t)blockIdx.y * state + u] : 0;
    for (int k0 = 0; k0 < a.c.chunks; k0 += AT_ONCE) {
        T opened[AT_ONCE], top[AT_ONCE][NP], msb[AT_ONCE][NP], w[AT_ONCE];
        size_t at[AT_ONCE];
        int L[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int step = min(k0 + k, a.c.chunks - 1), chunk = a.reverse ? a.c.chunks - 1 - step : step;
            L[k] = tokens_in(a.c, length, chunk);
            w[k] = weight(a.decay, h, a.c.chunk, L[k]) << a.c.f;
            at[k] = ((size_t)blockIdx.y * a.c.chunks + chunk) * state + u;
            opened[k] = once(a.opened + at[k]);
#pragma unroll
            for (int i = 0; i < NP; ++i) top[k][i] = once(a.t.r_top + i * each + at[k]), msb[k][i] = once(a.t.r_msb + i * each + at[k]);
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            if (k0 + k >= a.c.chunks) break;
            Opened<T> c{a.c.f + a.c.g};
            c.add(opened[k]);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                c.add(w[k] * S[i]);
                a.states[i * each + at[k]] = S[i];
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) S[i] = L[k] ? c.truncated(i, top[k][i], msb[k][i]) : S[i];
        }
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) a.last[i * one + (size_t)blockIdx.y * state + u] = S[i];
}

// ---- a single token -----------------------------------------------------------------------------------------
// A workgroup has `wide` columns of one head's state (a power of two), a thread one of them and every (kStepBlock / wide)-th row: all words of a state element are read and
// written once, 7 a party, and what q . S' takes of them is added in registers, then in LDS.  Bound by trips to memory one after another: the factors', then a thread's rows' (no
// load goes before the last row's stores, which may be to its words), a row's in two batches of three parties and six of five, since the first words are added before the last are
// asked for.  3 parties: 16 heads of 64 x 64, four rows a thread, 8.5 us, 6.9 of them in the kernel; 512 of 128 x 128, 32 rows a thread, 254 us, 4.6 TB/s (a seventh of it written).
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
template <int NP, class T, int TILE, class Kernel, class Args>
inline spin_status launch_products(Kernel kernel, const Args &a, int rows, int columns, OncePerDevice &lds_flags, hipStream_t s)
{
    const spin_status st = allow_dynamic_lds((const void *)kernel, product_lds<NP, T, TILE>, lds_flags);
    const int tiles = ((rows + TILE - 1) / TILE) * ((columns + TILE - 1) / TILE);
    if (st == SPIN_OK) kernel<<<grid_of(workgroups(a.c, tiles)), kProductBlock<TILE>, product_lds<NP, T, TILE>, s>>>(a);
    return st;
}
// Tiles of 64 read and split every factor half as often, tiles of 32 are four times as many.  3 parties, 2 x 16 heads of 128, 4096 tokens in chunks of 128 (64-bit words): a prompt
// 2.70 ms by 64, 2.99 by 32; 8 heads of 64, 300 tokens (40 tiles of 64): 98 us by 64, 55 by 32; 2 parties' training step of 16 heads of 64, 1024 tokens (256 tiles) 307
// and 336.  By the number of tiles of 64, heads and chunks of 64, 3 parties, us of scores, states, outputs by 64 : by 32 (a tile of 64 takes a CU, so that the 257th begins a second
// round):
//     100    31 : 22     32 : 27     45 : 33            300    67 : 52     73 : 64    110 : 90            512    90 : 91    102 : 109   133 : 146
//     200    37 : 37     43 : 46     57 : 64            400    78 : 74     88 : 90    115 : 120           600   116 : 107   129 : 126   175 : 168
//     256    43 : 42     52 : 53     67 : 74            768   133 : 136   154 : 160   195 : 214          1024   176 : 178   202 : 210   265 : 277
// 2 parties alike; 5, which read masks twice by 64 and wait for every party by 32: 100 51 : 45, 52 : 49, 86 : 82; 256 76 : 101, 85 : 110, 125 : 178; 300 122 : 119, 123 : 128, 199 : 216;
// 1024 300 : 383, 331 : 414, 468 : 690.  So between one round and about 350 tiles the rule loses up to a quarter with few parties.
// 32-bit words have tiles of 32 only: before others were left out, 24 heads of 80 and 48, chunks of 32, took 94 us by 64 and 73 by 32; longer chunks were not measured.
constexpr long kWantedTiles = 256;
template <class T, class F> inline void for_tile(const ChunkView &c, int rows, int columns, F &&fn)
{
    if constexpr (sizeof(T) == 8) {
        if (rows > 32 && columns > 32 && (long)c.batch * c.heads * c.chunks * ((rows + 63) / 64) * ((columns + 63) / 64) >= kWantedTiles)
            return fn(std::integral_constant<int, 64>());
    }
    fn(std::integral_constant<int, 32>());
}

}  // namespace

template <class T> spin_status launch_linattn_scores(const ScoresArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_LINATTN, s);
    spin_status st = SPIN_OK;
    for_party_count(a.c.n, [&](auto np) {
        for_tile<T>(a.c, a.c.chunk, a.c.chunk, [&](auto tile) {
            constexpr int NP = decltype(np)::value, TILE = decltype(tile)::value;
            static OncePerDevice lds_flags;
            st = launch_products<NP, T, TILE>(scores_kernel<NP, T, TILE>, a, a.c.chunk, a.c.chunk, lds_flags, s);
        });
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
        for_tile<T>(a.c, a.rows, a.columns, [&](auto tile) {
            constexpr int TILE = decltype(tile)::value;
            static OncePerDevice lds_flags;
            st = launch_products<NP, T, TILE>(sums_kernel<NP, T, TILE>, a, a.rows, a.columns, lds_flags, s);
        });
        if (st == SPIN_OK) scan_kernel<NP, T><<<dim3(blocks, a.c.batch * a.c.heads), kBlock, 0, s>>>(a);
    });
    return st != SPIN_OK ? st : check_launch("spin_linattn_states");
}

template <class T> spin_status launch_linattn_outputs(const OutputsArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_LINATTN, s);
    spin_status st = SPIN_OK;
    for_party_count(a.c.n, [&](auto np) {
        for_tile<T>(a.c, a.c.chunk, a.columns, [&](auto tile) {
            constexpr int NP = decltype(np)::value, TILE = decltype(tile)::value;
            static OncePerDevice lds_flags;
            st = launch_products<NP, T, TILE>(outputs_kernel<NP, T, TILE>, a, a.c.chunk, a.columns, lds_flags, s);
        });
    });
    return st != SPIN_OK ? st : check_launch("spin_linattn_outputs");
}

template <class T> spin_status launch_linattn_step(const StepArgs<T> &a, hipStream_t s)
{
    KernelTimer timer(SPIN_KERNEL_LINATTN, s);
    const bool streamed = (size_t)a.n * a.batch * a.heads * a.rows * a.columns * sizeof(T) >= kStreamingBytes;
    // Full lines where the CUs have enough of them: 3 parties, 512 heads of 128, 254 us by 64, 270 by 16, 490 by 8; 16 heads of 64 21.7, 8.5 and 8.7; 2 parties over Z_2^32, 45 heads
    // of 40 and 72, 9.4, 6.2 and 7.8.
    int wide = 64;
    while (wide > 16 && (long)a.batch * a.heads * ((a.columns + wide - 1) / wide) < 1024) wide /= 2;
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
