// Products of new tokens with the paged cache of shares (spin_cache_scores, spin_cache_values), on int8 MFMA.
//
// A ring word is rewritten as ND balanced digits of eight bits (limb_common.hpp); a product of words is the sum over digit pairs i + j < ND on
// v_mfma_i32_16x16x64_i8, pairs of one diagonal sharing an accumulator: 36 int8 products a multiply-add of 64-bit words, 10 of 32-bit ones.
// The cache stays in ring words, read once from HBM into the registers of the wave that multiplies them and split there.  A lane's 16 k of a
// fragment may be any 16 as long as both factors take the same, here two of the 16-byte pieces of each line of 128,
//     k(j, h, e) = 4 W j + W h + e       (W words in 16 bytes, h = lane / 16, e < W).  The new tokens' factor (E and every A_i, 16 rows) is split once a workgroup
// into LDS, in fragment order.
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

// The digits of two or four words, the e-th of them at byte q + e of lane `lane`, into the ND fragments at `frag`.
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
template <class T> __device__ inline void put_digits(char *frag, int lane, int q, const T (&w)[4])
{
#pragma unroll
    for (int half = 0; half < (int)sizeof(T) / 4; ++half) {
        u32 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (u32)(to_digits<T>(w[k]) >> (32 * half));
        const u32 t0 = __builtin_amdgcn_perm(v[1], v[0], 0x05010400u), t1 = __builtin_amdgcn_perm(v[1], v[0], 0x07030602u);
        const u32 t2 = __builtin_amdgcn_perm(v[3], v[2], 0x05010400u), t3 = __builtin_amdgcn_perm(v[3], v[2], 0x07030602u);
        char *at = frag + 4 * half * kFrag + lane * 16 + q;
        *(u32 *)(at) = __builtin_amdgcn_perm(t2, t0, 0x05040100u);
        *(u32 *)(at + kFrag) = __builtin_amdgcn_perm(t2, t0, 0x07060302u);
        *(u32 *)(at + 2 * kFrag) = __builtin_amdgcn_perm(t3, t1, 0x05040100u);
        *(u32 *)(at + 3 * kFrag) = __builtin_amdgcn_perm(t3, t1, 0x07060302u);
    }
}

// acc += left0 . right0 + left1 . right1 over all digit pairs that count; left: ND fragments in LDS, this lane's 16 bytes of the first.  One fragment is read
// ahead: left alone the compiler reads all of them first, into 64 registers.
template <class T> __device__ inline void multiply(v4i (&acc)[sizeof(T)], const char *left0, const v4i (&right0)[sizeof(T)], const char *left1, const v4i (&right1)[sizeof(T)])
{
    constexpr int ND = sizeof(T);
    v4i ahead = *(const v4i *)left0;
#pragma unroll
    for (int p = 0; p < 2 * ND; ++p) {
        const v4i a = ahead;
        if (p + 1 < 2 * ND) ahead = *(const v4i *)(p + 1 < ND ? left0 + (p + 1) * kFrag : left1 + (p + 1 - ND) * kFrag);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i + p % ND < ND; ++i)
            acc[i + p % ND] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, p < ND ? right0[i] : right1[i], acc[i + p % ND], 0, 0, 0);
    }
    // Multiplied here: put off to where the sums are used, the fragments of all parties would be kept until then.
#pragma unroll
    for (int d = 0; d < ND; ++d) asm volatile("" : "+v"(acc[d]));
}

// The word whose diagonals are acc[..][r].
template <class T> __device__ inline T recombine(const v4i (&acc)[sizeof(T)], int r)
{
    T v = 0;
#pragma unroll
    for (int d = (int)sizeof(T) - 1; d >= 0; --d) v = (v << 8) + (T)(std::make_signed_t<T>)acc[d][r];
    return v;
}

// The run or range of tokens and the first row of a workgroup, which has `rows` of them.  Row groups of one run are eight workgroup ids apart: on one XCD, next to each other in time, so
// that its L2 serves all but the first.  Which XCD has a run goes round with the head and the sequence: short sequences have the first runs only.
__device__ inline void place_of(int row_groups, int rows, int &block, int &row0)
{
    const int strip = blockIdx.x / (kXcds * row_groups), within = blockIdx.x % (kXcds * row_groups);
    block = strip * kXcds + (within + blockIdx.y + blockIdx.z * gridDim.y) % kXcds;
    row0 = within / kXcds * rows;
}

// A word at a scalar address and a lane's bytes from there (rows have at most kMostColumns words, so 32 of them are within 2^32 bytes): no register a lane but
// those 32 bits goes into addresses.
template <bool NT = false, class T> __device__ inline T at_bytes(const T *scalar, u32 bytes)
{
    const T *p = (const T *)((const char *)scalar + bytes);
    return NT ? __builtin_nontemporal_load(p) : *p;
}
template <class T> __device__ inline void put_at_bytes(T *scalar, u32 bytes, T v) { *(T *)((char *)scalar + bytes) = v; }

// ---- scores -----------------------------------------------------------------------------------------------------
// A workgroup: 16 rows (query heads of one cached head, times nodes) against runs of 64 cached tokens, 16 a wave, one k-tile of 64 elements after
// another; `held` k-tiles of the rows' digits are in LDS: all of them, or (heads so long and parties so many that they do not fit) the one at hand.
//
// Every party's two products go into the same diagonals where the result is truncated (SUM): what the parties open is the sum of their masked shares,
// and no share of Z is asked for by itself.  (8 pairs x 2 products x 256 elements x 8 parties x 2^14 = 2^29 fits an int32.)  Without truncation a workgroup
// has one party.
//
// HBM bounds it (a tile of 16 rows of three parties takes 64 KB of cache and 432 MFMA, a sixth of the time), if enough is in flight: a wave has the loads of
// two slots in flight, over the ends of k-tiles and runs, and reads all of a score's triple and tuple words at once.  A load instruction takes whole lines, eight lanes a
// row, and each line is turned in LDS to the four lanes that an MFMA wants of a row: with four lanes a row in the loads themselves 64 bytes are asked for at a time, by
// 16 lanes in 16 lines, and a token of 4 x 4 heads of 128 over up to 2000 (3 parties) takes 27 us, not 18.  3 parties, four sequences of up to 32768, one token: 8 heads of 128
// 365 us, 6.0 TB/s; 16 heads over 8 403 us, 5.65.  Calls with work for one round of workgroups wait for its beginning and end: trees of 8, 16 heads over 4, two sequences
// of up to 8192 111 us (118 with four lanes a row; two row tiles a workgroup the same); one token over two of up to 700, 8 heads of 64, 8.4 us.
constexpr int kScoreWanted = 2048;     // workgroups
constexpr int kScoreWaves = 4, kScoreBlock = 64 * kScoreWaves;
constexpr int kTurn = kTile * 128;     // bytes of a line of 16 rows
constexpr double kKept = 256 << 20;    // bytes of the Infinity Cache: a cache that is larger and read once is read with non-temporal loads
// Up to two rows a cached head are multiplied on the vector unit: no digits.  3 parties, a token, 4 cached heads of 128, four sequences of up to 2000, 64-bit words: one
// row 17.9 us, by matrix units 26.0; two 21.6 and 26.0; four 29.3 and 27.4.  32-bit words: one 11.4 and 14.3; four 15.8 and 15.0.
constexpr int kFewRows = 2;

template <int NP, class T, bool SUM, bool FEW, bool NT>
__global__ __launch_bounds__(kScoreBlock, sizeof(T) == 8 ? 2 : NP < (FEW ? 6 : 5) ? 4 : 3) void scores_kernel(AttentionArgs<T> a, int runs, int held)
{
    using L = Lane<T>;
    constexpr int ND = L::ND, W = L::W, STEPS = SUM ? NP + 1 : 2;
    typedef T vec __attribute__((ext_vector_type(L::W)));
    extern __shared__ __align__(16) char lds[];
    __shared__ u64 row_tree[kTile];                        // of this workgroup's rows: what they see, their places behind the context, their bias far from the keys
    __shared__ int row_place[kTile];
    __shared__ T row_far[NP][kTile];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane / 16;
    const int b = SUM ? blockIdx.z : blockIdx.z / NP, party = SUM ? 0 : blockIdx.z % NP;
    const int share = a.heads / a.c.heads, R = share * a.d.nodes, row_tiles = (R + kTile - 1) / kTile;
    int block, row0;
    place_of(row_tiles, kTile, block, row0);
    const int g = blockIdx.y;
    auto place = [&](int node) { return a.depth ? a.depth[(size_t)b * a.d.nodes + node] : node; };
    const size_t rows = (size_t)a.batch * a.heads * a.d.nodes, first_row = ((size_t)b * a.heads + (size_t)g * share) * a.d.nodes + row0;
    const int context = a.d.context[b], dim = a.c.dim;
    const int limit = context < 0 ? 0 : (int)min((long)a.d.columns, (long)context + a.d.nodes);
    const int k_tiles = (dim + kDepth - 1) / kDepth, begin = block * runs * kDepth;
    if (begin >= a.d.columns) return;

    auto stage = [&](int kt0, int count) __attribute__((always_inline)) {                // digits of E and A_i of k-tiles kt0 .. kt0 + count - 1
        const int per_row = count * (kDepth / W);
#pragma unroll 2
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
            const int p = part % (kDepth / W), to = (p % 4) * 16 + (row % 4 * 4 + row / 4), byte = p / 4 * W;    // row 4 r + h in the place 4 h + r
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
    // The same as words for the vector unit: [slot][row][k].
    const int row_words = k_tiles * kDepth, few_words = R * row_words;
    auto stage_words = [&]() __attribute__((always_inline)) {
        for (int c = threadIdx.x; c < few_words / W; c += kScoreBlock) {
            const int row = c * W / row_words, at = c * W % row_words;
            const bool there = at < dim;
            const size_t from = (first_row + row) * dim + (there ? at : 0);
            vec q[NP], m[NP], e;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                q[i] = *(const vec *)(a.x + i * rows * dim + from);
                m[i] = *(const vec *)(a.A + i * rows * dim + from);
            }
#pragma unroll
            for (int k = 0; k < W; ++k) {
                e[k] = 0;
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    e[k] += there ? q[i][k] - m[i][k] : 0;
                    m[i][k] = there ? m[i][k] : 0;
                }
            }
            ((vec *)lds)[c] = e;
#pragma unroll
            for (int i = 0; i < NP; ++i) ((vec *)lds)[(i + 1) * (few_words / W) + c] = m[i];
        }
    };
    const size_t slot = ((size_t)a.c.pages * a.c.heads << a.c.shift) * dim;
    const T *slots = a.pool + (SUM ? 0 : party * slot);    // the one that party's slot comes after
    const u32 lane_row = lane / 8 * dim * sizeof(T), lane_at = lane_row + lane % 8 * W * sizeof(T);  // 16 tokens are on one page: a scalar address and these bytes
    vec raw[FEW ? 3 : 2][L::loads];
    // The words of a step; past a row's end the rows' digits are zero, whatever is read.  No load stands behind a branch: its register would be copied where the
    // branches meet, and a copy waits for the load.
    auto load = [&](vec (&v)[L::loads], int s, int kt, size_t key) __attribute__((always_inline)) {
        const char *from = (const char *)((s == 0 ? a.pool : slots + s * slot) + key);
        int begin_of = kt * kDepth;
        asm volatile("" : "+s"(begin_of));                 // addresses are made here, not carried along for every slot and j
#pragma unroll
        for (int j = 0; j < L::loads; ++j) {
            const int at = begin_of + j / 2 * (8 * W);     // a row's end is a multiple of 8
            const vec *const piece = (const vec *)(from + (j % 2 * 8 * dim + (at < dim ? at : 0)) * sizeof(T) + (at + lane % 8 * W < dim ? lane_at : lane_row));
            v[j] = NT ? __builtin_nontemporal_load(piece) : *piece;
        }
    };
    int page = 0;
    auto key_of = [&](int first) __attribute__((always_inline)) {                        // where this wave's tile starts in slot 0
        const int t0 = first + wave * kTile;
        page = __builtin_amdgcn_readfirstlane(page_of(a.c, b, t0));
        return row_at(a.c, 0, max(page, 0), g, t0);
    };
    // What the first loads need is looked up before the context has come, the first run's words of rows 0 to 3 are under way before the products (up to three parties': 8
    // registers each), and the rows' own lookups go on behind the digits: a short call is a chain of such waits.
    const int my_row = min(row0 + (int)threadIdx.x % kTile, R - 1);
    const u64 my_tree = tree_row(a.d, b, my_row % a.d.nodes);
    const int my_place = place(my_row % a.d.nodes), my_bucket = a.bias.table ? bucket_at(a.bias, -a.bias.reach) : -1;
    const bool whole = FEW || held >= k_tiles;
    // Where a wave turns a line of 16 rows: piece p of row r in place p ^ (r / 2 % 8), which keeps 16 lanes off each other's banks both ways.
    char *const turn = lds + (NP + 1) * held * (ND * kFrag) + wave * kTurn;
    const u32 turn_in = lane / 8 * 128 + ((lane % 8) ^ (lane / 16)) * 16, turn_in8 = lane / 8 * 128 + ((lane % 8) ^ (4 + lane / 16)) * 16;
    const u32 turn_out = lane % 16 * 128 + (h ^ (lane % 16 / 2)) * 16;
    size_t key = key_of(begin);
    const int active = begin < limit ? min(runs, (limit - begin + kDepth - 1) / kDepth) : 0;   // runs with something to see
    const size_t each = rows * a.d.columns;
    auto near_of = [&](int first) __attribute__((always_inline)) { return min(first + wave * kTile, a.d.columns - 1); };      // a wave's first token, within the row
    auto word_at = [&](int row, int first) __attribute__((always_inline)) {                    // bytes from there to this lane's word of a row
        const int t = first + wave * kTile + lane % 16;
        return row0 + row < R && t < a.d.columns ? ((u32)row * a.d.columns + (t - near_of(first))) * (u32)sizeof(T) : 0;
    };
    constexpr bool kPre = SUM && NP <= 3;
    T pre[4][kPre ? NP : 1];
    if (active) {
        load(raw[0], 0, 0, key);
        load(raw[1], 1, 0, key);
        if constexpr (kPre) {
            const size_t corner = first_row * a.d.columns + near_of(begin);
            const u32 at = word_at(h, begin);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                pre[0][i] = at_bytes(a.C + (i * each + corner), at);
                pre[1][i] = at_bytes(a.r + (i * each + corner), at);
                pre[2][i] = at_bytes(a.r_top + (i * each + corner), at);
                pre[3][i] = at_bytes(a.r_msb + (i * each + corner), at);
            }
        }
        if constexpr (FEW) {
            if constexpr (STEPS > 2) load(raw[2], 2, 0, key);
            stage_words();
        } else if (whole) {
            stage(0, k_tiles);
        }
    }
    if (threadIdx.x < kTile) {
        row_tree[threadIdx.x] = my_tree;
        row_place[threadIdx.x] = my_place;
#pragma unroll
        for (int i = 0; i < NP; ++i)
            row_far[i][threadIdx.x] = my_bucket < 0 ? 0 : ((const T *)a.bias.table)[((size_t)i * a.heads + g * share + my_row / a.d.nodes) * a.bias.buckets + my_bucket];
    }
    __syncthreads();
    int nearest = row_place[0];                            // of the rows' places
    for (int k = 1; k < kTile; ++k) nearest = min(nearest, row_place[k]);
    nearest = __builtin_amdgcn_readfirstlane(nearest);
    v4i acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) acc[d] = v4i{0, 0, 0, 0};
    T z_few[kFewRows][2] = {};                             // tokens lane / 8 and 8 further
    int kt = 0, here = page;
    size_t next = 0;
    // One loop over k-tiles and runs, so that the loads of the next k-tile's first two steps are under way whichever run it belongs to; behind the last one
    // they read the pool's first rows, which every workgroup does.  Two buffers serve any number of steps: with an odd one the last step's is filled a
    // step before it is needed, the others' two.
    for (int run = 0; run < active;) {
        if (kt == 0) {
            here = page;
            next = run + 1 < active ? key_of(begin + (run + 1) * kDepth) : 0;
        }
        const int kt1 = kt + 1 == k_tiles ? 0 : kt + 1;
        const size_t key1 = kt1 ? key : next;
        if (!whole) {
            __syncthreads();
            stage(kt, 1);
            __syncthreads();
        }
        if constexpr (FEW) {
            const vec *left = (const vec *)lds + kt * (kDepth / W) + lane % 8;
#pragma unroll
            for (int s = 1; s < STEPS; ++s) {
                vec (&w)[L::loads] = raw[2 - s % 2];
                const vec *mask = left + (SUM ? s : party + 1) * (few_words / W);
#pragma unroll
                for (int r = 0; r < kFewRows; ++r) {
                    if (r >= R) break;
#pragma unroll
                    for (int j = 0; j < L::loads / 2; ++j) {
                        const vec e = left[r * (row_words / W) + 8 * j], m = mask[r * (row_words / W) + 8 * j];
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
#pragma unroll
                            for (int k = 0; k < W; ++k) z_few[r][g] += e[k] * w[2 * j + g][k] + m[k] * raw[0][2 * j + g][k];
                            computed_here(z_few[r][g]);
                        }
                        if (j % 2) __builtin_amdgcn_sched_barrier(0);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);         // these registers are the loads' from here on
                if (s + 2 < STEPS) load(w, s + 2, kt, key);
                else load(w, 2 - s % 2, kt1, key1);
                if (s + 1 == STEPS) load(raw[0], 0, kt1, key1);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        const char *left = lds + (whole ? kt : 0) * (ND * kFrag) + lane * 16;
        v4i f[ND], right[ND];
#pragma unroll
        for (int s = 0; s < (FEW ? 0 : STEPS); ++s) {
            T w[16];
#pragma unroll
            for (int j = 0; j < L::loads; j += 2) {        // 16 lines: eight lanes a row in, four lanes a row out; the wave's own LDS, whose accesses stay in order
                *(vec *)(turn + turn_in) = raw[s % 2][j];
                *(vec *)(turn + 8 * 128 + turn_in8) = raw[s % 2][j + 1];
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                const vec low = *(const vec *)(turn + turn_out), high = *(const vec *)(turn + (turn_out ^ 64));
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
                for (int k = 0; k < W; ++k) w[j * W + k] = low[k], w[(j + 1) * W + k] = high[k];
            }
            split<T>(w, s == 0 ? f : right);
            __builtin_amdgcn_sched_barrier(0);             // these registers are the loads' of two steps on
            if (s + 2 < STEPS) load(raw[s % 2], s + 2, kt, key);
            else load(raw[s % 2], s % 2, kt1, key1);
            __builtin_amdgcn_sched_barrier(0);
            if (s > 0) multiply<T>(acc, left, right, left + (SUM ? s : party + 1) * held * (ND * kFrag), f);
        }
        kt = kt1;
        if (kt) continue;
        key = next;
        const int first = begin + run * kDepth, t0 = first + wave * kTile, t = t0 + lane % 16;
        const size_t corner = first_row * a.d.columns + near_of(first);
        // All of the tile is seen; and so far behind all rows that they have one bucket (without a bias, its words are zero).
        const bool past = t0 + kTile <= context, far = !a.bias.table || (past && (long)t0 + kTile - 1 - context - nearest <= -(long)a.bias.reach);
        ++run;
        // Rows 4 r + quarter, token t: few rows are spread over the lanes.  What follows from the rows is computed anew for every run: kept over the products
        // it takes 50 registers.
        int quarter = h;
        asm volatile("" : "+v"(quarter));
#pragma unroll
        for (int r = 0; r < (FEW ? 1 : 4); ++r) {
            if (NP > 3) __builtin_amdgcn_sched_barrier(0); // a score's words at a time
            if (row0 + 4 * r >= R) break;
            const int row = row0 + 4 * r + quarter;
            const bool mine = row < R && t < a.d.columns;
            const bool seen = mine && here >= 0 && (past || sees(row_tree[4 * r + quarter], a.d.nodes, context, t));
            const u32 at = word_at(4 * r + quarter, first);
            int bucket = -1;
            const T *bias = (const T *)a.bias.table + (size_t)(g * share + row / a.d.nodes) * a.bias.buckets;
            if (a.bias.table && !far && seen) {
                const long away = (t < context ? (long)t - context : place(t - context)) - (long)row_place[4 * r + quarter];
                bucket = bucket_at(a.bias, (int)min(max(away, -(long)a.bias.reach), (long)a.bias.reach));
            }
            // What party i's share gets, of a place that is seen.
            auto bias_of = [&](int i) __attribute__((always_inline)) {
                return far ? row_far[i][4 * r + quarter] : bucket < 0 ? 0 : bias[(size_t)i * a.heads * a.bias.buckets + bucket];
            };
            T z = 0;
            if constexpr (FEW) {
#pragma unroll
                for (int k = 0; k < kFewRows; ++k) {
                    if (k >= R) break;
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        T v = z_few[k][g];                 // the eight lanes of a token have an eighth of k each
#pragma unroll
                        for (int by = 1; by < 8; by *= 2) v += __shfl_xor(v, by);
                        v = __shfl(v, lane % 8 * 8);
                        z = h == k && lane % 16 / 8 == g ? v : z;
                        z_few[k][g] = 0;
                    }
                }
            } else {
                z = recombine<T>(acc, r);
            }
            if constexpr (SUM) {
                Opened<T> c{a.f};
                c.add(z);
                T top[NP], msb[NP];
                if (kPre && r == 0 && run == 1) {
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        const int k = kPre ? i : 0;
                        c.add(pre[0][k] + pre[1][k]);
                        top[i] = pre[2][k], msb[i] = pre[3][k];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        c.add(at_bytes(a.C + (i * each + corner), at) + at_bytes(a.r + (i * each + corner), at));
                        top[i] = at_bytes(a.r_top + (i * each + corner), at);
                        msb[i] = at_bytes(a.r_msb + (i * each + corner), at);
                    }
                }
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const T y = c.truncated(i, top[i], msb[i]) + bias_of(i);
                    if (mine) put_at_bytes(a.out + (i * each + corner), at, seen ? y : i == 0 ? a.masked : 0);
                }
            } else if (mine) {
                z += at_bytes(a.C + (party * each + corner), at) + bias_of(party);
                put_at_bytes(a.out + (party * each + corner), at, seen ? z : party == 0 ? a.masked : 0);
            }
        }
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[d] = v4i{0, 0, 0, 0};
    }
    // Runs that nothing of is seen.
    const int left_over = min(a.d.columns, begin + runs * kDepth) - (begin + active * kDepth);
    for (int c = threadIdx.x; c < left_over * min(kTile, R - row0); c += kScoreBlock) {
        const size_t at = (first_row + c / left_over) * a.d.columns + begin + active * kDepth + c % left_over;
        if constexpr (SUM) {
#pragma unroll
            for (int i = 0; i < NP; ++i) a.out[i * rows * a.d.columns + at] = i == 0 ? a.masked : 0;
        } else {
            a.out[party * rows * a.d.columns + at] = party == 0 ? a.masked : 0;
        }
    }
}

// ---- values -----------------------------------------------------------------------------------------------------
// A workgroup: 16 rows and WAVES x 16 columns, a tile a wave, over a range of cached tokens, 64 at a time.  A wave reads its column tile word by word (16 lanes
// side by side, 128 or 64 bytes), so here a lane's 16 k are the tokens 16 j + 4 h + e, e < 4, whatever the word: four words of a row of P or A are read and their
// digits written by one thread.  The rows' digits of the next 64 tokens are split into the other half of LDS while the matrix cores work on these; a wave has the loads
// of two slots in flight, over the turns' ends.  Sums as above; eight pairs and two products of at most 2^14 a token and party, so a range is at
// most kMostTokens long (16 x 8 x 512 x 2^14 = 2^30).
//
// HBM bounds long calls (few rows: below).  With more rows it is the digits of P and A, which
// all column blocks make anew: 2 parties' 32-bit trees of 7, 20 heads over 8 x 4 x 80, up to 3008 cached, 39 us, 5 of them the join of the ranges.
constexpr int kMostTokens = 512 * SPIN_MAX_PARTIES;        // times parties

// One element of the result whose parties' products sum to z, truncated.
template <int NP, class T> __device__ inline void finish(const AttentionArgs<T> &a, size_t at, size_t each, T z)
{
    Opened<T> c{a.f};
    c.add(z);
    T top[NP], msb[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        c.add(a.C[i * each + at] + a.r[i * each + at]);
        top[i] = a.r_top[i * each + at];
        msb[i] = a.r_msb[i * each + at];
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) a.out[i * each + at] = c.truncated(i, top[i], msb[i]);
}

template <int NP, class T, bool SUM, int WAVES, int TILES, bool NT>
__global__ __launch_bounds__(64 * WAVES, sizeof(T) == 8 || NP > 6 ? 2 : 4) void values_kernel(AttentionArgs<T> a, int range, T *partial)
{
    constexpr int ND = sizeof(T), STEPS = SUM ? NP + 1 : 2, kRows = kTile * TILES, kTileBytes = (NP + 1) * ND * kFrag, kStage = TILES * kTileBytes;
    constexpr int kPieces = kTile * kDepth / 4;            // of four tokens of a row
    static_assert(kPieces == 4 * 64 && WAVES >= 4 * TILES, "a piece a thread of four waves");
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), h = lane / 16;
    const int share = a.heads / a.c.heads, R = share * a.d.nodes, row_groups = (R + kRows - 1) / kRows, dim = a.c.dim;
    const int b = SUM ? blockIdx.z : blockIdx.z / NP, party = SUM ? 0 : blockIdx.z % NP;
    int block, row0;
    place_of(row_groups, kRows, block, row0);
    const int column_blocks = (dim + WAVES * kTile - 1) / (WAVES * kTile);
    const int col0 = (blockIdx.y % column_blocks * WAVES + wave) * kTile, g = blockIdx.y / column_blocks;
    const size_t rows = (size_t)a.batch * a.heads * a.d.nodes, first_row = ((size_t)b * a.heads + (size_t)g * share) * a.d.nodes + row0;
    const int context = a.d.context[b];
    const int limit = context < 0 ? 0 : (int)min((long)a.d.columns, (long)context + a.d.nodes);
    if ((long)block * range >= a.d.columns) return;
    const int begin = block * range, end = min(begin + range, limit);
    const int my_tile = TILES > 1 ? wave / 4 : 0;          // whose digits this wave writes
    // The table's entry for position t, or its last one.
    auto listed = [&](int t) __attribute__((always_inline)) { return a.c.table[(size_t)b * a.c.table_pages + min(t >> a.c.shift, a.c.table_pages - 1)]; };
    // Digits of E and A_i of this thread's row and four tokens, zero where nothing is seen.  Eight waves share the tiles, or the slots of the one: the first four
    // have E, which takes all parties' words, and `firsts` of the A_i.
    constexpr bool kShared = WAVES > 4 && TILES == 1;
    constexpr int firsts = kShared ? (NP - 1) / 2 : NP;
    auto stage = [&](int t0, char *to) __attribute__((always_inline)) {
        int c = threadIdx.x % kPieces;
        asm volatile("" : "+v"(c));                        // what follows from the piece's place is not kept over the products
        const int row = my_tile * kTile + c / 16, p = c % 16, t = t0 + 4 * p, at = (p % 4) * 16 + (row + 4 * (p % 4)) % 16;
        to += my_tile * kTileBytes;
        const int page = listed(t);                        // a page holds a multiple of four tokens
        const bool there = row0 + row < R && (unsigned)page < (unsigned)a.c.pages && t >> a.c.shift < a.c.table_pages;
        const u32 from = (u32)(row0 + row < R ? row : 0) * a.d.columns;
        const int past = min(t, a.d.columns - 4), over = min(t, a.d.columns - 1) - past;              // read at `past`: rows end anywhere, but have four words
        auto read = [&](const T *v, T (&w)[4]) __attribute__((always_inline)) {
            typedef T pair __attribute__((ext_vector_type(sizeof(T) == 8 ? 2 : 4), aligned(sizeof(T))));
            constexpr int per = sizeof(pair) / sizeof(T);
#pragma unroll
            for (int k = 0; k < 4 / per; ++k) {
                const pair u = *(const pair *)((const char *)v + (from + past + k * per) * (u32)sizeof(T));
#pragma unroll
                for (int e = 0; e < per; ++e) w[k * per + e] = u[e];
            }
            // the last words of a row are those behind `over` others
            w[0] = over & 1 ? w[1] : w[0], w[1] = over & 1 ? w[2] : w[1], w[2] = over & 1 ? w[3] : w[2];
            w[0] = over & 2 ? w[2] : w[0], w[1] = over & 2 ? w[3] : w[1];
        };
        u64 tree = 0;                                      // looked up where drafted tokens are
        if (t + 3 >= context) tree = tree_row(a.d, b, (row0 + row < R ? row0 + row : 0) % a.d.nodes);
        bool seen[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) seen[e] = there && t + e < end && sees(tree, a.d.nodes, context, t + e);
        T m[NP][4];
        auto put = [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) m[i][e] = seen[e] ? m[i][e] : 0;
            put_digits<T>(to + (i + 1) * (ND * kFrag), at, p / 4 * 4, m[i]);
        };
        if (!kShared || wave < 4) {
            T sum[4] = {0, 0, 0, 0};
#pragma unroll
            for (int first = 0; first < NP; first += 4) {                  // four parties' words at a time
                T x[4][4];
#pragma unroll
                for (int i = first; i < min(first + 4, NP); ++i) {
                    read(a.x + (i * rows + first_row) * a.d.columns, x[i - first]);
                    read(a.A + (i * rows + first_row) * a.d.columns, m[i]);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
#pragma unroll
                    for (int i = first; i < min(first + 4, NP); ++i) sum[e] += seen[e] ? x[i - first][e] - m[i][e] : 0;
                    if (NP > 4) computed_here(sum[e]);
                }
            }
            put_digits<T>(to, at, p / 4 * 4, sum);
#pragma unroll
            for (int i = 0; i < firsts; ++i) put(i);
        } else {
#pragma unroll
            for (int i = firsts; i < NP; ++i) read(a.A + (i * rows + first_row) * a.d.columns, m[i]);
#pragma unroll
            for (int i = firsts; i < NP; ++i) put(i);
        }
    };
    const u32 lane_at = (h * 4 * dim + min(col0 + lane % 16, dim - 1)) * sizeof(T);            // bytes; a column past the row's end reads the last one and is not stored
    const int lane_left = (h * 16 + (lane % 16 + 4 * h) % 16) * 16;        // rows are turned on by four from h to h, which keeps the staging threads off each other's banks
    const size_t slot = ((size_t)a.c.pages * a.c.heads << a.c.shift) * dim;
    const T *slots = a.pool + (SUM ? 0 : party * slot);
    size_t base[4];                                        // of 16 tokens, which are on one page
    int next[4];                                           // that page of the next turn
    // (The table is not written here, so it may be read as constant memory: by scalar loads, into scalar registers.)
    const auto *table = (const __attribute__((address_space(4))) int32_t *)(uintptr_t)(a.c.table + (size_t)b * a.c.table_pages);
    auto look_up = [&](int t0) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) next[j] = table[min((t0 + j * 16) >> a.c.shift, a.c.table_pages - 1)];
    };
    auto find = [&](bool wanted, int t0) __attribute__((always_inline)) {                      // the pool's first rows if not, as for scores
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = t0 + j * 16, page = next[j];
            const bool there = (unsigned)page < (unsigned)a.c.pages;       // if not, or past the table, some page's rows: they are not seen
            base[j] = wanted ? row_at(a.c, 0, there ? page : 0, g, t) : 0;
        }
    };
    T raw[2][16];
    auto load = [&](T (&w)[16], int s) __attribute__((always_inline)) {
        const T *from = s == 0 ? a.pool : slots + s * slot;
#pragma unroll
        for (int j = 0; j < 16; ++j) w[j] = at_bytes<NT>(from + (base[j / 4] + j % 4 * dim), lane_at);
    };
    v4i acc[TILES][ND];
#pragma unroll
    for (int u = 0; u < TILES; ++u)
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[u][d] = v4i{0, 0, 0, 0};
    look_up(begin);                                        // while the context comes
    if (begin < end) {
        if (col0 < dim) {
            find(true, begin);
            load(raw[0], 0);
            load(raw[1], 1);
        }
        stage(begin, lds);
    }
    __syncthreads();
    for (int t0 = begin, half = 0; t0 < end; t0 += kDepth, half ^= 1) {
        const bool more = t0 + kDepth < end;
        look_up(t0 + kDepth);
        if (col0 < dim) {
            const char *left = lds + half * kStage + lane_left;
            v4i f[ND], right[ND];
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                split<T>(raw[s % 2], s == 0 ? f : right);
                __builtin_amdgcn_sched_barrier(0);         // these registers are the loads' of two steps on
                if (s + 2 == STEPS) find(more, t0 + kDepth);
                load(raw[s % 2], s + 2 < STEPS ? s + 2 : s % 2);
                __builtin_amdgcn_sched_barrier(0);
                if (s == 0) continue;
#pragma unroll
                for (int u = 0; u < TILES; ++u)
                    multiply<T>(acc[u], left + u * kTileBytes, right, left + u * kTileBytes + (SUM ? s : party + 1) * (ND * kFrag), f);
            }
        }
        if (more) stage(t0 + kDepth, lds + (half ^ 1) * kStage);
        __syncthreads();
    }
    const int col = col0 + lane % 16;
    if (col >= dim) return;
    const size_t each = rows * dim;
#pragma unroll
    for (int r = 0; r < 4 * TILES; ++r) {
        const int row = r / 4 * kTile + 4 * h + r % 4;
        if (row0 + row >= R) continue;
        const size_t at = (first_row + row) * dim + col;
        const T z = recombine<T>(acc[r / 4], r % 4);
        if (partial) partial[((size_t)block * (SUM ? 1 : NP) + party) * each + at] = z;
        else if constexpr (SUM) finish<NP, T>(a, at, each, z);
        else a.out[party * each + at] = a.C[party * each + at] + z;
    }
}

// Up to few_value_rows() rows a cached head: on the vector unit, a lane 16 bytes of a cached row, so that a load takes whole rows: `tokens` of them where they are short (up to 16,
// of one page).  A wave has every fourth group of tokens of 64; the rows' words of the next 64 are put into LDS, E and the A_i of a token side by side, behind the products
// of these.  HBM bounds it: 3 parties, a token, four sequences of up to 32769, 16 heads over 8 of 128 355 us, 6.1 TB/s, by matrix units 378; two parties' 8 heads, eight of up
// to 4097 81 and 111; of up to 2000, 3 parties' 4 heads 20.5 and 29.9, four rows a head 27.6 and 31.1, 32-bit words 17.4 and 15.0; 2 x 4 heads of 64 over 101 9.7 and 12.3.
// Two sets of buffers: the loads of the next kAtOnce groups are under way during the products of the last.
constexpr int few_value_rows(int word_bytes) { return word_bytes == 8 ? 4 : 2; }
template <int NP, class T, bool SUM, bool NT>
__global__ __launch_bounds__(kScoreBlock, 3) void row_values_kernel(AttentionArgs<T> a, int range, T *partial)
{
    constexpr int kMost = few_value_rows(sizeof(T));
    constexpr int W = 16 / sizeof(T), SLOTS = SUM ? NP + 1 : 2, kAtOnce = SLOTS <= 4 ? 2 : 1, kWords = 2 * kDepth * kMost * (NP + 1), kSums = kScoreBlock * kMost * W;
    typedef T vec __attribute__((ext_vector_type(W)));
    __shared__ __align__(16) T lds[kWords > kSums ? kWords : kSums];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int b = SUM ? blockIdx.z : blockIdx.z / NP, party = SUM ? 0 : blockIdx.z % NP, dim = a.c.dim;
    const int share = a.heads / a.c.heads, R = share * a.d.nodes, all = dim / W, column_blocks = (all + 63) / 64, lanes = min(all, 64);
    int block, row0;
    place_of(1, kMost, block, row0);
    const int g = blockIdx.y / column_blocks, col = (blockIdx.y % column_blocks * 64 + lane % lanes) * W;
    const size_t rows = (size_t)a.batch * a.heads * a.d.nodes, first_row = ((size_t)b * a.heads + (size_t)g * share) * a.d.nodes;
    const int context = a.d.context[b];
    const int limit = context < 0 ? 0 : (int)min((long)a.d.columns, (long)context + a.d.nodes);
    if ((long)block * range >= a.d.columns) return;
    const int begin = block * range, end = min(begin + range, limit);
    const int tokens = min(1 << (31 - __clz(64 / lanes)), kTile), steps = kTile / tokens, batches = (steps + kAtOnce - 1) / kAtOnce;       // a wave and 64 tokens
    const int sub = lane / lanes;
    const bool mine = sub < tokens && col < dim;
    const u32 lane_at = mine ? (sub * dim + col) * (u32)sizeof(T) : 0;

    auto stage = [&](int t0, T *to) __attribute__((always_inline)) {
        const int row = threadIdx.x / kDepth, t = t0 + threadIdx.x % kDepth;
        if (row >= R) return;
        const bool seen = t < end && page_of(a.c, b, t) >= 0 && sees(tree_row(a.d, b, row % a.d.nodes), a.d.nodes, context, t);
        const size_t from = (first_row + row) * a.d.columns + min(t, a.d.columns - 1);
        T x[NP], m[NP], e = 0;
#pragma unroll
        for (int i = 0; i < NP; ++i) x[i] = a.x[i * rows * a.d.columns + from], m[i] = a.A[i * rows * a.d.columns + from];
        to += (threadIdx.x % kDepth * R + row) * (NP + 1);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            e += seen ? x[i] - m[i] : 0;
            to[i + 1] = seen ? m[i] : 0;
        }
        to[0] = e;
    };
    const size_t slot = ((size_t)a.c.pages * a.c.heads << a.c.shift) * dim;
    const T *slots = a.pool + (SUM ? 0 : party * slot);
    const auto *table = (const __attribute__((address_space(4))) int32_t *)(uintptr_t)(a.c.table + (size_t)b * a.c.table_pages);
    // The groups of a batch; behind the last one, and where a page is not there, some rows of the pool, which are multiplied by zero or not at all.
    auto load = [&](vec (&v)[kAtOnce][SLOTS], int t0, int batch) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int t = t0 + (min(batch * kAtOnce + j, steps - 1) * kScoreWaves + wave) * tokens, page = table[min(t >> a.c.shift, a.c.table_pages - 1)];
            const size_t base = row_at(a.c, 0, (unsigned)page < (unsigned)a.c.pages ? page : 0, g, t);
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) {
                const vec *p = (const vec *)((const char *)((s == 0 ? a.pool : slots + s * slot) + base) + lane_at);
                v[j][s] = NT ? __builtin_nontemporal_load(p) : *p;
            }
        }
    };
    T z[kMost][W] = {};
    auto multiply_words = [&](const vec (&v)[kAtOnce][SLOTS], const T *from, int batch) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (batch * kAtOnce + j >= steps) break;
            const T *factors = from + (((batch * kAtOnce + j) * kScoreWaves + wave) * tokens + min(sub, tokens - 1)) * R * (NP + 1);
#pragma unroll
            for (int r = 0; r < kMost; ++r) {
                if (r >= R) break;
                const T e = factors[r * (NP + 1)];
#pragma unroll
                for (int s = 1; s < SLOTS; ++s) {
                    const T m = factors[r * (NP + 1) + (SUM ? s : party + 1)];
#pragma unroll
                    for (int k = 0; k < W; ++k) z[r][k] += e * v[j][s][k] + m * v[j][0][k];
                }
#pragma unroll
                for (int k = 0; k < W; ++k) computed_here(z[r][k]);
            }
        }
    };
    vec raw[2][kAtOnce][SLOTS];
    if (begin < end) {
        load(raw[0], begin, 0);
        stage(begin, lds);
    }
    int t0 = begin, batch = 0, half = 0;
    __syncthreads();
    // Two batches a turn of the loop, so that each set of buffers has its place in registers.
    while (t0 < end) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (t0 >= end) break;
            const bool last = batch + 1 == batches;
            __builtin_amdgcn_sched_barrier(0);
            load(raw[1 - k], last ? min(t0 + kDepth, end - 1 & ~(kDepth - 1)) : t0, last ? 0 : batch + 1);
            __builtin_amdgcn_sched_barrier(0);
            multiply_words(raw[k], lds + half * (kWords / 2), batch);
            ++batch;
            if (last) {
                t0 += kDepth;
                batch = 0;
                half ^= 1;
                if (t0 < end) stage(t0, lds + half * (kWords / 2));
                __syncthreads();
            }
        }
    }
    // The waves' and groups' sums.
    const size_t each = rows * dim;
#pragma unroll
    for (int r = 0; r < kMost; ++r)
#pragma unroll
        for (int k = 0; k < W; ++k) lds[(r * W + k) * kScoreBlock + threadIdx.x] = mine ? z[r][k] : 0;
    __syncthreads();
    for (int c = threadIdx.x; c < R * W * lanes; c += kScoreBlock) {
        const int part = c / lanes, l = c % lanes, column = (blockIdx.y % column_blocks * 64 + l) * W + part % W;
        if (column >= dim) continue;
        T sum = 0;
        for (int w = 0; w < kScoreWaves; ++w)
            for (int k = 0; k < tokens; ++k) sum += lds[part * kScoreBlock + w * 64 + k * lanes + l];
        const size_t at = (first_row + part / W) * dim + column;
        if (partial) partial[((size_t)block * (SUM ? 1 : NP) + party) * each + at] = sum;
        else if constexpr (SUM) finish<NP, T>(a, at, each, sum);
        else a.out[party * each + at] = a.C[party * each + at] + sum;
    }
}

// Adds the ranges' parts: kJoinRows threads an element (of one party where SUM is false), each every kJoinRows-th range.
constexpr int kJoinRows = 4, kJoinBlock = 256;
template <int NP, class T, bool SUM> __global__ __launch_bounds__(kJoinBlock) void join_kernel(AttentionArgs<T> a, int ranges, const T *partial)
{
    constexpr int kElements = kJoinBlock / kJoinRows;
    __shared__ T sums[kJoinBlock];
    const size_t each = (size_t)a.batch * a.heads * a.d.nodes * a.c.dim, count = SUM ? each : NP * each;
    const size_t at = (blockIdx.x + (size_t)blockIdx.y * gridDim.x) * kElements + threadIdx.x % kElements;
    T z = 0;
    if (at < count) {
#pragma unroll 8
        for (int p = threadIdx.x / kElements; p < ranges; p += kJoinRows) z += partial[p * count + at];
    }
    sums[threadIdx.x] = z;
    __syncthreads();
    if (threadIdx.x >= kElements || at >= count) return;
#pragma unroll
    for (int k = 1; k < kJoinRows; ++k) z += sums[threadIdx.x + k * kElements];
    if constexpr (SUM) finish<NP, T>(a, at, each, z);
    else a.out[at] = a.C[at] + z;
}

// A few tokens at most: one thread an element of the result, on the vector unit.  blockIdx.y = head and node, blockIdx.z = sequence.
constexpr int kFewTokens = 3, kFewBlock = 64;
template <int NP, class T> __global__ __launch_bounds__(kFewBlock) void few_values_kernel(AttentionArgs<T> a)
{
    const int d = blockIdx.x * kFewBlock + threadIdx.x, b = blockIdx.z, h = blockIdx.y / a.d.nodes, m = blockIdx.y % a.d.nodes;
    if (d >= a.c.dim) return;
    const size_t rows = (size_t)a.batch * a.heads * a.d.nodes, row = (size_t)b * a.heads * a.d.nodes + blockIdx.y;
    const size_t slot = ((size_t)a.c.pages * a.c.heads << a.c.shift) * a.c.dim, each = rows * a.c.dim, at = row * a.c.dim + d;
    const int context = a.d.context[b];
    const u64 tree = tree_row(a.d, b, m);
    T z[NP], sum = 0;
#pragma unroll
    for (int i = 0; i < NP; ++i) z[i] = 0;
    for (int t = 0; t < a.d.columns; ++t) {
        const int page = page_of(a.c, b, t);
        if (page < 0 || !sees(tree, a.d.nodes, context, t)) continue;
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
#pragma unroll
        for (int i = 0; i < NP; ++i) sum += z[i];
        finish<NP, T>(a, at, each, sum);
    } else {
#pragma unroll
        for (int i = 0; i < NP; ++i) a.out[i * each + at] = a.C[i * each + at] + z[i];
    }
}

constexpr double kFewSlots = 3;        // workgroups a CU of row_values_kernel
inline int value_waves(int dim) { return dim <= 4 * kTile ? 4 : 8; }
// Tiles of 16 rows a workgroup: two where there are more rows than one has, and registers and LDS for it.  2 parties' 16 heads over 4 cached ones, 16 nodes, two
// sequences of up to 6016: 95 us, 110 by single tiles; 32-bit words, 35 rows of eight sequences: 40 and 44; 20 and 32 rows of 3 parties: 78 and 78, 96 and 96.
constexpr bool two_value_tiles(int n, int word_bytes) { return n <= (word_bytes == 8 ? 3 : 2); }
inline int value_tiles(int n, int rows, int dim, int word_bytes) { return rows > kTile && value_waves(dim) == 8 && two_value_tiles(n, word_bytes) ? 2 : 1; }

// Tokens a workgroup, by an estimate: the chip holds `slots` workgroups, of each of which a beginning takes 0.7 of a turn, and with sequences of any length the
// last round of them is half empty on either side.  us by matrix units and ranges of 1, 2, 4, 8 turns, the chosen one in brackets: 3 parties' 2 x 8 heads of 64 over 701 tokens
// [13.9] 18.6 28.9 50.2; 4 x 8 heads of 128 over up to 32769 569 471 422 [402] (16: 487); 2 parties' 8 x 8 over up to 4097 138 112 [111] 176, 32-bit
// words, 8 x 4 heads of 80 and 35 rows over up to 3008 54 [44] 47 46.  By words the same with 2 to 4 workgroups a CU.
int value_range(int n, int batch, int heads, int cached_heads, int nodes, int columns, int dim, int word_bytes)
{
    const bool few = heads / cached_heads * nodes <= few_value_rows(word_bytes);
    const int waves = value_waves(dim), width = waves * kTile, rows = kTile * value_tiles(n, heads / cached_heads * nodes, dim, word_bytes);
    const double groups = (double)batch * cached_heads * ((heads / cached_heads * nodes + rows - 1) / rows) * ((dim + width - 1) / width);
    const double few_groups = (double)batch * cached_heads * ((dim * word_bytes / 16 + 63) / 64);
    const double slots = few ? 256.0 * kFewSlots : 256.0 * (8 / waves) * (8 / word_bytes);
    const int turns = (columns + kDepth - 1) / kDepth, most = kMostTokens / n / kDepth;
    int best = 1;
    double least = 0;
    for (int r = 1; r <= most && (r == 1 || r < 2 * turns); r *= 2) {
        const double time = ((few ? few_groups : groups) * ((turns + r - 1) / r) / slots + 1) * (0.7 + r);
        if (r == 1 || time < least) best = r, least = time;
    }
    return best * kDepth;
}

}  // namespace

size_t cache_values_workspace(int n, int batch, int heads, int cached_heads, int nodes, int columns, int dim, int word_bytes)
{
    const int range = value_range(n, batch, heads, cached_heads, nodes, columns, dim, word_bytes);
    const size_t ranges = ((size_t)columns + range - 1) / range;
    return 256 + (ranges > 1 ? ranges * n * batch * heads * nodes * dim * word_bytes : 0);
}

// The third axis of a launch: sequences, and without truncation, where a workgroup has one party, those times parties.
template <class T> inline long third_axis(const AttentionArgs<T> &a) { return (long)a.batch * (a.f ? 1 : a.n); }

template <class T> spin_status launch_cache_scores(const AttentionArgs<T> &a, hipStream_t s)
{
    if (third_axis(a) > kMaxGrid) return SPIN_ERANGE;
    KernelTimer timer(SPIN_KERNEL_ATTENTION, s);
    constexpr int kMostLds = 150 << 10;                    // and up to 1.2 KB for what belongs to the rows
    const int R = a.heads / a.c.heads * a.d.nodes, row_tiles = (R + kTile - 1) / kTile, k_tiles = (a.c.dim + kDepth - 1) / kDepth;
    // 3 parties, a token, four sequences of up to 32768: 8 heads of 128 366 us, 408 with ordinary loads; 32-bit words 191 and 214.  Read twice (two row tiles) 120 and 117.
    const bool streamed = row_tiles == 1 && (double)(a.n + 1) * a.batch * a.c.heads * a.d.columns * a.c.dim * sizeof(T) > kKept;
    spin_status st = SPIN_OK;
    for_party_count(a.n, [&](auto np) {
        constexpr int NP = decltype(np)::value, kSlots = (NP + 1) * (int)sizeof(T) * kFrag;
        const int held = k_tiles * kSlots <= kMostLds ? k_tiles : 1;
        const bool few = R <= kFewRows;
        const long blocks = ((long)a.d.columns + kDepth - 1) / kDepth, groups = (long)row_tiles * a.c.heads * a.batch;
        long runs = blocks * groups / kScoreWanted;
        runs = runs < 1 ? 1 : runs > 16 ? 16 : runs;
        const long strips = ((blocks + runs - 1) / runs + kXcds - 1) / kXcds;
        auto go = [&](auto sum, auto by_words, auto nt) {
            constexpr bool SUM = decltype(sum)::value, FEW = decltype(by_words)::value, NT = decltype(nt)::value;
            static OncePerDevice lds_flags;
            st = allow_dynamic_lds((const void *)scores_kernel<NP, T, SUM, FEW, NT>, kMostLds + kScoreWaves * kTurn, lds_flags);
            if (st != SPIN_OK) return;
            const dim3 grid((unsigned)(strips * kXcds * row_tiles), a.c.heads, SUM ? a.batch : a.batch * NP);
            const int bytes = FEW ? (NP + 1) * R * k_tiles * kDepth * (int)sizeof(T) : held * kSlots + kScoreWaves * kTurn;
            scores_kernel<NP, T, SUM, FEW, NT><<<grid, kScoreBlock, bytes, s>>>(a, (int)runs, held);
        };
        auto with = [&](auto sum) {
            if constexpr (decltype(sum)::value) {
                if (streamed) return few ? go(sum, std::true_type(), std::true_type()) : go(sum, std::false_type(), std::true_type());
            }
            if (few) go(sum, std::true_type(), std::false_type());
            else go(sum, std::false_type(), std::false_type());
        };
        if (a.f) with(std::true_type());
        else with(std::false_type());
    });
    return st != SPIN_OK ? st : check_launch("spin_cache_scores");
}

template <class T> spin_status launch_cache_values(const AttentionArgs<T> &a, hipStream_t s)
{
    const int R = a.heads / a.c.heads * a.d.nodes, width = R <= few_value_rows(sizeof(T)) ? 64 * 16 / (int)sizeof(T) : value_waves(a.c.dim) * kTile;
    const long second_axis = (long)((a.c.dim + width - 1) / width) * a.c.heads;
    if (a.d.columns > kFewTokens && (third_axis(a) > kMaxGrid || second_axis > kMaxGrid)) return SPIN_ERANGE;
    KernelTimer timer(SPIN_KERNEL_ATTENTION, s);
    const int range = value_range(a.n, a.batch, a.heads, a.c.heads, a.d.nodes, a.d.columns, a.c.dim, sizeof(T));
    const int ranges = (a.d.columns - 1) / range + 1, strips = (ranges + kXcds - 1) / kXcds;
    T *partial = ranges > 1 ? (T *)a.workspace : nullptr;
    // By digits, non-temporal where a wave's 16 words are whole cache lines (64-bit words, rows of whole tiles; 32-bit ones, half a line, lose a tenth) and no other row
    // tile reads them.  3 parties' 4 x 8 heads, four rows over up to 16384 226 us, 235 with ordinary loads; 16 rows over up to 9008 162 and 168.
    const bool large = (double)(a.n + 1) * a.batch * a.c.heads * a.d.columns * a.c.dim * sizeof(T) > kKept;
    const bool streamed = R <= kTile && a.c.dim % kTile == 0 && large;
    spin_status st = SPIN_OK;
    for_party_count(a.n, [&](auto np) {
        constexpr int NP = decltype(np)::value;
        if (a.d.columns <= kFewTokens) {
            const dim3 grid((a.c.dim + kFewBlock - 1) / kFewBlock, a.heads * a.d.nodes, a.batch);
            few_values_kernel<NP, T><<<grid, kFewBlock, 0, s>>>(a);
            return;
        }
        auto by_words = [&](auto sum, auto nt) {
            constexpr bool SUM = decltype(sum)::value, NT = decltype(nt)::value;
            const dim3 grid(strips * kXcds, (unsigned)second_axis, SUM ? a.batch : a.batch * NP);
            row_values_kernel<NP, T, SUM, NT><<<grid, kScoreBlock, 0, s>>>(a, range, partial);
            if (!partial) return;
            const size_t count = (size_t)a.batch * a.heads * a.d.nodes * a.c.dim * (SUM ? 1 : NP), each = kJoinBlock / kJoinRows;
            join_kernel<NP, T, SUM><<<grid_of((count + each - 1) / each), kJoinBlock, 0, s>>>(a, ranges, partial);
        };
        auto go = [&](auto sum, auto waves, auto tiles, auto nt) {
            constexpr bool SUM = decltype(sum)::value, NT = decltype(nt)::value;
            constexpr int WAVES = decltype(waves)::value, TILES = decltype(tiles)::value, kRows = kTile * TILES, kLds = 2 * TILES * (NP + 1) * (int)sizeof(T) * kFrag;
            static OncePerDevice lds_flags;
            st = allow_dynamic_lds((const void *)values_kernel<NP, T, SUM, WAVES, TILES, NT>, kLds, lds_flags);
            if (st != SPIN_OK) return;
            const dim3 grid(strips * kXcds * ((R + kRows - 1) / kRows), (unsigned)second_axis, SUM ? a.batch : a.batch * NP);
            values_kernel<NP, T, SUM, WAVES, TILES, NT><<<grid, 64 * WAVES, kLds, s>>>(a, range, partial);
            if (!partial) return;
            const size_t count = (size_t)a.batch * a.heads * a.d.nodes * a.c.dim * (SUM ? 1 : NP), each = kJoinBlock / kJoinRows;
            join_kernel<NP, T, SUM><<<grid_of((count + each - 1) / each), kJoinBlock, 0, s>>>(a, ranges, partial);
        };
        auto with = [&](auto sum) {
            if constexpr (decltype(sum)::value && two_value_tiles(NP, sizeof(T))) {
                if (value_tiles(NP, R, a.c.dim, sizeof(T)) == 2) return go(sum, std::integral_constant<int, 8>(), std::integral_constant<int, 2>(), std::false_type());
            }
            const std::integral_constant<int, 1> one;
            if (value_waves(a.c.dim) == 4) return go(sum, std::integral_constant<int, 4>(), one, std::false_type());
            if constexpr (decltype(sum)::value && sizeof(T) == 8) {
                if (streamed) return go(sum, std::integral_constant<int, 8>(), one, std::true_type());
            }
            go(sum, std::integral_constant<int, 8>(), one, std::false_type());
        };
        if (R <= few_value_rows(sizeof(T))) {
            if (a.f && large) by_words(std::true_type(), std::true_type());
            else if (a.f) by_words(std::true_type(), std::false_type());
            else by_words(std::false_type(), std::false_type());
            return;
        }
        if (a.f) with(std::true_type());
        else with(std::false_type());
    });
    return st != SPIN_OK ? st : check_launch("spin_cache_values");
}

template spin_status launch_cache_scores<u64>(const AttentionArgs<u64> &, hipStream_t);
template spin_status launch_cache_scores<u32>(const AttentionArgs<u32> &, hipStream_t);
template spin_status launch_cache_values<u64>(const AttentionArgs<u64> &, hipStream_t);
template spin_status launch_cache_values<u32>(const AttentionArgs<u32> &, hipStream_t);

}  // namespace spin
