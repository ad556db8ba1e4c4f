// What the kernels for generating token by token share: the paged cache as kernels see it, what a drafted token sees, and the
// truncation of shares held in registers.  Interface: spin_cache_* and spin_relbias_* in include/spin.h.
#pragma once
#include "common.hpp"

namespace spin {

struct CacheView {                     // of one pool
    int pages, heads, dim, table_pages, shift;           // page_tokens = 1 << shift
    const int32_t *table;
};
constexpr int kMostColumns = 1 << 24;   // of a row of scores
struct DraftView {                     // who sees what
    int nodes, columns;
    const int32_t *context;
    const u64 *tree;
};
struct BiasView {
    int buckets, reach;
    const int32_t *bucket_of;
    const void *table;
};

template <class T> struct AttentionArgs {
    CacheView c;
    DraftView d;
    BiasView bias;                     // scores only; table null: none
    const int32_t *depth;
    int n, batch, heads, f;
    const T *pool, *x, *A, *C, *r, *r_top, *r_msb;       // x: Q or P
    T masked;
    T *out;
    void *workspace;
};
template <class T> struct AppendArgs {
    CacheView c;
    int n, batch, rows;
    const int32_t *start, *count;
    const T *x[2], *b[2];
    T *pool[2];
};
template <class T> struct PairArgs {   // scores as whole matrices
    BiasView bias;
    int n, batch, heads, Q, K, first, causal, f;
    const int32_t *lengths;
    const T *x, *r, *r_top, *r_msb;
    T masked;
    T *out;
};

// T = u32 or u64
template <class T> spin_status launch_cache_append(const AppendArgs<T> &a, hipStream_t s);
template <class T> spin_status launch_cache_copy(const CacheView &c, int n, int pairs, const int32_t *src, const int32_t *dst, T *K, T *V, hipStream_t s);
template <class T>
spin_status launch_cache_compact(const CacheView &c, int n, int batch, int nodes, const int32_t *context, const int32_t *kept, const int32_t *kept_count,
                                 T *K, T *V, hipStream_t s);
template <class T> spin_status launch_cache_scores(const AttentionArgs<T> &a, hipStream_t s);
template <class T> spin_status launch_cache_values(const AttentionArgs<T> &a, hipStream_t s);
size_t cache_values_workspace(int n, int batch, int heads, int cached_heads, int nodes, int columns, int dim, int word_bytes);
template <class T> spin_status launch_relbias_trunc(const PairArgs<T> &a, hipStream_t s);
template <class T> spin_status launch_relbias_grad(const PairArgs<T> &a, hipStream_t s);

namespace {

constexpr int kMaxGrid = 65535;        // of a launch grid's second and third axes
constexpr int kXcds = 8;               // workgroups go to the XCDs in turn

// blockIdx.x, turned on from row to row of the grid so that every XCD meets all of its values: left alone a width that divides into the XCDs gives each of them
// the same few columns, and where some columns have more work than others (masks, diagonals of different lengths) half of the chip waits.
__device__ inline int turned_x()
{
    const unsigned row = blockIdx.y + blockIdx.z * gridDim.y;
    return (int)((blockIdx.x + row * gridDim.x / kXcds) % gridDim.x);
}

// A grid of at least `blocks` workgroups of up to 256 threads on two axes: one axis holds fewer than 2^32 threads.
inline dim3 grid_of(size_t blocks)
{
    constexpr size_t kMost = (size_t)1 << 22;
    const size_t rows = (blocks + kMost - 1) / kMost;
    return dim3((unsigned)((blocks + rows - 1) / rows), (unsigned)rows);
}

// The page of position `pos` of sequence b, or -1 where there is none.  pos may be anything.
__host__ __device__ inline int page_of(const CacheView &c, int b, long pos)
{
    if (pos < 0 || (pos >> c.shift) >= c.table_pages) return -1;
    const int p = c.table[(size_t)b * c.table_pages + (pos >> c.shift)];
    return (unsigned)p < (unsigned)c.pages ? p : -1;
}
// Word offset of a cached row.
__host__ __device__ inline size_t row_at(const CacheView &c, int slot, int page, int head, long pos)
{
    return (((((size_t)slot * c.pages + page) * c.heads + head) << c.shift) + (pos & ((1l << c.shift) - 1))) * c.dim;
}
// The nodes that node m of sequence b sees, as bits.
__host__ __device__ inline u64 tree_row(const DraftView &d, int b, int m) { return d.tree ? d.tree[(size_t)b * d.nodes + m] : ((u64)2 << m) - 1; }
__host__ __device__ inline bool sees(u64 row, int nodes, int context, int pos)
{
    const long at = (long)pos - context;
    return context >= 0 && (at < 0 || (at < nodes && (row >> at & 1)));
}

// Truncation (Section 4.4; steps as listed at spin_trunc) of one element: every party's y + r is added to the opened value, which then tells every
// party its share of the result.
template <class T> struct Opened {
    static constexpr int L = 8 * sizeof(T);
    int f;
    T c = (T)1 << (L - 2);
    __device__ void add(T masked) { c += masked; }
    __device__ T truncated(int party, T r_top, T r_msb) const
    {
        const T c_msb = c >> (L - 1), y = ((r_msb - 2 * c_msb * r_msb) << (L - 1 - f)) - r_top;
        return party ? y : y + (c_msb << (L - 1 - f)) + ((c >> f) & (((T)1 << (L - 1 - f)) - 1)) - ((T)1 << (L - 2 - f));
    }
};
template <int NP, class T> __device__ inline void truncate_shares(T (&y)[NP], const T (&r)[NP], const T (&r_top)[NP], const T (&r_msb)[NP], int f)
{
    Opened<T> c{f};
#pragma unroll
    for (int i = 0; i < NP; ++i) c.add(y[i] + r[i]);
#pragma unroll
    for (int i = 0; i < NP; ++i) y[i] = c.truncated(i, r_top[i], r_msb[i]);
}

// Bucket of a distance, or -1 where it has none.
__host__ __device__ inline int bucket_at(const BiasView &v, int distance)
{
    const int b = v.bucket_of[(distance < -v.reach ? -v.reach : distance > v.reach ? v.reach : distance) + v.reach];
    return (unsigned)b < (unsigned)v.buckets ? b : -1;
}

// The rows of [q0, q1) whose score on the diagonal k - q = away is there are [from, to): none where to <= from.  Lengths may be anything;
// |away| and |first| are below 2^30.
struct DiagonalRows { int from, to; };
__host__ __device__ inline DiagonalRows rows_of_diagonal(int away, int q0, int q1, int K, int length, bool causal, int first)
{
    length = length < 0 ? 0 : length > K ? K : length;     // left negative, the subtraction below can pass 32 bits
    const int from = q0 > -away ? q0 : -away;
    if (causal && away > first) return {from, from};
    return {from, q1 < length - away ? q1 : length - away};
}

}  // namespace
}  // namespace spin
