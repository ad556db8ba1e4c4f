// What the kernels of linear attention and layer norm share: their arguments as kernels see them.  Interface: spin_linattn_* and spin_layernorm* in
// include/spin.h.
#pragma once
#include "generation.hpp"

namespace spin {

template <class T> struct Masked { const T *x, *a; };
template <class T> struct Tuple { const T *r, *r_top, *r_msb; };

struct ChunkView {                     // tokens and their chunks
    int n, batch, heads, tokens, chunk, chunks, f, g;
    const int32_t *lengths;
};
// Products of rows within chunks.
template <class T> struct ScoresArgs {
    ChunkView c;
    const T *decay;
    int dim;
    Masked<T> x, y;
    const T *C;
    Tuple<T> t;
    T *out;
};
template <class T> struct StatesArgs {
    ChunkView c;
    const T *decay;
    int rows, columns;
    bool reverse;
    Masked<T> x, y;
    const T *C;
    Tuple<T> t;
    const T *first;
    T *states, *last, *opened;         // opened: workspace, a word an element of states
};
template <class T> struct OutputsArgs {
    ChunkView c;
    const T *decay;
    int rows, columns;
    bool reverse, transposed;
    Masked<T> P, y, x, S;
    const T *C;
    Tuple<T> t;
    T *out;
};
template <class T> struct StepArgs {
    int n, batch, heads, f, g, rows, columns;
    const T *decay;
    const int32_t *active;
    const T *S, *S_mask, *CS, *CO;
    Masked<T> q, k, v;
    Tuple<T> tS, tO;
    T *S_out, *out;
};
template <class T> struct NormArgs {
    int n, rows, dim, f, shift, iterations;
    T inv, offset, slope, eps;
    const T *x, *beta, *C1, *C2, *row_words;
    const T *mask_x, *mask_xhat;
    Masked<T> gamma;
    Tuple<T> t1, t2;
    T *out, *xhat, *rstd;
};
template <class T> struct NormGradArgs {
    int n, rows, dim, f, shift;
    T inv;
    Masked<T> dy, xhat, gamma;
    const T *rstd, *mask_g, *C1, *C2, *row_words, *column_words;
    Tuple<T> t1, t2;
    T *dx, *dgamma, *dbeta;
    void *workspace;
};

// T = u32 or u64
template <class T> spin_status launch_linattn_scores(const ScoresArgs<T> &a, hipStream_t s);
template <class T> spin_status launch_linattn_states(const StatesArgs<T> &a, hipStream_t s);
template <class T> spin_status launch_linattn_outputs(const OutputsArgs<T> &a, hipStream_t s);
template <class T> spin_status launch_linattn_step(const StepArgs<T> &a, hipStream_t s);
template <class T> spin_status launch_layernorm(const NormArgs<T> &a, hipStream_t s);
template <class T> spin_status launch_layernorm_grad(const NormGradArgs<T> &a, hipStream_t s);
size_t layernorm_grad_workspace(int n, int rows, int dim, int word_bytes);

constexpr int kNormWords = 15, kNormGradWords = 22;        // of a row: a Newton step's (and as many besides), the gradient's
constexpr int kMostDim = 8192;
// Waves a row: as many as hold its words in registers, four words a thread.  The gradient of 1568 rows of 256, 5 parties: 52 us by one wave, 62 by four, 140 by 16; forward, 3
// parties: 4096 rows of 1024 287 by four, 303 by 16.  Few rows get more waves than they need where all CUs are busy: 2 rows of 1024 14.3 by four, 12.2 by 16.
constexpr int norm_waves(int rows, int dim) { return dim <= 256 ? 1 : dim <= 1024 && rows > 256 ? 4 : 16; }

// The gradient's rows: of one wave or workgroup (`run` successive ones), and how many groups of rows have sums of their own: those of a workgroup.  As many as are on the chip at
// once: more groups only add sums to be written and joined (16 waves: one workgroup a CU).
struct NormRuns { int run, groups; };
constexpr int norm_rows_at_once(int rows, int dim) { return norm_waves(rows, dim) == 1 ? 4 : 1; }
constexpr int norm_wanted_groups(int rows, int dim) { return norm_waves(rows, dim) == 16 ? 256 : 1024; }
constexpr NormRuns norm_runs(int rows, int dim)
{
    const long at_once = norm_rows_at_once(rows, dim), wanted = norm_wanted_groups(rows, dim) * at_once, run = (rows + wanted - 1) / wanted;
    return {(int)run, (int)((rows + run * at_once - 1) / (run * at_once))};
}
// At least as many groups, and never fewer for more rows: 1025 rows in runs of two have half the groups of 1024, and a workspace for the largest batch has to do for all.
constexpr int norm_most_groups(int rows, int dim)
{
    const int at_once = norm_rows_at_once(rows, dim), all = (int)(((long)rows + at_once - 1) / at_once), wanted = norm_wanted_groups(rows, dim);
    return all < wanted ? all : wanted;
}

namespace {

// A word that is read once, by nobody else: what the dealer gave for one element.
template <class T> __device__ inline T once(const T *p) { return __builtin_nontemporal_load(p); }

// Results far larger than the caches, all parties', are written past them.
constexpr size_t kStreamingBytes = (size_t)64 << 20;
template <class T> __device__ inline void put(bool streamed, T *p, T v)
{
    if (streamed) __builtin_nontemporal_store(v, p);
    else *p = v;
}

// Tokens of a sequence of `length` that are in a chunk.  The length may be anything.
__host__ __device__ inline int tokens_in(const ChunkView &c, int length, int chunk)
{
    const int all = length < 0 ? 0 : length < c.tokens ? length : c.tokens, left = all - chunk * c.chunk;      // chunk * c.chunk < c.tokens
    return left < 0 ? 0 : left < c.chunk ? left : c.chunk;
}

}  // namespace
}  // namespace spin
