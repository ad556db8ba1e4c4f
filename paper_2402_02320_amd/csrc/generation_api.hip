// The C ABI of spin_cache_* and spin_relbias_* (include/spin.h): argument validation, then dispatch to the launchers.  Validation
// touches no HIP call.
#include "generation.hpp"

using namespace spin;

namespace {

inline bool bad_ptr(const void *p) { return p == nullptr || ((uintptr_t)p & 15) != 0; }
inline bool bad_list(const int32_t *p) { return p == nullptr || ((uintptr_t)p & 3) != 0; }
inline bool bad_n(int n) { return n < 1 || n > SPIN_MAX_PARTIES; }
constexpr double kMaxWords = (double)((size_t)1 << 40);  // of any one tensor; offsets are 64 bits

int log2_of(int v)
{
    int k = 0;
    while ((1 << k) < v) ++k;
    return k;
}

// Everything about the cache but its pools; with the table where the call looks at it.
spin_status check_cache(const spin_cache *c, bool table)
{
    if (c == nullptr || bad_n(c->n) || c->pages < 1 || c->heads < 1) return SPIN_EINVAL;
    if (c->page_tokens < 16 || c->page_tokens > 4096 || (c->page_tokens & (c->page_tokens - 1)) != 0) return SPIN_EINVAL;
    if (c->dim < 8 || c->dim > 256 || c->dim % 8 != 0) return SPIN_EINVAL;
    if ((double)(c->n + 1) * c->pages * c->heads * c->page_tokens * c->dim > kMaxWords || c->heads > kMaxGrid) return SPIN_ERANGE;
    if (!table) return SPIN_OK;
    if (c->batch < 1 || c->table_pages < 1 || bad_list(c->table)) return SPIN_EINVAL;
    if ((long)c->batch * c->heads > kMaxGrid) return SPIN_ERANGE;
    return SPIN_OK;
}

CacheView view_of(const spin_cache &c) { return CacheView{c.pages, c.heads, c.dim, c.table_pages, log2_of(c.page_tokens), c.table}; }

template <class T>
spin_status append(const spin_cache *c, int rows, const int32_t *start, const int32_t *count, const T *Kx, const T *Kb, const T *Vx, const T *Vb, spin_stream stream)
{
    const spin_status st = check_cache(c, true);
    if (st != SPIN_OK) return st;
    if (rows < 1 || bad_list(start) || (count && bad_list(count)) || bad_ptr(c->K) || bad_ptr(c->V) || bad_ptr(Kx) || bad_ptr(Kb) || bad_ptr(Vx) || bad_ptr(Vb))
        return SPIN_EINVAL;
    if (rows > (1 << 24) || (double)c->n * c->batch * c->heads * rows * c->dim > kMaxWords) return SPIN_ERANGE;
    return launch_cache_append<T>(AppendArgs<T>{view_of(*c), c->n, c->batch, rows, start, count, {Kx, Vx}, {Kb, Vb}, {(T *)c->K, (T *)c->V}}, (hipStream_t)stream);
}

template <class T> spin_status copy(const spin_cache *c, int pairs, const int32_t *src, const int32_t *dst, spin_stream stream)
{
    const spin_status st = check_cache(c, false);
    if (st != SPIN_OK) return st;
    if (pairs < 1 || bad_list(src) || bad_list(dst) || bad_ptr(c->K) || bad_ptr(c->V)) return SPIN_EINVAL;
    if (pairs > kMaxGrid) return SPIN_ERANGE;
    return launch_cache_copy<T>(view_of(*c), c->n, pairs, src, dst, (T *)c->K, (T *)c->V, (hipStream_t)stream);
}

template <class T>
spin_status compact(const spin_cache *c, int nodes, const int32_t *context, const int32_t *kept, const int32_t *kept_count, spin_stream stream)
{
    const spin_status st = check_cache(c, true);
    if (st != SPIN_OK) return st;
    if (nodes < 1 || nodes > SPIN_MAX_NODES || bad_list(context) || bad_list(kept) || bad_list(kept_count) || bad_ptr(c->K) || bad_ptr(c->V)) return SPIN_EINVAL;
    return launch_cache_compact<T>(view_of(*c), c->n, c->batch, nodes, context, kept, kept_count, (T *)c->K, (T *)c->V, (hipStream_t)stream);
}

spin_status check_attention(const spin_cache *c, int heads, int nodes, int columns)
{
    const spin_status st = check_cache(c, true);
    if (st != SPIN_OK) return st;
    if (heads < 1 || heads % c->heads != 0 || nodes < 1 || nodes > SPIN_MAX_NODES || columns < 1) return SPIN_EINVAL;
    if (columns > kMostColumns || (long)heads * nodes > kMaxGrid || (double)c->n * c->batch * heads * nodes * columns > kMaxWords) return SPIN_ERANGE;
    return SPIN_OK;
}

bool bad_bias(const spin_relbias *b, bool table)
{
    return b == nullptr || b->buckets < 1 || b->buckets > 1024 || b->reach < 0 || b->reach > 65535 || bad_list(b->bucket_of) || (table && bad_ptr(b->table));
}

template <class T>
spin_status attend(bool scores, const spin_cache *c, int heads, int nodes, int columns, int f, const int32_t *context, const u64 *tree, const T *x, const T *A,
                   const T *C, const T *r, const T *r_top, const T *r_msb, T masked, const spin_relbias *bias, const int32_t *depth, T *out, void *workspace,
                   size_t workspace_bytes, spin_stream stream)
{
    const spin_status st = check_attention(c, heads, nodes, columns);
    if (st != SPIN_OK) return st;
    const void *pool = scores ? c->K : c->V;
    if (f < 0 || f > 8 * (int)sizeof(T) - 3 || bad_list(context) || (tree && ((uintptr_t)tree & 7) != 0)) return SPIN_EINVAL;
    if (bad_ptr(pool) || bad_ptr(x) || bad_ptr(A) || bad_ptr(C) || bad_ptr(out)) return SPIN_EINVAL;
    if (f > 0 && (bad_ptr(r) || bad_ptr(r_top) || bad_ptr(r_msb))) return SPIN_EINVAL;
    if (bias && (bad_bias(bias, true) || (depth && bad_list(depth)))) return SPIN_EINVAL;
    if (!scores) {
        const size_t need = cache_values_workspace(c->n, c->batch, heads, c->heads, nodes, columns, c->dim, sizeof(T));
        if (workspace == nullptr || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < need) return SPIN_EWORKSPACE;
    }
    AttentionArgs<T> a{view_of(*c), {nodes, columns, context, tree}, {0, 0, nullptr, nullptr}, bias ? depth : nullptr, c->n, c->batch, heads, f, (const T *)pool, x, A, C,
                       r, r_top, r_msb, masked, out, workspace};
    if (bias) a.bias = BiasView{bias->buckets, bias->reach, bias->bucket_of, bias->table};
    return scores ? launch_cache_scores<T>(a, (hipStream_t)stream) : launch_cache_values<T>(a, (hipStream_t)stream);
}

size_t values_workspace(const spin_cache *c, int heads, int nodes, int columns, int word_bytes)
{
    if (check_attention(c, heads, nodes, columns) != SPIN_OK) return 0;
    return cache_values_workspace(c->n, c->batch, heads, c->heads, nodes, columns, c->dim, word_bytes);
}

spin_status check_pairs(int n, int batch, int heads, int Q, int K, int first, const int32_t *lengths, int f, int most)
{
    if (bad_n(n) || batch < 1 || heads < 1 || Q < 1 || K < 1 || f < 0 || f > most || (lengths && bad_list(lengths))) return SPIN_EINVAL;
    if (Q > (1 << 24) || K > (1 << 24) || first < -(1 << 28) || first > (1 << 28)) return SPIN_ERANGE;
    if ((long)batch * heads > kMaxGrid || (double)n * batch * heads * Q * K > kMaxWords || (long)n * heads > kMaxGrid) return SPIN_ERANGE;
    return SPIN_OK;
}

template <class T>
spin_status relbias_trunc(int n, int batch, int heads, int Q, int K, int first, int causal, const int32_t *lengths, int f, const T *x, const T *r,
                          const T *r_top, const T *r_msb, T masked, const spin_relbias *bias, T *out, spin_stream stream)
{
    const spin_status st = check_pairs(n, batch, heads, Q, K, first, lengths, f, 8 * (int)sizeof(T) - 3);
    if (st != SPIN_OK) return st;
    if (bad_ptr(x) || bad_ptr(out) || bad_bias(bias, true) || (f > 0 && (bad_ptr(r) || bad_ptr(r_top) || bad_ptr(r_msb)))) return SPIN_EINVAL;
    return launch_relbias_trunc<T>(PairArgs<T>{{bias->buckets, bias->reach, bias->bucket_of, bias->table}, n, batch, heads, Q, K, first, causal != 0, f, lengths,
                                               x, r, r_top, r_msb, masked, out}, (hipStream_t)stream);
}

template <class T>
spin_status relbias_grad(int n, int batch, int heads, int Q, int K, int first, int causal, const int32_t *lengths, const T *dS, const spin_relbias *bias, T *grad,
                         spin_stream stream)
{
    const spin_status st = check_pairs(n, batch, heads, Q, K, first, lengths, 0, 0);
    if (st != SPIN_OK) return st;
    if (bad_ptr(dS) || bad_ptr(grad) || bad_bias(bias, false)) return SPIN_EINVAL;
    return launch_relbias_grad<T>(PairArgs<T>{{bias->buckets, bias->reach, bias->bucket_of, nullptr}, n, batch, heads, Q, K, first, causal != 0, 0, lengths,
                                              dS, nullptr, nullptr, nullptr, 0, grad}, (hipStream_t)stream);
}

}  // namespace

extern "C" {

spin_status spin_cache_append(const spin_cache *c, int rows, const int32_t *start, const int32_t *count, const uint64_t *Kx, const uint64_t *Kb,
                              const uint64_t *Vx, const uint64_t *Vb, spin_stream stream)
{
    return append<uint64_t>(c, rows, start, count, Kx, Kb, Vx, Vb, stream);
}

spin_status spin_cache_copy(const spin_cache *c, int pairs, const int32_t *src, const int32_t *dst, spin_stream stream)
{
    return copy<uint64_t>(c, pairs, src, dst, stream);
}

spin_status spin_cache_compact(const spin_cache *c, int nodes, const int32_t *context, const int32_t *kept, const int32_t *kept_count, spin_stream stream)
{
    return compact<uint64_t>(c, nodes, context, kept, kept_count, stream);
}

spin_status spin_cache_scores(const spin_cache *c, int heads, int nodes, int columns, int f, const int32_t *context, const uint64_t *tree, const uint64_t *Q,
                              const uint64_t *A, const uint64_t *C, const uint64_t *r, const uint64_t *r_top, const uint64_t *r_msb,
                              uint64_t masked, const spin_relbias *bias, const int32_t *depth, uint64_t *out, spin_stream stream)
{
    return attend<uint64_t>(true, c, heads, nodes, columns, f, context, tree, Q, A, C, r, r_top, r_msb, masked, bias, depth, out, nullptr, 0, stream);
}

spin_status spin_cache_values(const spin_cache *c, int heads, int nodes, int columns, int f, const int32_t *context, const uint64_t *tree, const uint64_t *P,
                              const uint64_t *A, const uint64_t *C, const uint64_t *r, const uint64_t *r_top, const uint64_t *r_msb, uint64_t *out,
                              void *workspace, size_t workspace_bytes, spin_stream stream)
{
    return attend<uint64_t>(false, c, heads, nodes, columns, f, context, tree, P, A, C, r, r_top, r_msb, 0, nullptr, nullptr, out, workspace, workspace_bytes, stream);
}

size_t spin_cache_values_workspace_bytes(const spin_cache *c, int heads, int nodes, int columns)
{
    return values_workspace(c, heads, nodes, columns, sizeof(uint64_t));
}

spin_status spin_relbias_trunc(int n, int batch, int heads, int Q, int K, int first, int causal, const int32_t *lengths, int f, const uint64_t *x,
                               const uint64_t *r, const uint64_t *r_top, const uint64_t *r_msb, uint64_t masked, const spin_relbias *bias, uint64_t *out,
                               spin_stream stream)
{
    return relbias_trunc<uint64_t>(n, batch, heads, Q, K, first, causal, lengths, f, x, r, r_top, r_msb, masked, bias, out, stream);
}

spin_status spin_relbias_grad(int n, int batch, int heads, int Q, int K, int first, int causal, const int32_t *lengths, const uint64_t *dS,
                              const spin_relbias *bias, uint64_t *grad, spin_stream stream)
{
    return relbias_grad<uint64_t>(n, batch, heads, Q, K, first, causal, lengths, dS, bias, grad, stream);
}

spin_status spin32_cache_append(const spin_cache *c, int rows, const int32_t *start, const int32_t *count, const uint32_t *Kx, const uint32_t *Kb,
                              const uint32_t *Vx, const uint32_t *Vb, spin_stream stream)
{
    return append<uint32_t>(c, rows, start, count, Kx, Kb, Vx, Vb, stream);
}

spin_status spin32_cache_copy(const spin_cache *c, int pairs, const int32_t *src, const int32_t *dst, spin_stream stream)
{
    return copy<uint32_t>(c, pairs, src, dst, stream);
}

spin_status spin32_cache_compact(const spin_cache *c, int nodes, const int32_t *context, const int32_t *kept, const int32_t *kept_count, spin_stream stream)
{
    return compact<uint32_t>(c, nodes, context, kept, kept_count, stream);
}

spin_status spin32_cache_scores(const spin_cache *c, int heads, int nodes, int columns, int f, const int32_t *context, const uint64_t *tree, const uint32_t *Q,
                              const uint32_t *A, const uint32_t *C, const uint32_t *r, const uint32_t *r_top, const uint32_t *r_msb,
                              uint32_t masked, const spin_relbias *bias, const int32_t *depth, uint32_t *out, spin_stream stream)
{
    return attend<uint32_t>(true, c, heads, nodes, columns, f, context, tree, Q, A, C, r, r_top, r_msb, masked, bias, depth, out, nullptr, 0, stream);
}

spin_status spin32_cache_values(const spin_cache *c, int heads, int nodes, int columns, int f, const int32_t *context, const uint64_t *tree, const uint32_t *P,
                              const uint32_t *A, const uint32_t *C, const uint32_t *r, const uint32_t *r_top, const uint32_t *r_msb, uint32_t *out,
                              void *workspace, size_t workspace_bytes, spin_stream stream)
{
    return attend<uint32_t>(false, c, heads, nodes, columns, f, context, tree, P, A, C, r, r_top, r_msb, 0, nullptr, nullptr, out, workspace, workspace_bytes, stream);
}

size_t spin32_cache_values_workspace_bytes(const spin_cache *c, int heads, int nodes, int columns)
{
    return values_workspace(c, heads, nodes, columns, sizeof(uint32_t));
}

spin_status spin32_relbias_trunc(int n, int batch, int heads, int Q, int K, int first, int causal, const int32_t *lengths, int f, const uint32_t *x,
                               const uint32_t *r, const uint32_t *r_top, const uint32_t *r_msb, uint32_t masked, const spin_relbias *bias, uint32_t *out,
                               spin_stream stream)
{
    return relbias_trunc<uint32_t>(n, batch, heads, Q, K, first, causal, lengths, f, x, r, r_top, r_msb, masked, bias, out, stream);
}

spin_status spin32_relbias_grad(int n, int batch, int heads, int Q, int K, int first, int causal, const int32_t *lengths, const uint32_t *dS,
                              const spin_relbias *bias, uint32_t *grad, spin_stream stream)
{
    return relbias_grad<uint32_t>(n, batch, heads, Q, K, first, causal, lengths, dS, bias, grad, stream);
}

}  // extern "C"
