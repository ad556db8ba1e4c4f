// The C ABI of spin_linattn_* and spin_layernorm* (include/spin.h): argument validation, then dispatch to the launchers.  Validation
// touches no HIP call.
#include "linear.hpp"

using namespace spin;

namespace {

inline bool bad_ptr(const void *p) { return p == nullptr || ((uintptr_t)p & 15) != 0; }
inline bool bad_list(const int32_t *p) { return ((uintptr_t)p & 3) != 0; }
inline bool bad_n(int n) { return n < 1 || n > SPIN_MAX_PARTIES; }
inline bool bad(const spin_masked *m) { return m == nullptr || bad_ptr(m->value) || bad_ptr(m->mask); }
inline bool bad(const spin_tuple *t) { return t == nullptr || bad_ptr(t->r) || bad_ptr(t->r_top) || bad_ptr(t->r_msb); }
inline bool bad_dim(int d) { return d < 8 || d > 256 || d % 8 != 0; }
inline bool bad_workspace(const void *p, size_t have, size_t need) { return p == nullptr || ((uintptr_t)p & 255) != 0 || have < need; }
constexpr double kMaxWords = (double)((size_t)1 << 40);    // of any one tensor; offsets are 64 bits
template <class T> constexpr int most_bits = 8 * (int)sizeof(T) - 3;

template <class T> Masked<T> of(const spin_masked *m) { return {(const T *)m->value, (const T *)m->mask}; }
template <class T> Tuple<T> of(const spin_tuple *t) { return {(const T *)t->r, (const T *)t->r_top, (const T *)t->r_msb}; }

// What every call looks at: parties, heads, bits, the decay.
spin_status check_heads(const spin_linattn *s, int most)
{
    if (s == nullptr || bad_n(s->n) || s->batch < 1 || s->heads < 1 || s->f < 1 || s->g < 0 || s->f > most || s->g > most || s->f + s->g > most) return SPIN_EINVAL;
    if ((s->decay == nullptr && s->g != 0) || (s->decay && bad_ptr(s->decay)) || bad_list(s->lengths)) return SPIN_EINVAL;
    return (long)s->batch * s->heads > kMaxGrid ? SPIN_ERANGE : SPIN_OK;
}

// And the chunks; `words` a token and `square` a chunk are those of the call's largest tensors.
spin_status check_chunks(const spin_linattn *s, int most, double words, double square)
{
    const spin_status st = check_heads(s, most);
    if (st != SPIN_OK) return st;
    if (s->tokens < 1 || (s->chunk != 32 && s->chunk != 64 && s->chunk != 128)) return SPIN_EINVAL;
    if (s->tokens > (1 << 24)) return SPIN_ERANGE;
    const double rows = (double)s->n * s->batch * s->heads, chunks = (s->tokens + s->chunk - 1) / s->chunk;
    return rows * s->tokens * words > kMaxWords || rows * chunks * square > kMaxWords ? SPIN_ERANGE : SPIN_OK;
}

ChunkView view_of(const spin_linattn &s)
{
    return ChunkView{s.n, s.batch, s.heads, s.tokens, s.chunk, (s.tokens + s.chunk - 1) / s.chunk, s.f, s.g, s.lengths};
}

template <class T>
spin_status run_scores(const spin_linattn *s, int dim, const spin_masked *x, const spin_masked *y, const T *C, const spin_tuple *t, T *out, spin_stream stream)
{
    if (bad_dim(dim)) return SPIN_EINVAL;
    const spin_status st = check_chunks(s, most_bits<T>, dim, s ? (double)s->chunk * s->chunk : 0);
    if (st != SPIN_OK) return st;
    if (bad(x) || bad(y) || bad(t) || bad_ptr(C) || bad_ptr(out)) return SPIN_EINVAL;
    return launch_linattn_scores<T>({view_of(*s), (const T *)s->decay, dim, of<T>(x), of<T>(y), C, of<T>(t), out}, (hipStream_t)stream);
}

spin_status check_states(const spin_linattn *s, int rows, int columns, int most)
{
    if (bad_dim(rows) || bad_dim(columns)) return SPIN_EINVAL;
    return check_chunks(s, most, rows > columns ? rows : columns, (double)rows * columns);
}

size_t states_workspace(const spin_linattn *s, int rows, int columns, int word_bytes)
{
    if (check_states(s, rows, columns, 8 * word_bytes - 3) != SPIN_OK) return 0;
    return (size_t)s->batch * s->heads * ((s->tokens + s->chunk - 1) / s->chunk) * rows * columns * word_bytes;
}

template <class T>
spin_status run_states(const spin_linattn *s, int rows, int columns, int reverse, const spin_masked *x, const spin_masked *y, const T *C, const spin_tuple *t, const T *first,
                   T *all, T *last, void *workspace, size_t workspace_bytes, spin_stream stream)
{
    const spin_status st = check_states(s, rows, columns, most_bits<T>);
    if (st != SPIN_OK) return st;
    if (bad(x) || bad(y) || bad(t) || bad_ptr(C) || (first && bad_ptr(first)) || bad_ptr(all) || bad_ptr(last)) return SPIN_EINVAL;
    if (bad_workspace(workspace, workspace_bytes, states_workspace(s, rows, columns, sizeof(T)))) return SPIN_EWORKSPACE;
    return launch_linattn_states<T>({view_of(*s), (const T *)s->decay, rows, columns, reverse != 0, of<T>(x), of<T>(y), C, of<T>(t), first, all, last, (T *)workspace},
                                    (hipStream_t)stream);
}

template <class T>
spin_status run_outputs(const spin_linattn *s, int rows, int columns, int reverse, int transposed, const spin_masked *P, const spin_masked *y, const spin_masked *x,
                    const spin_masked *S, const T *C, const spin_tuple *t, T *out, spin_stream stream)
{
    if (bad_dim(rows) || bad_dim(columns)) return SPIN_EINVAL;
    const double state = (double)rows * columns, pairs = s ? (double)s->chunk * s->chunk : 0;
    const spin_status st = check_chunks(s, most_bits<T>, rows > columns ? rows : columns, state > pairs ? state : pairs);
    if (st != SPIN_OK) return st;
    if (bad(P) || bad(y) || bad(x) || bad(S) || bad(t) || bad_ptr(C) || bad_ptr(out)) return SPIN_EINVAL;
    return launch_linattn_outputs<T>({view_of(*s), (const T *)s->decay, rows, columns, reverse != 0, transposed != 0, of<T>(P), of<T>(y), of<T>(x), of<T>(S), C, of<T>(t),
                                      out}, (hipStream_t)stream);
}

template <class T>
spin_status run_step(const spin_linattn *s, int rows, int columns, const T *S, const spin_masked *q, const spin_masked *k, const spin_masked *v, const T *S_mask, const T *CS,
                 const spin_tuple *tS, const T *CO, const spin_tuple *tO, T *S_out, T *out, spin_stream stream)
{
    if (bad_dim(rows) || bad_dim(columns)) return SPIN_EINVAL;
    const spin_status st = check_heads(s, most_bits<T>);
    if (st != SPIN_OK) return st;
    if (bad_ptr(S) || bad(q) || bad(k) || bad(v) || bad_ptr(S_mask) || bad_ptr(CS) || bad(tS) || bad_ptr(CO) || bad(tO) || bad_ptr(S_out) || bad_ptr(out)) return SPIN_EINVAL;
    return launch_linattn_step<T>({s->n, s->batch, s->heads, s->f, s->g, rows, columns, (const T *)s->decay, s->lengths, S, S_mask, CS, CO, of<T>(q), of<T>(k), of<T>(v),
                                   of<T>(tS), of<T>(tO), S_out, out}, (hipStream_t)stream);
}

spin_status check_norm(const spin_norm *s, int most)
{
    if (s == nullptr || bad_n(s->n) || s->rows < 1 || s->dim < 1 || s->dim > kMostDim || s->f < 1 || s->f >= most || s->shift < 1 || s->shift > most) return SPIN_EINVAL;
    // a launch has fewer than 2^32 threads
    if (s->rows > (1 << 24) || (double)s->rows * norm_waves(s->rows, s->dim) * 64 > (double)(1u << 31)) return SPIN_ERANGE;
    return (double)s->n * s->rows * s->dim > kMaxWords ? SPIN_ERANGE : SPIN_OK;
}

template <class T> T inverse(const spin_norm &s) { return (T)((((uint64_t)1 << s.shift) + s.dim / 2) / s.dim); }

size_t norm_grad_workspace(const spin_norm *s, int word_bytes)
{
    return check_norm(s, 8 * word_bytes - 3) == SPIN_OK ? layernorm_grad_workspace(s->n, s->rows, s->dim, word_bytes) : 0;
}

template <class T>
spin_status run_norm(const spin_norm *s, int iterations, T offset, T slope, T eps, const T *x, const spin_masked *gamma, const T *beta, const T *mask_x, const T *mask_xhat,
                 const T *C1, const spin_tuple *t1, const T *C2, const spin_tuple *t2, const T *row_words, T *out, T *xhat, T *rstd, spin_stream stream)
{
    const spin_status st = check_norm(s, most_bits<T>);
    if (st != SPIN_OK) return st;
    if (iterations < 0 || iterations > SPIN_MAX_NORM_ITERATIONS || bad_ptr(x) || bad(gamma) || bad_ptr(beta) || bad_ptr(mask_x) || bad_ptr(mask_xhat) || bad_ptr(C1) ||
        bad(t1) || bad_ptr(C2) || bad(t2) || bad_ptr(row_words) || bad_ptr(out) || (xhat && bad_ptr(xhat)) || (rstd && bad_ptr(rstd)))
        return SPIN_EINVAL;
    return launch_layernorm<T>({s->n, s->rows, s->dim, s->f, s->shift, iterations, inverse<T>(*s), offset, slope, eps, x, beta, C1, C2, row_words, mask_x, mask_xhat,
                                of<T>(gamma), of<T>(t1), of<T>(t2), out, xhat, rstd}, (hipStream_t)stream);
}

template <class T>
spin_status run_norm_grad(const spin_norm *s, const spin_masked *dy, const spin_masked *xhat, const T *rstd, const spin_masked *gamma, const T *mask_g, const T *C1,
                      const spin_tuple *t1, const T *C2, const spin_tuple *t2, const T *row_words, const T *column_words, T *dx, T *dgamma, T *dbeta, void *workspace,
                      size_t workspace_bytes, spin_stream stream)
{
    const spin_status st = check_norm(s, most_bits<T>);
    if (st != SPIN_OK) return st;
    if (bad(dy) || bad(xhat) || bad_ptr(rstd) || bad(gamma) || bad_ptr(mask_g) || bad_ptr(C1) || bad(t1) || bad_ptr(C2) || bad(t2) || bad_ptr(row_words) ||
        bad_ptr(column_words) || bad_ptr(dx) || bad_ptr(dgamma) || bad_ptr(dbeta))
        return SPIN_EINVAL;
    if (bad_workspace(workspace, workspace_bytes, layernorm_grad_workspace(s->n, s->rows, s->dim, sizeof(T)))) return SPIN_EWORKSPACE;
    return launch_layernorm_grad<T>({s->n, s->rows, s->dim, s->f, s->shift, inverse<T>(*s), of<T>(dy), of<T>(xhat), of<T>(gamma), rstd, mask_g, C1, C2, row_words,
                                     column_words, of<T>(t1), of<T>(t2), dx, dgamma, dbeta, workspace}, (hipStream_t)stream);
}

}  // namespace

extern "C" {

spin_status spin_linattn_scores(const spin_linattn *s, int dim, const spin_masked *x, const spin_masked *y, const uint64_t *C, const spin_tuple *t, uint64_t *out,
                                spin_stream stream)
{
    return run_scores<uint64_t>(s, dim, x, y, C, t, out, stream);
}

spin_status spin_linattn_states(const spin_linattn *s, int rows, int columns, int reverse, const spin_masked *x, const spin_masked *y, const uint64_t *C,
                                const spin_tuple *t, const uint64_t *first, uint64_t *states, uint64_t *last, void *workspace, size_t workspace_bytes,
                                spin_stream stream)
{
    return run_states<uint64_t>(s, rows, columns, reverse, x, y, C, t, first, states, last, workspace, workspace_bytes, stream);
}

size_t spin_linattn_states_workspace_bytes(const spin_linattn *s, int rows, int columns)
{
    return states_workspace(s, rows, columns, sizeof(uint64_t));
}

spin_status spin_linattn_outputs(const spin_linattn *s, int rows, int columns, int reverse, int transposed, const spin_masked *P, const spin_masked *y,
                                 const spin_masked *x, const spin_masked *S, const uint64_t *C, const spin_tuple *t, uint64_t *out, spin_stream stream)
{
    return run_outputs<uint64_t>(s, rows, columns, reverse, transposed, P, y, x, S, C, t, out, stream);
}

spin_status spin_linattn_step(const spin_linattn *s, int rows, int columns, const uint64_t *S, const spin_masked *q, const spin_masked *k, const spin_masked *v,
                              const uint64_t *S_mask, const uint64_t *CS, const spin_tuple *tS, const uint64_t *CO, const spin_tuple *tO, uint64_t *S_out,
                              uint64_t *out, spin_stream stream)
{
    return run_step<uint64_t>(s, rows, columns, S, q, k, v, S_mask, CS, tS, CO, tO, S_out, out, stream);
}

spin_status spin_layernorm(const spin_norm *s, int iterations, uint64_t offset, uint64_t slope, uint64_t eps, const uint64_t *x, const spin_masked *gamma,
                           const uint64_t *beta, const uint64_t *mask_x, const uint64_t *mask_xhat, const uint64_t *C1, const spin_tuple *t1, const uint64_t *C2,
                           const spin_tuple *t2, const uint64_t *row_words, uint64_t *out, uint64_t *xhat, uint64_t *rstd, spin_stream stream)
{
    return run_norm<uint64_t>(s, iterations, offset, slope, eps, x, gamma, beta, mask_x, mask_xhat, C1, t1, C2, t2, row_words, out, xhat, rstd, stream);
}

spin_status spin_layernorm_grad(const spin_norm *s, const spin_masked *dy, const spin_masked *xhat, const uint64_t *rstd, const spin_masked *gamma,
                                const uint64_t *mask_g, const uint64_t *C1, const spin_tuple *t1, const uint64_t *C2, const spin_tuple *t2,
                                const uint64_t *row_words, const uint64_t *column_words, uint64_t *dx, uint64_t *dgamma, uint64_t *dbeta, void *workspace,
                                size_t workspace_bytes, spin_stream stream)
{
    return run_norm_grad<uint64_t>(s, dy, xhat, rstd, gamma, mask_g, C1, t1, C2, t2, row_words, column_words, dx, dgamma, dbeta, workspace, workspace_bytes, stream);
}

size_t spin_layernorm_grad_workspace_bytes(const spin_norm *s)
{
    return norm_grad_workspace(s, sizeof(uint64_t));
}

spin_status spin32_linattn_scores(const spin_linattn *s, int dim, const spin_masked *x, const spin_masked *y, const uint32_t *C, const spin_tuple *t, uint32_t *out,
                                  spin_stream stream)
{
    return run_scores<uint32_t>(s, dim, x, y, C, t, out, stream);
}

spin_status spin32_linattn_states(const spin_linattn *s, int rows, int columns, int reverse, const spin_masked *x, const spin_masked *y, const uint32_t *C,
                                  const spin_tuple *t, const uint32_t *first, uint32_t *states, uint32_t *last, void *workspace, size_t workspace_bytes,
                                  spin_stream stream)
{
    return run_states<uint32_t>(s, rows, columns, reverse, x, y, C, t, first, states, last, workspace, workspace_bytes, stream);
}

size_t spin32_linattn_states_workspace_bytes(const spin_linattn *s, int rows, int columns)
{
    return states_workspace(s, rows, columns, sizeof(uint32_t));
}

spin_status spin32_linattn_outputs(const spin_linattn *s, int rows, int columns, int reverse, int transposed, const spin_masked *P, const spin_masked *y,
                                   const spin_masked *x, const spin_masked *S, const uint32_t *C, const spin_tuple *t, uint32_t *out, spin_stream stream)
{
    return run_outputs<uint32_t>(s, rows, columns, reverse, transposed, P, y, x, S, C, t, out, stream);
}

spin_status spin32_linattn_step(const spin_linattn *s, int rows, int columns, const uint32_t *S, const spin_masked *q, const spin_masked *k, const spin_masked *v,
                                const uint32_t *S_mask, const uint32_t *CS, const spin_tuple *tS, const uint32_t *CO, const spin_tuple *tO, uint32_t *S_out,
                                uint32_t *out, spin_stream stream)
{
    return run_step<uint32_t>(s, rows, columns, S, q, k, v, S_mask, CS, tS, CO, tO, S_out, out, stream);
}

spin_status spin32_layernorm(const spin_norm *s, int iterations, uint32_t offset, uint32_t slope, uint32_t eps, const uint32_t *x, const spin_masked *gamma,
                             const uint32_t *beta, const uint32_t *mask_x, const uint32_t *mask_xhat, const uint32_t *C1, const spin_tuple *t1, const uint32_t *C2,
                             const spin_tuple *t2, const uint32_t *row_words, uint32_t *out, uint32_t *xhat, uint32_t *rstd, spin_stream stream)
{
    return run_norm<uint32_t>(s, iterations, offset, slope, eps, x, gamma, beta, mask_x, mask_xhat, C1, t1, C2, t2, row_words, out, xhat, rstd, stream);
}

spin_status spin32_layernorm_grad(const spin_norm *s, const spin_masked *dy, const spin_masked *xhat, const uint32_t *rstd, const spin_masked *gamma,
                                  const uint32_t *mask_g, const uint32_t *C1, const spin_tuple *t1, const uint32_t *C2, const spin_tuple *t2,
                                  const uint32_t *row_words, const uint32_t *column_words, uint32_t *dx, uint32_t *dgamma, uint32_t *dbeta, void *workspace,
                                  size_t workspace_bytes, spin_stream stream)
{
    return run_norm_grad<uint32_t>(s, dy, xhat, rstd, gamma, mask_g, C1, t1, C2, t2, row_words, column_words, dx, dgamma, dbeta, workspace, workspace_bytes, stream);
}

size_t spin32_layernorm_grad_workspace_bytes(const spin_norm *s)
{
    return norm_grad_workspace(s, sizeof(uint32_t));
}

}  // extern "C"
