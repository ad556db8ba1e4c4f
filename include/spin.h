/*
 * spin.h -- C ABI of the MI355X (gfx950) library for the per-party local work
 * of additive-secret-sharing multiplication over the ring Z_2^64:
 * sharing, opening, the Beaver-triple share update for matrix and elementwise
 * products, and fixed-point truncation (spin_share, spin_open,
 * spin_beaver_matmul, spin_beaver_mul, spin_trunc).  Further down: the same
 * over Z_2^32 and Z_2^128 (spin32_*, spin128_*), binary shares (spin_b*),
 * a public linear combination with fused truncation, and for generating token by
 * token a paged cache of shared keys and values, the attention products of a tree
 * of drafted tokens over it and a relative position bias (spin_cache_*,
 * spin_relbias_*), and for blocks without softmax linear attention with a decay
 * and layer norm, forward and backward (spin_linattn_*, spin_layernorm*).
 * Measurement aids (per-kernel event timing, an MFMA rate probe) are declared
 * in spin_bench.h.
 *
 * Conventions that hold for every entry point
 * -------------------------------------------
 *  - Ring elements are uint64_t unless a section says otherwise; all arithmetic
 *    wraps mod 2^64.  Read as signed they are the range [-2^63, 2^63-1] of
 *    Section 4.1 (Notations).
 *  - All n parties live on the one GPU.  Share tensors are party-major:
 *    T[i] is party i's share, contiguous, so a tensor of `count` elements is
 *    laid out [n][count].  Party 0 is the paper's party 1: it holds residual
 *    shares and adds every public term.
 *  - Every data pointer is a DEVICE pointer, 16-byte aligned (the widest vector
 *    access any kernel makes; workspaces 256-byte), owned by the caller; the
 *    entry points of this header never allocate, free or keep a pointer.
 *    Buffers must not overlap unless a function says an output may alias an
 *    input.
 *  - Calls are asynchronous: work is enqueued on `stream` (a hipStream_t; NULL
 *    is the default stream) and the function returns without synchronising.
 *  - Errors are return codes.  Arguments are validated before anything is
 *    launched, so SPIN_EINVAL / SPIN_ERANGE / SPIN_EWORKSPACE never leave
 *    partial work behind.  Nothing throws across the boundary.
 *  - 1 <= n <= SPIN_MAX_PARTIES.
 */
#ifndef SPIN_H
#define SPIN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SPIN_MAX_PARTIES 8

typedef enum {
    SPIN_OK = 0,
    SPIN_EINVAL = 1,     /* null pointer, n out of range, non-positive size, f out of range, misaligned */
    SPIN_ERANGE = 2,     /* a size whose element count or padded extent does not fit the index types  */
    SPIN_EWORKSPACE = 3, /* workspace missing or smaller than spin_beaver_matmul_workspace_bytes()    */
    SPIN_EHIP = 4        /* a launch failed; spin_last_hip_error() holds the runtime's message        */
} spin_status;

/* The `path` argument of the matmul calls.  It is passed as an int so that a value outside the
 * enumeration is refused with SPIN_EINVAL instead of being undefined behaviour on the library's side. */
typedef enum {
    SPIN_GEMM_LIMB_MFMA = 0, /* exact 8-bit-limb decomposition on int8 MFMA, int32 accumulation */
    SPIN_GEMM_VALU = 1       /* 64-bit multiply-add on the vector ALU (baseline)                */
} spin_gemm_path;

typedef void *spin_stream; /* hipStream_t */

/* Synthetic randomness.  The paper's parties draw masks and triples in an
 * OT-based offline phase (Section 4.2); here a stateless counter generator
 * stands in:  mix(z) is the SplitMix64 finaliser, absorb(h,v) =
 * mix(h + (v+1)*0x9E3779B97F4A7C15), and
 *   rand64(seed, stream_id, party, idx) =
 *       absorb(absorb(absorb(absorb(0, seed), stream_id), party), idx).
 * out[k] = rand64(seed, stream_id, party, first_idx + k), k < count.          */
spin_status spin_random(uint64_t *out, size_t count, uint64_t seed, uint64_t stream_id,
                        uint64_t party, uint64_t first_idx, spin_stream stream);

/* n-out-of-n arithmetic sharing (Section 4.1): x = sum_i x_i.
 * shares[i][k] = rand64(seed, stream_id, i, k) for i >= 1 and
 * shares[0][k] = x[k] - sum_{i>=1} shares[i][k].
 * x: [count] in; shares: [n][count] out.                                      */
spin_status spin_share(const uint64_t *x, size_t count, int n, uint64_t seed, uint64_t stream_id,
                       uint64_t *shares, spin_stream stream);

/* Opening (Section 4.1 reconstruction; with a mask, the E = X - A opening of
 * Section 4.3 Multiplication): out[k] = sum_i (shares[i][k] - mask[i][k]).
 * The network exchange of the paper is a reduction over the party axis here.
 * shares, mask: [n][count] in (mask may be NULL = zeros); out: [count].       */
spin_status spin_open(const uint64_t *shares, const uint64_t *mask, size_t count, int n,
                      uint64_t *out, spin_stream stream);

/* Online phase of matrix multiplication with a matrix Beaver triple
 * (Section 4.3 Multiplication; batched as in Section 7.4).  For every batch
 * entry: E = sum_i (X_i - A_i), F = sum_i (Y_i - B_i), then
 *     Z_i = C_i + E.B_i + A_i.F   and party 0 adds E.F once.
 * Row-major operands: X, A [n][batch][M][K]; Y, B [n][batch][K][N];
 * C, Z [n][batch][M][N].  Z may alias C.  For a right operand that is stored
 * transposed (Q.K^T) see spin_beaver_matmul_nt.
 * workspace: device scratch of at least
 * spin_beaver_matmul_workspace_bytes(n,batch,M,N,K,path) bytes, 256-byte
 * aligned; its contents are overwritten.  Any K is accepted: the limb path
 * splits the inner dimension so that no int32 partial sum can overflow.       */
spin_status spin_beaver_matmul(int n, int batch, int M, int N, int K,
                               const uint64_t *X, const uint64_t *Y,
                               const uint64_t *A, const uint64_t *B, const uint64_t *C,
                               uint64_t *Z, int path,
                               void *workspace, size_t workspace_bytes, spin_stream stream);

/* The same with the right operands stored transposed, the layout of K in the attention product
 * Q.K^T (Section 7.4 multiplies such pairs head by head): Yt, Bt are [n][batch][N][K] row-major and
 * Z = X . Yt^T.  Everything else, including the workspace size, as for spin_beaver_matmul; the
 * transposition costs no pass over memory (the right-hand fragments are read along rows).       */
spin_status spin_beaver_matmul_nt(int n, int batch, int M, int N, int K,
                                  const uint64_t *X, const uint64_t *Yt,
                                  const uint64_t *A, const uint64_t *Bt, const uint64_t *C,
                                  uint64_t *Z, int path,
                                  void *workspace, size_t workspace_bytes, spin_stream stream);

/* An array of Beaver matmuls of different shapes in one call (Section 7.4's PMatMul takes arrays of
 * matrices and multiplies them in parallel; products of one shape go into the batch dimension of a group,
 * different shapes into different groups).  desc: HOST array of `groups` descriptors, read before the call
 * returns; every group is what spin_beaver_matmul (y_transposed == 0) or spin_beaver_matmul_nt (!= 0) would
 * be given, with the common party count n.  On the limb path the groups share launches -- the operand packs
 * of all groups first, then their GEMMs, a handful of launches whatever the number of groups -- and every
 * group has its own part of the workspace, so the workspace must hold the SUM of the groups' needs
 * (the baseline path enqueues the groups one after another and needs the largest):
 * spin_beaver_matmul_grouped_workspace_bytes(n, groups, desc, path), 0 if a descriptor is invalid.  All
 * descriptors are validated before the first launch.  The Z of different groups must not overlap (their
 * GEMMs run concurrently).  1 <= groups <= SPIN_MAX_GROUPS.                                       */
#define SPIN_MAX_GROUPS 64
typedef struct {
    int batch, M, N, K;
    const uint64_t *X, *Y, *A, *B, *C;
    uint64_t *Z;
    int y_transposed;
} spin_matmul_group;
spin_status spin_beaver_matmul_grouped(int n, int groups, const spin_matmul_group *desc, int path,
                                       void *workspace, size_t workspace_bytes, spin_stream stream);
size_t spin_beaver_matmul_grouped_workspace_bytes(int n, int groups, const spin_matmul_group *desc,
                                                  int path);

/* Bytes of workspace spin_beaver_matmul needs; 0 if the arguments are invalid. */
size_t spin_beaver_matmul_workspace_bytes(int n, int batch, int M, int N, int K, int path);

/* Bytes of workspace with which spin_beaver_matmul (and _nt) is fastest; never less than it needs, 0 if the
 * arguments are invalid.  Large products run on residues modulo 18 pairwise coprime numbers of at most eight bits (36 for
 * spin128_beaver_matmul), whose operand copies take 18 (36) bytes an element; with less than this workspace such a product
 * is computed in more blocks, or by the digit kernels.  The result is the same words either way.                  */
size_t spin_beaver_matmul_preferred_workspace_bytes(int n, int batch, int M, int N, int K, int path);

/* spin_beaver_matmul for callers that cannot allocate device memory, and so cannot bring a workspace:
 * code running under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
 * operands, result and checks as spin_beaver_matmul; the workspace is an array of
 * SPIN_STATIC_WORKSPACE_BYTES inside the library's device image (each GPU the library runs on holds its
 * copy until the process ends).  The call allocates and frees nothing -- no device or host memory, no
 * event objects (per-kernel timing is not recorded for it) -- and only enqueues kernels on `stream`.
 * Returns SPIN_EWORKSPACE, before anything is launched, when
 * spin_beaver_matmul_workspace_bytes(n, batch, M, N, K, path) exceeds SPIN_STATIC_WORKSPACE_BYTES.
 * All calls on one GPU share that GPU's array: two calls whose kernels may overlap in time (different
 * streams, or two replays of graphs that contain it) race and give wrong results; calls on one stream,
 * one after another, are safe.  The first call on a device looks the array's address up.          */
#define SPIN_STATIC_WORKSPACE_BYTES (64u << 20)
spin_status spin_beaver_matmul_static(int n, int batch, int M, int N, int K,
                                      const uint64_t *X, const uint64_t *Y,
                                      const uint64_t *A, const uint64_t *B, const uint64_t *C,
                                      uint64_t *Z, int path, spin_stream stream);

/* Online phase of elementwise multiplication with scalar triples (Section 4.3;
 * the "batch multiplication" of Section 7.3):
 *     e = sum_i (x_i - a_i), f = sum_i (y_i - b_i),
 *     z_i = c_i + e*b_i + a_i*f  (+ e*f for i = 0).
 * x, y, a, b, c: [n][count] in; z: [n][count] out; z may alias any input.     */
spin_status spin_beaver_mul(int n, size_t count,
                            const uint64_t *x, const uint64_t *y,
                            const uint64_t *a, const uint64_t *b, const uint64_t *c,
                            uint64_t *z, spin_stream stream);

/* The same with one factor tiled, the batch multiplication E * R of Section 7.3 in which the smaller
 * array is repeated along one axis up to the size of the other (and its downsized form R * V).  The
 * large operands y, b, c and the result z are [n][outer][mid][inner]; the small factor x and its mask a
 * are [n][outer][mid] when over_inner != 0 (one factor per row, repeated along inner) and
 * [n][outer][inner] when over_inner == 0 (one factor per column, repeated along mid).  With xt, at the
 * tiled arrays, z equals spin_beaver_mul(n, outer*mid*inner, xt, y, at, b, c); the triple satisfies
 * sum_i c_i = (tiled sum_i a_i) * (sum_i b_i).  The tiled arrays are never formed: 4n instead of 6n
 * words move per element.  z may alias y, b or c.                                                   */
spin_status spin_beaver_mul_bcast(int n, size_t outer, size_t mid, size_t inner, int over_inner,
                                  const uint64_t *x, const uint64_t *y,
                                  const uint64_t *a, const uint64_t *b, const uint64_t *c,
                                  uint64_t *z, spin_stream stream);

/* Signed probabilistic truncation by f bits (Section 4.4 Truncation):
 * Truncate(x,f) = UnsignedTruncate(x + 2^62, 64, f) - 2^(62-f), correct up to
 * one unit for x in [-2^62, 2^62-1] and undefined (not an error) outside.
 * The dealer tuple per element is a random ring element r with sharings of r,
 * of r_top = bits f..62 of r and of r_msb = bit 63 of r.  Steps:
 *     c = sum_i (x_i + r_i) + 2^62;  c_msb = c >> 63;  c' = bits f..62 of c;
 *     b_i   = r_msb_i + [i=0] c_msb - 2 c_msb r_msb_i;
 *     out_i = [i=0] c' - r_top_i + 2^(63-f) b_i - [i=0] 2^(62-f).
 * x, r, r_top, r_msb: [n][count] in; out: [n][count], may alias x.
 * 1 <= f <= 61.                                                               */
spin_status spin_trunc(int n, size_t count, int f, const uint64_t *x,
                       const uint64_t *r, const uint64_t *r_top, const uint64_t *r_msb,
                       uint64_t *out, spin_stream stream);

/* Fixed-point multiplication in one pass: spin_beaver_mul followed by spin_trunc of its result
 * (a product carries twice the precision, Section 4.3; Truncate brings it back, Section 4.4), with
 * the product shares kept in registers instead of written and read again.  out equals
 * spin_trunc(n, count, f, z, r, r_top, r_msb) of z = spin_beaver_mul(n, count, x, y, a, b, c) word
 * for word.  Shapes and aliasing as for those two calls; out may alias any input.  1 <= f <= 61. */
spin_status spin_beaver_mul_trunc(int n, size_t count, int f,
                                  const uint64_t *x, const uint64_t *y,
                                  const uint64_t *a, const uint64_t *b, const uint64_t *c,
                                  const uint64_t *r, const uint64_t *r_top, const uint64_t *r_msb,
                                  uint64_t *out, spin_stream stream);

/* Public-coefficient linear combination followed by one truncation: the local
 * part of Scale and Add (Section 4.3) and the single deferred truncation of
 * polynomial evaluation (Section 4.4, Polynomial evaluation; the fused
 * (p+6)-bit truncation of Section 7.2, Eq. (4)):
 *     y_i   = sum_j coef[j] * in[j]_i  +  [i=0] constant          (local)
 *     out   = f > 0 ? Truncate(y, f) : y                           (as spin_trunc)
 * in:   HOST array of `terms` DEVICE pointers, each a [n][count] share tensor;
 * coef: HOST array of `terms` public ring coefficients; 1 <= terms <= SPIN_MAX_TERMS.
 * r, r_top, r_msb: truncation tuple as in spin_trunc (ignored, may be NULL,
 * when f = 0).  out: [n][count], may alias any input.  0 <= f <= 61.          */
#define SPIN_MAX_TERMS 8
spin_status spin_lincomb_trunc(int n, size_t count, int terms, const uint64_t *const *in,
                               const uint64_t *coef, uint64_t constant, int f,
                               const uint64_t *r, const uint64_t *r_top, const uint64_t *r_msb,
                               uint64_t *out, spin_stream stream);

/* The completed-square quartic of Section 7.2, Eq. (4), in one pass, word for word what these calls give:
 *     u   = x + [i=0] t3                                   (spin_lincomb_trunc, f = 0)
 *     v   = Truncate(u * u, f[0]) + [i=0] t2               (spin_beaver_mul_trunc; spin_lincomb_trunc, f = 0)
 *     out = Truncate(v * v + lin x + [i=0] t0, f[1])       (spin_beaver_mul; spin_lincomb_trunc)
 * triples, tuples: HOST arrays of six DEVICE pointers, a, b, c of the first square, then of the second; r, r_top, r_msb
 * of the first truncation, then of the second; f: HOST array of two.  All tensors [n][count]; out may alias any input.
 * 1 <= f[k] <= 61.                                                                                                  */
spin_status spin_completed_square_trunc(int n, size_t count, const uint64_t *x, uint64_t t3, uint64_t t2, uint64_t lin,
                                        uint64_t t0, const uint64_t *const *triples, const uint64_t *const *tuples,
                                        const int *f, uint64_t *out, spin_stream stream);

/* Binary sharing (Section 4.1): 64 independent bit positions per word,
 * x = XOR_i x_i.  XOR of sharings is local (Section 4.3 Addition); AND consumes
 * a bit triple (a, b, c = a AND b) and is the GF(2) form of the Beaver update.
 *   spin_bshare:     shares[i][k] = rand64(seed, stream_id, i, k) for i >= 1,
 *                    shares[0][k] = x[k] XOR (XOR of the others).
 *   spin_bopen:      out[k] = XOR_i (shares[i][k] XOR mask[i][k]); mask may be NULL.
 *   spin_beaver_and: e = XOR_i (x_i ^ a_i), f = XOR_i (y_i ^ b_i),
 *                    z_i = c_i ^ (e & b_i) ^ (a_i & f)  (^ (e & f) for i = 0).
 * Layouts as for the arithmetic calls: [n][count] words; z may alias an input. */
spin_status spin_bshare(const uint64_t *x, size_t count, int n, uint64_t seed, uint64_t stream_id,
                        uint64_t *shares, spin_stream stream);
spin_status spin_bopen(const uint64_t *shares, const uint64_t *mask, size_t count, int n,
                       uint64_t *out, spin_stream stream);
spin_status spin_beaver_and(int n, size_t count,
                            const uint64_t *x, const uint64_t *y,
                            const uint64_t *a, const uint64_t *b, const uint64_t *c,
                            uint64_t *z, spin_stream stream);

/* The same calls over the ring Z_2^128 (the paper's second ring width, Section 6: "64-bit or
 * 128-bit"; its own kernels multiply __int128, Section 6.1).  A ring element is 16 bytes,
 * little-endian: two uint64_t words, low word first (the layout of unsigned __int128).  Pointers
 * are passed as uint64_t* to those words; `count` and the matrix dimensions count ring elements;
 * tensors are party-major as before.  A 128-bit generator word is the pair of 64-bit generator
 * outputs at indices 2k (low) and 2k+1 (high).  spin128_trunc: Truncate(x,f) =
 * UnsignedTruncate(x + 2^126, 128, f) - 2^(126-f), tuple fields r_top = bits f..126 and
 * r_msb = bit 127 of r, 1 <= f <= 125.  Everything else as documented at the 64-bit call.       */
spin_status spin128_share(const uint64_t *x, size_t count, int n, uint64_t seed, uint64_t stream_id,
                          uint64_t *shares, spin_stream stream);
spin_status spin128_open(const uint64_t *shares, const uint64_t *mask, size_t count, int n,
                         uint64_t *out, spin_stream stream);
spin_status spin128_beaver_matmul(int n, int batch, int M, int N, int K,
                                  const uint64_t *X, const uint64_t *Y,
                                  const uint64_t *A, const uint64_t *B, const uint64_t *C,
                                  uint64_t *Z, int path,
                                  void *workspace, size_t workspace_bytes, spin_stream stream);
size_t spin128_beaver_matmul_workspace_bytes(int n, int batch, int M, int N, int K, int path);
size_t spin128_beaver_matmul_preferred_workspace_bytes(int n, int batch, int M, int N, int K, int path);
spin_status spin128_beaver_mul(int n, size_t count,
                               const uint64_t *x, const uint64_t *y,
                               const uint64_t *a, const uint64_t *b, const uint64_t *c,
                               uint64_t *z, spin_stream stream);
spin_status spin128_trunc(int n, size_t count, int f, const uint64_t *x,
                          const uint64_t *r, const uint64_t *r_top, const uint64_t *r_msb,
                          uint64_t *out, spin_stream stream);

/* The same calls over the ring Z_2^32, the Fixed32 representation of Section 7.1 (mixing bit
 * lengths): steps that do not need 64 bits run on 32-bit shares at half the bytes.  Ring elements
 * are uint32_t, tensors party-major as before.  A 32-bit generator word is the low half of
 * rand64 at the same index.  spin32_trunc: Truncate(x,f) = UnsignedTruncate(x + 2^30, 32, f) -
 * 2^(30-f), tuple fields r_top = bits f..30 and r_msb = bit 31 of r, 1 <= f <= 29.  The limb
 * path of spin32_beaver_matmul uses four digits (10 digit pairs) and never splits the inner
 * dimension.  Everything else as documented at the 64-bit call.
 *
 * spin_cast_64_to_32 is the local Fixed64 -> Fixed32 cast of Section 7.1: out[k] = low 32 bits
 * of in[k], applied by every party to its own share (pass all n*count share words at once);
 * the opened value is preserved while it lies in [-2^31, 2^31).  in: [count] uint64_t,
 * out: [count] uint32_t, must not overlap.                                                      */
spin_status spin32_share(const uint32_t *x, size_t count, int n, uint64_t seed, uint64_t stream_id,
                         uint32_t *shares, spin_stream stream);
spin_status spin32_open(const uint32_t *shares, const uint32_t *mask, size_t count, int n,
                        uint32_t *out, spin_stream stream);
spin_status spin32_beaver_matmul(int n, int batch, int M, int N, int K,
                                 const uint32_t *X, const uint32_t *Y,
                                 const uint32_t *A, const uint32_t *B, const uint32_t *C,
                                 uint32_t *Z, int path,
                                 void *workspace, size_t workspace_bytes, spin_stream stream);
size_t spin32_beaver_matmul_workspace_bytes(int n, int batch, int M, int N, int K, int path);
/* With it large products run by Strassen's recursion, in fewer multiplications; the same words with less.           */
size_t spin32_beaver_matmul_preferred_workspace_bytes(int n, int batch, int M, int N, int K, int path);
spin_status spin32_beaver_mul(int n, size_t count,
                              const uint32_t *x, const uint32_t *y,
                              const uint32_t *a, const uint32_t *b, const uint32_t *c,
                              uint32_t *z, spin_stream stream);
spin_status spin32_trunc(int n, size_t count, int f, const uint32_t *x,
                         const uint32_t *r, const uint32_t *r_top, const uint32_t *r_msb,
                         uint32_t *out, spin_stream stream);
spin_status spin_cast_64_to_32(const uint64_t *in, size_t count, uint32_t *out, spin_stream stream);

/* ---- A paged cache of shared keys and values, and what reads it --------------------------------------
 * Generating token by token multiplies the same K and V again in every step.  A row of K or V is therefore
 * opened once, against a mask b dealt for it, and kept: F = sum_i (x_i - b_i) is public, and every later product
 * with that row needs only its own fresh mask of the other factor (Section 4.3's update with F fixed).
 * A cached row takes n + 1 words an element: slot 0 holds F, slot 1 holds b_0 + F (which folds party 0's public term E.F
 * into its product) and slot 1 + i holds b_i.  Slots 1 to n are themselves a sharing of the row.
 *
 * Rows live in pages of page_tokens positions; table[b][j] is the page that holds positions j * page_tokens and on of
 * sequence b.  Sequences may share pages (a fork) as long as none of them writes there.  table, contexts, counts and page lists are
 * DEVICE arrays of int32_t (4-byte aligned); what is wrong in them cannot be refused by the call and never makes a kernel
 * leave the buffers: an entry outside [0, pages) is a page that is not there, whose rows are not written and not visible, and
 * neither are positions past the end of the table.  Entry points spin32_* take the same structure with pools of uint32_t.        */
typedef struct {
    int n;                 /* parties                                                                            */
    int pages;             /* pages of each pool                                                                 */
    int heads;             /* cached heads                                                                       */
    int page_tokens;       /* positions a page: a power of two, 16 to 4096                                       */
    int dim;               /* elements of a head's row: a multiple of 8, 8 to 256                                */
    void *K, *V;           /* pools, each [n + 1][pages][heads][page_tokens][dim] ring elements                  */
    int batch;             /* sequences                                                                          */
    int table_pages;       /* entries of a sequence in the table                                                 */
    const int32_t *table;  /* [batch][table_pages]                                                               */
} spin_cache;

/* A learned relative position bias: one shared word a head and bucket, added to scores of precision f after truncation.
 * bucket_of[d + reach] is the bucket of distance d = key position - query position, distances beyond reach count as reach;
 * entries outside [0, buckets) add nothing.                                                                                  */
typedef struct {
    int buckets;               /* 1 to 1024                                                                      */
    int reach;                 /* 0 to 65535                                                                     */
    const int32_t *bucket_of;  /* device, [2 * reach + 1]                                                        */
    const void *table;         /* device, shares [n][heads][buckets] of ring elements                            */
} spin_relbias;

/* Opens new rows of keys and values and writes them into their pages: row s < count[b] of sequence b goes to position
 * start[b] + s.  Kx, Vx: shares, Kb, Vb: their masks, all [n][batch][heads][rows][dim].  count: [batch], or NULL for `rows` each.
 * Rows whose page is not there, or whose position is negative, are left out.                                              */
spin_status spin_cache_append(const spin_cache *c, int rows, const int32_t *start, const int32_t *count,
                              const uint64_t *Kx, const uint64_t *Kb, const uint64_t *Vx, const uint64_t *Vb, spin_stream stream);

/* Copies whole pages of both pools, src[p] to dst[p] for p < pairs (a fork about to be written, a pool being compacted).  The
 * table is not looked at.  Pairs with a page that is not there are left out; no page may be written twice, or read and written, in one call.  */
spin_status spin_cache_copy(const spin_cache *c, int pairs, const int32_t *src, const int32_t *dst, spin_stream stream);

/* Keeps the accepted ones of `nodes` drafted tokens: the row at position context[b] + kept[b][j] moves to context[b] + j, for
 * j < kept_count[b], in both pools.  kept: [batch][nodes], strictly ascending in every sequence.  Nothing moves where
 * context[b] < 0; indices outside [0, nodes) are left out.  1 <= nodes <= 64.                                                              */
#define SPIN_MAX_NODES 64
spin_status spin_cache_compact(const spin_cache *c, int nodes, const int32_t *context, const int32_t *kept,
                               const int32_t *kept_count, spin_stream stream);

/* Scores of `nodes` new tokens a sequence over the cache.  The tokens, a single one or a tree of drafted ones, stand
 * in the cache at positions context[b] .. context[b] + nodes - 1; node m sees all positions below context[b], and drafted node j where
 * bit j of tree[b][m] is set (tree NULL: the nodes up to itself).  A sequence with context[b] < 0 sees nothing.  For every
 * query head h (cached head h / (heads / c->heads)) and node m, with E = sum_i (Q_i - A_i), at every visible position t < columns:
 *     Z_i = C_i + E . slot(1 + i)[t] + A_i . slot(0)[t],     out = f > 0 ? Truncate(Z, f) : Z,     out_i += bias_i[h][bucket]
 * and everywhere else the public constant `masked` (party 0 holds it, the others 0).
 * Q, A: [n][batch][heads][nodes][dim]; C, r, r_top, r_msb, out: [n][batch][heads][nodes][columns].  Triples satisfy sum_i C_i = (sum A_i)(sum b_i)
 * with the masks that the rows were opened with.  tuple pointers are ignored when f = 0; out may alias C, and r, r_top or r_msb.
 * bias may be NULL (depth is then not looked at); with it depth ([batch][nodes] or NULL: 0, 1, ..) is the distance of a node behind the context: its position is
 * context[b] + depth[b][m] as query and as key.  heads is a multiple of c->heads; c->V is not looked at.  0 <= f <= 61.  Refused (SPIN_ERANGE), here
 * and below, are more than 2^24 columns and more than 65535 of heads * nodes, of batch * c->heads or, if f = 0, of batch * c->n (in spin_cache_values
 * over more than three columns, which refuses more than 32767 cached heads of more than 128 64-bit words as well).                    */
spin_status spin_cache_scores(const spin_cache *c, int heads, int nodes, int columns, int f, const int32_t *context,
                              const uint64_t *tree, const uint64_t *Q, const uint64_t *A, const uint64_t *C,
                              const uint64_t *r, const uint64_t *r_top, const uint64_t *r_msb, uint64_t masked,
                              const spin_relbias *bias, const int32_t *depth, uint64_t *out, spin_stream stream);

/* The weighted sums of cached values: with E = sum_i (P_i - A_i), over the positions t < columns that node m sees (as above),
 *     Z_i = C_i + sum_t E[t] slot(1 + i)[t] + A_i[t] slot(0)[t],     out = f > 0 ? Truncate(Z, f) : Z.
 * P and A count as zero where nothing is seen, whatever they hold there; a node that sees nothing gives Z = C.
 * P, A: [n][batch][heads][nodes][columns]; C, r, r_top, r_msb, out: [n][batch][heads][nodes][dim].  c->K is not looked at.
 * workspace: device scratch of spin_cache_values_workspace_bytes() bytes (0 if the arguments are invalid), 256-byte aligned.   */
spin_status spin_cache_values(const spin_cache *c, int heads, int nodes, int columns, int f, const int32_t *context,
                              const uint64_t *tree, const uint64_t *P, const uint64_t *A, const uint64_t *C,
                              const uint64_t *r, const uint64_t *r_top, const uint64_t *r_msb, uint64_t *out,
                              void *workspace, size_t workspace_bytes, spin_stream stream);
size_t spin_cache_values_workspace_bytes(const spin_cache *c, int heads, int nodes, int columns);

/* Whole matrices of scores: truncation, relative position bias and mask in one pass.  For x [n][batch][heads][Q][K],
 *     out = f > 0 ? Truncate(x, f) : x,     out_i += bias_i[h][bucket of k - (q + first)]
 * where k < lengths[b] (lengths NULL: everywhere) and, if causal != 0, k <= q + first; elsewhere the public constant `masked`.
 * out may alias any input but the bias.  0 <= f <= 61.                                                                       */
spin_status spin_relbias_trunc(int n, int batch, int heads, int Q, int K, int first, int causal, const int32_t *lengths, int f,
                               const uint64_t *x, const uint64_t *r, const uint64_t *r_top, const uint64_t *r_msb,
                               uint64_t masked, const spin_relbias *bias, uint64_t *out, spin_stream stream);

/* The gradient of that bias: grad_i[h][b] = sum of dS_i[..][h][q][k] over the batch and the positions that are there (as above) and have
 * bucket b.  dS: [n][batch][heads][Q][K]; grad: [n][heads][buckets], overwritten.  bias->table is not looked at.  (The gradient with
 * respect to x is dS where the position is there.)                                                                            */
spin_status spin_relbias_grad(int n, int batch, int heads, int Q, int K, int first, int causal, const int32_t *lengths,
                              const uint64_t *dS, const spin_relbias *bias, uint64_t *grad, spin_stream stream);

/* The same over Z_2^32 (pools and tables of uint32_t; f <= 29).                                                               */
spin_status spin32_cache_append(const spin_cache *c, int rows, const int32_t *start, const int32_t *count,
                                const uint32_t *Kx, const uint32_t *Kb, const uint32_t *Vx, const uint32_t *Vb, spin_stream stream);
spin_status spin32_cache_copy(const spin_cache *c, int pairs, const int32_t *src, const int32_t *dst, spin_stream stream);
spin_status spin32_cache_compact(const spin_cache *c, int nodes, const int32_t *context, const int32_t *kept,
                                 const int32_t *kept_count, spin_stream stream);
spin_status spin32_cache_scores(const spin_cache *c, int heads, int nodes, int columns, int f, const int32_t *context,
                                const uint64_t *tree, const uint32_t *Q, const uint32_t *A, const uint32_t *C,
                                const uint32_t *r, const uint32_t *r_top, const uint32_t *r_msb, uint32_t masked,
                                const spin_relbias *bias, const int32_t *depth, uint32_t *out, spin_stream stream);
spin_status spin32_cache_values(const spin_cache *c, int heads, int nodes, int columns, int f, const int32_t *context,
                                const uint64_t *tree, const uint32_t *P, const uint32_t *A, const uint32_t *C,
                                const uint32_t *r, const uint32_t *r_top, const uint32_t *r_msb, uint32_t *out,
                                void *workspace, size_t workspace_bytes, spin_stream stream);
size_t spin32_cache_values_workspace_bytes(const spin_cache *c, int heads, int nodes, int columns);
spin_status spin32_relbias_trunc(int n, int batch, int heads, int Q, int K, int first, int causal, const int32_t *lengths, int f,
                                 const uint32_t *x, const uint32_t *r, const uint32_t *r_top, const uint32_t *r_msb,
                                 uint32_t masked, const spin_relbias *bias, uint32_t *out, spin_stream stream);
spin_status spin32_relbias_grad(int n, int batch, int heads, int Q, int K, int first, int causal, const int32_t *lengths,
                                const uint32_t *dS, const spin_relbias *bias, uint32_t *grad, spin_stream stream);

/* ---- Linear attention with a decay, and layer norm ----------------------------------------------------
 * What a transformer block without softmax multiplies.  A secret x is opened once, E = sum_i (x_i - a_i) against the mask a dealt for it, and
 * every product with it takes the same E: beside the dealt share C_i of the masks' product party i adds E . b_i + a_i . F, and party 0 E . F.  T(z, f)
 * is the truncation of spin_trunc by f bits, and as there z has to be from -2^62 to 2^62 - 1 (spin32_*: -2^30 to 2^30 - 1): attention's scores, states and results
 * have to stay below 2^(62 - 2f - g) (2^(30 - 2f - g): 64 at f = 9, g = 6).  Entry points spin32_* take the same structures over arrays of uint32_t.  */
typedef struct { const void *value, *mask; } spin_masked;          /* shares and the masks that they are opened against, of one shape */
typedef struct { const void *r, *r_top, *r_msb; } spin_tuple;      /* a truncation tuple, of the result's shape                       */

/* Linear attention takes `tokens` in chunks of `chunk`, the last of them cut; chunks = ceil(tokens / chunk).  A head's decay is public: w[j] is
 * round(lambda^j 2^g).  Sequence b has lengths[b] tokens (at most `tokens`; below zero counts as none), L of which are in the chunk at hand; what stands behind
 * them is not looked at.  lengths is a device array of int32_t (4-byte aligned).                                             */
typedef struct {
    int n, batch, heads;
    int tokens;
    int chunk;               /* 32, 64 or 128                                                                        */
    int f, g;                /* fractional bits of the factors (1 or more) and of w (0 or more), f + g <= 61 (29)    */
    const void *decay;       /* device, [heads][chunk + 1] public ring words w, or NULL: all 1, and g is 0           */
    const int32_t *lengths;  /* [batch], or NULL: all have `tokens`                                                  */
} spin_linattn;

/* Scores within a chunk, for j <= i < L of its tokens:   out[i][j] = T(C[i][j] + w[i - j] x_i . y_j, f + g),   0 elsewhere.
 * x, y: [n][batch][heads][tokens][dim]; C, t, out: [n][batch][heads][chunks][chunk][chunk]; the masks satisfy sum C = w[i - j] (sum a_i . sum b_j).
 * out may alias C or an array of t.  dim here, and rows and columns below, are multiples of 8 from 8 to 256.  Attention takes them of queries and keys; the gradient of
 * the scores, of the result's gradient and the values.                                                                      */
spin_status spin_linattn_scores(const spin_linattn *s, int dim, const spin_masked *x, const spin_masked *y, const uint64_t *C,
                                const spin_tuple *t, uint64_t *out, spin_stream stream);

/* States from chunk to chunk.  states[c] is the state S before chunk c is taken, `last` the one behind all; S begins as `first` (NULL: zeros), and a chunk
 * with L > 0 tokens makes    S <- T(C[c] + 2^f w[L] S + sum_j w[L - 1 - j] x_j (x) y_j, f + g);   one without leaves it.
 * reverse != 0 takes the chunks from the last to the first and weighs by w[j + 1]: the gradient of the states, of queries and the result's gradient; states[c] is then
 * the gradient of what chunk c leaves, `last` that of `first`.  x: [n][batch][heads][tokens][rows]; y: [..][tokens][columns]; C, t, states:
 * [n][batch][heads][chunks][rows][columns]; first, last: [n][batch][heads][rows][columns].  sum C = sum_j w (sum a_j) (x) (sum b_j).  states may alias C or an array
 * of t, last may alias first.  workspace: device scratch of spin_linattn_states_workspace_bytes() bytes (0 if the arguments are invalid), 256-byte aligned.     */
spin_status spin_linattn_states(const spin_linattn *s, int rows, int columns, int reverse, const spin_masked *x, const spin_masked *y,
                                const uint64_t *C, const spin_tuple *t, const uint64_t *first, uint64_t *states, uint64_t *last,
                                void *workspace, size_t workspace_bytes, spin_stream stream);
size_t spin_linattn_states_workspace_bytes(const spin_linattn *s, int rows, int columns);

/* Rows i < L of every chunk:    out_i = T(C_i + 2^g sum_j P_ij y_j + w[i + 1] x_i . S, f + g),    j <= i;   0 behind them.
 * reverse != 0 takes P_ji, i <= j < L, and w[L - 1 - i].  P and its mask count as zero where no score is, whatever they hold there.
 * P: [n][batch][heads][chunks][chunk][chunk]; y, C, t, out: [n][batch][heads][tokens][columns]; x: [..][tokens][rows]; S: [n][batch][heads][chunks][rows][columns],
 * or [columns][rows] last where transposed != 0.  sum C is the same expression in the masks.  out may alias C or an array of t.  With the scores P of (Q, K), dP of (dO, V), the
 * states S of (K, V), their gradients dS of (Q, dO):   O: (P, V, Q, S);   dQ: (dP, K, dO, S transposed);   dK: (dP, Q, V, dS transposed) reverse;
 * dV: (P, dO, K, dS) reverse.                                                                                               */
spin_status spin_linattn_outputs(const spin_linattn *s, int rows, int columns, int reverse, int transposed, const spin_masked *P,
                                 const spin_masked *y, const spin_masked *x, const spin_masked *S, const uint64_t *C, const spin_tuple *t,
                                 uint64_t *out, spin_stream stream);

/* One token of every sequence b with active[b] > 0 (active NULL: all):   S' = T(CS + 2^f w[1] S + w[0] k (x) v, f + g),   out = T(CO + q . S', f),
 * S' being opened against S_mask; sum CS = w[0] (sum a_k) (x) (sum a_v), sum CO = (sum a_q) . (sum S_mask).  Of the others S' = S and out = 0.
 * s->tokens and s->chunk are not looked at, s->lengths is `active`, and decay is [heads][2].
 * q, k: [n][batch][heads][rows]; v, CO, tO, out: [n][batch][heads][columns]; S, S_mask, CS, tS, S_out: [n][batch][heads][rows][columns].  S_out may alias S, S_mask, CS or
 * an array of tS; out CO or an array of tO.                                                                                 */
spin_status spin_linattn_step(const spin_linattn *s, int rows, int columns, const uint64_t *S, const spin_masked *q, const spin_masked *k,
                              const spin_masked *v, const uint64_t *S_mask, const uint64_t *CS, const spin_tuple *tS, const uint64_t *CO,
                              const spin_tuple *tO, uint64_t *S_out, uint64_t *out, spin_stream stream);

/* Layer norm of rows of `dim` words at f fractional bits.  Means are sums times inv = (2^shift + dim / 2) / dim, truncated by `shift`: the larger the
 * more exact, as long as a sum of dim words times inv stays where T is exact: means and variances below 2^(62 - f - shift) (2^(30 - f - shift)).  So do all sums of products, at 2f
 * bits: a row's squares, its g xhat, a column's dy xhat have to stay below 2^(62 - 2f) (2^(30 - 2f): 4096 at f = 9).  dim: 1 to 8192.               */
typedef struct {
    int n, rows, dim;
    int f;                   /* 1 to 60 (28)                                                                         */
    int shift;               /* 1 to 61 (29)                                                                         */
} spin_norm;

/* Forward.  row_words [n][15 (iterations + 1)][rows] holds, a row of words each, what belongs to whole rows; t(k) are its words k, k + 1, k + 2 as a tuple:
 *     mu  = T(inv sum x, shift), t(0);     xc = x - mu, opened against mask_x
 *     q   = word 3 + sum xc^2;   v = T(inv T(q, f), shift) + [party 0] eps, t(4) and t(7);   y = T(2^f offset - slope v, f), t(10);   v is opened against word 13
 *     for each iteration, k = 14, 29, ..:   y is opened against word k,  u = T(word k+1 + y y, f), t(k+2), against word k+5,
 *         h = 3 2^f - T(word k+6 + u v, f), t(k+7), against word k+10,  y <- T(word k+11 + y h, f + 1), t(k+12)
 *     rstd = y, opened against the last word;   xhat = T(C1 + xc rstd, f), t1, opened against mask_xhat;   out = T(C2 + xhat gamma, f) + beta, t2
 * so 1 / sqrt(v) is Newton's, from the public line offset - slope v (ring words at f bits); it converges where that first guess y has 0 < v y^2 < 3.
 * The words 3, k+1, k+6, k+11 and C1, C2 are the dealt shares of the masks' products.  x, mask_x, mask_xhat, C1, C2, t1, t2, out, xhat: [n][rows][dim]; gamma, beta:
 * [n][dim]; rstd: [n][rows].  xhat and rstd, which the gradient takes, may be NULL.  out may alias C2 or an array of t2, xhat C1 or one of t1.
 * 0 <= iterations <= 16.                                                                                                                       */
#define SPIN_MAX_NORM_ITERATIONS 16
spin_status spin_layernorm(const spin_norm *s, int iterations, uint64_t offset, uint64_t slope, uint64_t eps, const uint64_t *x,
                           const spin_masked *gamma, const uint64_t *beta, const uint64_t *mask_x, const uint64_t *mask_xhat,
                           const uint64_t *C1, const spin_tuple *t1, const uint64_t *C2, const spin_tuple *t2, const uint64_t *row_words,
                           uint64_t *out, uint64_t *xhat, uint64_t *rstd, spin_stream stream);

/* Gradients from dy, that of the result.  column_words: [n][4][dim]; row_words: [n][22][rows], t(k) as above:
 *     g      = T(C1 + dy gamma, f), t1;   dy, xhat and g are opened against their masks
 *     dgamma = T(column word 0 + sum_rows dy xhat, f), column words 1 to 3;     dbeta = sum_rows dy
 *     m1 = T(inv sum g, shift), t(0);   m2 = T(inv T(word 3 + sum g xhat, f), shift), t(4) and t(7);   rstd is opened against word 10
 *     k1 = T(word 12 + m1 rstd, f), m1 against word 11, t(13);   k2 = T(word 17 + m2 rstd, f), m2 against word 16, t(18);   k2 is opened against word 21
 *     dx = T(C2 + g rstd - xhat k2, f) - k1, t2
 * Column word 0, words 3, 12, 17 and C1, C2 (of g rstd - xhat k2) are the dealt shares of the masks' products.  dy, xhat, C1, C2, t1, t2, dx: [n][rows][dim]; gamma, dgamma,
 * dbeta: [n][dim]; rstd: [n][rows].  xhat's mask may be the forward pass's.  dx may alias C2 or an array of t2.  workspace: device scratch of
 * spin_layernorm_grad_workspace_bytes() bytes (0 if the arguments are invalid), 256-byte aligned.  The size does not shrink as n or, for one dim, rows grow: that of the
 * largest batch does for all.                                                                                                                       */
spin_status spin_layernorm_grad(const spin_norm *s, const spin_masked *dy, const spin_masked *xhat, const uint64_t *rstd, const spin_masked *gamma,
                                const uint64_t *mask_g, const uint64_t *C1, const spin_tuple *t1, const uint64_t *C2, const spin_tuple *t2,
                                const uint64_t *row_words, const uint64_t *column_words, uint64_t *dx, uint64_t *dgamma, uint64_t *dbeta,
                                void *workspace, size_t workspace_bytes, spin_stream stream);
size_t spin_layernorm_grad_workspace_bytes(const spin_norm *s);

/* The same over Z_2^32.                                                                                                          */
spin_status spin32_linattn_scores(const spin_linattn *s, int dim, const spin_masked *x, const spin_masked *y, const uint32_t *C,
                                const spin_tuple *t, uint32_t *out, spin_stream stream);
spin_status spin32_linattn_states(const spin_linattn *s, int rows, int columns, int reverse, const spin_masked *x, const spin_masked *y,
                                const uint32_t *C, const spin_tuple *t, const uint32_t *first, uint32_t *states, uint32_t *last,
                                void *workspace, size_t workspace_bytes, spin_stream stream);
size_t spin32_linattn_states_workspace_bytes(const spin_linattn *s, int rows, int columns);
spin_status spin32_linattn_outputs(const spin_linattn *s, int rows, int columns, int reverse, int transposed, const spin_masked *P,
                                 const spin_masked *y, const spin_masked *x, const spin_masked *S, const uint32_t *C, const spin_tuple *t,
                                 uint32_t *out, spin_stream stream);
spin_status spin32_linattn_step(const spin_linattn *s, int rows, int columns, const uint32_t *S, const spin_masked *q, const spin_masked *k,
                              const spin_masked *v, const uint32_t *S_mask, const uint32_t *CS, const spin_tuple *tS, const uint32_t *CO,
                              const spin_tuple *tO, uint32_t *S_out, uint32_t *out, spin_stream stream);
spin_status spin32_layernorm(const spin_norm *s, int iterations, uint32_t offset, uint32_t slope, uint32_t eps, const uint32_t *x,
                           const spin_masked *gamma, const uint32_t *beta, const uint32_t *mask_x, const uint32_t *mask_xhat,
                           const uint32_t *C1, const spin_tuple *t1, const uint32_t *C2, const spin_tuple *t2, const uint32_t *row_words,
                           uint32_t *out, uint32_t *xhat, uint32_t *rstd, spin_stream stream);
spin_status spin32_layernorm_grad(const spin_norm *s, const spin_masked *dy, const spin_masked *xhat, const uint32_t *rstd, const spin_masked *gamma,
                                const uint32_t *mask_g, const uint32_t *C1, const spin_tuple *t1, const uint32_t *C2, const spin_tuple *t2,
                                const uint32_t *row_words, const uint32_t *column_words, uint32_t *dx, uint32_t *dgamma, uint32_t *dbeta,
                                void *workspace, size_t workspace_bytes, spin_stream stream);
size_t spin32_layernorm_grad_workspace_bytes(const spin_norm *s);

/* Static description of a status code. */
const char *spin_status_string(int status);

/* Message of the most recent HIP failure seen by this thread ("" if none). */
const char *spin_last_hip_error(void);

#ifdef __cplusplus
}
#endif
#endif /* SPIN_H */
