/*
 * slowmo_operators.h -- C ABI of the operators that a worker's local step needs
 * around a Transformer's matrices, for one AMD MI355X (gfx950); in the same
 * library as slowmo.h, with its status codes, element types and conventions:
 *
 *  - slowmo_orthogonalize / slowmo_momentum_orthogonalize: an update, or the
 *    direction of the SGD row of Table C.1, replaced by (nearly) the closest
 *    matrix with orthonormal rows or columns, by Newton-Schulz products.  What
 *    they write is handed to slowmo_local_step as the gradient.
 *  - slowmo_head_norm_rotary and its backward pass: the norm of queries and
 *    keys for each head with the position rotation in the same pass, for
 *    positions along one axis (text) or several (time, height, width).
 *
 * Conventions
 *  - Pointers named "device" are HIP device pointers; everything else is host
 *    memory that may be freed as soon as the call returns.
 *  - Calls enqueue work on `stream` (a hipStream_t, NULL = the default stream)
 *    and return without synchronizing; they allocate nothing on the device,
 *    copy nothing from the host and clear nothing by memset, so all but
 *    slowmo_orth_create may be recorded into a HIP graph.
 *  - Errors: every entry point returns a slowmo_status; nothing aborts or
 *    throws.  Arguments are checked before anything is launched;
 *    slowmo_last_error(NULL) has the message of the last failure on this thread.
 */
#ifndef SLOWMO_OPERATORS_H
#define SLOWMO_OPERATORS_H

#include "slowmo.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- norm of queries and keys for each head, with the position rotation ---- */

#define SLOWMO_MAX_HEAD_DIM 512
#define SLOWMO_MAX_AXES 4

/* What the heads of one call have in common. */
typedef struct {
  int32_t dtype;       /* slowmo_dtype of every element of slowmo_heads */
  int32_t head_dim;    /* D, 1..SLOWMO_MAX_HEAD_DIM */
  int32_t rotary_dim;  /* R, even, 0..D: the first R elements of a head are turned */
  int32_t interleaved; /* pair i is elements (2i, 2i+1) if 1, (i, i + R/2) if 0 */
  int32_t norm;        /* 1: divide by sqrt(mean(x^2) + eps) and multiply by the weight; 0: turn only */
  float eps;           /* >= 0 */
  int32_t n_axes;      /* 1..SLOWMO_MAX_AXES */
  const uint8_t *pair_axis; /* host: the axis (0..n_axes-1) of each of the R/2 pairs; NULL: axis 0 */
  const float *q_weight;    /* device, D floats; NULL: ones (must be NULL without norm) */
  const float *k_weight;
  const float *table;       /* device, [table_rows][2][R/2]: cos, then sin, of the angle of a pair at a
                               position; 4-byte aligned */
  int64_t table_rows;
  const int64_t *positions; /* device, [n_axes][tokens]: row of the table for each axis and token; -1: the
                               axis's pairs are not turned.  Any other place outside the table is not
                               read and gives NaN in the axis's pairs and nothing else (backward, with
                               norm: in the token's heads, and in the pairs' weight gradients) */
  int64_t position_stride;  /* elements from one axis to the next, >= tokens; 0: all axes have the same positions */
} slowmo_head_config;

/* A [tokens][heads][D] array; the D elements of a head are contiguous.  Strides in
 * elements, >= 0, and no array longer than 2^50 elements; data aligned to its element size. */
typedef struct {
  void *data;      /* device; may be NULL if heads == 0 */
  int32_t heads;   /* >= 0 */
  int64_t token_stride, head_stride;
} slowmo_heads;

/*
 * For every token and every head of q and k,
 *   x^ = w * x / sqrt(mean(x^2) + eps)           (x^ = x without norm)
 *   pair (u, v), at the token's position along the pair's axis:
 *   (u, v) <- (u cos - v sin, u sin + v cos)
 * in one pass: fp32 inside, one rounding at the end.
 *   q_out, k_out : as q and k; may be q and k themselves (same data and strides),
 *                  and must not overlap them otherwise.
 *   k_slots      : device, `tokens` entries, or NULL.  Token t's keys go to row
 *                  k_slots[t] of k_out, which has k_rows rows (a cache); to no
 *                  row where the entry lies outside 0..k_rows-1.  Entries inside
 *                  must differ.  k_rows is ignored without k_slots.
 * Errors: ARG, ALIGN, HIP.
 */
slowmo_status slowmo_head_norm_rotary(const slowmo_head_config *cfg, int64_t tokens,
                                      const slowmo_heads *q, const slowmo_heads *k,
                                      const slowmo_heads *q_out, const slowmo_heads *k_out,
                                      const int64_t *k_slots, int64_t k_rows, void *stream);

/*
 * The gradient of slowmo_head_norm_rotary (without slots) for q, k and the weights.
 * With g the output's gradient turned back and x^ = x / sqrt(mean(x^2) + eps):
 *   dx = (g w - x^ mean(g w x^)) / sqrt(mean(x^2) + eps),   dw = sum over tokens and heads of g x^
 * (dx = g without norm).
 *   gq, gk : gradients of q_out and k_out
 *   q, k   : the inputs of the forward call
 *   dq, dk : written; may be gq, gk (same data and strides)
 *   dq_weight, dk_weight : device, D floats each; NULL: not wanted (must be NULL
 *            without norm).  Zeros if there are no tokens or heads.
 *   workspace : device, 16-byte aligned, slowmo_head_backward_bytes() long; NULL if
 *            that is 0.  Sums run in an order fixed by the sizes, strides, alignment and pair_axis.
 * Errors: ARG, ALIGN, NOMEM (workspace too small), HIP.
 */
size_t slowmo_head_backward_bytes(const slowmo_head_config *cfg, int64_t tokens, int32_t q_heads,
                                  int32_t k_heads);
slowmo_status slowmo_head_norm_rotary_backward(const slowmo_head_config *cfg, int64_t tokens,
                                               const slowmo_heads *gq, const slowmo_heads *gk,
                                               const slowmo_heads *q, const slowmo_heads *k,
                                               const slowmo_heads *dq, const slowmo_heads *dk,
                                               float *dq_weight, float *dk_weight, void *workspace,
                                               size_t workspace_bytes, void *stream);

/* ---- orthogonalised updates ------------------------------------------------ */

typedef struct slowmo_orth slowmo_orth; /* opaque */

/* The factor s on the result for a matrix of `rows` by `cols`. */
typedef enum {
  SLOWMO_SCALE_NONE = 0,  /* 1 */
  SLOWMO_SCALE_SHAPE = 1, /* sqrt(max(1, rows / cols)): the same change of outputs for all shapes */
  SLOWMO_SCALE_RMS = 2    /* 0.2 sqrt(max(rows, cols)): elements as large as Adam's */
} slowmo_orth_scale;

#define SLOWMO_MAX_ORTH_STEPS 16

typedef struct {
  int32_t in_dtype;   /* slowmo_dtype of the matrices read */
  int32_t out_dtype;  /* slowmo_dtype of the results.  It decides how the products are formed: of
                         11-bit halves for bf16 results, of pairs of halves (22 bits) for fp32,
                         whatever in_dtype is.  Off from 64 bits, Frobenius norms: bf16 results 0.8e-3 to
                         2.5e-3 (few rows) beside their own rounding of 1.65e-3, up to 2.9e-3 where the
                         rank is deficient; fp32 results 2e-6, 1.6e-5 */
  int32_t steps;      /* Newton-Schulz steps, 1..SLOWMO_MAX_ORTH_STEPS */
  int32_t scale;      /* slowmo_orth_scale */
  float eps;          /* added to the Frobenius norm, >= 0 */
  const float *coefficients; /* host, [steps][3]: a, b, c of every step, finite; NULL: (3.4445, -4.7750, 2.0315).
                                Refused if some singular value of 0..1 comes to 7.5 or more after a step, where each
                                step from s adds up to (|a| s + |b| s^3 + |c| s^5) / 1024 for rounding: X's elements
                                have to stay in a half's range.  (Steps that are steep at the largest values that
                                reach them need a safety factor, as the roundings grow there) */
} slowmo_orth_config;

/*
 * Orthogonalising a list of matrices.  For each one, U with n <= k its shorter and
 * longer side,
 *   X_0 = U / (|U|_F + eps)     (as n x k: transposed if it has more rows than columns)
 *   A = X X^T;   X <- a X + (b A + c A A) X,   `steps` times
 *   O = s X                     (in U's own orientation)
 * U's bits count in full however small |U| is beside eps (unless a step's a is 0: X then shrinks with
 * its cube and may come to zeros).
 * A matrix of zeros gives zeros; one that holds a NaN or an infinity gives NaN
 * everywhere.  A handle is made for a list of shapes and keeps a workspace:
 *   rows, cols : host, n_matrices entries each, >= 0 (an empty matrix is skipped),
 *                at most 65536 a side
 *   ld         : host, elements from one row to the next (>= cols), for inputs and
 *                results alike; NULL: cols
 *   workspace  : device, 256-byte aligned, at least slowmo_orth_bytes() long; owned by
 *                the caller, kept until slowmo_orth_destroy.
 * slowmo_orth_create waits for `stream`; slowmo_orth_bytes returns 0 for bad arguments and is
 * host-only.  Calls on one handle must be issued on one stream or be ordered by the caller.
 * Errors: ARG, ALIGN, NOMEM, HIP.
 */
size_t slowmo_orth_bytes(const slowmo_orth_config *cfg, int32_t n_matrices, const int64_t *rows,
                         const int64_t *cols, const int64_t *ld);
slowmo_status slowmo_orth_create(slowmo_orth **out, const slowmo_orth_config *cfg,
                                 int32_t n_matrices, const int64_t *rows, const int64_t *cols,
                                 const int64_t *ld, void *workspace, size_t workspace_bytes,
                                 void *stream);

/*
 * out[i] <- the orthogonalised in[i].  `in` and `out` are host arrays of n_matrices device
 * pointers, aligned to their element size; out[i] may be in[i] where the types are the same, and
 * results overlap nothing else.
 * Errors: ARG, ALIGN, HIP.
 */
slowmo_status slowmo_orthogonalize(slowmo_orth *h, const void *const *in, void *const *out,
                                   void *stream);

/*
 * The same behind the momentum of the SGD row of Table C.1:
 *   M <- mu M + G,   U = G + mu M (nesterov) or M,   out <- the orthogonalised U.
 *   momentum : host array of n_matrices device pointers to fp32 matrices (row distance ld), updated
 *              in place; zeros at the start.  It is the caller's: slowmo_outer_step's buffer policies
 *              (reset, maintain, average) and slowmo_export_state do not reach it.  Left alone it is
 *              maintained; to reset it, zero it after the outer step.
 *   mu       : 0 <= mu < 1
 * Errors: ARG, ALIGN, HIP.
 */
slowmo_status slowmo_momentum_orthogonalize(slowmo_orth *h, const void *const *grads,
                                            float *const *momentum, void *const *out, float mu,
                                            int32_t nesterov, void *stream);

/* Frees the handle's host memory; never the workspace.  NULL is accepted. */
slowmo_status slowmo_orth_destroy(slowmo_orth *h);

#ifdef __cplusplus
}
#endif
#endif /* SLOWMO_OPERATORS_H */
