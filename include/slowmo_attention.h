/*
 * slowmo_attention.h -- C ABI of what reads the queries and keys that
 * slowmo_head_norm_rotary turns, for one AMD MI355X (gfx950); in the same library as
 * slowmo.h and slowmo_operators.h, with their status codes, element types and arrays:
 *
 *  - slowmo_attention and its backward pass: attention over packed sequences, with a
 *    sliding window and first keys that stay visible beside it, for training and prompts.
 *  - slowmo_cache_append: new keys and values to their places in a paged cache, turned
 *    by their positions on the way.
 *  - slowmo_paged_attention: attention of each sequence's newest tokens, one or many,
 *    over that cache, under the same mask.
 *
 * Conventions: those of slowmo_operators.h.  Every call may be recorded into a HIP graph.
 * A workspace belongs to one call at a time: calls that may run at once, captured ones
 * included, need one each.  Offsets, lengths and pages are read on the device: what they
 * hold is not checked before the launch, and the kernels read and write nothing outside
 * the arrays that the call names whatever they hold.
 */
#ifndef SLOWMO_ATTENTION_H
#define SLOWMO_ATTENTION_H

#include "slowmo_operators.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SLOWMO_MAX_ATTENTION_DIM 256
#define SLOWMO_MAX_PAGE 65536

/* What a call's sequences have in common.  Query i of a sequence of n queries and m keys
 * is at position p = i + m - n (the last query beside the last key); it sees key j if
 *   (j <= p or not causal)  and  (window = 0  or  |p - j| < window  or  j < sinks). */
typedef struct {
  int32_t dtype;      /* slowmo_dtype of queries, keys, values, results and gradients */
  int32_t head_dim;   /* D, 1..SLOWMO_MAX_ATTENTION_DIM, of queries, keys and values */
  int32_t causal;     /* 0 or 1 */
  int32_t clear_rest; /* rows of results behind the last sequence: 1 set to zero (lse: -infinity), 0 left as they are */
  float scale;        /* of the products, finite and > 0 */
  int64_t window;     /* >= 0; 0: none */
  int64_t sinks;      /* >= 0; without a window of no effect */
} slowmo_attention_config;

/*
 * Attention over packed sequences.  With s_ij = scale q_i . k_j over the keys that query i
 * sees, P_ij = exp(s_ij - lse_i):
 *   lse_i = log sum_j exp(s_ij),   out_i = sum_j P_ij v_j.
 * A query that sees no key: out 0, lse -infinity.  What a key or value that a query does not see
 * holds, NaN and infinities too, has no part in its result.  Query heads share key heads in groups:
 * query head h has key head h / (q heads / k heads).  Products of the matrix cores (bf16: P is
 * rounded to bf16, statistics and sums are fp32; f32: products and sums fp32).
 *   batch     : number of sequences, 0..2^20
 *   q_offsets : device, batch + 1 entries, ascending from 0: sequence b has query rows
 *               q_offsets[b] .. q_offsets[b+1]-1
 *   k_offsets : the same for keys and values; NULL: q_offsets
 *   tokens, keys : rows of q and out, rows of k and v, each 0..2^30
 *   q, k, v   : q heads a multiple of k heads, at most 2^12 times as many, tokens times q
 *               heads at most 2^36; v has k's heads
 *   out       : as q; may not overlap an input
 *   lse       : device, [tokens][q heads] floats, or NULL
 * Errors: ARG, ALIGN, HIP.
 */
slowmo_status slowmo_attention(const slowmo_attention_config *cfg, int32_t batch, const int64_t *q_offsets,
                               const int64_t *k_offsets, int64_t tokens, int64_t keys, const slowmo_heads *q,
                               const slowmo_heads *k, const slowmo_heads *v, const slowmo_heads *out, float *lse,
                               void *stream);

/*
 * The gradient of slowmo_attention.  With g the gradient of out and P as above:
 *   dV = P^T g,   dS = P (g V^T - rowsum(g out)),   dQ = scale dS K,   dK = scale dS^T Q,
 * dK and dV summed over the query heads that share a key head.  All sums run in an order
 * fixed by the sizes.  g out is taken of the rounded result and mended by the sum of the row's dS: bf16 in every row, fp32
 * where it is more than 2^-21 of the sum of |dS|.
 *   g, q, k, v, out, lse : of the forward call (lse is wanted here), over these very keys: a row's P sums to 1
 *   dq, dk, dv : written; may overlap no input and not one another.  Keys that no query sees: zeros
 *   workspace  : device, 16-byte aligned, slowmo_attention_backward_bytes() long
 * Errors: ARG, ALIGN, NOMEM (workspace too small), HIP.
 */
size_t slowmo_attention_backward_bytes(const slowmo_attention_config *cfg, int32_t batch, int64_t tokens, int64_t keys,
                                       int32_t q_heads, int32_t k_heads);
slowmo_status slowmo_attention_backward(const slowmo_attention_config *cfg, int32_t batch, const int64_t *q_offsets,
                                        const int64_t *k_offsets, int64_t tokens, int64_t keys, const slowmo_heads *g,
                                        const slowmo_heads *q, const slowmo_heads *k, const slowmo_heads *v,
                                        const slowmo_heads *out, const float *lse, const slowmo_heads *dq,
                                        const slowmo_heads *dk, const slowmo_heads *dv, void *workspace,
                                        size_t workspace_bytes, void *stream);

/* ---- a paged cache of keys or values ---- */

/* A [pages][page][heads][D] array; the D elements of a head are contiguous.  Strides in elements, >= 0,
 * and no array longer than 2^50 elements; data aligned to its element size. */
typedef struct {
  void *data;     /* device */
  int32_t heads;  /* >= 1 */
  int32_t page;   /* positions of a page: a power of two, 1..SLOWMO_MAX_PAGE */
  int64_t pages;  /* 0..2^31-1 */
  int64_t page_stride, token_stride, head_stride;
} slowmo_cache;

/* Which pages the sequences of a call have.  Position j of sequence b lies in row j mod page of page
 * pages[b * stride + j / page]. */
typedef struct {
  int32_t batch;           /* 0..2^20 */
  int32_t columns;         /* pages of a row of the table, 0..2^30 */
  int64_t stride;          /* elements from one row to the next, >= columns */
  const int32_t *pages;    /* device */
  const int64_t *lengths;  /* device, [batch]: positions of each sequence, the call's new tokens, its last ones, included */
  const int64_t *offsets;  /* device, [batch + 1], ascending from 0: sequence b has the new tokens offsets[b] .. offsets[b+1]-1 */
} slowmo_pages;

/* What slowmo_cache_append turns.  New token i of n of a sequence of length m is at position i + m - n. */
typedef struct {
  int32_t dtype;        /* slowmo_dtype of every array */
  int32_t head_dim;     /* D, 1..SLOWMO_MAX_HEAD_DIM */
  int32_t rotary_dim;   /* R, even, 0..D: the first R elements of a head are turned */
  int32_t interleaved;  /* pair i is elements (2i, 2i+1) if 1, (i, i + R/2) if 0 */
  int32_t clear_rest;   /* rows of q_out behind the last sequence: 1 set to zero, 0 left as they are */
  const float *table;   /* device, [table_rows][2][R/2]: cos, then sin; 4-byte aligned */
  int64_t table_rows;   /* a position outside the table gives NaN in the turned pairs */
} slowmo_append_config;

/*
 * For every new token: its key, turned by its position, to its place in k_cache; its value to its
 * place in v_cache; its query, turned the same way, to q_out.  fp32 inside, one rounding.
 *   tokens : rows of k, v and q, 0..2^30.  Rows behind the last sequence are not read
 *   k, v   : heads as the caches have (k's and v's may differ)
 *   q, q_out : may be NULL, both; q_out may be q itself (same data and strides)
 * A token whose position is negative, or past the table's columns, or whose page lies outside the cache is not
 * appended (its query is turned).  Pages that two sequences share must not be written by both.
 * All other places of the caches stay as they are.
 * Errors: ARG, ALIGN, HIP.
 */
slowmo_status slowmo_cache_append(const slowmo_append_config *cfg, const slowmo_pages *pages, int64_t tokens,
                                  const slowmo_heads *k, const slowmo_heads *v, const slowmo_cache *k_cache,
                                  const slowmo_cache *v_cache, const slowmo_heads *q, const slowmo_heads *q_out,
                                  void *stream);

/*
 * slowmo_attention of each sequence's new tokens over all its lengths[b] positions, read from the caches
 * (which hold the new tokens' keys and values too).  causal is 1 as a rule.
 *   k_cache, v_cache : the same heads and page
 *   lse       : device, [tokens][q heads] floats, or NULL
 *   workspace : device, 16-byte aligned, slowmo_paged_attention_bytes() long; NULL if that is 0
 * Pages that no query sees are not looked at.  A query that sees a position whose page lies outside the
 * cache, or past the table's columns, has NaN, and so has its lse.  Lengths past 2^30 count as 2^30, below 0 as 0.
 * Errors: ARG, ALIGN, NOMEM, HIP.
 */
size_t slowmo_paged_attention_bytes(const slowmo_attention_config *cfg, const slowmo_pages *pages, int64_t tokens,
                                    int32_t q_heads, const slowmo_cache *k_cache);
slowmo_status slowmo_paged_attention(const slowmo_attention_config *cfg, const slowmo_pages *pages, int64_t tokens,
                                     const slowmo_heads *q, const slowmo_cache *k_cache, const slowmo_cache *v_cache,
                                     const slowmo_heads *out, float *lse, void *workspace, size_t workspace_bytes,
                                     void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SLOWMO_ATTENTION_H */
