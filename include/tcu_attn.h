/*
 * tcu_attn.h -- C ABI of the attention operators of libtcu_dft.so: the norm of
 * each head of queries and keys with the rotation by position in the same
 * pass, and attention over a sliding window and a sequence's first tokens;
 * each with its gradient, and for single tokens.
 *
 * Attention is the third way to mix positions beside convolutions
 * (tcu_dft.h) and recurrences (tcu_seq.h): weights that come from pairs of
 * tokens.  Over a window of a fixed length its cost and its cache stay
 * bounded as a recurrence's do, so layers of both alternate in one model.
 *
 *   norm_rotate  n = x / sqrt(mean(x^2) + eps) weight       (per head, `dim` values)
 *                pairs (n_p, n_{p+turned}), p < turned, of adjacent pairs (n_2p,
 *                n_{2p+1}) with `interleaved`, turned by the angle
 *                position rates[p]:  (a cos - b sin, a sin + b cos)
 *                values from 2 turned on are only normalised
 *   attention    y_i = sum_j p_ij v_j, p_i the softmax of scale q_i.k_j over the
 *                visible j of the same sequence: j <= i and (i - j < window or
 *                j < sinks), rows counted from the sequence's first.  Query head
 *                h reads key head h kv_heads / heads.
 *
 * Layout: as in tcu_seq.h; a row of q and y holds heads x dim adjacent values,
 * one of k and v kv_heads x dim.  Rows behind the last packed sequence are
 * left as they are in outputs, and their gradients are zeros.
 *
 * Statistics, sums and products are accumulated in fp32 and rounded once, on
 * storing; attention over prompts rounds its weights, and in the gradient the
 * scores' gradients, to the rows' type before the products that take them (fp16:
 * times powers of two for each row or key, so that nothing is lost to its range;
 * single tokens: in two parts).  The same call gives the same bits every time.
 * Angles are 2^-25 turns off at most, at any position: the turns of a position
 * are a 64-bit product that wraps, 2^-31 off for rates up to 2^32, and round to
 * fp32.  Pairs whose rate is not finite become no numbers.
 *
 * Calls and statuses are as in tcu_seq.h.  Every wait inside a kernel of
 * attention ends after two seconds; what a block then stores is no number,
 * while the call, which returned before, has given OK.  Outputs must not
 * overlap inputs or themselves, but y_q and y_k may be q and k, with the same
 * strides.
 */
#ifndef TCU_ATTN_H
#define TCU_ATTN_H

#include "tcu_seq.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { TCU_ATTN_MAX_NORM_DIM = 256, TCU_ATTN_MAX_DIM = 128 };

/* Norm and rotation.  dim is even, at most TCU_ATTN_MAX_NORM_DIM; 1 <= turned <=
 * dim / 2; rates: turned values; weights: dim values or NULL.  positions: one
 * for each row, batch entries x rows, or NULL: the row's place in its
 * sequence. */
typedef struct {
  int32_t type, sequences, heads, kv_heads, dim, turned, interleaved;
  float eps;
  int64_t rows;
  const int32_t *offsets, *positions;
  tcu_seq_rows q, k, y_q, y_k;
  const float *rates, *q_weight, *k_weight;
  tcu_seq_rows dy_q, dy_k, dq, dk;
  float *dq_weight, *dk_weight;
  void *workspace;
  int64_t workspace_bytes;
} tcu_norm_rotate_args;

/* q, k, rates [...] -> y_q, y_k. */
int tcu_norm_rotate(const tcu_norm_rotate_args *a, void *stream);
/* dy_q, dy_k and the inputs -> dq, dk [, dq_weight, dk_weight], through
 * workspace. */
int tcu_norm_rotate_grad(const tcu_norm_rotate_args *a, void *stream);
int64_t tcu_norm_rotate_grad_workspace(const tcu_norm_rotate_args *a);

/* Window attention.  type: bf16 or fp16.  dim is a multiple of 8, at most
 * TCU_ATTN_MAX_DIM; heads a multiple of kv_heads; window >= 1, sinks >= 0,
 * scale > 0.  Rows of q, k, v, y and of their gradients start at multiples of
 * 16 bytes and do not overlap.  lse: the log of each row's sum of
 * exponentials, batch entries x rows x heads, written by the prompt call when
 * not NULL and read by the gradient.
 *
 * A cache of keys and one of values: num_slots entries of sinks + window rows
 * of kv_heads x dim values, contiguous, 16-byte aligned.  Position p of a
 * sequence is row p of its entry if p < sinks, else row sinks + (p - sinks) %
 * window: what a token sees is what its entry holds. */
typedef struct {
  int32_t type, sequences, heads, kv_heads, dim, window, sinks;
  float scale;
  int64_t rows;
  const int32_t *offsets;
  tcu_seq_rows q, k, v, y;
  float *lse;
  tcu_seq_rows dy, dq, dk, dv;
  void *workspace;
  int64_t workspace_bytes;
  void *cache_k, *cache_v;
  const int32_t *slots, *positions;
  int64_t num_slots;
} tcu_window_attention_args;

/* q, k, v [, offsets] -> y [, lse]. */
int tcu_window_attention(const tcu_window_attention_args *a, void *stream);
/* dy, q, k, v, y, lse -> dq, dk, dv, through workspace. */
int tcu_window_attention_grad(const tcu_window_attention_args *a, void *stream);
int64_t tcu_window_attention_grad_workspace(const tcu_window_attention_args *a);
/* One row per sequence (rows = 1, dense), at positions[b] of its sequence: its
 * k and v enter entry slots[b] (entry b without slots) of the caches, and q
 * reads them -> y.  A position below zero or an entry outside [0, num_slots)
 * gives a row of zeros and changes no cache; no two rows may name one entry. */
int tcu_window_attention_step(const tcu_window_attention_args *a, void *stream);
/* The rows of whole prompts k and v that the next token of each sequence
 * sees, into its entry; entries outside [0, num_slots) are passed over, and no
 * two sequences may name one. */
int tcu_window_cache(const tcu_window_attention_args *a, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* TCU_ATTN_H */
