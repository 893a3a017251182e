/*
 * tcu_seq.h -- C ABI of the sequence operators of libtcu_dft.so: a short
 * causal convolution, a selective state-space scan and a gated linear
 * recurrence, each over whole prompts, with its gradient, and for one token.
 *
 * The 2-D convolutions and stencils of tcu_dft.h mix positions with weights
 * that are the same everywhere, so a DFT diagonalises them.  The scan's decay
 * and inputs depend on the position: it is the linear recurrence that remains
 * when they do (with constant coefficients it equals a causal convolution).
 *
 *   convolution  p_t = bias + sum_{k < width} w_k x_{t - (width-1) + k}
 *                y_t = p_t sigma(p_t) with silu, else p_t
 *   scan         d_t = softplus(dt_t + dt_bias)   (dt_t + dt_bias without softplus)
 *                h_t[n] = exp(d_t A[n]) h_{t-1}[n] + d_t u_t B_t[n]
 *                o_t = sum_n C_t[n] h_t[n] + skip u_t
 *                y_t = o_t g_t sigma(g_t) with a gate, else o_t
 *   recurrence   a_t = exp(-rate sigma(forget_t))
 *                h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigma(admit_t) x_t,  y_t = h_t
 * per sequence and channel, sigma(v) = 1 / (1 + exp(-v)).
 *
 * Layout.  Row tensors (x, u, dt, gate, forget, admit, y, their gradients) hold one row of
 * `channels` adjacent values per position; B and C one row of groups x states
 * adjacent values, group g serving channels [g channels/groups, (g+1)
 * channels/groups).  Every row tensor has its own strides, in elements,
 * between batch entries and between rows.  Dense: `sequences` batch entries
 * of `rows` rows each.  Packed (offsets != NULL): `rows` rows in all, sequence
 * s being rows [offsets[s], offsets[s+1]); offsets is a device array of
 * sequences + 1 values from 0 to rows, never falling; equal neighbours are an
 * empty sequence.  Packed offsets are read on the device only: values out of
 * order give unspecified results, never an access out of range.
 *
 * Row tensors and the convolution's states are of one type (tcu_seq_type);
 * the states of scan and recurrence, all parameters and their gradients are
 * fp32.  Sums,
 * states and gradients are accumulated in fp32 and rounded once, on storing;
 * the same call gives the same bits every time.  Exponentials and reciprocals
 * are the special function unit's (2^-22 of the result).
 *
 * Calls are asynchronous on `stream` (a cudaStream_t), allocate nothing, and
 * return a TCU_DFT_* status: ERR_INVALID (sizes, null pointers, alignment of
 * a pointer to its element, workspace too small, a single-token call's cache
 * over another argument), ERR_UNSUPPORTED (width or states beyond the limits,
 * more than 2^31 - 4097 rows, a row stride beyond 32 bits; a single-token
 * scan's batch stride beyond 32 bits, or more than 2^31 - 262141 entries; more
 * than 4,194,240 channels of a convolution; a grid of 2^31 blocks), ERR_CUDA.  On an argument error nothing is launched.
 * A wait between blocks of the recurrence ends after two seconds; what is then
 * stored is no number, while the call, which returned before, has given OK.
 * Outputs must not overlap inputs or themselves; y of a single-token call may
 * be its x, u, dt, gate, forget or admit, with the same strides.
 */
#ifndef TCU_SEQ_H
#define TCU_SEQ_H

#include <stdint.h>

#include "tcu_dft.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { TCU_SEQ_F32 = 0, TCU_SEQ_BF16 = 1, TCU_SEQ_F16 = 2 } tcu_seq_type;

enum { TCU_SEQ_MAX_WIDTH = 8, TCU_SEQ_MAX_STATES = 128 };

/* A row tensor: element (batch b, row t, channel c) is at
 * ptr[b * batch_stride + t * row_stride + c]. */
typedef struct {
  void *ptr;
  int64_t batch_stride, row_stride;
} tcu_seq_rows;

/* Short causal convolution.  Fields that a call does not name are ignored.
 * weight: channels x width, the last tap on the current row; bias: channels
 * or NULL.  state / last / dlast / dstate: sequences x (width-1) x channels,
 * oldest row first: the rows before the first, those a continuation needs,
 * and their gradients.  state == NULL is rows of zeros. */
typedef struct {
  int32_t type, width, silu, sequences;
  int64_t rows, channels;
  const int32_t *offsets;
  tcu_seq_rows x, y, dy, dx;
  const float *weight, *bias;
  const void *state, *dlast;
  void *last, *dstate;
  float *dweight, *dbias;
  void *workspace;
  int64_t workspace_bytes;
  const int32_t *slots; /* step: cache entry of each batch entry, or NULL */
  int64_t num_slots;
} tcu_short_conv_args;

/* x, weight [, bias, state, offsets] -> y [, last]. */
int tcu_short_conv(const tcu_short_conv_args *a, void *stream);
/* dy, x, weight [, bias, state, offsets, dlast] -> dx, dweight [, dbias,
 * dstate], through workspace (tcu_short_conv_grad_workspace bytes). */
int tcu_short_conv_grad(const tcu_short_conv_args *a, void *stream);
int64_t tcu_short_conv_grad_workspace(const tcu_short_conv_args *a);
/* One row per sequence (rows = 1, dense): x -> y, and the cache `last`
 * (num_slots x (width-1) x channels) advanced in place at entry slots[b]
 * (entry b without slots).  An entry outside [0, num_slots) gives a row of
 * zeros and changes no state; no two rows may name one entry. */
int tcu_short_conv_step(const tcu_short_conv_args *a, void *stream);

/* Selective scan.  A: channels x states; skip, dt_bias: channels or NULL;
 * state / last / dlast / dstate: sequences x channels x states (NULL state:
 * zeros).  marks: the state that enters every TCU_SEQ_MARK-th row, batch
 * entries x ceil(rows / TCU_SEQ_MARK) x channels x states (batch entries:
 * sequences when dense, 1 when packed), written by the scan when not NULL
 * and read by its gradient. */
enum { TCU_SEQ_MARK = 16 };
typedef struct {
  int32_t type, softplus, sequences, groups;
  int64_t rows, channels, states;
  const int32_t *offsets;
  tcu_seq_rows u, dt, gate, y, B, C; /* gate.ptr == NULL: no gate */
  const float *A, *skip, *dt_bias;
  const float *state, *dlast;
  float *last, *dstate, *marks;
  tcu_seq_rows dy, du, ddt, dgate, dB, dC;
  float *dA, *dskip, *ddt_bias;
  void *workspace;
  int64_t workspace_bytes;
  const int32_t *slots;
  int64_t num_slots;
} tcu_state_scan_args;

/* u, dt, A, B, C [...] -> y [, last, marks], through workspace. */
int tcu_state_scan(const tcu_state_scan_args *a, void *stream);
int64_t tcu_state_scan_workspace(const tcu_state_scan_args *a);
/* dy, marks and the scan's inputs -> du, ddt, dA, dB, dC [, dskip, dgate,
 * ddt_bias, dstate], through workspace. */
int tcu_state_scan_grad(const tcu_state_scan_args *a, void *stream);
/* Mostly shares of dB and dC, 1 byte for each row and channel at 16 states, 4
 * at 32, 16 at 64 and 64 at 128. */
int64_t tcu_state_scan_grad_workspace(const tcu_state_scan_args *a);
/* One row per sequence (rows = 1, dense): u, dt, B, C -> y, and the cache
 * `last` (num_slots x channels x states) advanced in place; slots as for
 * tcu_short_conv_step. */
int tcu_state_scan_step(const tcu_state_scan_args *a, void *stream);

/* Gated linear recurrence, one state a channel.  rate: channels, positive;
 * state / last / dlast / dstate: sequences x channels (NULL state: zeros).
 * marks: the state that enters every TCU_SEQ_GATED_MARK-th row, batch entries
 * x ceil(rows / TCU_SEQ_GATED_MARK) x channels, as the scan's.  Rows behind
 * the last packed sequence are left as they are in y, and their gradients are
 * zeros. */
enum { TCU_SEQ_GATED_MARK = 8 };
typedef struct {
  int32_t type, sequences;
  int64_t rows, channels;
  const int32_t *offsets;
  tcu_seq_rows x, forget, admit, y;
  const float *rate, *state, *dlast;
  float *last, *dstate, *marks;
  tcu_seq_rows dy, dx, dforget, dadmit;
  float *drate;
  void *workspace;
  int64_t workspace_bytes;
  const int32_t *slots;
  int64_t num_slots;
} tcu_gated_scan_args;

/* x, forget, admit, rate [, state, offsets] -> y [, last, marks], through
 * workspace. */
int tcu_gated_scan(const tcu_gated_scan_args *a, void *stream);
int64_t tcu_gated_scan_workspace(const tcu_gated_scan_args *a);
/* dy, marks and the recurrence's inputs [, dlast] -> dx, dforget, dadmit,
 * drate [, dstate], through workspace. */
int tcu_gated_scan_grad(const tcu_gated_scan_args *a, void *stream);
int64_t tcu_gated_scan_grad_workspace(const tcu_gated_scan_args *a);
/* One row per sequence (rows = 1, dense): x, forget, admit -> y, and the cache
 * `last` (num_slots x channels) advanced in place; slots as for
 * tcu_short_conv_step. */
int tcu_gated_scan_step(const tcu_gated_scan_args *a, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* TCU_SEQ_H */
