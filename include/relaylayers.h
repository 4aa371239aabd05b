/*
 * relaylayers.h -- layer operators for training n workers' models on one GPU
 * (librelaysum.so, beside the RelaySum step of relaysum.h).
 *
 * The step keeps one fp32 model row per worker; these calls run one layer of
 * all n models at once, forward and backward, and keep the activations that
 * the backward pass reads in 8 bits:
 *
 *   relay_rms_norm            h = x + r;  s = 1 / sqrt(mean(h^2) + eps);  xhat = h s;  y = xhat w
 *   relay_rms_norm_backward   u = dy w;  dx = s (u - xhat mean(u xhat)) + dh;  dw = sum_t dy xhat
 *   relay_gated               a = g sigma(g) u,  sigma(g) = 1 / (1 + exp(-g))
 *   relay_gated_backward      du = da g sigma(g);  dg = da u sigma(g) (1 + g (1 - sigma(g)));  a again
 *   relay_weight_grad         dW[o][i] = scale[i] sum_t dy[t][o] xhat[t][i]
 *   relay_block_norm          h = rho r + sigma(z) (x s_x) w_post;  y = h s_h w_pre,  s the norms' reciprocal roots
 *   relay_block_norm_backward its gradients
 *   relay_recurrence          h_t = f_t h_{t-1} + (1 - f_t) v_t,  f = sigma(gate)
 *   relay_recurrence_backward l_t = dh_t + f_{t+1} l_{t+1};  dv = l (1 - f);  dgate = l (h_{t-1} - v) f (1 - f)
 *   relay_orthogonalise       x = u / |u|, then x <- a x + (b g + c g g) x with g = x x^T, step by step
 *   relay_checkpoint_pack     any activation to 8 bits, and
 *   relay_checkpoint_unpack   back
 *
 * The norm's and the gated activation's checkpoints are what their own
 * backward passes and the next linear layer's weight gradient read: with
 * xhat of the norm in 8 bits, scale = w gives the gradient of a layer that
 * read y = xhat w.
 *
 * Conventions shared by every call:
 *   - Rows.  An activation is a view [n][tokens][d] of one of the types
 *     below, features next to one another, with a stride in elements from
 *     worker to worker and from token to token (relay_rows).  Inputs may
 *     repeat rows (stride 0); the rows of an output may not overlap.  All
 *     activations of a call have the same type.  Rows whose addresses and
 *     strides are multiples of 16 bytes and whose d is a multiple of 8 are
 *     moved 16 bytes at a time, others element by element.
 *   - Weights.  A norm's weight and its gradient, the column scale and the
 *     weight gradient are fp32 views with a stride from worker to worker, of
 *     any alignment: they lie in the workers' model rows and in rows beside
 *     them.  A weight that all workers share has stride 0, and a gradient
 *     per worker.
 *   - Arithmetic is in fp32, and each output is rounded once, to the nearest
 *     (y and xhat come from the unrounded h).  sigma of 16-bit gates is off by
 *     less than (3 + |g|) 2^-23 relative, by which an 8-bit code behind it can
 *     land beside the nearest one.  The results of a call are the
 *     same bits every time: no atomics.
 *   - Lengths.  Where a call sums over tokens or goes along them, `lengths`
 *     (device int32 [n], or NULL for all) says how many of each worker's rows
 *     count, clamped to 0 .. tokens.  Rows past it may hold anything, and the
 *     rows that the call writes there are zero.
 *   - Streams, ownership and errors are those of relaysum.h: caller-owned
 *     device buffers, nothing allocated, nothing synchronised, every argument
 *     checked before anything is enqueued.  The sizes that the library cannot
 *     see (of the buffers) are the caller's to get right.  An output may not
 *     be another argument's buffer, with the exceptions that a call names:
 *     `total` of relay_rms_norm and relay_block_norm may be the view of x or
 *     of the residual (the same rows at the same strides), the recurrence's
 *     outgoing state its incoming one, relay_orthogonalise's out its update.
 *     RELAY_EINVAL: NULL for something needed, a size or stride out of range
 *     (n < 1, tokens < 0, d < 1, overlapping output rows), an address that
 *     is not a multiple of its element's size, checkpoint or workspace
 *     addresses that are not multiples of 16, a workspace too small.
 *     RELAY_EUNSUPPORTED: n > RELAY_MAX_N (in the recurrence
 *     RELAY_RECURRENCE_MAX_N), n tokens >= 2^30, d > 2^24, in the norms d >
 *     RELAY_NORM_MAX_D, in the weight gradient inputs >
 *     RELAY_WEIGHT_GRAD_MAX_INPUTS, in the orthogonal update rows or columns
 *     > RELAY_ORTHOGONALISE_MAX.
 *
 * The 8-bit format.  A row of d features is blocks of 32 with one scale byte
 * c per block and one signed code q per feature:
 *
 *   value = q 2^(c - 133),  -127 <= q <= 127,  7 <= c <= 254
 *
 * c is the least that keeps |q| <= 127 when the block's values are rounded to
 * the nearest (ties to even); blocks below 2^-120 keep c = 7.  c = 255 says
 * that the block held an infinity, a NaN or a magnitude of 127.5 2^121 and
 * more, and all of it reads as NaN.  Scales that are powers of two make the
 * codes an exact function of the values, and the values exact in bf16 and
 * fp32.  Codes are int8 [n][tokens][pitch], scales uint8
 * [n][tokens][pitch / 32], pitch = relay_checkpoint_pitch(d) = d rounded up
 * to a multiple of 128; features past d are written as 0 (scale 7) and never
 * change a result.
 */
#ifndef RELAYLAYERS_H
#define RELAYLAYERS_H

#include <stdint.h>

#include "relaysum.h"

#ifdef __cplusplus
extern "C" {
#endif

#define RELAY_BF16 0
#define RELAY_FP16 1
#define RELAY_FP32 2

#define RELAY_NORM_MAX_D 32768
#define RELAY_WEIGHT_GRAD_MAX_INPUTS (1 << 22)
#define RELAY_RECURRENCE_MAX_N (1 << 20)
#define RELAY_ORTHOGONALISE_MAX 65536
#define RELAY_ORTHOGONALISE_MAX_STEPS 100

/* A view [n][tokens][d] of device memory: element (i, t, k) is at
 * data + i worker_stride + t token_stride + k, strides in elements, >= 0. */
typedef struct relay_rows {
    void *data;
    int64_t worker_stride;
    int64_t token_stride;
} relay_rows;

/* Codes per row of a checkpoint (scale bytes: a 32nd of it); RELAY_EINVAL for
 * d < 1. */
int64_t relay_checkpoint_pitch(int64_t d);

/* x to 8 bits. */
int relay_checkpoint_pack(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows *x, int8_t *codes,
                          uint8_t *scales, relay_stream_t stream);

/* 8 bits to `out`: exact in bf16 and fp32 (fp16: rounded, and held at its
 * largest finite magnitude). */
int relay_checkpoint_unpack(int32_t type, int32_t n, int64_t tokens, int64_t d, const int8_t *codes,
                            const uint8_t *scales, const relay_rows *out, relay_stream_t stream);

/* The sum, its root-mean-square norm and, where codes and scales are given,
 * xhat in 8 bits.  residual, total (h in the rows' type), rstd (s, fp32
 * [n][tokens]) and codes with scales may each be NULL.  eps > 0.  The squares
 * are summed in fp32: a row of which they pass 3.4e38 (values of 1e17 to 1e19
 * and more) has s = 0 and y = 0. */
int relay_rms_norm(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows *x,
                   const relay_rows *residual, const float *weight, int64_t weight_stride, float eps,
                   const relay_rows *total, const relay_rows *y, float *rstd, int8_t *codes, uint8_t *scales,
                   relay_stream_t stream);

/* Bytes of workspace for relay_rms_norm_backward, or a negative status. */
int64_t relay_rms_norm_backward_workspace(int32_t n, int64_t tokens, int64_t d);

/* Gradients of the norm: dx (of x and of the residual alike) and dweight (per
 * worker, overwritten).  xhat is read from codes and scales, or, where those
 * are NULL, formed from total and rstd.  dtotal: the gradient that reaches h
 * past the norm, or NULL. */
int relay_rms_norm_backward(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows *dy,
                            const relay_rows *dtotal, const float *weight, int64_t weight_stride, const float *rstd,
                            const relay_rows *total, const int8_t *codes, const uint8_t *scales,
                            const int32_t *lengths, const relay_rows *dx, float *dweight, int64_t dweight_stride,
                            void *workspace, int64_t workspace_bytes, relay_stream_t stream);

/* The gated activation; gate and up (rounded as given) in 8 bits too where
 * their codes and scales are given. */
int relay_gated(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows *gate, const relay_rows *up,
                const relay_rows *out, int8_t *gate_codes, uint8_t *gate_scales, int8_t *up_codes,
                uint8_t *up_scales, relay_stream_t stream);

/* Its gradients, from the rows (gate, up) or from their checkpoints: one of
 * the two is given and the other NULL.  Where out_codes and out_scales are
 * given, the activation is formed again and put there in 8 bits. */
int relay_gated_backward(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows *dout,
                         const relay_rows *gate, const relay_rows *up, const int8_t *gate_codes,
                         const uint8_t *gate_scales, const int8_t *up_codes, const uint8_t *up_scales,
                         const relay_rows *dgate, const relay_rows *dup, int8_t *out_codes, uint8_t *out_scales,
                         relay_stream_t stream);

/* Bytes of workspace for relay_weight_grad (may be 0), or a negative status.
 * dy: the rows that it will get, for which this is the exact size, or NULL for
 * any strides and alignment.  fp16 and fp32 rows, and bf16 rows that are not
 * 16-byte aligned or that repeat, are copied into it (2, 3 or 1 times 2 bytes
 * an element); the rest are the sums of splits of the tokens.  The size for
 * NULL is enough for every call of the type with the same n, outputs and
 * inputs and as many tokens or fewer, that for RELAY_FP32 and NULL for every
 * type. */
int64_t relay_weight_grad_workspace(int32_t type, int32_t n, int64_t tokens, int64_t outputs, int64_t inputs,
                                    const relay_rows *dy);

/* The weight gradient of a linear layer, per worker, from the gradient of its
 * outputs dy [n][tokens][outputs] and its inputs in 8 bits; overwrites
 * dweight: element (i, o, k) at dweight + i worker_stride + o row_stride + k.
 * column_scale (fp32, `inputs` per worker) may be NULL.  The kernel's waits
 * for copies and products end after about a second each; results that one of
 * them was for are NaN then. */
int relay_weight_grad(int32_t type, int32_t n, int64_t tokens, int64_t outputs, int64_t inputs, const relay_rows *dy,
                      const int8_t *codes, const uint8_t *scales, const float *column_scale,
                      int64_t column_scale_stride, const int32_t *lengths, float *dweight, int64_t worker_stride,
                      int64_t row_stride, void *workspace, int64_t workspace_bytes, relay_stream_t stream);

/* From one block to the next: the norm of the block's output x, its gate, its
 * addition to the residual r, and the norm of the sum for the next block:
 *   m = x s_x post;  h = scale r + sigma(gate) m;  y = h s_h pre
 * with s_x = 1 / sqrt(mean(x^2) + eps) and s_h likewise of the unrounded h.
 * gate (rows) and scale (fp32, per feature) may be NULL: 1.  total (h in the
 * rows' type), rstd (fp32 [2][n][tokens]: s_x, s_h) and codes with scales
 * (h s_h in 8 bits) may each be NULL.  total may be the view of x or of the
 * residual.  The squares are summed in fp32, as in relay_rms_norm. */
int relay_block_norm(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows *x, const relay_rows *gate,
                     const relay_rows *residual, const float *post, int64_t post_stride, const float *pre,
                     int64_t pre_stride, const float *scale, int64_t scale_stride, float eps, const relay_rows *total,
                     const relay_rows *y, float *rstd, int8_t *codes, uint8_t *scales, relay_stream_t stream);

/* Bytes of workspace for relay_block_norm_backward, or a negative status. */
int64_t relay_block_norm_backward_workspace(int32_t n, int64_t tokens, int64_t d);

/* Its gradients, from the rows of the forward pass and rstd (h is formed
 * again): of x, of the gate (given and asked for together), of the residual,
 * and per worker, overwritten, of post, pre and scale (dscale may be NULL).
 * dtotal: the gradient that reaches h past the second norm, or NULL.  Rows
 * past the lengths count nowhere and get gradients of 0.  The mean that dx
 * takes off is a difference of sums over the row, whose terms are those of
 * sigma(gate) x s_x post times h's gradient: off by what fp32 leaves of them,
 * also where dx itself is small. */
int relay_block_norm_backward(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows *dy,
                              const relay_rows *dtotal, const relay_rows *x, const relay_rows *gate,
                              const relay_rows *residual, const float *post, int64_t post_stride, const float *pre,
                              int64_t pre_stride, const float *scale, int64_t scale_stride, const float *rstd,
                              const int32_t *lengths, const relay_rows *dx, const relay_rows *dgate,
                              const relay_rows *dresidual, float *dpost, int64_t dpost_stride, float *dpre,
                              int64_t dpre_stride, float *dscale, int64_t dscale_stride, void *workspace,
                              int64_t workspace_bytes, relay_stream_t stream);

/* Bytes of workspace for relay_recurrence and relay_recurrence_backward (may
 * be 0), or a negative status. */
int64_t relay_recurrence_workspace(int32_t n, int64_t tokens, int64_t d);

/* The gated linear recurrence along the tokens of each of n workers (or of n
 * sequences, up to RELAY_RECURRENCE_MAX_N), every feature on its own:
 * h_t = f_t h_{t-1} + (1 - f_t) v_t with f = sigma(gate).  The state is fp32,
 * the rows `out` are h rounded.  initial (fp32 [n][d], stride from worker to
 * worker): the state before the first token, NULL for 0.  last (the same
 * shape, or NULL): the state behind the last token, for the call that goes on;
 * it may be `initial`, at the same stride.  begins (uint8 [n][tokens], or
 * NULL): not 0 at a token that begins a sequence, where h_{t-1} counts as 0
 * whatever it holds.  lengths: tokens past them leave the state as it is and
 * get rows of 0.  Behind an input that is not finite the states
 * are not finite up to the next beginning (an infinity may become NaN).  The
 * calls' waits for copies end after about a second each; results that one of
 * them was for are NaN then (in relay_block_norm and its backward pass too). */
int relay_recurrence(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows *gate,
                     const relay_rows *value, const float *initial, int64_t initial_stride, const uint8_t *begins,
                     const int32_t *lengths, const relay_rows *out, float *last, int64_t last_stride, void *workspace,
                     int64_t workspace_bytes, relay_stream_t stream);

/* Its gradients, from the rows of the forward pass: gate, value and out (whose
 * rounded values are taken as h).  dlast: the gradient of the last state, or
 * NULL; dinitial: that of the first one, or NULL (it may be dlast, at the same
 * stride).  begins, lengths and initial as in the forward pass; rows past the
 * lengths get gradients of 0. */
int relay_recurrence_backward(int32_t type, int32_t n, int64_t tokens, int64_t d, const relay_rows *dout,
                              const relay_rows *gate, const relay_rows *value, const relay_rows *out,
                              const float *initial, int64_t initial_stride, const float *dlast, int64_t dlast_stride,
                              const uint8_t *begins, const int32_t *lengths, const relay_rows *dgate,
                              const relay_rows *dvalue, float *dinitial, int64_t dinitial_stride, void *workspace,
                              int64_t workspace_bytes, relay_stream_t stream);

/* Bytes of workspace for relay_orthogonalise, or a negative status. */
int64_t relay_orthogonalise_workspace(int32_t n, int64_t rows, int64_t columns);

/* Makes n fp32 matrices [rows][columns] nearly orthogonal, each by itself, as
 * the update of a weight matrix: x = update / (|update| + eps) with the root of
 * the sum of squares |.|, then `steps` times
 *   g = x x^T;  x <- a x + (b g + c g g) x,  a = 3.4445, b = -4.7750, c = 2.0315,
 * or the same from the other side where rows outnumber columns; out = scale x.
 * Five steps bring singular values from 0.002 of |update| up to between 0.68
 * and 1.21.  Element (i, r, c) is at update + i worker_stride + r row_stride +
 * c; out likewise, and may be the view of update.  The coefficients are those
 * of the Muon optimiser (K. Jordan and others, 2024).  Operands are held in 22
 * to 23 bits and summed in fp32.  A matrix of zeros stays zero; one that holds a
 * value that is not finite becomes NaN, all of it.  rows, columns <=
 * RELAY_ORTHOGONALISE_MAX, steps in 1 .. RELAY_ORTHOGONALISE_MAX_STEPS, eps >=
 * 0.  The kernel's waits end after about a second each; results that one of
 * them was for are NaN then. */
int relay_orthogonalise(int32_t n, int64_t rows, int64_t columns, const float *update, int64_t worker_stride,
                        int64_t row_stride, int32_t steps, float eps, float scale, float *out,
                        int64_t out_worker_stride, int64_t out_row_stride, void *workspace, int64_t workspace_bytes,
                        relay_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* RELAYLAYERS_H */
