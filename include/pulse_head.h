/*
 * pulse_head.h -- C ABI of libpulse's operators at a model's output end.
 *
 * The weights whose changes the codec of pulse.h carries are trained and used
 * here: the trainer normalises the last hidden states, takes the cross entropy
 * of the head's logits and its gradient; a receiver multiplies its current
 * tokens with weights that it holds as FP8 or MXFP4 codes.
 *
 * Conventions: those of pulse.h (device pointers, a hipStream_t passed as
 * void*, work enqueued and not waited for, no device memory allocated,
 * PULSE_OK or a negative pulse_status with pulse_last_error()).  Unless said
 * otherwise:
 *   - matrices are row-major; a stride is the number of elements from one row
 *     to the next and at least the row's length;
 *   - dense pointers are 16-byte aligned (else PULSE_EALIGN);
 *   - outputs do not overlap inputs;
 *   - a workspace is 256-byte aligned, needs no initialisation, holds nothing
 *     between calls, and serves any calls ordered on one stream;
 *   - results are the same bits for the same inputs: every sum has a fixed
 *     order.
 * Sums, statistics and products are accumulated in FP32.
 */
#ifndef PULSE_HEAD_H
#define PULSE_HEAD_H

#include <stddef.h>
#include <stdint.h>

#include "pulse.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types beside PULSE_DTYPE_FP8_E4M3 and PULSE_DTYPE_MXFP4. */
#define PULSE_DTYPE_F32 3
#define PULSE_DTYPE_BF16 4

/* The largest row that the norm handles. */
#define PULSE_NORM_MAX_COLS 16384

/* Flag of the norm: no mean is taken off and none is written (RMS norm). */
#define PULSE_NORM_RMS 1u

/*
 * pulse_layer_norm_forward -- per row of x, with n = cols:
 *   mean = sum(x) / n (0 with PULSE_NORM_RMS),
 *   rstd = 1 / sqrt(sum((x - mean)^2) / n + eps),
 *   y = (x - mean) * rstd * weight + bias, rounded once to y's type.
 *   dtype         of x and y: PULSE_DTYPE_F32 or PULSE_DTYPE_BF16.
 *   weight, bias  [cols] of `param_dtype` (F32 or BF16); bias may be NULL.
 *   mean          FP32 [rows]; ignored with PULSE_NORM_RMS (may be NULL then).
 *   rstd          FP32 [rows].
 *   x_stride, y_stride   elements from row to row.
 * cols is 1 to PULSE_NORM_MAX_COLS.  Rows of 16-byte groups (cols and strides
 * multiples of 8) are moved 16 bytes at a time; any other row element by
 * element.
 */
int pulse_layer_norm_forward(int dtype, const void *x, uint64_t x_stride, int param_dtype,
                             const void *weight, const void *bias, void *y, uint64_t y_stride,
                             float *mean, float *rstd, uint64_t rows, uint32_t cols, float eps,
                             uint32_t flags, void *stream);

/* Workspace of pulse_layer_norm_backward for rows of `cols` elements. */
size_t pulse_layer_norm_workspace_bytes(uint32_t cols);

/*
 * pulse_layer_norm_backward -- the gradient of a forward pass that gave mean
 * and rstd.  With xh = (x - mean) * rstd and a = dy * weight, per row
 *   dx = rstd * (a - sum(a)/n - xh * sum(a * xh)/n)
 * (without the middle term with PULSE_NORM_RMS), rounded once to dx's type, and
 *   dweight = sum over rows of dy * xh,   dbias = sum over rows of dy.
 *   dweight, dbias  FP32 [cols]; dbias may be NULL.
 * rows == 0 sets dweight and dbias to zero.
 */
int pulse_layer_norm_backward(int dtype, const void *dy, uint64_t dy_stride, const void *x,
                              uint64_t x_stride, int param_dtype, const void *weight,
                              const float *mean, const float *rstd, void *dx, uint64_t dx_stride,
                              float *dweight, float *dbias, uint64_t rows, uint32_t cols,
                              uint32_t flags, void *workspace, size_t workspace_bytes,
                              void *stream);

/*
 * Softmax cross entropy of a head's logits, which are never stored: with
 *   z[t][v] = logit_scale * sum_k x[t][k] weight[v][k]      (products exact,
 *             summed in FP32),
 *   lse[t]  = log sum_v exp(z[t][v]),
 *   loss[t] = lse[t] - z[t][targets[t]];  0 where the target is ignored.
 * A target outside [0, vocab) is ignored, whatever its value: such a token has
 * an lse, no loss and no gradient, and what is in its row of x (NaN, say) reaches
 * no gradient of another token or of the weight.
 *   x         BF16 [tokens, hidden], rows x_stride apart.
 *   weight    BF16 [vocab, hidden], rows adjacent.
 *   targets   device int64 [tokens].
 * hidden is 1 to PULSE_CE_MAX_HIDDEN; tokens and vocab are below 2^31, vocab at
 * least 1; logit_scale is finite.  tokens == 0 writes no loss or lse (and a
 * zero dweight).  A hidden that is no multiple of 8 costs a copy of the weight
 * with padded rows in the workspace.
 */
#define PULSE_CE_MAX_HIDDEN 65536

/* A workspace for calls of any number of tokens up to `tokens`, both directions; 0 for
 * sizes that no call handles. */
size_t pulse_linear_ce_workspace_bytes(uint32_t tokens, uint32_t vocab, uint32_t hidden);

/* loss and lse: FP32 [tokens]. */
int pulse_linear_ce_forward(const uint16_t *x, uint64_t x_stride, const uint16_t *weight,
                            const int64_t *targets, uint32_t tokens, uint32_t vocab,
                            uint32_t hidden, float logit_scale, float *loss, float *lse,
                            void *workspace, size_t workspace_bytes, void *stream);

/*
 * pulse_linear_ce_backward -- the gradient for the upstream dloss (FP32
 * [tokens], e.g. a token's advantage over the number of tokens), with the
 * forward pass's lse.  Piece by piece of the vocabulary the logits are computed
 * again and G[t][v] = dloss[t] * (exp(z[t][v] - lse[t]) - [v == targets[t]]) is
 * rounded to BF16 for the two products
 *   dx = logit_scale * G weight,   dweight = logit_scale * G^T x,
 * which are summed in FP32 and rounded once to BF16.  What the rounding of G takes
 * is added back: to dx from large entries one by one and from the others through a
 * mean row of the weight, so that a direction which the weight's rows share cancels as
 * in the exact sum; to dweight from the targets' entries, and up to 128 tokens from
 * all.
 *   dx       BF16 [tokens, hidden], rows dx_stride apart.
 *   dweight  BF16 [vocab, hidden].
 */
int pulse_linear_ce_backward(const uint16_t *x, uint64_t x_stride, const uint16_t *weight,
                             const int64_t *targets, uint32_t tokens, uint32_t vocab,
                             uint32_t hidden, float logit_scale, const float *lse,
                             const float *dloss, uint16_t *dx, uint64_t dx_stride,
                             uint16_t *dweight, void *workspace, size_t workspace_bytes,
                             void *stream);

/*
 * pulse_lowp_matmul -- y = x W^T, W the receiver's copy of a [rows, cols]
 * weight as pulse_cast_lowp and pulse_apply_lowp_batch leave it (codes flat in
 * row order, an MXFP4 block any 32 consecutive values, so a block may span two
 * rows):
 *   W = code * 2^(scale - 127)  (MXFP4; a block with scale 0xFF is NaN),
 *   W = code / inv_scale        (FP8 E4M3, inv_scale as it was cast with).
 * Meant for the few tokens of a decoding step: the weight is read once for
 * every 16 or 32 tokens.  Products are exact, summed in FP32, rounded once to y.
 *   dtype    PULSE_DTYPE_MXFP4 (codes 4-byte aligned) or PULSE_DTYPE_FP8_E4M3
 *            (codes 8-byte aligned; scales unused).
 *   x        BF16 [tokens, cols]; y [tokens, rows] of `y_dtype` (F32 or BF16).
 * rows and cols are at least 1 and below 2^31; tokens at most 2^20; inv_scale
 * is finite and not zero for FP8.
 */
int pulse_lowp_matmul(int dtype, const uint8_t *codes, const uint8_t *scales, float inv_scale,
                      uint32_t rows, uint32_t cols, const uint16_t *x, uint64_t x_stride,
                      uint32_t tokens, int y_dtype, void *y, uint64_t y_stride, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* PULSE_HEAD_H */
