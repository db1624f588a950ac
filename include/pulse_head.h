/*
 * pulse_head.h -- C ABI of libpulse's operators at a model's output end and
 * between its blocks.
 *
 * The weights whose changes the codec of pulse.h carries are trained and used
 * here: the trainer normalises the last hidden states, takes the cross entropy
 * of the head's logits and its gradient; a receiver multiplies its current
 * tokens with weights that it holds as FP8 or MXFP4 codes.  Before that, on both
 * sides, blocks' outputs join the residual stream through norms and linear
 * layers; after it, drafted tokens are held against the target's probabilities.
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
 * Sums, statistics and products are accumulated in FP32 (the verification's in FP64).
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
 * pulse_block_norm_forward -- a block's output b joins the residual stream h, and
 * the stream is normalised for the next block; per row, with N_post and N the norms
 * of pulse_layer_norm_forward (PULSE_NORM_RMS for both) with the same eps,
 *   h_out = residual_scale * h + gate * N_post(b),
 *   y     = N(h_out)                    of the sum before it is rounded,
 * each rounded once.
 *   dtype         of b, h, h_out and y: PULSE_DTYPE_F32 or PULSE_DTYPE_BF16.
 *   weight, bias  of N, [cols] of `param_dtype` (F32 or BF16); bias may be NULL.
 *   post_weight, post_bias  of N_post; post_weight NULL: b is taken as it is
 *                 (and post_bias is NULL too); post_bias may be NULL.
 *   gate          [cols] of `param_dtype`, a factor per column; NULL: 1.
 *   h_out         may be h itself (the same pointer and stride).
 *   stats         FP32, rows of `rows` values stats_stride apart: rstd of N, rstd of
 *                 N_post, then (without PULSE_NORM_RMS) mean of N, mean of N_post;
 *                 N_post's are left as they were without post_weight.  NULL: not kept.
 * cols is 1 to PULSE_NORM_MAX_COLS, residual_scale finite.
 */
int pulse_block_norm_forward(int dtype, const void *b, uint64_t b_stride, const void *h,
                             uint64_t h_stride, float residual_scale, int param_dtype,
                             const void *weight, const void *bias, const void *post_weight,
                             const void *post_bias, const void *gate, void *y, uint64_t y_stride,
                             void *h_out, uint64_t h_out_stride, float *stats,
                             uint64_t stats_stride, uint64_t rows, uint32_t cols, float eps,
                             uint32_t flags, void *stream);

/* Workspace of pulse_block_norm_backward for rows of `cols` elements. */
size_t pulse_block_norm_workspace_bytes(uint32_t cols);

/*
 * pulse_block_norm_backward -- the gradient of a forward pass that gave h_out and
 * stats: with xh and bh the rows of h_out and b less their mean, times their rstd
 * (bh = b without post_weight), a = dy * weight and, per row,
 *   g  = dh_out + rstd * (a - sum(a)/n - xh * sum(a * xh)/n),
 *   c  = g * gate * post_weight,
 *   dh = residual_scale * g,
 *   db = post_rstd * (c - sum(c)/n - bh * sum(c * bh)/n)   (without post_weight: c)
 * (without the terms of sum(a) and sum(c) with PULSE_NORM_RMS), rounded once, and
 * summed over the rows, FP32 [cols],
 *   dweight = dy * xh,  dbias = dy,  dpost_weight = g * gate * bh,
 *   dpost_bias = g * gate,  dgate = g * N_post(b).
 *   dh_out   the gradient that reaches h_out elsewhere; NULL: none.
 *   b        may be NULL with neither post_weight nor gate.
 *   dbias, dpost_weight, dpost_bias, dgate  may each be NULL; dpost_weight,
 *            dpost_bias need post_weight, dgate needs gate.
 * rows == 0 sets the sums to zero.
 */
int pulse_block_norm_backward(int dtype, const void *dy, uint64_t dy_stride, const void *dh_out,
                              uint64_t dh_out_stride, const void *b, uint64_t b_stride,
                              const void *h_out, uint64_t h_out_stride, float residual_scale,
                              int param_dtype, const void *weight, const void *post_weight,
                              const void *post_bias, const void *gate, const float *stats,
                              uint64_t stats_stride, void *db, uint64_t db_stride, void *dh,
                              uint64_t dh_stride, float *dweight, float *dbias,
                              float *dpost_weight, float *dpost_bias, float *dgate, uint64_t rows,
                              uint32_t cols, uint32_t flags, void *workspace,
                              size_t workspace_bytes, void *stream);

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

/* The most drafted tokens of a sequence. */
#define PULSE_VERIFY_MAX_DRAFTS 128

/* A workspace for calls of up to `batch` sequences and `drafts` drafts each; 0 for sizes
 * that no call handles. */
size_t pulse_verify_drafts_workspace_bytes(uint32_t batch, uint32_t drafts, uint32_t vocab);

/*
 * pulse_verify_drafts -- which drafted tokens a target model keeps, and the token that
 * follows them, so that all are distributed as the target's own.  With, for the k-th
 * draft x of a sequence,
 *   p = softmax(scale * target row k),  q = softmax(draft_scale * draft row k),
 * the draft is taken if those before it were and u[k] * q(x) < p(x).  At the first that
 * is not taken, a token is drawn from max(p - q, 0); where all were, from p of the
 * next target row: the lowest v with
 *   sum of the weights of 0 ... v  >  u[drafts] * sum of all weights.
 * With drafts == 0 that is sampling from p.
 *   dtype    of the logits: PULSE_DTYPE_F32 or PULSE_DTYPE_BF16.
 *   target   [batch * (drafts + 1), vocab], a sequence's rows one after the other.
 *   draft    [batch * drafts, vocab]; NULL: q is 1 at the draft.
 *   tokens   int64 [batch, drafts]; one outside [0, vocab) is not taken.
 *   lengths  int32 [batch], a sequence's number of drafts, brought into 0 ... drafts;
 *            NULL: drafts of each.  Rows past them are not read.
 *   uniform  FP32 [batch, drafts + 1], in [0, 1).
 *   out      int64 [batch, drafts + 1]: the drafts taken, the token drawn, then -1.
 *   count    int32 [batch]: how many drafts were taken.
 *   logprob  FP32 [batch, drafts + 1]: log p of each token of `out`, 0 past them.
 * A logit of -inf has probability 0.  A row that is -inf throughout, or holds a NaN or
 * +inf, has p (or q) = 0 everywhere: where p has, the draft is refused, and where
 * nothing can be drawn the token is -1 and its logprob -inf.
 * Probabilities and their sums are FP64, and so are the scales: rounded to FP32 they
 * would move every border by some 1e-7.  drafts is at most PULSE_VERIFY_MAX_DRAFTS,
 * batch * (2 drafts + 1) and vocab are below 2^31, the scales from 1e-100 to 1e100.
 */
int pulse_verify_drafts(int dtype, const void *target, uint64_t target_stride, const void *draft,
                        uint64_t draft_stride, const int64_t *tokens, const int32_t *lengths,
                        const float *uniform, uint32_t batch, uint32_t drafts, uint32_t vocab,
                        double scale, double draft_scale, int64_t *out, int32_t *count,
                        float *logprob, void *workspace, size_t workspace_bytes, void *stream);

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

/* Activations; silu(v) = v / (1 + e^-v), gelu(v) = v (1 + erf(v / sqrt 2)) / 2,
 * gelu_tanh(v) = v (1 + tanh(sqrt(2 / pi) (v + 0.044715 v^3))) / 2.  At -inf and inf they
 * and their slopes are what they tend to: 0 and inf, 0 and 1. */
#define PULSE_ACT_NONE 0
#define PULSE_ACT_RELU 1
#define PULSE_ACT_SILU 2
#define PULSE_ACT_GELU 3
#define PULSE_ACT_GELU_TANH 4

/*
 * pulse_lowp_linear -- pulse_lowp_matmul with what follows it in a block, before the one
 * rounding:
 *   y = act(x W^T + bias) * times + residual.
 *   bias      [rows] of `bias_dtype` (F32 or BF16); NULL: none.
 *   times, residual  [tokens, rows] of `y_dtype`; NULL: none.  y may be one of them
 *             (the same pointer and stride), and is then brought up to date in place.
 */
int pulse_lowp_linear(int dtype, const uint8_t *codes, const uint8_t *scales, float inv_scale,
                      uint32_t rows, uint32_t cols, const uint16_t *x, uint64_t x_stride,
                      uint32_t tokens, int bias_dtype, const void *bias, int activation,
                      const void *times, uint64_t times_stride, const void *residual,
                      uint64_t residual_stride, int y_dtype, void *y, uint64_t y_stride,
                      void *stream);

/* The largest weight that pulse_linear handles, and the most tokens of a call. */
#define PULSE_LINEAR_MAX_WIDTH 1048576

/* Up to so many tokens pulse_linear_forward needs no workspace (which may be NULL). */
#define PULSE_LINEAR_FEW_TOKENS 16

/* A workspace for calls of any number of tokens up to `tokens`, both directions; 0 for
 * sizes that no call handles. */
size_t pulse_linear_workspace_bytes(uint32_t tokens, uint32_t rows, uint32_t cols);

/*
 * pulse_linear_forward -- y = act(x W^T + bias) * times + residual, as pulse_lowp_linear,
 * for a BF16 weight [rows, cols] (rows adjacent) and any number of tokens, with
 *   pre   [tokens, rows] of `y_dtype`: x W^T + bias, rounded, which the gradient asks
 *         for where there is an activation or a multiplier; NULL: not kept.
 * rows, cols and tokens are at most PULSE_LINEAR_MAX_WIDTH, rows and cols at least 1.
 * A cols that is no multiple of 8 costs, above PULSE_LINEAR_FEW_TOKENS, a copy of the weight with padded
 * rows in the workspace.
 */
int pulse_linear_forward(const uint16_t *x, uint64_t x_stride, const uint16_t *weight,
                         uint32_t tokens, uint32_t rows, uint32_t cols, int bias_dtype,
                         const void *bias, int activation, const void *times,
                         uint64_t times_stride, const void *residual, uint64_t residual_stride,
                         int y_dtype, void *y, uint64_t y_stride, void *pre, uint64_t pre_stride,
                         void *workspace, size_t workspace_bytes, void *stream);

/*
 * pulse_linear_backward -- the gradient at the forward pass's x, pre and times for the
 * upstream dy (the residual's gradient is dy itself): with
 *   d = dy * times * act'(pre),
 *   dx = d W,   dweight = d^T x,   dbias = sum over tokens of d,   dtimes = dy * act(pre).
 * The two products take d as the sum of two BF16 values, which leaves 2^-16 of it or
 * 2^-126 at most (nothing of a BF16 dy without multiplier and with no activation or relu); they
 * are summed in FP32 and rounded once to BF16.  dbias is summed from d as it is.  relu's
 * derivative at 0 is 0.
 *   dtype     of dy, pre, times and dtimes: F32 or BF16.
 *   pre       may be NULL with neither an activation nor times.
 *   dbias     FP32 [rows]; NULL: not asked for.
 *   dtimes    [tokens, rows]; NULL: not asked for.  dweight: BF16 [rows, cols].
 * tokens == 0 sets dweight and dbias to zero.
 */
int pulse_linear_backward(int dtype, const void *dy, uint64_t dy_stride, const uint16_t *x,
                          uint64_t x_stride, const uint16_t *weight, const void *pre,
                          uint64_t pre_stride, int activation, const void *times,
                          uint64_t times_stride, uint32_t tokens, uint32_t rows, uint32_t cols,
                          uint16_t *dx, uint64_t dx_stride, uint16_t *dweight, float *dbias,
                          void *dtimes, uint64_t dtimes_stride, void *workspace,
                          size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* PULSE_HEAD_H */
