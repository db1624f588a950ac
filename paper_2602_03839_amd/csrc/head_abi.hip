// head_abi.hip -- the extern "C" entry points declared in
// include/pulse_head.h: argument validation on the host, then the launches.
#include "../../include/pulse_head.h"

#include "abi_status.hpp"
#include "head.hpp"

namespace {

using pulse::aligned;
using pulse::aligned16;
using pulse::fail;
using pulse::hip_status;
using pulse::ok;

int check_space(const char* who, const void* ws, size_t bytes, size_t needed) {
  if (!ws) return fail(PULSE_EINVAL, "%s: workspace is NULL", who);
  if (!aligned(ws, 256)) return fail(PULSE_EALIGN, "%s: workspace is not 256-byte aligned", who);
  if (bytes < needed)
    return fail(PULSE_EINVAL, "%s: workspace has %zu bytes, needs %zu", who, bytes, needed);
  return PULSE_OK;
}

// what both directions of the norm ask of their arguments
int check_norm(const char* who, int dtype, int param_dtype, uint64_t rows, uint32_t cols, uint32_t flags,
               const void* weight, const float* mean, const float* rstd) {
  if (dtype != PULSE_DTYPE_F32 && dtype != PULSE_DTYPE_BF16)
    return fail(PULSE_EINVAL, "%s: dtype %d is neither F32 nor BF16", who, dtype);
  if (param_dtype != PULSE_DTYPE_F32 && param_dtype != PULSE_DTYPE_BF16)
    return fail(PULSE_EINVAL, "%s: param_dtype %d is neither F32 nor BF16", who, param_dtype);
  if (flags & ~PULSE_NORM_RMS) return fail(PULSE_EINVAL, "%s: unknown flags %#x", who, flags);
  if (cols == 0 || cols > PULSE_NORM_MAX_COLS)
    return fail(PULSE_EINVAL, "%s: %u columns, 1 to %d are handled", who, cols, PULSE_NORM_MAX_COLS);
  if (rows > 0x7FFFFFFFull) return fail(PULSE_EINVAL, "%s: more than 2^31 - 1 rows", who);
  if (!weight) return fail(PULSE_EINVAL, "%s: weight is NULL", who);
  if (rows && !rstd) return fail(PULSE_EINVAL, "%s: rstd is NULL", who);
  if (rows && !(flags & PULSE_NORM_RMS) && !mean) return fail(PULSE_EINVAL, "%s: mean is NULL", who);
  if (!aligned16(weight)) return fail(PULSE_EALIGN, "%s: weight not 16-byte aligned", who);
  if (!aligned(mean, 4) || !aligned(rstd, 4)) return fail(PULSE_EALIGN, "%s: mean/rstd not 4-byte aligned", who);
  return PULSE_OK;
}

int check_matrix(const char* who, const char* name, const void* p, uint64_t stride, uint64_t rows,
                 uint32_t cols) {
  if (rows == 0) return PULSE_OK;
  if (!p) return fail(PULSE_EINVAL, "%s: %s is NULL", who, name);
  if (!aligned16(p)) return fail(PULSE_EALIGN, "%s: %s not 16-byte aligned", who, name);
  if (stride < cols || stride > (1ull << 40))
    return fail(PULSE_EINVAL, "%s: %s stride %llu for rows of %u", who, name, (unsigned long long)stride,
                cols);
  return PULSE_OK;
}

// what both directions of the block norm ask of their arguments
int check_block_norm(const char* who, int dtype, int param_dtype, uint64_t rows, uint32_t cols, uint32_t flags,
                     float residual_scale, const void* weight, const void* post_weight, const void* post_bias,
                     const void* gate, const float* stats, uint64_t stats_stride) {
  // the statistics are checked apart: they may be absent
  const float* none = (const float*)(uintptr_t)16;
  if (int rc = check_norm(who, dtype, param_dtype, rows, cols, flags, weight, none, none)) return rc;
  if (!(residual_scale - residual_scale == 0.0f))
    return fail(PULSE_EINVAL, "%s: residual_scale is not finite", who);
  if (post_bias && !post_weight) return fail(PULSE_EINVAL, "%s: post_bias without post_weight", who);
  for (const void* v : {post_weight, post_bias, gate})
    if (!aligned16(v)) return fail(PULSE_EALIGN, "%s: post_weight, post_bias or gate not 16-byte aligned", who);
  if (!aligned(stats, 4)) return fail(PULSE_EALIGN, "%s: stats not 4-byte aligned", who);
  if (stats && (stats_stride < rows || stats_stride > (1ull << 40)))
    return fail(PULSE_EINVAL, "%s: stats stride %llu for %llu rows", who, (unsigned long long)stats_stride,
                (unsigned long long)rows);
  return PULSE_OK;
}

bool verify_handles(uint32_t batch, uint32_t drafts, uint32_t vocab) {
  return drafts <= PULSE_VERIFY_MAX_DRAFTS && vocab != 0 && vocab <= 0x7FFFFFFFu &&
         (uint64_t)batch * (2 * drafts + 1) <= 0x7FFFFFFFull;
}

bool linear_handles(uint32_t tokens, uint32_t rows, uint32_t cols) {
  return tokens <= PULSE_LINEAR_MAX_WIDTH && rows != 0 && rows <= PULSE_LINEAR_MAX_WIDTH && cols != 0 &&
         cols <= PULSE_LINEAR_MAX_WIDTH;
}

// what both directions of the linear layer ask of their arguments
int check_linear(const char* who, bool forward, const void* x, uint64_t x_stride, const void* weight, uint32_t tokens, uint32_t rows,
                 uint32_t cols, const void* ws, size_t ws_bytes) {
  if (!linear_handles(tokens, rows, cols))
    return fail(PULSE_EINVAL, "%s: %u tokens, a weight of %u x %u", who, tokens, rows, cols);
  if (tokens == 0) return PULSE_OK;
  if (int rc = check_matrix(who, "x", x, x_stride, tokens, cols)) return rc;
  if (!weight) return fail(PULSE_EINVAL, "%s: weight is NULL", who);
  if (!aligned16(weight)) return fail(PULSE_EALIGN, "%s: weight not 16-byte aligned", who);
  const uint64_t needs = pulse::linear_needs(forward, tokens, rows, cols);
  return needs ? check_space(who, ws, ws_bytes, needs) : PULSE_OK;
}

// what every product with codes asks of its arguments
int check_lowp(const char* who, int dtype, const void* codes, const void* scales, float inv_scale, uint32_t rows,
               uint32_t cols, const void* x, uint64_t x_stride, uint32_t tokens, int y_dtype, const void* y,
               uint64_t y_stride) {
  const bool mx = dtype == PULSE_DTYPE_MXFP4;
  if (!mx && dtype != PULSE_DTYPE_FP8_E4M3)
    return fail(PULSE_EINVAL, "%s: dtype %d is neither FP8_E4M3 nor MXFP4", who, dtype);
  if (y_dtype != PULSE_DTYPE_F32 && y_dtype != PULSE_DTYPE_BF16)
    return fail(PULSE_EINVAL, "%s: y_dtype %d is neither F32 nor BF16", who, y_dtype);
  if (rows == 0 || rows > 0x7FFFFFFFu || cols == 0 || cols > 0x7FFFFFFFu)
    return fail(PULSE_EINVAL, "%s: a weight of %u x %u", who, rows, cols);
  if (tokens > 1u << 20) return fail(PULSE_EINVAL, "%s: more than 2^20 tokens", who);
  if (tokens == 0) return PULSE_OK;
  if (!codes) return fail(PULSE_EINVAL, "%s: codes is NULL", who);
  if (mx && !scales) return fail(PULSE_EINVAL, "%s: scales is NULL", who);
  if (!aligned(codes, mx ? 4 : 8)) return fail(PULSE_EALIGN, "%s: codes not %d-byte aligned", who, mx ? 4 : 8);
  if (!mx && !(inv_scale - inv_scale == 0.0f && inv_scale != 0.0f))
    return fail(PULSE_EINVAL, "%s: inv_scale is zero or not finite", who);
  if (int rc = check_matrix(who, "x", x, x_stride, tokens, cols)) return rc;
  return check_matrix(who, "y", y, y_stride, tokens, rows);
}

pulse::LowpMatmulParams lowp_params(int dtype, const uint8_t* codes, const uint8_t* scales, float inv_scale,
                                    uint32_t rows, uint32_t cols, const uint16_t* x, uint64_t x_stride,
                                    uint32_t tokens, int y_dtype, void* y, uint64_t y_stride) {
  const uint64_t n = (uint64_t)rows * cols;
  return {codes, scales, inv_scale, rows, cols, dtype == PULSE_DTYPE_MXFP4 ? (n + 1) / 2 : n, (n + 31) / 32, x, x_stride,
          tokens, y, y_stride, y_dtype == PULSE_DTYPE_BF16, {}};
}

// The epilogue's arguments, checked, as `e` (whose `pre` is none).
int check_epilogue(const char* who, uint32_t rows, uint32_t tokens, int bias_dtype, const void* bias, int activation,
                   const void* times, uint64_t times_stride, const void* residual, uint64_t residual_stride,
                   int y_dtype, const void* y, uint64_t y_stride, pulse::Epilogue& e) {
  if (bias && bias_dtype != PULSE_DTYPE_F32 && bias_dtype != PULSE_DTYPE_BF16)
    return fail(PULSE_EINVAL, "%s: bias_dtype %d is neither F32 nor BF16", who, bias_dtype);
  if (!aligned16(bias)) return fail(PULSE_EALIGN, "%s: bias not 16-byte aligned", who);
  if (activation < 0 || activation >= pulse::kActs)
    return fail(PULSE_EINVAL, "%s: activation %d is not known", who, activation);
  if (times)
    if (int rc = check_matrix(who, "times", times, times_stride, tokens, rows)) return rc;
  if (residual)
    if (int rc = check_matrix(who, "residual", residual, residual_stride, tokens, rows)) return rc;
  if (tokens && ((times && y == times && y_stride != times_stride) ||
                 (residual && y == residual && y_stride != residual_stride)))
    return fail(PULSE_EINVAL, "%s: y is times or residual with another stride", who);
  e = {bias, bias_dtype == PULSE_DTYPE_BF16, activation, times, times_stride, residual, residual_stride, nullptr, 0,
       y_dtype == PULSE_DTYPE_BF16};
  return PULSE_OK;
}

bool ce_handles(uint32_t tokens, uint32_t vocab, uint32_t hidden) {
  return tokens <= 0x7FFFFFFFu && vocab != 0 && vocab <= 0x7FFFFFFFu && hidden != 0 && hidden <= PULSE_CE_MAX_HIDDEN;
}

int check_ce(const char* who, const void* x, uint64_t x_stride, const void* weight, const void* targets,
             uint32_t tokens, uint32_t vocab, uint32_t hidden, float logit_scale, const void* ws,
             size_t ws_bytes) {
  if (vocab == 0 || vocab > 0x7FFFFFFFu || tokens > 0x7FFFFFFFu)
    return fail(PULSE_EINVAL, "%s: %u tokens, vocabulary of %u", who, tokens, vocab);
  if (hidden == 0 || hidden > PULSE_CE_MAX_HIDDEN)
    return fail(PULSE_EINVAL, "%s: hidden size %u, 1 to %d are handled", who, hidden, PULSE_CE_MAX_HIDDEN);
  if (!(logit_scale - logit_scale == 0.0f)) return fail(PULSE_EINVAL, "%s: logit_scale is not finite", who);
  if (tokens == 0) return PULSE_OK;
  if (int rc = check_matrix(who, "x", x, x_stride, tokens, hidden)) return rc;
  if (!weight || !targets) return fail(PULSE_EINVAL, "%s: weight or targets is NULL", who);
  if (!aligned16(weight)) return fail(PULSE_EALIGN, "%s: weight not 16-byte aligned", who);
  if (!aligned(targets, 8)) return fail(PULSE_EALIGN, "%s: targets not 8-byte aligned", who);
  return check_space(who, ws, ws_bytes, pulse::linear_ce_needs(tokens, vocab, hidden));
}

}  // namespace

extern "C" {

int pulse_layer_norm_forward(int dtype, const void* x, uint64_t x_stride, int param_dtype,
                             const void* weight, const void* bias, void* y, uint64_t y_stride,
                             float* mean, float* rstd, uint64_t rows, uint32_t cols, float eps,
                             uint32_t flags, void* stream) {
  const char* who = "layer_norm forward";
  if (int rc = check_norm(who, dtype, param_dtype, rows, cols, flags, weight, mean, rstd)) return rc;
  if (int rc = check_matrix(who, "x", x, x_stride, rows, cols)) return rc;
  if (int rc = check_matrix(who, "y", y, y_stride, rows, cols)) return rc;
  if (!aligned16(bias)) return fail(PULSE_EALIGN, "%s: bias not 16-byte aligned", who);
  if (!(eps >= 0.0f)) return fail(PULSE_EINVAL, "%s: eps is negative or NaN", who);
  if (rows == 0) return ok();
  pulse::NormParams p = {x, x_stride, weight, bias, y, y_stride, flags & PULSE_NORM_RMS ? nullptr : mean,
                         rstd, rows, cols, eps, param_dtype == PULSE_DTYPE_BF16};
  return hip_status(pulse::launch_layer_norm(dtype == PULSE_DTYPE_BF16, p, (hipStream_t)stream),
                    "layer_norm launch");
}

size_t pulse_layer_norm_workspace_bytes(uint32_t cols) {
  return (size_t)pulse::kNormBlocks * cols * 2 * sizeof(float);
}

int pulse_layer_norm_backward(int dtype, const void* dy, uint64_t dy_stride, const void* x,
                              uint64_t x_stride, int param_dtype, const void* weight,
                              const float* mean, const float* rstd, void* dx, uint64_t dx_stride,
                              float* dweight, float* dbias, uint64_t rows, uint32_t cols,
                              uint32_t flags, void* workspace, size_t workspace_bytes,
                              void* stream) {
  const char* who = "layer_norm backward";
  if (int rc = check_norm(who, dtype, param_dtype, rows, cols, flags, weight, mean, rstd)) return rc;
  if (int rc = check_matrix(who, "dy", dy, dy_stride, rows, cols)) return rc;
  if (int rc = check_matrix(who, "x", x, x_stride, rows, cols)) return rc;
  if (int rc = check_matrix(who, "dx", dx, dx_stride, rows, cols)) return rc;
  if (!dweight) return fail(PULSE_EINVAL, "%s: dweight is NULL", who);
  if (!aligned(dweight, 4) || !aligned(dbias, 4))
    return fail(PULSE_EALIGN, "%s: dweight/dbias not 4-byte aligned", who);
  if (int rc = check_space(who, workspace, workspace_bytes, pulse_layer_norm_workspace_bytes(cols)))
    return rc;
  pulse::NormGradParams p = {dy, dy_stride, x, x_stride, weight,
                             flags & PULSE_NORM_RMS ? nullptr : mean, rstd, dx, dx_stride, dweight, dbias,
                             (float*)workspace, rows, cols, param_dtype == PULSE_DTYPE_BF16};
  return hip_status(pulse::launch_layer_norm_grad(dtype == PULSE_DTYPE_BF16, p, (hipStream_t)stream),
                    "layer_norm backward launch");
}

int pulse_block_norm_forward(int dtype, const void* b, uint64_t b_stride, const void* h, uint64_t h_stride,
                             float residual_scale, int param_dtype, const void* weight, const void* bias,
                             const void* post_weight, const void* post_bias, const void* gate, void* y,
                             uint64_t y_stride, void* h_out, uint64_t h_out_stride, float* stats,
                             uint64_t stats_stride, uint64_t rows, uint32_t cols, float eps, uint32_t flags,
                             void* stream) {
  const char* who = "block_norm forward";
  if (int rc = check_block_norm(who, dtype, param_dtype, rows, cols, flags, residual_scale, weight, post_weight,
                                post_bias, gate, stats, stats_stride))
    return rc;
  if (int rc = check_matrix(who, "b", b, b_stride, rows, cols)) return rc;
  if (int rc = check_matrix(who, "h", h, h_stride, rows, cols)) return rc;
  if (int rc = check_matrix(who, "y", y, y_stride, rows, cols)) return rc;
  if (int rc = check_matrix(who, "h_out", h_out, h_out_stride, rows, cols)) return rc;
  if (!aligned16(bias)) return fail(PULSE_EALIGN, "%s: bias not 16-byte aligned", who);
  if (!(eps >= 0.0f)) return fail(PULSE_EINVAL, "%s: eps is negative or NaN", who);
  if (rows == 0) return ok();
  if (h_out == h && h_out_stride != h_stride)
    return fail(PULSE_EINVAL, "%s: h_out is h with another stride", who);
  pulse::BlockNormParams p = {b, b_stride, h, h_stride, residual_scale, weight, bias, post_weight, post_bias, gate,
                              y, y_stride, h_out, h_out_stride, stats, stats_stride, rows, cols, eps,
                              param_dtype == PULSE_DTYPE_BF16, (flags & PULSE_NORM_RMS) != 0};
  return hip_status(pulse::launch_block_norm(dtype == PULSE_DTYPE_BF16, p, (hipStream_t)stream),
                    "block_norm launch");
}

size_t pulse_block_norm_workspace_bytes(uint32_t cols) {
  return (size_t)pulse::kBlockNormBlocks * cols * 4 * sizeof(float);
}

int pulse_block_norm_backward(int dtype, const void* dy, uint64_t dy_stride, const void* dh_out,
                              uint64_t dh_out_stride, const void* b, uint64_t b_stride, const void* h_out,
                              uint64_t h_out_stride, float residual_scale, int param_dtype, const void* weight,
                              const void* post_weight, const void* post_bias, const void* gate,
                              const float* stats, uint64_t stats_stride, void* db, uint64_t db_stride, void* dh,
                              uint64_t dh_stride, float* dweight, float* dbias, float* dpost_weight,
                              float* dpost_bias, float* dgate, uint64_t rows, uint32_t cols, uint32_t flags,
                              void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "block_norm backward";
  if (int rc = check_block_norm(who, dtype, param_dtype, rows, cols, flags, residual_scale, weight, post_weight,
                                post_bias, gate, stats, stats_stride))
    return rc;
  if (rows && !stats) return fail(PULSE_EINVAL, "%s: stats is NULL", who);
  if (int rc = check_matrix(who, "dy", dy, dy_stride, rows, cols)) return rc;
  if (dh_out)
    if (int rc = check_matrix(who, "dh_out", dh_out, dh_out_stride, rows, cols)) return rc;
  const bool reads_b = post_weight || gate;
  if (reads_b)
    if (int rc = check_matrix(who, "b", b, b_stride, rows, cols)) return rc;
  if (int rc = check_matrix(who, "h_out", h_out, h_out_stride, rows, cols)) return rc;
  if (int rc = check_matrix(who, "db", db, db_stride, rows, cols)) return rc;
  if (int rc = check_matrix(who, "dh", dh, dh_stride, rows, cols)) return rc;
  if (!dweight) return fail(PULSE_EINVAL, "%s: dweight is NULL", who);
  if ((dpost_weight || dpost_bias) && !post_weight)
    return fail(PULSE_EINVAL, "%s: dpost_weight or dpost_bias without post_weight", who);
  if (dgate && !gate) return fail(PULSE_EINVAL, "%s: dgate without gate", who);
  for (const void* v : {(const void*)dweight, (const void*)dbias, (const void*)dpost_weight,
                        (const void*)dpost_bias, (const void*)dgate})
    if (!aligned(v, 4)) return fail(PULSE_EALIGN, "%s: a parameter's gradient is not 4-byte aligned", who);
  if (int rc = check_space(who, workspace, workspace_bytes, pulse_block_norm_workspace_bytes(cols))) return rc;
  const bool biases = dbias || dpost_bias || (dgate && post_bias);
  pulse::BlockNormGradParams p = {dy, dy_stride, dh_out, dh_out_stride, reads_b ? b : nullptr, b_stride, h_out,
                                  h_out_stride, residual_scale, weight, post_weight, post_bias, gate, stats,
                                  stats_stride, db, db_stride, dh, dh_stride, dweight, dbias, dpost_weight,
                                  dpost_bias, dgate, (float*)workspace, rows, cols,
                                  param_dtype == PULSE_DTYPE_BF16, (flags & PULSE_NORM_RMS) != 0, biases};
  return hip_status(pulse::launch_block_norm_grad(dtype == PULSE_DTYPE_BF16, p, (hipStream_t)stream),
                    "block_norm backward launch");
}

size_t pulse_linear_ce_workspace_bytes(uint32_t tokens, uint32_t vocab, uint32_t hidden) {
  return tokens && ce_handles(tokens, vocab, hidden) ? pulse::linear_ce_bytes(tokens, vocab, hidden) : 0;
}

int pulse_linear_ce_forward(const uint16_t* x, uint64_t x_stride, const uint16_t* weight,
                            const int64_t* targets, uint32_t tokens, uint32_t vocab, uint32_t hidden,
                            float logit_scale, float* loss, float* lse, void* workspace,
                            size_t workspace_bytes, void* stream) {
  const char* who = "linear_ce forward";
  if (int rc = check_ce(who, x, x_stride, weight, targets, tokens, vocab, hidden, logit_scale, workspace,
                        workspace_bytes))
    return rc;
  if (tokens == 0) return ok();
  if (!loss || !lse) return fail(PULSE_EINVAL, "%s: loss or lse is NULL", who);
  if (!aligned(loss, 4) || !aligned(lse, 4)) return fail(PULSE_EALIGN, "%s: loss/lse not 4-byte aligned", who);
  pulse::LinearCeParams p = {x, x_stride, weight, targets, tokens, vocab, hidden, logit_scale, loss, lse};
  return hip_status(pulse::launch_linear_ce(p, (char*)workspace, (hipStream_t)stream), "linear_ce launch");
}

int pulse_linear_ce_backward(const uint16_t* x, uint64_t x_stride, const uint16_t* weight,
                             const int64_t* targets, uint32_t tokens, uint32_t vocab, uint32_t hidden,
                             float logit_scale, const float* lse, const float* dloss, uint16_t* dx,
                             uint64_t dx_stride, uint16_t* dweight, void* workspace,
                             size_t workspace_bytes, void* stream) {
  const char* who = "linear_ce backward";
  if (int rc = check_ce(who, x, x_stride, weight, targets, tokens, vocab, hidden, logit_scale, workspace,
                        workspace_bytes))
    return rc;
  if (!dweight) return fail(PULSE_EINVAL, "%s: dweight is NULL", who);
  if (!aligned16(dweight)) return fail(PULSE_EALIGN, "%s: dweight not 16-byte aligned", who);
  if (tokens == 0)
    return hip_status(pulse::launch_zero_bytes(dweight, (uint64_t)vocab * hidden * 2, (hipStream_t)stream),
                      "linear_ce launch");
  if (!lse || !dloss) return fail(PULSE_EINVAL, "%s: lse or dloss is NULL", who);
  if (!aligned(lse, 4) || !aligned(dloss, 4)) return fail(PULSE_EALIGN, "%s: lse/dloss not 4-byte aligned", who);
  if (int rc = check_matrix(who, "dx", dx, dx_stride, tokens, hidden)) return rc;
  pulse::LinearCeGradParams p = {x, x_stride, weight, targets, tokens, vocab, hidden, logit_scale, lse, dloss,
                                 dx, dx_stride, dweight};
  return hip_status(pulse::launch_linear_ce_grad(p, (char*)workspace, (hipStream_t)stream),
                    "linear_ce backward launch");
}

size_t pulse_verify_drafts_workspace_bytes(uint32_t batch, uint32_t drafts, uint32_t vocab) {
  return batch && verify_handles(batch, drafts, vocab) ? pulse::verify_workspace(batch, drafts, vocab) : 0;
}

int pulse_verify_drafts(int dtype, const void* target, uint64_t target_stride, const void* draft,
                        uint64_t draft_stride, const int64_t* tokens, const int32_t* lengths, const float* uniform,
                        uint32_t batch, uint32_t drafts, uint32_t vocab, double scale, double draft_scale,
                        int64_t* out, int32_t* count, float* logprob, void* workspace, size_t workspace_bytes,
                        void* stream) {
  const char* who = "verify_drafts";
  if (dtype != PULSE_DTYPE_F32 && dtype != PULSE_DTYPE_BF16)
    return fail(PULSE_EINVAL, "%s: dtype %d is neither F32 nor BF16", who, dtype);
  if (!verify_handles(batch, drafts, vocab))
    return fail(PULSE_EINVAL, "%s: %u sequences of %u drafts, vocabulary of %u", who, batch, drafts, vocab);
  for (double v : {scale, draft_scale})
    if (!(v >= 1e-100 && v <= 1e100)) return fail(PULSE_EINVAL, "%s: a scale is not from 1e-100 to 1e100", who);
  if (batch == 0) return ok();
  // rows are read from any element on
  const uintptr_t size = dtype == PULSE_DTYPE_BF16 ? 2 : 4;
  if (!target || (drafts && !tokens) || !uniform) return fail(PULSE_EINVAL, "%s: target, tokens or uniform is NULL", who);
  if (!out || !count || !logprob) return fail(PULSE_EINVAL, "%s: out, count or logprob is NULL", who);
  if (target_stride < vocab || target_stride > (1ull << 40) ||
      (draft && (draft_stride < vocab || draft_stride > (1ull << 40))))
    return fail(PULSE_EINVAL, "%s: row strides %llu and %llu for a vocabulary of %u", who,
                (unsigned long long)target_stride, (unsigned long long)draft_stride, vocab);
  if (!aligned(target, size) || !aligned(draft, size) || !aligned(tokens, 8) || !aligned(out, 8) ||
      !aligned(lengths, 4) || !aligned(uniform, 4) || !aligned(count, 4) || !aligned(logprob, 4))
    return fail(PULSE_EALIGN, "%s: a pointer is not aligned to its elements", who);
  if (int rc = check_space(who, workspace, workspace_bytes, pulse::verify_workspace(batch, drafts, vocab))) return rc;
  const double log2e = 1.4426950408889634;
  pulse::VerifyParams p = {};
  p.target = target;
  p.target_stride = target_stride;
  p.draft = drafts ? draft : nullptr;
  p.draft_stride = draft_stride;
  p.tokens = tokens;
  p.lengths = lengths;
  p.uniform = uniform;
  p.batch = batch;
  p.drafts = drafts;
  p.vocab = vocab;
  p.scale = scale;
  p.by = scale * log2e;
  p.draft_by = draft_scale * log2e;
  p.floor = -1000.0 / p.by;
  p.draft_floor = -1000.0 / p.draft_by;
  p.out = out;
  p.count = count;
  p.logprob = logprob;
  return hip_status(pulse::launch_verify(dtype == PULSE_DTYPE_BF16, p, (char*)workspace, (hipStream_t)stream),
                    "verify_drafts launch");
}

int pulse_lowp_matmul(int dtype, const uint8_t* codes, const uint8_t* scales, float inv_scale,
                      uint32_t rows, uint32_t cols, const uint16_t* x, uint64_t x_stride,
                      uint32_t tokens, int y_dtype, void* y, uint64_t y_stride, void* stream) {
  const char* who = "lowp matmul";
  if (int rc = check_lowp(who, dtype, codes, scales, inv_scale, rows, cols, x, x_stride, tokens, y_dtype, y, y_stride))
    return rc;
  if (tokens == 0) return ok();
  return hip_status(pulse::launch_lowp_matmul(dtype == PULSE_DTYPE_MXFP4 ? pulse::kWeightMxfp4 : pulse::kWeightFp8, false,
                                              lowp_params(dtype, codes, scales, inv_scale, rows, cols, x, x_stride,
                                                          tokens, y_dtype, y, y_stride),
                                              (hipStream_t)stream),
                    "lowp matmul launch");
}

int pulse_lowp_linear(int dtype, const uint8_t* codes, const uint8_t* scales, float inv_scale, uint32_t rows,
                      uint32_t cols, const uint16_t* x, uint64_t x_stride, uint32_t tokens, int bias_dtype,
                      const void* bias, int activation, const void* times, uint64_t times_stride,
                      const void* residual, uint64_t residual_stride, int y_dtype, void* y, uint64_t y_stride,
                      void* stream) {
  const char* who = "lowp linear";
  if (int rc = check_lowp(who, dtype, codes, scales, inv_scale, rows, cols, x, x_stride, tokens, y_dtype, y, y_stride))
    return rc;
  pulse::Epilogue e;
  if (int rc = check_epilogue(who, rows, tokens, bias_dtype, bias, activation, times, times_stride, residual,
                              residual_stride, y_dtype, y, y_stride, e))
    return rc;
  if (tokens == 0) return ok();
  pulse::LowpMatmulParams p = lowp_params(dtype, codes, scales, inv_scale, rows, cols, x, x_stride, tokens, y_dtype, y,
                                          y_stride);
  p.e = e;
  return hip_status(pulse::launch_lowp_matmul(dtype == PULSE_DTYPE_MXFP4 ? pulse::kWeightMxfp4 : pulse::kWeightFp8, true,
                                              p, (hipStream_t)stream),
                    "lowp linear launch");
}

size_t pulse_linear_workspace_bytes(uint32_t tokens, uint32_t rows, uint32_t cols) {
  return tokens && linear_handles(tokens, rows, cols) ? pulse::linear_bytes(tokens, rows, cols) : 0;
}

int pulse_linear_forward(const uint16_t* x, uint64_t x_stride, const uint16_t* weight, uint32_t tokens, uint32_t rows,
                         uint32_t cols, int bias_dtype, const void* bias, int activation, const void* times,
                         uint64_t times_stride, const void* residual, uint64_t residual_stride, int y_dtype, void* y,
                         uint64_t y_stride, void* pre, uint64_t pre_stride, void* workspace, size_t workspace_bytes,
                         void* stream) {
  const char* who = "linear forward";
  if (int rc = check_linear(who, true, x, x_stride, weight, tokens, rows, cols, workspace, workspace_bytes)) return rc;
  if (y_dtype != PULSE_DTYPE_F32 && y_dtype != PULSE_DTYPE_BF16)
    return fail(PULSE_EINVAL, "%s: y_dtype %d is neither F32 nor BF16", who, y_dtype);
  if (int rc = check_matrix(who, "y", y, y_stride, tokens, rows)) return rc;
  pulse::LinearParams p = {x, x_stride, weight, tokens, rows, cols, y, y_stride, {}};
  if (int rc = check_epilogue(who, rows, tokens, bias_dtype, bias, activation, times, times_stride, residual,
                              residual_stride, y_dtype, y, y_stride, p.e))
    return rc;
  if (pre)
    if (int rc = check_matrix(who, "pre", pre, pre_stride, tokens, rows)) return rc;
  if (tokens == 0) return ok();
  p.e.pre = pre;
  p.e.pre_stride = pre_stride;
  return hip_status(pulse::launch_linear(p, (char*)workspace, (hipStream_t)stream), "linear launch");
}

int pulse_linear_backward(int dtype, const void* dy, uint64_t dy_stride, const uint16_t* x, uint64_t x_stride,
                          const uint16_t* weight, const void* pre, uint64_t pre_stride, int activation,
                          const void* times, uint64_t times_stride, uint32_t tokens, uint32_t rows, uint32_t cols,
                          uint16_t* dx, uint64_t dx_stride, uint16_t* dweight, float* dbias, void* dtimes,
                          uint64_t dtimes_stride, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "linear backward";
  if (dtype != PULSE_DTYPE_F32 && dtype != PULSE_DTYPE_BF16)
    return fail(PULSE_EINVAL, "%s: dtype %d is neither F32 nor BF16", who, dtype);
  if (activation < 0 || activation >= pulse::kActs)
    return fail(PULSE_EINVAL, "%s: activation %d is not known", who, activation);
  if (int rc = check_linear(who, false, x, x_stride, weight, tokens, rows, cols, workspace, workspace_bytes)) return rc;
  if (!dweight) return fail(PULSE_EINVAL, "%s: dweight is NULL", who);
  if (!aligned16(dweight)) return fail(PULSE_EALIGN, "%s: dweight not 16-byte aligned", who);
  if (!aligned(dbias, 4)) return fail(PULSE_EALIGN, "%s: dbias not 4-byte aligned", who);
  if (tokens == 0) {
    hipError_t e = pulse::launch_zero_bytes(dweight, (uint64_t)rows * cols * 2, (hipStream_t)stream);
    if (e == hipSuccess && dbias) e = pulse::launch_zero_bytes(dbias, (uint64_t)rows * 4, (hipStream_t)stream);
    return hip_status(e, "linear backward launch");
  }
  if (int rc = check_matrix(who, "dy", dy, dy_stride, tokens, rows)) return rc;
  if (activation || times)
    if (int rc = check_matrix(who, "pre", pre, pre_stride, tokens, rows)) return rc;
  if (times)
    if (int rc = check_matrix(who, "times", times, times_stride, tokens, rows)) return rc;
  if (dtimes && !times) return fail(PULSE_EINVAL, "%s: dtimes without times", who);
  if (dtimes)
    if (int rc = check_matrix(who, "dtimes", dtimes, dtimes_stride, tokens, rows)) return rc;
  if (int rc = check_matrix(who, "dx", dx, dx_stride, tokens, cols)) return rc;
  pulse::LinearGradParams p = {dy, dy_stride, x, x_stride, weight, pre, pre_stride, times, times_stride, activation,
                               dtype == PULSE_DTYPE_BF16, tokens, rows, cols, dx, dx_stride, dweight, dbias, dtimes,
                               dtimes_stride};
  return hip_status(pulse::launch_linear_grad(p, (char*)workspace, (hipStream_t)stream), "linear backward launch");
}

}  // extern "C"
