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

int pulse_lowp_matmul(int dtype, const uint8_t* codes, const uint8_t* scales, float inv_scale,
                      uint32_t rows, uint32_t cols, const uint16_t* x, uint64_t x_stride,
                      uint32_t tokens, int y_dtype, void* y, uint64_t y_stride, void* stream) {
  const char* who = "lowp matmul";
  const bool mx = dtype == PULSE_DTYPE_MXFP4;
  if (!mx && dtype != PULSE_DTYPE_FP8_E4M3)
    return fail(PULSE_EINVAL, "%s: dtype %d is neither FP8_E4M3 nor MXFP4", who, dtype);
  if (y_dtype != PULSE_DTYPE_F32 && y_dtype != PULSE_DTYPE_BF16)
    return fail(PULSE_EINVAL, "%s: y_dtype %d is neither F32 nor BF16", who, y_dtype);
  if (rows == 0 || rows > 0x7FFFFFFFu || cols == 0 || cols > 0x7FFFFFFFu)
    return fail(PULSE_EINVAL, "%s: a weight of %u x %u", who, rows, cols);
  if (tokens > 1u << 20) return fail(PULSE_EINVAL, "%s: more than 2^20 tokens", who);
  if (tokens == 0) return ok();
  if (!codes) return fail(PULSE_EINVAL, "%s: codes is NULL", who);
  if (mx && !scales) return fail(PULSE_EINVAL, "%s: scales is NULL", who);
  if (!aligned(codes, mx ? 4 : 8)) return fail(PULSE_EALIGN, "%s: codes not %d-byte aligned", who, mx ? 4 : 8);
  if (!mx && !(inv_scale - inv_scale == 0.0f && inv_scale != 0.0f))
    return fail(PULSE_EINVAL, "%s: inv_scale is zero or not finite", who);
  if (int rc = check_matrix(who, "x", x, x_stride, tokens, cols)) return rc;
  if (int rc = check_matrix(who, "y", y, y_stride, tokens, rows)) return rc;
  const uint64_t n = (uint64_t)rows * cols;
  pulse::LowpMatmulParams p = {codes, scales, inv_scale, rows, cols, mx ? (n + 1) / 2 : n, (n + 31) / 32,
                               x, x_stride, tokens, y, y_stride, y_dtype == PULSE_DTYPE_BF16};
  return hip_status(pulse::launch_lowp_matmul(mx, p, (hipStream_t)stream), "lowp matmul launch");
}

}  // extern "C"
