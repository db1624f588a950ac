// head.hpp -- parameter blocks, launchers and device helpers of the operators
// at a model's output end (include/pulse_head.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace pulse {

// ---------------------------------------------------------------- norm

constexpr uint32_t kNormMaxCols = 16384;
constexpr uint32_t kNormBlocks = 512;  // blocks of the backward pass, each with its column sums

struct NormParams {
  const void* x;
  uint64_t x_stride;
  const void* weight;
  const void* bias;  // may be null
  void* y;
  uint64_t y_stride;
  float* mean;  // null: RMS form
  float* rstd;
  uint64_t rows;
  uint32_t cols;
  float eps;
  int param_bf16;
};

struct NormGradParams {
  const void* dy;
  uint64_t dy_stride;
  const void* x;
  uint64_t x_stride;
  const void* weight;
  const float* mean;  // null: RMS form
  const float* rstd;
  void* dx;
  uint64_t dx_stride;
  float* dweight;
  float* dbias;    // may be null
  float* partial;  // [blocks][cols] of dweight, then of dbias
  uint64_t rows;
  uint32_t cols;
  int param_bf16;
};

hipError_t launch_layer_norm(bool bf16, const NormParams& p, hipStream_t stream);
hipError_t launch_layer_norm_grad(bool bf16, const NormGradParams& p, hipStream_t stream);

// ---------------------------------------------------------------- block norm

constexpr uint32_t kBlockNormBlocks = 512;  // blocks of the backward pass, each with its column sums

struct BlockNormParams {
  const void* b;
  uint64_t b_stride;
  const void* h;
  uint64_t h_stride;
  float residual_scale;
  const void* weight;
  const void* bias;         // may be null
  const void* post_weight;  // null: b is not normalised
  const void* post_bias;    // may be null
  const void* gate;         // may be null
  void* y;
  uint64_t y_stride;
  void* h_out;  // h itself, or elsewhere
  uint64_t h_out_stride;
  float* stats;  // rows of rstd, post_rstd, mean, post_mean; null: not kept
  uint64_t stats_stride;
  uint64_t rows;
  uint32_t cols;
  float eps;
  int param_bf16;
  bool rms;
  bool stream;  // set by the launcher, as below
};

struct BlockNormGradParams {
  const void* dy;
  uint64_t dy_stride;
  const void* dh_out;  // null: zeros
  uint64_t dh_out_stride;
  const void* b;  // null where nothing asks for it: neither post norm nor gate
  uint64_t b_stride;
  const void* h_out;
  uint64_t h_out_stride;
  float residual_scale;
  const void* weight;
  const void* post_weight;
  const void* post_bias;
  const void* gate;
  const float* stats;
  uint64_t stats_stride;
  void* db;
  uint64_t db_stride;
  void* dh;
  uint64_t dh_stride;
  float* dweight;
  float* dbias;  // this and the following may be null
  float* dpost_weight;
  float* dpost_bias;
  float* dgate;
  float* partial;  // [blocks][cols] of dy xh, then of g bh, dy and g
  uint64_t rows;
  uint32_t cols;
  int param_bf16;
  bool rms, biases;  // biases: the sums of dy and g are asked for
  // set by the launcher
  bool stream;   // the results are more than the caches keep
  float* means;  // of wide rows: the means of a and of a xh
  uint64_t means_stride;
};

hipError_t launch_block_norm(bool bf16, const BlockNormParams& p, hipStream_t stream);
hipError_t launch_block_norm_grad(bool bf16, const BlockNormGradParams& p, hipStream_t stream);

// ---------------------------------------------------------------- products with an epilogue

enum Activation { kActNone, kActRelu, kActSilu, kActGelu, kActGeluTanh, kActs };

// y = act(product + bias) * times + residual; what is null is left out.  times, residual
// and pre are rows of y's type, [tokens][rows of the weight].
struct Epilogue {
  const void* bias;
  int bias_bf16;
  int act;
  const void* times;
  uint64_t times_stride;
  const void* residual;
  uint64_t residual_stride;
  void* pre;  // product + bias, kept for the gradient
  uint64_t pre_stride;
  int out_bf16;
};

// ---------------------------------------------------------------- few-token products

enum WeightForm { kWeightFp8, kWeightMxfp4, kWeightBf16 };

struct LowpMatmulParams {
  const uint8_t* codes;   // BF16: the weight itself
  const uint8_t* scales;  // MXFP4
  float inv_scale;        // FP8
  uint32_t rows, cols;
  uint64_t code_bytes, scale_bytes;
  const uint16_t* x;
  uint64_t x_stride;
  uint32_t tokens;
  void* y;
  uint64_t y_stride;
  int y_bf16;
  Epilogue e;
};

constexpr uint32_t kBf16Tokens = 16;  // the most that a BF16 weight is multiplied with here

// `epilogue`: e is looked at; always so for BF16 weights.
hipError_t launch_lowp_matmul(WeightForm form, bool epilogue, const LowpMatmulParams& p, hipStream_t stream);

// ---------------------------------------------------------------- linear

constexpr uint32_t kLinearFewTokens = 16;  // up to here the forward pass needs no workspace
static_assert(kLinearFewTokens <= kBf16Tokens, "they are launch_lowp_matmul's");

struct LinearParams {
  const uint16_t* x;
  uint64_t x_stride;
  const uint16_t* weight;
  uint32_t tokens, rows, cols;
  void* y;
  uint64_t y_stride;
  Epilogue e;
};

struct LinearGradParams {
  const void* dy;
  uint64_t dy_stride;
  const uint16_t* x;
  uint64_t x_stride;
  const uint16_t* weight;
  const void* pre;  // null: neither activation nor multiplier
  uint64_t pre_stride;
  const void* times;  // may be null
  uint64_t times_stride;
  int act, bf16;  // bf16: type of dy, pre, times and dtimes
  uint32_t tokens, rows, cols;
  uint16_t* dx;
  uint64_t dx_stride;
  uint16_t* dweight;
  float* dbias;  // may be null
  void* dtimes;  // may be null
  uint64_t dtimes_stride;
};

uint64_t linear_needs(bool forward, uint32_t tokens, uint32_t rows, uint32_t cols);  // one call's workspace
// a workspace for any call of up to `tokens` tokens
uint64_t linear_bytes(uint32_t tokens, uint32_t rows, uint32_t cols);
hipError_t launch_linear(const LinearParams& p, char* ws, hipStream_t stream);
hipError_t launch_linear_grad(const LinearGradParams& p, char* ws, hipStream_t stream);

// ---------------------------------------------------------------- cross entropy

constexpr uint32_t kCeMaxHidden = 65536;

struct LinearCeParams {
  const uint16_t* x;
  uint64_t x_stride;
  const uint16_t* weight;
  const int64_t* targets;
  uint32_t tokens, vocab, hidden;
  float logit_scale;
  float* loss;
  float* lse;
};

struct LinearCeGradParams {
  const uint16_t* x;
  uint64_t x_stride;
  const uint16_t* weight;
  const int64_t* targets;
  uint32_t tokens, vocab, hidden;
  float logit_scale;
  const float* lse;
  const float* dloss;
  uint16_t* dx;
  uint64_t dx_stride;
  uint16_t* dweight;
};

hipError_t launch_zero_bytes(void* p, uint64_t bytes, hipStream_t stream);  // an even number of them
uint64_t linear_ce_needs(uint32_t tokens, uint32_t vocab, uint32_t hidden);  // one call's workspace
// a workspace for any call of up to `tokens` tokens
uint64_t linear_ce_bytes(uint32_t tokens, uint32_t vocab, uint32_t hidden);
hipError_t launch_linear_ce(const LinearCeParams& p, char* ws, hipStream_t stream);
hipError_t launch_linear_ce_grad(const LinearCeGradParams& p, char* ws, hipStream_t stream);

// ---------------------------------------------------------------- drafts

constexpr uint32_t kVerifyMaxDrafts = 128;

struct VerifyPart {  // of a row's segment: the sum of exponentials below its largest logit
  double sum;
  float top;
};

// A row's distribution: entry z has the probability 2^((z - top) by) inv; all of them 0
// where inv is, that is, where the logits' exponentials have no finite positive sum.
struct VerifyRow {
  double by, inv;
  float top;
};

// What is decided for a sequence: the rows at its first draft that is not taken.
struct VerifyDecision {
  VerifyRow p, q;
  uint32_t taken, length;
};

struct VerifyParams {
  const void* target;  // [batch][drafts + 1] rows
  uint64_t target_stride;
  const void* draft;  // [batch][drafts] rows; null: q is 1 at the draft
  uint64_t draft_stride;
  const int64_t* tokens;   // [batch][drafts]
  const int32_t* lengths;  // [batch]; null: drafts of each
  const float* uniform;    // [batch][drafts + 1]
  uint32_t batch, drafts, vocab;
  double scale, by, draft_by;  // the latter log2(e) times the scales
  double floor, draft_floor;   // the difference of logits that these take to -1000
  int64_t* out;
  int32_t* count;
  float* logprob;
  // set by the launcher
  uint32_t rows;        // of a sequence
  uint32_t segments;    // of a row
  uint32_t rest_count;  // 512 entries each
  VerifyPart* parts;    // [batch][rows][segments]
  double* rests;        // [batch][rest_count]: sums of max(p - q, 0)
  VerifyDecision* decisions;
};

uint64_t verify_workspace(uint32_t batch, uint32_t drafts, uint32_t vocab);
hipError_t launch_verify(bool bf16, const VerifyParams& p, char* ws, hipStream_t stream);

// ---------------------------------------------------------------- device helpers

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// The wave's sum in every lane: within rows of 16 lanes by DPP, then the four
// rows' sums through scalar registers.  A fixed order, no LDS.
__device__ __forceinline__ float wave_sum(float v) {
  auto add = [&](auto ctrl) {
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xF,
                                                    0xF, true));
  };
  add(std::integral_constant<int, 0xB1>{});   // quad_perm 1,0,3,2
  add(std::integral_constant<int, 0x4E>{});   // quad_perm 2,3,0,1
  add(std::integral_constant<int, 0x141>{});  // row_half_mirror
  add(std::integral_constant<int, 0x140>{});  // row_mirror
  auto row = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };
  return (row(0) + row(16)) + (row(32) + row(48));
}

// 16 bytes at any address of a 2-byte type (such an access is one instruction here).
struct __attribute__((packed, aligned(2))) Unaligned16 {
  uint32_t w[4];
};

__device__ __forceinline__ uint4 load16_any(const void* p) {
  const Unaligned16 u = *reinterpret_cast<const Unaligned16*>(p);
  return make_uint4(u.w[0], u.w[1], u.w[2], u.w[3]);
}

__device__ __forceinline__ void store16_any(void* p, uint4 v) {
  *reinterpret_cast<Unaligned16*>(p) = Unaligned16{{v.x, v.y, v.z, v.w}};
}

}  // namespace pulse
