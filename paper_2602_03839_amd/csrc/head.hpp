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

// ---------------------------------------------------------------- low-bit products

struct LowpMatmulParams {
  const uint8_t* codes;
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
};

hipError_t launch_lowp_matmul(bool mxfp4, const LowpMatmulParams& p, hipStream_t stream);

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
