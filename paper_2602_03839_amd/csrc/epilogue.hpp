// epilogue.hpp -- what follows a product's sum before it is stored: bias, activation,
// multiplier and residual, in FP32 and in this order; and the activations' derivatives.
//
//   silu(v) = v s(v), s(v) = 1 / (1 + e^-v)
//   gelu(v) = v (1 + erf(v / sqrt 2)) / 2 = v erfc(-v / sqrt 2) / 2
//   gelu_tanh(v) = v (1 + tanh y) / 2 = v s(2 y), y = sqrt(2 / pi) (v + 0.044715 v^3)
// Exponentials and reciprocals are the hardware's (1 ulp each).  An exponential makes of its
// argument's rounding a relative error: silu is off by (6 + 2 |v|) 2^-24 of itself at most,
// gelu by (36 + 3 v^2) 2^-24, gelu_tanh by (6 + 12 |y|) 2^-24; what is below 2e-36 may be 0.
// (1 + erf cancels: 4% off at v = -5, and 0 from -5.5 on.  4,096 tokens, 4,864 x 896: 87 us
// with it, 95 with erfc; 18,944 x 3,584: 600 with either.)
#pragma once

#include <cfloat>

#include "device_common.hpp"
#include "head.hpp"

namespace pulse {

namespace {

__device__ __forceinline__ float sigmoid_of(float v) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * v));
}

constexpr float kGeluA = 0.7978845608028654f;  // sqrt(2 / pi)
constexpr float kGeluB = 0.044715f;

// The logistic function's argument for gelu_tanh, whose cube would overflow far from 0:
// from 30 on it is 0 or 1 in FP32 anyway.
__device__ __forceinline__ float near_zero(float v) { return __builtin_fminf(__builtin_fmaxf(v, -30.0f), 30.0f); }
__device__ __forceinline__ float gelu_tanh_gate(float v) {
  const float u = near_zero(v);
  return v == v ? sigmoid_of(2.0f * kGeluA * __builtin_fmaf(kGeluB * u * u, u, u)) : v;
}

// Factors beside one that is 0 where v is infinite: -inf and what is far below 0 give 0, the
// activations' limit there, and a slope has its limits 0 and 1 (a NaN comes from the other factor).
__device__ __forceinline__ float not_minus_inf(float v) { return __builtin_fmaxf(v, -FLT_MAX); }
__device__ __forceinline__ float not_inf(float v) { return __builtin_fminf(not_minus_inf(v), FLT_MAX); }

__device__ __forceinline__ float activate(int act, float v) {
  switch (act) {
    case kActRelu: return v < 0.0f ? 0.0f : v;  // a NaN stays one
    case kActSilu: return not_minus_inf(v) * sigmoid_of(v);
    case kActGelu: return 0.5f * not_minus_inf(v) * erfcf(-0.7071067811865476f * v);
    case kActGeluTanh: return not_minus_inf(v) * gelu_tanh_gate(v);
    default: return v;
  }
}

// An activation and its derivative.
__device__ __forceinline__ float2 activate2(int act, float v) {
  switch (act) {
    case kActRelu: return make_float2(v < 0.0f ? 0.0f : v, v > 0.0f ? 1.0f : v == v ? 0.0f : v);
    case kActSilu: {
      const float s = sigmoid_of(v);
      return make_float2(not_minus_inf(v) * s, s * __builtin_fmaf(not_inf(v), 1.0f - s, 1.0f));
    }
    case kActGelu: {
      const float h = 0.5f * erfcf(-0.7071067811865476f * v);
      const float d = 0.3989422804014327f * __builtin_amdgcn_exp2f(-0.7213475204444817f * v * v);
      return make_float2(not_minus_inf(v) * h, __builtin_fmaf(not_inf(v), d, h));
    }
    case kActGeluTanh: {
      const float s = gelu_tanh_gate(v), u = near_zero(v);
      const float y = 2.0f * kGeluA * __builtin_fmaf(3.0f * kGeluB * u, u, 1.0f);
      return make_float2(not_minus_inf(v) * s, __builtin_fmaf(u * s * (1.0f - s), y, s));
    }
    default: return make_float2(v, 1.0f);
  }
}

__device__ __forceinline__ float load_f32(const void* p, uint64_t at, int bf16) {
  return bf16 ? __uint_as_float((uint32_t)((const uint16_t*)p)[at] << 16) : ((const float*)p)[at];
}

// Four adjacent values from element `at` on, of which `left` are there (the others 0).
__device__ __forceinline__ f32x4_t load_four(const void* p, uint64_t at, int bf16, uint32_t left) {
  f32x4_t v = {0.0f, 0.0f, 0.0f, 0.0f};
  if (left >= 4 && at % 4 == 0) {
    if (!bf16) return *(const f32x4_t*)((const float*)p + at);
    const uint2 w = *(const uint2*)((const uint16_t*)p + at);
    return f32x4_t{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                   __uint_as_float(w.y & 0xFFFF0000u)};
  }
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i)
    if (i < left) v[i] = load_f32(p, at + i, bf16);
  return v;
}

// The four values from row `row` on of `rows` at element `at`.  (Of comparisons in 64 bits
// come the shorter stores: FP8 18,944 x 3,584, 5 tokens, 14.1 us from how many are left, 13.9 so.)
__device__ __forceinline__ void store_four(void* p, uint64_t at, int bf16, uint64_t row, uint64_t rows,
                                           f32x4_t v) {
  if (bf16) {
    uint16_t* const y = (uint16_t*)p + at;
    const uint2 o = make_uint2(bf16x2_rne(__float_as_uint(v[0]), __float_as_uint(v[1])),
                               bf16x2_rne(__float_as_uint(v[2]), __float_as_uint(v[3])));
    if (at % 4 == 0 && row + 4 <= rows) {
      *(uint2*)y = o;
    } else {
      const uint32_t w[2] = {o.x, o.y};
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
        if (row + i < rows) y[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
  } else {
    float* const y = (float*)p + at;
    if (at % 4 == 0 && row + 4 <= rows) {
      *(f32x4_t*)y = v;
    } else {
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
        if (row + i < rows) y[i] = v[i];
    }
  }
}

// The operands of the four features from `row` on of token t (`left` of them are there).
struct FourOperands {
  f32x4_t bias, times, residual;
};

__device__ __forceinline__ FourOperands load_operands(const Epilogue& e, uint64_t t, uint64_t row, uint32_t left) {
  FourOperands o = {};
  if (e.bias) o.bias = load_four(e.bias, row, e.bias_bf16, left);
  if (e.times) o.times = load_four(e.times, t * e.times_stride + row, e.out_bf16, left);
  if (e.residual) o.residual = load_four(e.residual, t * e.residual_stride + row, e.out_bf16, left);
  return o;
}

// What is stored as y; `pre`, if it is kept, is stored here.
__device__ __forceinline__ f32x4_t finish_four(const Epilogue& e, const FourOperands& o, f32x4_t v, uint64_t t,
                                               uint64_t row, uint32_t left) {
  if (e.bias) v += o.bias;
  if (e.pre) store_four(e.pre, t * e.pre_stride + row, e.out_bf16, 0, left, v);
  if (e.act) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = activate(e.act, v[i]);
  }
  if (e.times) v *= o.times;
  if (e.residual) v += o.residual;
  return v;
}

__device__ __forceinline__ float finish_one(const Epilogue& e, float v, uint64_t t, uint64_t row) {
  if (e.bias) v += load_f32(e.bias, row, e.bias_bf16);
  if (e.pre) {
    const uint64_t at = t * e.pre_stride + row;
    if (e.out_bf16) ((uint16_t*)e.pre)[at] = (uint16_t)bf16x2_rne(__float_as_uint(v), 0u);
    else ((float*)e.pre)[at] = v;
  }
  v = activate(e.act, v);
  if (e.times) v *= load_f32(e.times, t * e.times_stride + row, e.out_bf16);
  if (e.residual) v += load_f32(e.residual, t * e.residual_stride + row, e.out_bf16);
  return v;
}

}  // namespace

}  // namespace pulse
