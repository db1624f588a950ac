// norm_rows.hpp -- how the norms hold a row: in the registers of G lanes, E elements
// each, groups of 8 side by side (rows of 16-byte groups, or any rows) or element by
// element, and the sums over those lanes.
#pragma once

#include <type_traits>

#include "device_common.hpp"
#include "head.hpp"

namespace pulse {

namespace {

template <typename T>
constexpr bool kIsBf16 = std::is_same<T, uint16_t>::value;

__device__ __forceinline__ float from_bits(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float from_bits(float v) { return v; }

// 8 elements as they lie in memory, and as FP32.
template <typename T>
struct Raw8 {
  uint4 v[sizeof(T) / 2];
};

template <bool STREAM, typename T>
__device__ __forceinline__ void load8(const T* p, Raw8<T>& r) {
#pragma unroll
  for (size_t i = 0; i < sizeof(T) / 2; ++i)
    r.v[i] = STREAM ? load16_stream(p + 16 / sizeof(T) * i) : load16(p + 16 / sizeof(T) * i);
}

__device__ __forceinline__ void unpack8(const Raw8<uint16_t>& r, float* v) {
  const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

__device__ __forceinline__ void unpack8(const Raw8<float>& r, float* v) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(get_u32(r.v[i / 4], i & 3));
}

template <bool STREAM>
__device__ __forceinline__ void store8(uint16_t* p, const float* v) {
  uint4 o;
  o.x = bf16x2_rne(__float_as_uint(v[0]), __float_as_uint(v[1]));
  o.y = bf16x2_rne(__float_as_uint(v[2]), __float_as_uint(v[3]));
  o.z = bf16x2_rne(__float_as_uint(v[4]), __float_as_uint(v[5]));
  o.w = bf16x2_rne(__float_as_uint(v[6]), __float_as_uint(v[7]));
  if (STREAM) store16_stream(p, o);
  else store16(p, o);
}

template <bool STREAM>
__device__ __forceinline__ void store8(float* p, const float* v) {
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    const uint4 o = make_uint4(__float_as_uint(v[i]), __float_as_uint(v[i + 1]),
                               __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3]));
    if (STREAM) store16_stream(p + i, o);
    else store16(p + i, o);
  }
}

__device__ __forceinline__ void store1(uint16_t* p, float v) {
  *p = (uint16_t)bf16x2_rne(__float_as_uint(v), 0u);
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }

// Where a lane's elements lie in the row: groups of 8, G lanes side by side
// (VEC), or single elements.  A group beyond the row holds zeros; `in` tells.
template <int E, int G, bool VEC>
struct Row {
  static constexpr int kStep = VEC ? 8 : 1;
  static __device__ __forceinline__ uint32_t at(int j, uint32_t t) { return (uint32_t)(j * G + t) * kStep; }

  // a row's elements as they lie in memory, zeros past its end
  template <typename T>
  struct Raw {
    typename std::conditional<VEC, Raw8<T>, T>::type v[E / kStep];
  };
  template <bool STREAM, typename T>
  static __device__ __forceinline__ void load(const T* p, uint32_t cols, uint32_t t, Raw<T>& r) {
#pragma unroll
    for (int j = 0; j < E / kStep; ++j) {
      const uint32_t c = at(j, t);
      if constexpr (VEC) {
        if (c < cols) load8<STREAM>(p + c, r.v[j]);
        else
#pragma unroll
          for (size_t i = 0; i < sizeof(T) / 2; ++i) r.v[j].v[i] = make_uint4(0, 0, 0, 0);
      } else {
        r.v[j] = c < cols ? p[c] : (T)0;
      }
    }
  }
  template <typename T>
  static __device__ __forceinline__ void unpack(const Raw<T>& r, float (&v)[E]) {
#pragma unroll
    for (int j = 0; j < E / kStep; ++j) {
      if constexpr (VEC) unpack8(r.v[j], v + 8 * j);
      else v[j] = from_bits(r.v[j]);
    }
  }
  template <bool STREAM, typename T>
  static __device__ __forceinline__ void load(const T* p, uint32_t cols, uint32_t t, float (&v)[E]) {
    Raw<T> r;
    load<STREAM>(p, cols, t, r);
    unpack(r, v);
  }
  template <bool STREAM = false, typename T>
  static __device__ __forceinline__ void store(T* p, uint32_t cols, uint32_t t, const float (&v)[E]) {
#pragma unroll
    for (int j = 0; j < E / kStep; ++j) {
      const uint32_t c = at(j, t);
      if (c < cols) {
        if constexpr (VEC) store8<STREAM>(p + c, v + 8 * j);
        else store1(p + c, v[j]);
      }
    }
  }
  static __device__ __forceinline__ bool in(int e, uint32_t cols, uint32_t t) {
    return at(e / kStep, t) < cols;
  }
  static __device__ __forceinline__ void params(const void* p, int bf16, uint32_t cols, uint32_t t,
                                                float (&v)[E]) {
    if (bf16) load<false>((const uint16_t*)p, cols, t, v);
    else load<false>((const float*)p, cols, t, v);
  }
};

// Groups of 8 of a row of any length and alignment: loaded 16 bytes at a time wherever
// they lie, but for the row's last one, which may be cut short.
template <int E, int G>
struct AnyRow {
  static __device__ __forceinline__ uint32_t at(int j, uint32_t t) { return (uint32_t)(j * G + t) * 8; }

  template <typename T>
  struct Raw {
    Raw8<T> v[E / 8];
  };
  template <bool STREAM, typename T>
  static __device__ __forceinline__ void load(const T* p, uint32_t cols, uint32_t t, Raw<T>& r) {
    constexpr int kPer = 16 / sizeof(T);
#pragma unroll
    for (int j = 0; j < E / 8; ++j) {
      const uint32_t c = at(j, t);
      if (c + 8 <= cols) {
#pragma unroll
        for (size_t i = 0; i < sizeof(T) / 2; ++i) r.v[j].v[i] = load16_any(p + c + kPer * i);
        continue;
      }
      uint32_t w[2 * sizeof(T)] = {};
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i)
        if (c + i < cols) {
          if constexpr (sizeof(T) == 2) w[i >> 1] |= (uint32_t)p[c + i] << (16 * (i & 1));
          else w[i] = __float_as_uint(p[c + i]);
        }
#pragma unroll
      for (size_t i = 0; i < sizeof(T) / 2; ++i)
        r.v[j].v[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    }
  }
  template <typename T>
  static __device__ __forceinline__ void unpack(const Raw<T>& r, float (&v)[E]) {
#pragma unroll
    for (int j = 0; j < E / 8; ++j) unpack8(r.v[j], v + 8 * j);
  }
  static __device__ __forceinline__ void store_group(uint16_t* p, uint32_t left, const float* v) {
    uint4 o;
    o.x = bf16x2_rne(__float_as_uint(v[0]), __float_as_uint(v[1]));
    o.y = bf16x2_rne(__float_as_uint(v[2]), __float_as_uint(v[3]));
    o.z = bf16x2_rne(__float_as_uint(v[4]), __float_as_uint(v[5]));
    o.w = bf16x2_rne(__float_as_uint(v[6]), __float_as_uint(v[7]));
    if (left >= 8) return store16_any(p, o);
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (i < left) p[i] = (uint16_t)(get_u32(o, i >> 1) >> (16 * (i & 1)));
  }
  static __device__ __forceinline__ void store_group(float* p, uint32_t left, const float* v) {
    if (left >= 8) {
#pragma unroll
      for (int i = 0; i < 8; i += 4)
        store16_any(p + i, make_uint4(__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]),
                                      __float_as_uint(v[i + 3])));
      return;
    }
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (i < left) p[i] = v[i];
  }
  template <bool STREAM = false, typename T>
  static __device__ __forceinline__ void store(T* p, uint32_t cols, uint32_t t, const float (&v)[E]) {
#pragma unroll
    for (int j = 0; j < E / 8; ++j) {
      const uint32_t c = at(j, t);
      if (c < cols) store_group(p + c, cols - c, v + 8 * j);
    }
  }
  static __device__ __forceinline__ bool in(int e, uint32_t cols, uint32_t t) { return at(e / 8, t) + e % 8 < cols; }
  static __device__ __forceinline__ void params(const void* p, int bf16, uint32_t cols, uint32_t t, float (&v)[E]) {
    if (bf16) {
      Raw<uint16_t> r;
      load<false>((const uint16_t*)p, cols, t, r);
      unpack(r, v);
    } else {
      Raw<float> r;
      load<false>((const float*)p, cols, t, r);
      unpack(r, v);
    }
  }
};

constexpr int block_of(int g) { return g < 256 ? 256 : g; }

// The G lanes' sums of two values in each of them, with one barrier (none for a
// wave).  `s` holds a pair per wave and is free again after the next call's barrier,
// so callers alternate between two.
template <int G>
__device__ __forceinline__ float2 group_sum2(float a, float b, float2* s) {
  a = wave_sum(a);
  b = wave_sum(b);
  if constexpr (G == 64) return make_float2(a, b);
  const int wave = threadIdx.x >> 6, first = wave & ~(G / 64 - 1);
  if (lane_id() == 0) s[wave] = make_float2(a, b);
  __syncthreads();
  float2 r = make_float2(0.0f, 0.0f);
#pragma unroll
  for (int i = 0; i < G / 64; ++i) {
    r.x += s[first + i].x;
    r.y += s[first + i].y;
  }
  return r;
}

}  // namespace

}  // namespace pulse
