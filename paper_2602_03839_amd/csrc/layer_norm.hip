// layer_norm.hip -- layer norm and RMS norm, forward and backward.
//
// A row lies in the registers of G lanes, E elements each, so that x (and dy)
// are read once: the mean, then the sum of squares about it, then the result.
// Both passes are bound by HBM: forward x in, y out; backward x and dy in, dx
// out.
//
// The gradients of weight and bias are sums down the columns.  A lane owns the
// same columns of every row that its block takes, so it keeps their sums in
// registers over all its rows; each block writes one row of sums to the
// workspace and a second kernel adds those.  No atomics: the order of each sum
// is fixed by the sizes alone.
#include <type_traits>

#include "device_common.hpp"
#include "head.hpp"

namespace pulse {

namespace {

template <typename T>
constexpr bool kIsBf16 = std::is_same<T, uint16_t>::value;

__device__ __forceinline__ float from_bits(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float from_bits(float v) { return v; }

__device__ __forceinline__ void load8(const uint16_t* p, float* v) {
  const uint4 a = load16(p);
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

__device__ __forceinline__ void load8(const float* p, float* v) {
  const uint4 a = load16(p), b = load16(p + 4);
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
}

__device__ __forceinline__ void store8(uint16_t* p, const float* v) {
  uint4 o;
  o.x = bf16x2_rne(__float_as_uint(v[0]), __float_as_uint(v[1]));
  o.y = bf16x2_rne(__float_as_uint(v[2]), __float_as_uint(v[3]));
  o.z = bf16x2_rne(__float_as_uint(v[4]), __float_as_uint(v[5]));
  o.w = bf16x2_rne(__float_as_uint(v[6]), __float_as_uint(v[7]));
  store16(p, o);
}

__device__ __forceinline__ void store8(float* p, const float* v) {
#pragma unroll
  for (int i = 0; i < 8; i += 4)
    store16(p + i, make_uint4(__float_as_uint(v[i]), __float_as_uint(v[i + 1]),
                              __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3])));
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

  template <typename T>
  static __device__ __forceinline__ void load(const T* p, uint32_t cols, uint32_t t, float (&v)[E]) {
#pragma unroll
    for (int j = 0; j < E / kStep; ++j) {
      const uint32_t c = at(j, t);
      if (c < cols) {
        if constexpr (VEC) load8(p + c, v + 8 * j);
        else v[j] = from_bits(p[c]);
      } else {
#pragma unroll
        for (int i = 0; i < kStep; ++i) v[kStep * j + i] = 0.0f;
      }
    }
  }
  template <typename T>
  static __device__ __forceinline__ void store(T* p, uint32_t cols, uint32_t t, const float (&v)[E]) {
#pragma unroll
    for (int j = 0; j < E / kStep; ++j) {
      const uint32_t c = at(j, t);
      if (c < cols) {
        if constexpr (VEC) store8(p + c, v + 8 * j);
        else store1(p + c, v[j]);
      }
    }
  }
  static __device__ __forceinline__ bool in(int e, uint32_t cols, uint32_t t) {
    return at(e / kStep, t) < cols;
  }
  static __device__ __forceinline__ void params(const void* p, int bf16, uint32_t cols, uint32_t t,
                                                float (&v)[E]) {
    if (bf16) load((const uint16_t*)p, cols, t, v);
    else load((const float*)p, cols, t, v);
  }
};

constexpr int block_of(int g) { return g < 256 ? 256 : g; }

// The G lanes' sum of v in each of them (G a multiple of 64; `s` holds one
// float per wave and is free again after the next call's first barrier, so
// callers alternate between two).
template <int G>
__device__ __forceinline__ float group_sum(float v, float* s) {
  v = wave_sum(v);
  if constexpr (G == 64) return v;
  const int wave = threadIdx.x >> 6;
  if (lane_id() == 0) s[wave] = v;
  __syncthreads();
  float r = 0.0f;
#pragma unroll
  for (int i = 0; i < G / 64; ++i) r += s[i];
  return r;
}

template <typename T, int E, int G, bool VEC>
__global__ __launch_bounds__(block_of(G)) void norm_kernel(NormParams p) {
  typedef Row<E, G, VEC> R;
  constexpr int kRows = block_of(G) / G;
  __shared__ float s[2][16];
  const uint32_t t = threadIdx.x % G;
  const uint64_t row = (uint64_t)blockIdx.x * kRows + threadIdx.x / G;
  if (row >= p.rows) return;  // whole waves: G is 64 where a block has several rows
  const float inv_n = 1.0f / (float)p.cols;
  float v[E];
  R::load((const T*)p.x + row * p.x_stride, p.cols, t, v);
  float mean = 0.0f;
  if (p.mean) {
    float a = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) a += v[e];
    mean = group_sum<G>(a, s[0]) * inv_n;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = R::in(e, p.cols, t) ? v[e] - mean : 0.0f;
  }
  float q = 0.0f;
#pragma unroll
  for (int e = 0; e < E; ++e) q = __builtin_fmaf(v[e], v[e], q);
  const float rstd = 1.0f / __builtin_sqrtf(group_sum<G>(q, s[1]) * inv_n + p.eps);
  float w[E];
  R::params(p.weight, p.param_bf16, p.cols, t, w);
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = v[e] * rstd * w[e];
  if (p.bias) {
    R::params(p.bias, p.param_bf16, p.cols, t, w);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] += w[e];
  }
  R::store((T*)p.y + row * p.y_stride, p.cols, t, v);
  if (t == 0) {
    if (p.mean) p.mean[row] = mean;
    p.rstd[row] = rstd;
  }
}

template <typename T, int E, int G, bool VEC>
__global__ __launch_bounds__(block_of(G)) void norm_grad_kernel(NormGradParams p) {
  typedef Row<E, G, VEC> R;
  constexpr int kRows = block_of(G) / G;
  __shared__ float s[2][2][16];
  const uint32_t t = threadIdx.x % G;
  const uint64_t first = (uint64_t)blockIdx.x * kRows + threadIdx.x / G;
  const float inv_n = 1.0f / (float)p.cols;
  float w[E], dw[E], db[E];
  R::params(p.weight, p.param_bf16, p.cols, t, w);
#pragma unroll
  for (int e = 0; e < E; ++e) dw[e] = db[e] = 0.0f;
  int turn = 0;
  for (uint64_t row = first; row < p.rows; row += (uint64_t)gridDim.x * kRows, turn ^= 1) {
    float x[E], dy[E];
    R::load((const T*)p.x + row * p.x_stride, p.cols, t, x);
    R::load((const T*)p.dy + row * p.dy_stride, p.cols, t, dy);
    const float rstd = p.rstd[row], mean = p.mean ? p.mean[row] : 0.0f;
    float sa = 0.0f, sax = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      x[e] = (x[e] - mean) * rstd;  // past the row: meets dy = w = 0
      dw[e] = __builtin_fmaf(dy[e], x[e], dw[e]);
      db[e] += dy[e];
      dy[e] *= w[e];
      sa += dy[e];
      sax = __builtin_fmaf(dy[e], x[e], sax);
    }
    sax = group_sum<G>(sax, s[turn][0]) * inv_n;
    sa = p.mean ? group_sum<G>(sa, s[turn][1]) * inv_n : 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = (dy[e] - sa - x[e] * sax) * rstd;
    R::store((T*)p.dx + row * p.dx_stride, p.cols, t, x);
  }
  // one row of sums for each group of lanes
  const uint64_t mine = first, all = (uint64_t)gridDim.x * kRows;
  float* out = p.partial + mine * p.cols;
  R::store(out, p.cols, t, dw);
  if (p.dbias) R::store(out + all * p.cols, p.cols, t, db);
}

// The sums of the n partial rows: 64 columns a block, its 16 waves a slice of
// the rows each.
__global__ __launch_bounds__(1024) void norm_columns_kernel(const float* partial, uint32_t n,
                                                            uint32_t cols, float* dweight,
                                                            float* dbias) {
  __shared__ float s[16][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint32_t c = blockIdx.x * 64 + lane;
  const float* from = partial + (blockIdx.y ? (uint64_t)n * cols : 0);
  float a = 0.0f;
  if (c < cols) {
#pragma unroll 4
    for (uint32_t r = wave; r < n; r += 16) a += from[(uint64_t)r * cols + c];
  }
  s[wave][lane] = a;
  __syncthreads();
  if (wave == 0 && c < cols) {
    a = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) a += s[i][lane];
    (blockIdx.y ? dbias : dweight)[c] = a;
  }
}

template <typename F>
void by_shape(uint32_t cols, F f) {
  typedef std::integral_constant<int, 8> E8;
  typedef std::integral_constant<int, 16> E16;
  typedef std::integral_constant<int, 64> G64;
  typedef std::integral_constant<int, 256> G256;
  typedef std::integral_constant<int, 1024> G1024;
  if (cols <= 512) f(E8{}, G64{});
  else if (cols <= 1024) f(E16{}, G64{});
  else if (cols <= 2048) f(E8{}, G256{});
  else if (cols <= 4096) f(E16{}, G256{});
  else if (cols <= 8192) f(E8{}, G1024{});
  else f(E16{}, G1024{});
}

}  // namespace

hipError_t launch_layer_norm(bool bf16, const NormParams& p, hipStream_t stream) {
  const bool vec = p.cols % 8 == 0 && p.x_stride % 8 == 0 && p.y_stride % 8 == 0;
  by_shape(p.cols, [&](auto e, auto g) {
    constexpr int E = decltype(e)::value, G = decltype(g)::value;
    const dim3 block(block_of(G)), grid((uint32_t)((p.rows + block_of(G) / G - 1) / (block_of(G) / G)));
    if (bf16) {
      if (vec) hipLaunchKernelGGL((norm_kernel<uint16_t, E, G, true>), grid, block, 0, stream, p);
      else hipLaunchKernelGGL((norm_kernel<uint16_t, E, G, false>), grid, block, 0, stream, p);
    } else {
      if (vec) hipLaunchKernelGGL((norm_kernel<float, E, G, true>), grid, block, 0, stream, p);
      else hipLaunchKernelGGL((norm_kernel<float, E, G, false>), grid, block, 0, stream, p);
    }
  });
  return hipGetLastError();
}

hipError_t launch_layer_norm_grad(bool bf16, const NormGradParams& p, hipStream_t stream) {
  const bool vec = p.cols % 8 == 0 && p.x_stride % 8 == 0 && p.dy_stride % 8 == 0 && p.dx_stride % 8 == 0;
  uint32_t sums = 0;
  by_shape(p.cols, [&](auto e, auto g) {
    constexpr int E = decltype(e)::value, G = decltype(g)::value;
    constexpr uint32_t kRows = block_of(G) / G;
    uint64_t blocks = (p.rows + kRows - 1) / kRows;
    if (blocks > kNormBlocks / kRows) blocks = kNormBlocks / kRows;
    sums = (uint32_t)blocks * kRows;
    if (blocks == 0) return;
    const dim3 block(block_of(G)), grid((uint32_t)blocks);
    if (bf16) {
      if (vec) hipLaunchKernelGGL((norm_grad_kernel<uint16_t, E, G, true>), grid, block, 0, stream, p);
      else hipLaunchKernelGGL((norm_grad_kernel<uint16_t, E, G, false>), grid, block, 0, stream, p);
    } else {
      if (vec) hipLaunchKernelGGL((norm_grad_kernel<float, E, G, true>), grid, block, 0, stream, p);
      else hipLaunchKernelGGL((norm_grad_kernel<float, E, G, false>), grid, block, 0, stream, p);
    }
  });
  if (hipError_t e = hipGetLastError()) return e;
  hipLaunchKernelGGL(norm_columns_kernel, dim3((p.cols + 63) / 64, p.dbias ? 2 : 1), dim3(1024), 0,
                     stream, p.partial, sums, p.cols, p.dweight, p.dbias);
  return hipGetLastError();
}

}  // namespace pulse
