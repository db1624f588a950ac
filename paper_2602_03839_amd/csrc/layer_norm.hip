// layer_norm.hip -- layer norm and RMS norm, forward and backward.
//
// A row lies in the registers of G lanes, E elements each, so that x (and dy)
// are read once: the mean, then the sum of squares about it, then the result.
// Both passes are bound by HBM: forward x in, y out; backward x and dy in, dx
// out.  Two forms fall short of that: the gradient of few rows reads x and dy a second
// time, from a cache (below), and that of rows of more than 8,192 elements keeps 31 (BF16)
// to 104 (FP32, element by element) of a lane's values in scratch memory, since 1,024
// threads have 128 registers each.
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
    if (bf16) load<false>((const uint16_t*)p, cols, t, v);
    else load<false>((const float*)p, cols, t, v);
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

// N rows at a time by each group of G lanes, and no loop: short-lived blocks.  Two rows
// share the parameters' loads and the barriers of their sums, and both are on their
// way at once; one where the rows are too few to fill the chip that way.
// 16,384 x 3,584 in BF16: 43 us with two (5.4 TB/s), 53 with one.
template <typename T, int E, int G, bool VEC, int N>
__global__ __launch_bounds__(block_of(G)) void norm_kernel(NormParams p) {
  typedef Row<E, G, VEC> R;
  constexpr int kRows = block_of(G) / G * N;
  __shared__ float2 s[2][16];
  const uint32_t t = threadIdx.x % G;
  const uint64_t row = (uint64_t)blockIdx.x * kRows + threadIdx.x / G * N;
  if (row >= p.rows) return;  // whole waves: G is 64 where a block has several groups
  const uint64_t last = p.rows - 1;
  const float inv_n = 1.0f / (float)p.cols;
  float v[N][E];
  {
    typename R::template Raw<T> raw[N];
#pragma unroll
    for (int k = 0; k < N; ++k)
      R::template load<true>((const T*)p.x + (row + k < p.rows ? row + k : last) * p.x_stride, p.cols, t, raw[k]);
#pragma unroll
    for (int k = 0; k < N; ++k) R::unpack(raw[k], v[k]);
  }
  float mean[2] = {0.0f, 0.0f}, a[2] = {0.0f, 0.0f};
  if (p.mean) {
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) a[k] += v[k][e];
    const float2 sum = group_sum2<G>(a[0], a[1], s[0]);
    mean[0] = sum.x * inv_n;
    mean[1] = sum.y * inv_n;
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) v[k][e] = R::in(e, p.cols, t) ? v[k][e] - mean[k] : 0.0f;
  }
  a[0] = a[1] = 0.0f;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) a[k] = __builtin_fmaf(v[k][e], v[k][e], a[k]);
  const float2 sum = group_sum2<G>(a[0], a[1], s[1]);
  const float rstd[2] = {1.0f / __builtin_sqrtf(sum.x * inv_n + p.eps), 1.0f / __builtin_sqrtf(sum.y * inv_n + p.eps)};
  float w[E];
  R::params(p.weight, p.param_bf16, p.cols, t, w);
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) v[k][e] = v[k][e] * rstd[k] * w[e];
  if (p.bias) {
    R::params(p.bias, p.param_bf16, p.cols, t, w);
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) v[k][e] += w[e];
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    if (row + k > last) break;
    R::store((T*)p.y + (row + k) * p.y_stride, p.cols, t, v[k]);
    if (t == 0) {
      if (p.mean) p.mean[row + k] = mean[k];
      p.rstd[row + k] = rstd[k];
    }
  }
}

constexpr int grad_block_of(int g) { return g == 64 ? 256 : g == 256 ? 512 : 1024; }

// Each block has several groups of G lanes and each group a row at a time, the next
// one's x and dy on their way: a row alone is too little in flight to
// cover the way to HBM and the sums in between (16,384 x 3,584 in BF16: 119 us
// without, 67 with).  SUMS: the columns' sums are kept as well.
template <typename T, int E, int G, bool VEC, bool SUMS>
__device__ __forceinline__ void grad_rows(const NormGradParams& p, uint64_t first, uint64_t step,
                                          float (&dw)[E], float (&db)[E]) {
  typedef Row<E, G, VEC> R;
  __shared__ float2 s[2][16];
  const uint32_t t = threadIdx.x % G;
  const float inv_n = 1.0f / (float)p.cols;
  float w[E];
  R::params(p.weight, p.param_bf16, p.cols, t, w);
  // every group of the block makes the same number of turns: there are barriers
  const uint64_t turns = first - threadIdx.x / G < p.rows ? (p.rows - (first - threadIdx.x / G) + step - 1) / step : 0;
  typename R::template Raw<T> nx, ndy;
  float nrstd = 0.0f, nmean = 0.0f;
  auto fetch = [&](uint64_t row) {
    if (row >= p.rows) row = p.rows - 1;
    R::template load<SUMS>((const T*)p.x + row * p.x_stride, p.cols, t, nx);
    R::template load<SUMS>((const T*)p.dy + row * p.dy_stride, p.cols, t, ndy);
    nrstd = p.rstd[row];
    nmean = p.mean ? p.mean[row] : 0.0f;
  };
  if (turns) fetch(first);
  for (uint64_t k = 0; k < turns; ++k) {
    const uint64_t row = first + k * step;
    const bool valid = row < p.rows;
    float x[E], dy[E];
    R::unpack(nx, x);
    R::unpack(ndy, dy);
    const float rstd = nrstd, mean = nmean;
    if (k + 1 < turns) fetch(row + step);
    float sa = 0.0f, sax = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      // past the row a zero, which meets dy = 0: mean * rstd may be out of range
      x[e] = (x[e] - (R::in(e, p.cols, t) ? mean : 0.0f)) * rstd;
      if (SUMS && valid) {
        dw[e] = __builtin_fmaf(dy[e], x[e], dw[e]);
        db[e] += dy[e];
      }
      dy[e] *= w[e];
      sa += dy[e];
      sax = __builtin_fmaf(dy[e], x[e], sax);
    }
    const float2 sum = group_sum2<G>(sa, sax, s[k & 1]);
    sa = p.mean ? sum.x * inv_n : 0.0f;
    sax = sum.y * inv_n;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = (dy[e] - sa - x[e] * sax) * rstd;
    if (valid) R::store((T*)p.dx + row * p.dx_stride, p.cols, t, x);
  }
}

template <typename T, int E, int G, bool VEC>
__global__ __launch_bounds__(grad_block_of(G)) void norm_grad_kernel(NormGradParams p) {
  typedef Row<E, G, VEC> R;
  constexpr int kGroups = grad_block_of(G) / G;
  __shared__ float s_sum[kGroups > 1 ? G * E : 1];
  const uint32_t t = threadIdx.x % G, group = threadIdx.x / G;
  float dw[E], db[E];
#pragma unroll
  for (int e = 0; e < E; ++e) dw[e] = db[e] = 0.0f;
  grad_rows<T, E, G, VEC, true>(p, (uint64_t)blockIdx.x * kGroups + group, (uint64_t)gridDim.x * kGroups, dw, db);
  // the groups' sums one after the other, then one row of sums for the block
  if constexpr (kGroups > 1) {
    for (int what = 0; what < (p.dbias ? 2 : 1); ++what)
      for (uint32_t k = 1; k < kGroups; ++k) {
        __syncthreads();
        if (group == k) {
#pragma unroll
          for (int e = 0; e < E; ++e) s_sum[e * G + t] = what ? db[e] : dw[e];
        }
        __syncthreads();
        if (group == 0) {
#pragma unroll
          for (int e = 0; e < E; ++e) (what ? db[e] : dw[e]) += s_sum[e * G + t];
        }
      }
  }
  if (group != 0) return;
  float* out = p.partial + (uint64_t)blockIdx.x * p.cols;
  R::store(out, p.cols, t, dw);
  if (p.dbias) R::store(out + (uint64_t)gridDim.x * p.cols, p.cols, t, db);
}

// Few rows: one launch, whose blocks past the first `row_blocks` sum kStrip columns
// each over all rows, a wave 8 rows at a time.  mean and rstd are given, so these
// sums need nothing of the other blocks; x and dy are read twice, the second time
// from a cache.
constexpr int kStrip = 8;

constexpr int few_block_of(int g) { return g == 1024 ? 1024 : 512; }

template <typename T, int E, int G, bool VEC>
__global__ __launch_bounds__(few_block_of(G)) void norm_grad_few_kernel(NormGradParams p, uint32_t row_blocks) {
  constexpr int kBlock = few_block_of(G), kGroups = kBlock / G;
  if (blockIdx.x < row_blocks) {
    float none[E];
    grad_rows<T, E, G, VEC, false>(p, (uint64_t)blockIdx.x * kGroups + threadIdx.x / G,
                                   (uint64_t)row_blocks * kGroups, none, none);
    return;
  }
  constexpr uint32_t kRows = kBlock / kStrip;
  __shared__ float s[2][kBlock];
  const uint32_t c = (blockIdx.x - row_blocks) * kStrip + threadIdx.x % kStrip, r0 = threadIdx.x / kStrip;
  float dw = 0.0f, db = 0.0f;
  if (c < p.cols) {
#pragma unroll 8
    for (uint32_t r = r0; r < (uint32_t)p.rows; r += kRows) {
      const float dy = from_bits(((const T*)p.dy)[r * p.dy_stride + c]);
      const float x = from_bits(((const T*)p.x)[r * p.x_stride + c]);
      dw = __builtin_fmaf(dy, (x - (p.mean ? p.mean[r] : 0.0f)) * p.rstd[r], dw);
      db += dy;
    }
  }
  s[0][threadIdx.x] = dw;
  s[1][threadIdx.x] = db;
  __syncthreads();
  if (threadIdx.x >= 2 * kStrip) return;
  const uint32_t what = threadIdx.x / kStrip, lane = threadIdx.x % kStrip;
  const uint32_t col = (blockIdx.x - row_blocks) * kStrip + lane;
  if (col >= p.cols || (what && !p.dbias)) return;
  float a = 0.0f;
#pragma unroll 8
  for (uint32_t k = 0; k < kRows; ++k) a += s[what][k * kStrip + lane];
  (what ? p.dbias : p.dweight)[col] = a;
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

constexpr uint64_t kNormFewRows = 1280;

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

namespace {

void run_layer_norm(bool bf16, const NormParams& p, hipStream_t stream) {
  const bool vec = p.cols % 8 == 0 && p.x_stride % 8 == 0 && p.y_stride % 8 == 0;
  by_shape(p.cols, [&](auto e, auto g) {
    constexpr int E = decltype(e)::value, G = decltype(g)::value;
    // two rows a group where that still leaves eight blocks for every CU
    const uint64_t two = 2 * block_of(G) / G;
    const bool pairs = p.rows >= two * 2048;
    const uint64_t rows = pairs ? two : two / 2;
    const dim3 block(block_of(G)), grid((uint32_t)((p.rows + rows - 1) / rows));
    auto run = [&](auto type, auto v) {
      typedef decltype(type) T;
      constexpr bool V = decltype(v)::value;
      if (pairs) hipLaunchKernelGGL((norm_kernel<T, E, G, V, 2>), grid, block, 0, stream, p);
      else hipLaunchKernelGGL((norm_kernel<T, E, G, V, 1>), grid, block, 0, stream, p);
    };
    if (bf16 && vec) run(uint16_t{}, std::true_type{});
    else if (bf16) run(uint16_t{}, std::false_type{});
    else if (vec) run(float{}, std::true_type{});
    else run(float{}, std::false_type{});
  });
}

// A launch has fewer than 2^32 threads; the widest form takes 512 for a row.
constexpr uint64_t kNormRowsAtOnce = 1u << 22;

}  // namespace

hipError_t launch_layer_norm(bool bf16, const NormParams& p, hipStream_t stream) {
  const uint64_t size = bf16 ? 2 : 4;
  for (uint64_t first = 0; first < p.rows; first += kNormRowsAtOnce) {
    NormParams q = p;
    q.rows = p.rows - first < kNormRowsAtOnce ? p.rows - first : kNormRowsAtOnce;
    q.x = (const char*)p.x + first * p.x_stride * size;
    q.y = (char*)p.y + first * p.y_stride * size;
    if (p.mean) q.mean = p.mean + first;
    q.rstd = p.rstd + first;
    run_layer_norm(bf16, q, stream);
  }
  return hipGetLastError();
}

hipError_t launch_layer_norm_grad(bool bf16, const NormGradParams& p, hipStream_t stream) {
  const bool vec = p.cols % 8 == 0 && p.x_stride % 8 == 0 && p.dy_stride % 8 == 0 && p.dx_stride % 8 == 0;
  // one launch for few rows: the second one costs its 3 us on the host and as much
  // again on the GPU, a strip of columns 0.5 us for every 128 rows
  const bool few = p.rows > 0 && p.rows <= kNormFewRows;
  uint32_t sums = 0;
  by_shape(p.cols, [&](auto e, auto g) {
    constexpr int E = decltype(e)::value, G = decltype(g)::value;
    const uint32_t size = few ? few_block_of(G) : grad_block_of(G), groups = size / G;
    uint64_t blocks = (p.rows + groups - 1) / groups;
    if (blocks > kNormBlocks) blocks = kNormBlocks;
    sums = (uint32_t)blocks;
    if (blocks == 0) return;
    const dim3 block(size), grid((uint32_t)blocks + (few ? (p.cols + kStrip - 1) / kStrip : 0));
    auto run = [&](auto type, auto v) {
      typedef decltype(type) T;
      constexpr bool V = decltype(v)::value;
      if (few) hipLaunchKernelGGL((norm_grad_few_kernel<T, E, G, V>), grid, block, 0, stream, p, (uint32_t)blocks);
      else hipLaunchKernelGGL((norm_grad_kernel<T, E, G, V>), grid, block, 0, stream, p);
    };
    if (bf16 && vec) run(uint16_t{}, std::true_type{});
    else if (bf16) run(uint16_t{}, std::false_type{});
    else if (vec) run(float{}, std::true_type{});
    else run(float{}, std::false_type{});
  });
  if (hipError_t e = hipGetLastError()) return e;
  if (few) return hipSuccess;
  hipLaunchKernelGGL(norm_columns_kernel, dim3((p.cols + 63) / 64, p.dbias ? 2 : 1), dim3(1024), 0,
                     stream, p.partial, sums, p.cols, p.dweight, p.dbias);
  return hipGetLastError();
}

}  // namespace pulse
