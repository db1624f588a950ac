// block_norm.hip -- a block's output joins the residual stream, and the stream is
// normalised for the next block, in one pass; and the gradient of that.
//
//   u  = post_norm(b) * gate       (each if there is one)
//   h' = residual_scale * h + u
//   y  = norm(h')                  of the sum before it is rounded
//
// Bound by HBM: forward b and h in, h' and y out; backward dy, dh', h' and b in, dh
// and db out (16,384 x 3,584 BF16: 82 us, 5.8 TB/s, and 134, 5.3).  A row lies in the registers of G lanes as in layer_norm.hip, so that
// everything in between stays there.
//
// Backward, with xh and bh the normalised rows of h' and b and a = dy * weight:
//   g  = dh' + rstd (a - mean(a) - xh mean(a xh)),     dh = residual_scale * g
//   c  = g * gate * post_weight,  db = post_rstd (c - mean(c) - bh mean(c bh))
// The five parameter gradients are made of four sums down the columns,
//   dy xh, dy, S1 = g bh and S2 = g,
// since gate and post_weight are the same in every row: dpost_weight = gate S1,
// dpost_bias = gate S2, dgate = post_weight S1 + post_bias S2.  So a lane keeps two
// sums a column (four with biases) and one product of parameters.  Each block writes
// its sums to the workspace, a second kernel adds those in a fixed order.
#include "norm_rows.hpp"

namespace pulse {

namespace {

// VEC: rows of 16-byte groups.  Other rows in groups from any address or, up to 4,096,
// element by element, where that is faster: us with groups and with single elements,
// forward, 8,192 x 3,585 BF16 49 and 95, FP32 106 and 97; backward, BF16 124 and 86,
// 8,192 x 5,121 199 and 319.
template <typename T, int E, int G, bool VEC, bool GRAD>
using RowOf = typename std::conditional<VEC || (E * G <= 4096 && (GRAD || !kIsBf16<T>)), Row<E, G, VEC>, AnyRow<E, G>>::type;

// The mean of each group's row (0 in the RMS form), taken off, and its rstd.
template <typename T, int E, int G, bool VEC, int N>
__device__ __forceinline__ void normalise(float (&v)[N][E], const BlockNormParams& p, uint32_t t, float inv_n,
                                          float2 (&s)[2][16], float (&mean)[2], float (&rstd)[2]) {
  typedef RowOf<T, E, G, VEC, false> R;
  float a[2] = {0.0f, 0.0f};
  mean[0] = mean[1] = 0.0f;
  if (!p.rms) {
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
  // the RMS form has one sum a norm: two norms in a row take one buffer each
  const float2 sum = group_sum2<G>(a[0], a[1], s[1]);
  rstd[0] = 1.0f / __builtin_sqrtf(sum.x * inv_n + p.eps);
  rstd[1] = 1.0f / __builtin_sqrtf(sum.y * inv_n + p.eps);
}

// stream: rows that the caches will not keep until they are read again are written past
// them (16,384 x 3,584 BF16: forward 87 us, 82 so, backward 142 and 134).
template <typename R, typename T, int E>
__device__ __forceinline__ void store_row(bool stream, T* p, uint32_t cols, uint32_t t, const float (&v)[E]) {
  if (stream) R::template store<true>(p, cols, t, v);
  else R::store(p, cols, t, v);
}

// N rows at a time by each group of G lanes, and no loop, as the layer norm's.
template <typename T, int E, int G, bool VEC, int N>
__global__ __launch_bounds__(block_of(G)) void block_norm_kernel(BlockNormParams p) {
  typedef RowOf<T, E, G, VEC, false> R;
  constexpr int kRows = block_of(G) / G * N;
  __shared__ float2 s_post[2][16], s[2][16];
  const uint32_t t = threadIdx.x % G;
  const uint64_t row = (uint64_t)blockIdx.x * kRows + threadIdx.x / G * N;
  if (row >= p.rows) return;  // whole waves: G is 64 where a block has several groups
  const uint64_t last = p.rows - 1;
  const float inv_n = 1.0f / (float)p.cols;
  float u[N][E], w[E], mean[2], rstd[2];
  typename R::template Raw<T> raw[N];
  {
    typename R::template Raw<T> first[N];
#pragma unroll
    for (int k = 0; k < N; ++k)
      R::template load<true>((const T*)p.b + (row + k < p.rows ? row + k : last) * p.b_stride, p.cols, t, first[k]);
#pragma unroll
    for (int k = 0; k < N; ++k)
      R::template load<true>((const T*)p.h + (row + k < p.rows ? row + k : last) * p.h_stride, p.cols, t, raw[k]);
#pragma unroll
    for (int k = 0; k < N; ++k) R::unpack(first[k], u[k]);
  }
  if (p.post_weight) {
    normalise<T, E, G, VEC, N>(u, p, t, inv_n, s_post, mean, rstd);
    if (t == 0 && p.stats) {
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (row + k <= last) {
          p.stats[p.stats_stride + row + k] = rstd[k];
          if (!p.rms) p.stats[3 * p.stats_stride + row + k] = mean[k];
        }
    }
    R::params(p.post_weight, p.param_bf16, p.cols, t, w);
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) u[k][e] = u[k][e] * rstd[k] * w[e];
    if (p.post_bias) {
      R::params(p.post_bias, p.param_bf16, p.cols, t, w);
#pragma unroll
      for (int k = 0; k < N; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) u[k][e] += w[e];
    }
  }
  if (p.gate) {
    R::params(p.gate, p.param_bf16, p.cols, t, w);
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) u[k][e] *= w[e];
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    float h[E];
    R::unpack(raw[k], h);
#pragma unroll
    for (int e = 0; e < E; ++e)
      // past the row's end zeros, whatever rstd is
      u[k][e] = R::in(e, p.cols, t) ? __builtin_fmaf(p.residual_scale, h[e], u[k][e]) : 0.0f;
    // where h_out is h these lanes have read what they write
    if (row + k <= last) store_row<R>(p.stream, (T*)p.h_out + (row + k) * p.h_out_stride, p.cols, t, u[k]);
  }
  normalise<T, E, G, VEC, N>(u, p, t, inv_n, s, mean, rstd);
  R::params(p.weight, p.param_bf16, p.cols, t, w);
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) u[k][e] = u[k][e] * rstd[k] * w[e];
  if (p.bias) {
    R::params(p.bias, p.param_bf16, p.cols, t, w);
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) u[k][e] += w[e];
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    if (row + k > last) break;
    store_row<R>(p.stream, (T*)p.y + (row + k) * p.y_stride, p.cols, t, u[k]);
    if (t == 0 && p.stats) {
      p.stats[row + k] = rstd[k];
      if (!p.rms) p.stats[2 * p.stats_stride + row + k] = mean[k];
    }
  }
}

constexpr int block_grad_of(int g) { return g < 256 ? 256 : g; }

// Each group of G lanes takes a row at a time, the next one on its way where there are
// registers for that: 8,192 x 5,120 layer norms, 177 us with it, 128 without.  BIASES:
// the sums of dy and g are kept as well.  SUMS: else none are, and the two means of a row
// are written for the kernel below.
template <typename T, int E, int G, bool VEC, bool BIASES, bool SUMS>
__global__ __launch_bounds__(block_grad_of(G)) void block_norm_grad_kernel(BlockNormGradParams p) {
  typedef RowOf<T, E, G, VEC, true> R;
  constexpr int kGroups = block_grad_of(G) / G;
  constexpr bool kAhead = G < 512 || (G * E <= 4096) || (kIsBf16<T> && !BIASES && SUMS);
  __shared__ float2 s[2][16];
  __shared__ float s_sum[kGroups > 1 ? G * E : 1];
  const uint32_t t = threadIdx.x % G, group = threadIdx.x / G;
  const float inv_n = 1.0f / (float)p.cols;
  const bool post = p.post_weight != nullptr;
  float w[E], by[E];  // the norm's weight; gate * post_weight
  auto load_weight = [&] { R::params(p.weight, p.param_bf16, p.cols, t, w); };
  auto load_by = [&] {
#pragma unroll
    for (int e = 0; e < E; ++e) by[e] = 1.0f;
    if (p.gate) R::params(p.gate, p.param_bf16, p.cols, t, by);
    if (post) {
      float v[E];
      R::params(p.post_weight, p.param_bf16, p.cols, t, v);
#pragma unroll
      for (int e = 0; e < E; ++e) by[e] *= v[e];
    }
  };
  if constexpr (SUMS) {  // for all rows; else there is no room to keep them
    load_weight();
    load_by();
  }
  float dw[SUMS ? E : 1] = {}, s1[SUMS ? E : 1] = {}, db[BIASES ? E : 1] = {}, s2[BIASES ? E : 1] = {};
  const uint64_t block_first = (uint64_t)blockIdx.x * kGroups, step = (uint64_t)gridDim.x * kGroups;
  // every group of the block makes the same number of turns: there are barriers
  const uint64_t turns = block_first < p.rows ? (p.rows - block_first + step - 1) / step : 0;
  typename R::template Raw<T> nx, ndy, ndh, nb;
  float nrstd = 0.0f, nmean = 0.0f, npr = 0.0f, npm = 0.0f;
  auto fetch = [&](uint64_t row) {
    if (row >= p.rows) row = p.rows - 1;
    R::template load<true>((const T*)p.h_out + row * p.h_out_stride, p.cols, t, nx);
    R::template load<true>((const T*)p.dy + row * p.dy_stride, p.cols, t, ndy);
    if (p.dh_out) R::template load<true>((const T*)p.dh_out + row * p.dh_out_stride, p.cols, t, ndh);
    if (p.b) R::template load<true>((const T*)p.b + row * p.b_stride, p.cols, t, nb);
    nrstd = p.stats[row];
    if (!p.rms) nmean = p.stats[2 * p.stats_stride + row];
    if (post) {
      npr = p.stats[p.stats_stride + row];
      if (!p.rms) npm = p.stats[3 * p.stats_stride + row];
    }
  };
  if (kAhead && turns) fetch(block_first + group);
  for (uint64_t k = 0; k < turns; ++k) {
    const uint64_t row = block_first + group + k * step;
    const bool valid = row < p.rows;
    if (!kAhead) fetch(row);
    float x[E], g[E], bh[E];
    R::unpack(nx, x);
    float dy[E];
    R::unpack(ndy, dy);
    // as they lie in memory until they are needed
    const typename R::template Raw<T> raw_dh = ndh, raw_b = nb;
    const float rstd = nrstd, mean = nmean, pr = npr, pm = npm;
    if (kAhead && k + 1 < turns) fetch(row + step);
    float sa = 0.0f, sax = 0.0f;
    if constexpr (!SUMS) load_weight();
#pragma unroll
    for (int e = 0; e < E; ++e) {
      // past the row a zero, which meets dy = 0: mean * rstd may be out of range
      x[e] = R::in(e, p.cols, t) ? (x[e] - mean) * rstd : 0.0f;
      if (SUMS && valid) {
        dw[e] = __builtin_fmaf(dy[e], x[e], dw[e]);
        if constexpr (BIASES) db[e] += dy[e];
      }
      g[e] = dy[e] * w[e];
      sa += g[e];
      sax = __builtin_fmaf(g[e], x[e], sax);
    }
    float2 sum = group_sum2<G>(sa, sax, s[0]);
    sa = p.rms ? 0.0f : sum.x * inv_n;
    sax = sum.y * inv_n;
    if (!SUMS && valid && t == 0) {
      p.means[row] = sa;
      p.means[p.means_stride + row] = sax;
    }
    float dh[E];
    if (p.dh_out) {
      R::unpack(raw_dh, dh);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) dh[e] = 0.0f;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
      g[e] = R::in(e, p.cols, t) ? __builtin_fmaf(g[e] - sa - x[e] * sax, rstd, dh[e]) : 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = g[e] * p.residual_scale;
    if (valid) store_row<R>(p.stream, (T*)p.dh + row * p.dh_stride, p.cols, t, x);
    float sc = 0.0f, scb = 0.0f;
    if (p.b) {
      R::unpack(raw_b, bh);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) bh[e] = 0.0f;
    }
    if (post) {
#pragma unroll
      for (int e = 0; e < E; ++e) bh[e] = R::in(e, p.cols, t) ? (bh[e] - pm) * pr : 0.0f;
    }
    if constexpr (!SUMS) load_by();
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (SUMS && valid) {
        s1[e] = __builtin_fmaf(g[e], bh[e], s1[e]);
        if constexpr (BIASES) s2[e] += g[e];
      }
      g[e] *= by[e];
    }
    if (post) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        sc += g[e];
        scb = __builtin_fmaf(g[e], bh[e], scb);
      }
    }
    // also where nothing is summed: the barrier frees s[0] for the next row
    sum = group_sum2<G>(sc, scb, s[1]);
    if (post) {
      sc = p.rms ? 0.0f : sum.x * inv_n;
      scb = sum.y * inv_n;
#pragma unroll
      for (int e = 0; e < E; ++e) g[e] = (g[e] - sc - bh[e] * scb) * pr;
    }
    if (valid) store_row<R>(p.stream, (T*)p.db + row * p.db_stride, p.cols, t, g);
  }
  if constexpr (!SUMS) return;
  // the groups' sums one after the other, then one row of each sum for the block
  auto join = [&](auto& v) {
    if constexpr (kGroups > 1) {
      for (uint32_t k = 1; k < kGroups; ++k) {
        __syncthreads();
        if (group == k) {
#pragma unroll
          for (int e = 0; e < E; ++e) s_sum[e * G + t] = v[e];
        }
        __syncthreads();
        if (group == 0) {
#pragma unroll
          for (int e = 0; e < E; ++e) v[e] += s_sum[e * G + t];
        }
      }
    }
  };
  if constexpr (SUMS) {
    const uint64_t apart = (uint64_t)gridDim.x * p.cols;
    float* const out = p.partial + (uint64_t)blockIdx.x * p.cols;
    join(dw);
    if (p.b) join(s1);
    if constexpr (BIASES) {
      join(db);
      join(s2);
    }
    if (group != 0) return;
    R::store(out, p.cols, t, dw);
    if (p.b) R::store(out + apart, p.cols, t, s1);
    if constexpr (BIASES) {
      R::store(out + 2 * apart, p.cols, t, db);
      R::store(out + 3 * apart, p.cols, t, s2);
    }
  }
}

// Wide rows, for whose sums there are no registers: the four sums of 64 columns and a
// chunk of rows, whose means are given, a wave every 16th row.  Everything is read a second
// time, which is less than what the sums would be moved in and out of scratch memory:
// 4,096 x 12,000 BF16 layer norms 4,070 us that way, 409 this way.
template <typename T>
__global__ __launch_bounds__(1024) void block_norm_wide_sums_kernel(BlockNormGradParams p, uint32_t chunk,
                                                                    uint32_t first, uint32_t all) {
  __shared__ float s[4][16][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint32_t c = blockIdx.x * 64 + lane;
  const uint64_t begin = (uint64_t)blockIdx.y * chunk, end = begin + chunk < p.rows ? begin + chunk : p.rows;
  const bool post = p.post_weight != nullptr;
  float dw = 0.0f, s1 = 0.0f, db = 0.0f, s2 = 0.0f;
  if (c < p.cols) {
    const float w = p.param_bf16 ? from_bits(((const uint16_t*)p.weight)[c]) : ((const float*)p.weight)[c];
#pragma unroll 4
    for (uint64_t r = begin + wave; r < end; r += 16) {
      const float dy = from_bits(((const T*)p.dy)[r * p.dy_stride + c]);
      float x = from_bits(((const T*)p.h_out)[r * p.h_out_stride + c]);
      const float dh = p.dh_out ? from_bits(((const T*)p.dh_out)[r * p.dh_out_stride + c]) : 0.0f;
      float bh = p.b ? from_bits(((const T*)p.b)[r * p.b_stride + c]) : 0.0f;
      const float rstd = p.stats[r];
      x = (x - (p.rms ? 0.0f : p.stats[2 * p.stats_stride + r])) * rstd;
      if (post) bh = (bh - (p.rms ? 0.0f : p.stats[3 * p.stats_stride + r])) * p.stats[p.stats_stride + r];
      const float g = __builtin_fmaf(dy * w - p.means[r] - x * p.means[p.means_stride + r], rstd, dh);
      dw = __builtin_fmaf(dy, x, dw);
      db += dy;
      s1 = __builtin_fmaf(g, bh, s1);
      s2 += g;
    }
  }
  s[0][wave][lane] = dw;
  s[1][wave][lane] = s1;
  s[2][wave][lane] = db;
  s[3][wave][lane] = s2;
  __syncthreads();
  if (wave >= 4 || c >= p.cols) return;
  float a = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) a += s[wave][i][lane];
  p.partial[((uint64_t)wave * all + first + blockIdx.y) * p.cols + c] = a;
}

// The sums of the n partial rows, 64 columns a block, its 16 waves a slice of the rows
// each; y = 0: dy xh and dy, y = 1: S1 and S2 and what is made of them.
__global__ __launch_bounds__(1024) void block_norm_columns_kernel(BlockNormGradParams p, uint32_t n) {
  __shared__ float s[2][16][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint32_t c = blockIdx.x * 64 + lane;
  const uint64_t apart = (uint64_t)n * p.cols;
  const float* const first = p.partial + (blockIdx.y ? apart : 0);
  const bool sums = !blockIdx.y || p.b, biases = p.biases;
  float a = 0.0f, b = 0.0f;
  if (c < p.cols) {
    if (sums) {
#pragma unroll 4
      for (uint32_t r = wave; r < n; r += 16) a += first[(uint64_t)r * p.cols + c];
    }
    if (biases) {
#pragma unroll 4
      for (uint32_t r = wave; r < n; r += 16) b += first[2 * apart + (uint64_t)r * p.cols + c];
    }
  }
  s[0][wave][lane] = a;
  s[1][wave][lane] = b;
  __syncthreads();
  if (wave != 0 || c >= p.cols) return;
  a = b = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    a += s[0][i][lane];
    b += s[1][i][lane];
  }
  auto param = [&](const void* v) { return p.param_bf16 ? from_bits(((const uint16_t*)v)[c]) : ((const float*)v)[c]; };
  if (blockIdx.y == 0) {
    p.dweight[c] = a;
    if (p.dbias) p.dbias[c] = b;
    return;
  }
  const float gate = p.gate ? param(p.gate) : 1.0f;
  if (p.dpost_weight) p.dpost_weight[c] = gate * a;
  if (p.dpost_bias) p.dpost_bias[c] = gate * b;
  if (p.dgate) {
    float v = p.post_weight ? param(p.post_weight) * a : a;
    if (p.post_bias) v = __builtin_fmaf(param(p.post_bias), b, v);
    p.dgate[c] = v;
  }
}

template <int E, int G>
struct Lanes {
  static constexpr int kE = E, kG = G;
};

// f(Lanes) for rows of `cols`.
template <typename F>
void forward_lanes(uint32_t cols, F f) {
  if (cols <= 512) f(Lanes<8, 64>{});
  else if (cols <= 1024) f(Lanes<16, 64>{});
  else if (cols <= 2048) f(Lanes<8, 256>{});
  else if (cols <= 4096) f(Lanes<16, 256>{});
  else if (cols <= 8192) f(Lanes<8, 1024>{});
  else f(Lanes<16, 1024>{});
}

// The gradient keeps up to eleven values an element in registers, rows on their way among
// them, which with 16 elements a lane leaves one wave for a SIMD where those are FP32 or
// loaded one by one (HEAVY): half as many elements then.  us with 16 and 8: 1,027 x 897
// FP32 layer norms 26 and 20, 8,192 x 3,585 BF16 133 and 90; 16,384 x 896 BF16 (not
// heavy) 37.5 and 42, 4,096 x 3,584 38.4 and 41.4.
template <bool HEAVY, typename F>
void grad_lanes(uint32_t cols, F f) {  // cols up to 8,192
  if (cols <= 512) f(Lanes<8, 64>{});
  else if (cols <= 1024) f(Lanes<HEAVY ? 8 : 16, HEAVY ? 128 : 64>{});
  else if (cols <= 2048) f(Lanes<8, 256>{});
  else if (cols <= 4096) f(Lanes<HEAVY ? 8 : 16, HEAVY ? 512 : 256>{});
  else f(Lanes<16, 512>{});
}

template <typename F>
void by_type(bool bf16, bool vec, F f) {
  if (bf16 && vec) f(uint16_t{}, std::true_type{});
  else if (bf16) f(uint16_t{}, std::false_type{});
  else if (vec) f(float{}, std::true_type{});
  else f(float{}, std::false_type{});
}

void run_block_norm(bool bf16, const BlockNormParams& p, hipStream_t stream) {
  const bool vec = p.cols % 8 == 0 && p.b_stride % 8 == 0 && p.h_stride % 8 == 0 && p.y_stride % 8 == 0 &&
                   p.h_out_stride % 8 == 0;
  forward_lanes(p.cols, [&](auto lanes) {
    constexpr int E = decltype(lanes)::kE, G = decltype(lanes)::kG;
    // two rows a group where that still leaves eight blocks for every CU
    const uint64_t two = 2 * block_of(G) / G;
    const bool pairs = p.rows >= two * 2048;
    const uint64_t rows = pairs ? two : two / 2;
    const dim3 block(block_of(G)), grid((uint32_t)((p.rows + rows - 1) / rows));
    by_type(bf16, vec, [&](auto type, auto v) {
      typedef decltype(type) T;
      constexpr bool V = decltype(v)::value;
      if (pairs) hipLaunchKernelGGL((block_norm_kernel<T, E, G, V, 2>), grid, block, 0, stream, p);
      else hipLaunchKernelGGL((block_norm_kernel<T, E, G, V, 1>), grid, block, 0, stream, p);
    });
  });
}

constexpr uint64_t kStreamBytes = 64ull << 20;  // of one matrix

// A launch has fewer than 2^32 threads; the widest form takes 512 for a row.
constexpr uint64_t kRowsAtOnce = 1u << 22;

}  // namespace

hipError_t launch_block_norm(bool bf16, const BlockNormParams& all, hipStream_t stream) {
  const uint64_t size = bf16 ? 2 : 4;
  BlockNormParams p = all;
  p.stream = p.rows * p.cols * size >= kStreamBytes;
  for (uint64_t first = 0; first < p.rows; first += kRowsAtOnce) {
    BlockNormParams q = p;
    q.rows = p.rows - first < kRowsAtOnce ? p.rows - first : kRowsAtOnce;
    q.b = (const char*)p.b + first * p.b_stride * size;
    q.h = (const char*)p.h + first * p.h_stride * size;
    q.y = (char*)p.y + first * p.y_stride * size;
    q.h_out = (char*)p.h_out + first * p.h_out_stride * size;
    if (p.stats) q.stats = p.stats + first;
    run_block_norm(bf16, q, stream);
  }
  return hipGetLastError();
}

namespace {

// Wide rows: the rows' gradients and means, as many rows at a time as the workspace has
// room for means, then their columns' sums.  Returns the number of partial rows.
template <typename T, bool VEC>
uint32_t run_wide_grad(const BlockNormGradParams& p, hipStream_t stream) {
  // half of the workspace for the sums, half for the means
  constexpr uint32_t kChunks = kBlockNormBlocks / 2;
  const uint64_t at_once = (uint64_t)kChunks * p.cols * 4 / 2;
  const uint64_t slabs = p.rows ? (p.rows - 1) / at_once + 1 : 0;
  if (slabs > kChunks) return ~0u;  // rows of more memory than there is
  const uint32_t strips = (p.cols + 63) / 64;
  auto chunks_of = [&](uint64_t rows) -> uint32_t {
    const uint32_t most = kChunks / (uint32_t)slabs, wanted = 2048 / strips + 1;
    const uint64_t fit = (rows + 63) / 64;  // four turns of the waves at least
    return (uint32_t)(fit < most && fit < wanted ? fit : wanted < most ? wanted : most);
  };
  uint32_t all = 0, done = 0;
  for (uint64_t first = 0; first < p.rows; first += at_once)
    all += chunks_of(p.rows - first < at_once ? p.rows - first : at_once);
  for (uint64_t first = 0; first < p.rows; first += at_once) {
    BlockNormGradParams q = p;
    q.rows = p.rows - first < at_once ? p.rows - first : at_once;
    q.means = p.partial + (uint64_t)kChunks * p.cols * 4;
    q.means_stride = q.rows;
    q.dy = (const T*)p.dy + first * p.dy_stride;
    q.h_out = (const T*)p.h_out + first * p.h_out_stride;
    if (p.dh_out) q.dh_out = (const T*)p.dh_out + first * p.dh_out_stride;
    if (p.b) q.b = (const T*)p.b + first * p.b_stride;
    q.db = (T*)p.db + first * p.db_stride;
    q.dh = (T*)p.dh + first * p.dh_stride;
    q.stats = p.stats + first;
    const dim3 grid((uint32_t)(q.rows < 4096 ? q.rows : 4096));
    hipLaunchKernelGGL((block_norm_grad_kernel<T, 16, 1024, VEC, false, false>), grid, dim3(1024), 0, stream, q);
    const uint32_t chunks = chunks_of(q.rows), chunk = (uint32_t)((q.rows + chunks - 1) / chunks);
    // what is rounded up leaves the last chunks without rows: their sums are zero
    hipLaunchKernelGGL(block_norm_wide_sums_kernel<T>, dim3(strips, chunks), dim3(1024), 0, stream, q, chunk, done, all);
    done += chunks;
  }
  return all;
}

}  // namespace

hipError_t launch_block_norm_grad(bool bf16, const BlockNormGradParams& all, hipStream_t stream) {
  BlockNormGradParams p = all;
  p.stream = p.rows * p.cols * (bf16 ? 2 : 4) >= kStreamBytes;
  const bool vec = p.cols % 8 == 0 && p.dy_stride % 8 == 0 && p.h_out_stride % 8 == 0 && p.dh_stride % 8 == 0 &&
                   p.db_stride % 8 == 0 && (!p.dh_out || p.dh_out_stride % 8 == 0) && (!p.b || p.b_stride % 8 == 0);
  uint32_t sums = 0;
  by_type(bf16, vec, [&](auto type, auto v) {
    typedef decltype(type) T;
    constexpr bool V = decltype(v)::value;
    if (p.cols > 8192) {
      sums = run_wide_grad<T, V>(p, stream);
      return;
    }
    grad_lanes<!kIsBf16<T> || !V>(p.cols, [&](auto lanes) {
      constexpr int E = decltype(lanes)::kE, G = decltype(lanes)::kG;
      constexpr uint32_t kGroups = block_grad_of(G) / G, kMost = G < 512 ? kBlockNormBlocks : kBlockNormBlocks / 2;
      uint64_t blocks = (p.rows + kGroups - 1) / kGroups;
      // two turns of a block rather than a second one for a CU, whose sums are read again
      if (blocks > kMost / 2) blocks = blocks / 2 + 1 < kMost / 2 ? kMost / 2 : blocks / 2 + 1;
      sums = blocks < kMost ? (uint32_t)blocks : kMost;
      if (blocks == 0) return;
      const dim3 block(block_grad_of(G)), grid(sums);
      if (p.biases) hipLaunchKernelGGL((block_norm_grad_kernel<T, E, G, V, true, true>), grid, block, 0, stream, p);
      else hipLaunchKernelGGL((block_norm_grad_kernel<T, E, G, V, false, true>), grid, block, 0, stream, p);
    });
  });
  if (sums == ~0u) return hipErrorInvalidValue;
  if (hipError_t e = hipGetLastError()) return e;
  const bool more = p.dpost_weight || p.dpost_bias || p.dgate;
  hipLaunchKernelGGL(block_norm_columns_kernel, dim3((p.cols + 63) / 64, more ? 2 : 1), dim3(1024), 0, stream, p, sums);
  return hipGetLastError();
}

}  // namespace pulse
