// linear.hip -- y = act(x W^T + bias) * times + residual for a BF16 weight and BF16
// tokens, and its gradient.
//
// Up to 16 tokens the weight's way from HBM bounds it: lowp_matmul.hip, which reads it
// once for every 16 (18,944 x 3,584, 16 tokens: 27 us; 24 tokens took 35 that way, and 33
// tokens take 28 by tiles).  For more, the matrix cores: tiles of gemm_tile.hpp, whose sums
// go through LDS as FP32 rows, so that multiplier, residual and results move 16 bytes a lane
// and whole lines at a time, and the epilogue's code is there once, not once per
// accumulator.  4,096 tokens, 18,944 x 3,584: forward 412 us (1.35 PFLOP/s), with silu, multiplier and pre-activation 500 to
// 515 for the 466 MB that these move; dx 444 and dW 498 (1.25 and 1.12) for a d of one part.
//
// Backward, with d = dy * times * act'(pre):
//   dx = d W,   dW = d^T x,   dbias = sum over tokens of d,   dtimes = dy * act(pre).
// The matrix cores take BF16, which would cut d to 8 bits: dx and dW 0.0023 off where
// their own rounding is 0.0017, and a direction that the rows of W (or x) share would not
// cancel in sums over d.  So d is two BF16 values, both products have twice the steps, and
// 2^-16 of d is what is left out (4,096 tokens, 18,944 x 3,584: 1,920 us, 1,020 with one).
// For a BF16 dy without multiplier, and no activation or relu, one holds it.
// One elementwise kernel makes d, dtimes and parts of dbias (172 us there: 931 MB at 5.4
// TB/s).
//
// Where the tiles are too few for the chip, k is split over blocks, whose FP32 sums are
// added by a further kernel, with the epilogue.  Tile and split are chosen by a cost.
#include "device_common.hpp"
#include "epilogue.hpp"
#include "gemm_tile.hpp"
#include "head.hpp"

namespace pulse {

namespace {

// out[n][m] = sum_k A[m][k] B[n][k], then the epilogue, whose tokens are n and rows m.
struct ProductParams {
  GemmOperand a, b;
  uint32_t m, n, k;
  uint32_t tiles_m, tiles_n, first_tile;
  uint32_t k_split;  // a multiple of 64
  float* sums;       // null: no split; [splits][n][m_ld]
  uint32_t m_ld;     // a multiple of 4
  void* out;
  uint64_t out_ld;
  uint64_t low;  // PAIRS: bytes from b's upper parts to its lower ones
  bool wide;    // every row of the epilogue starts at 16 bytes
  bool stream;  // what is read and written there is more than the caches keep
  Epilogue e;
};

__device__ __forceinline__ void unpack_eight(const uint4& w, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    v[e] = __uint_as_float(e & 1 ? get_u32(w, e >> 1) & 0xFFFF0000u : get_u32(w, e >> 1) << 16);
}

// Eight adjacent values from element `at` on, `left` of them there.
__device__ __forceinline__ void load_eight(const void* p, uint64_t at, int bf16, bool wide, uint32_t left,
                                           float (&v)[8]) {
  if (wide && left >= 8) {
    if (bf16) {
      unpack_eight(load16((const uint16_t*)p + at), v);
    } else {
      const uint4 a = load16((const float*)p + at), b = load16((const float*)p + at + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = __uint_as_float(get_u32(a, e));
        v[4 + e] = __uint_as_float(get_u32(b, e));
      }
    }
    return;
  }
#pragma unroll
  for (uint32_t e = 0; e < 8; ++e) v[e] = e < left ? load_f32(p, at + e, bf16) : 0.0f;
}

__device__ __forceinline__ uint4 pack_eight(const float (&v)[8]) {
  uint4 o;
  o.x = bf16x2_rne(__float_as_uint(v[0]), __float_as_uint(v[1]));
  o.y = bf16x2_rne(__float_as_uint(v[2]), __float_as_uint(v[3]));
  o.z = bf16x2_rne(__float_as_uint(v[4]), __float_as_uint(v[5]));
  o.w = bf16x2_rne(__float_as_uint(v[6]), __float_as_uint(v[7]));
  return o;
}

__device__ __forceinline__ void store_eight(void* p, uint64_t at, int bf16, bool wide, bool stream, uint32_t left,
                                            const float (&v)[8]) {
  if (bf16) {
    uint16_t* const y = (uint16_t*)p + at;
    const uint4 o = pack_eight(v);
    if (wide && left >= 8) {
      if (stream) store16_stream(y, o);
      else store16(y, o);
    } else if (left >= 8) {
      store16_any(y, o);
    } else {
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e)
        if (e < left) y[e] = (uint16_t)(get_u32(o, e >> 1) >> (16 * (e & 1)));
    }
  } else {
    float* const y = (float*)p + at;
    if (wide && left >= 8) {
      *(f32x4_t*)y = f32x4_t{v[0], v[1], v[2], v[3]};
      *(f32x4_t*)(y + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e)
        if (e < left) y[e] = v[e];
    }
  }
}

// Multiplier and residual of eight features, fetched before the sums are there.
struct Fetched {
  uint4 times, residual;
};

// Token t's eight features from `row` on, from their sums to what is stored.  FETCHED: `f`
// holds the operands, of whole eights of BF16.  act: p.e.act, where it is known a
// constant, so that the others' code is not there.
template <bool FETCHED>
__device__ __forceinline__ void finish_eight(const ProductParams& p, const Fetched& f, int act, float (&v)[8],
                                             uint64_t t, uint32_t row) {
  const Epilogue& e = p.e;
  const uint32_t left = p.m - row;
  float bias[8], times[8], residual[8];
  if (e.bias) load_eight(e.bias, row, e.bias_bf16, true, left, bias);
  if (e.times) {
    if (FETCHED && left >= 8) unpack_eight(f.times, times);
    else load_eight(e.times, t * e.times_stride + row, e.out_bf16, p.wide, left, times);
  }
  if (e.residual) {
    if (FETCHED && left >= 8) unpack_eight(f.residual, residual);
    else load_eight(e.residual, t * e.residual_stride + row, e.out_bf16, p.wide, left, residual);
  }
  if (e.bias) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += bias[i];
  }
  if (e.pre) store_eight(e.pre, t * e.pre_stride + row, e.out_bf16, p.wide, p.stream, left, v);
  if (act) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = activate(act, v[i]);
  }
  if (e.times) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= times[i];
  }
  if (e.residual) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += residual[i];
  }
  store_eight(p.out, t * p.out_ld + row, e.out_bf16, p.wide, p.stream, left, v);
}

// Block `id` of a product's tiles, and its split's share of k.  ACT: the epilogue's
// activation, or kPlain: there is no epilogue.
constexpr int kPlain = -1;

template <typename T, bool AK, bool BK, int ACT, bool PAIRS>
__device__ __forceinline__ void product_block(const ProductParams& p, char* lds, uint32_t id, uint32_t split) {
  // the tile's FP32 rows pass through LDS, as many fragments' columns at a time as fit
  constexpr int kFit = T::kLds / (T::BM * 4 * 16 * T::WN), kAtOnce = kFit < T::FN ? kFit : T::FN;
  static_assert(kFit >= 1 && (T::FN == kAtOnce || T::FN == 2 * kAtOnce), "in one or two passes");
  uint32_t tm, tn;
  gemm_tile_of(id, p.tiles_m, p.tiles_n, 8, tm, tn);
  const uint32_t m0 = tm * T::BM, n0 = tn * T::BN;
  const GemmOperand a = {p.a.p + (AK ? (uint64_t)m0 : m0 * p.a.ld), p.a.ld, p.a.limit - m0};
  const GemmOperand b = {p.b.p + (BK ? (uint64_t)n0 : n0 * p.b.ld), p.b.ld, p.b.limit - n0};
  const uint32_t k0 = p.sums ? split * p.k_split : 0;
  // a split past the end has no k and gives zeros
  const uint32_t k1 = !p.sums ? p.k : k0 >= p.k ? k0 : p.k - k0 < p.k_split ? p.k : k0 + p.k_split;
  typename T::Acc acc;
  T::template run<PAIRS>(lds, a, b, k0, k1, acc, p.low);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (p.sums) {
    float* const sums = p.sums + (uint64_t)split * p.n * p.m_ld;
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
      const uint32_t n = n0 + T::n_of(j, lane, wave);
#pragma unroll
      for (int i = 0; i < T::FM; ++i) {
        const uint32_t m = m0 + T::m_of(i, lane, wave);
        if (n < p.n && m < p.m) *(f32x4_t*)(sums + (uint64_t)n * p.m_ld + m) = acc[i][j];
      }
    }
    return;
  }
  // The operands of all of a thread's eights leave together and before the sums are
  // staged: one after the other they took as long as the bytes of seven (4,096 tokens,
  // 18,944 x 3,584, silu and multiplier: 515 us, 458 so).
  constexpr uint32_t kRows = kAtOnce * 16 * T::WN, kEights = T::BM / 8, kItems = kRows * kEights / T::kThreads;
  const bool fetch = ACT != kPlain && p.wide && p.e.out_bf16 && (p.e.times || p.e.residual);
  auto pass = [&](auto first) {
    constexpr int j0 = decltype(first)::value;
    // a thread's i-th eight: row r of the staged ones, which is this token of the tile
    auto place = [&](uint32_t i, uint32_t& r, uint32_t& g, uint32_t& n, uint32_t& m) {
      const uint32_t q = threadIdx.x + i * T::kThreads;
      r = q / kEights;
      g = q % kEights;
      n = n0 + r / (kAtOnce * 16) * (T::FN * 16) + j0 * 16 + r % (kAtOnce * 16);
      m = m0 + g * 8;
      return n < p.n && m < p.m;
    };
    Fetched f[kItems];
    if (fetch) {
#pragma unroll
      for (uint32_t i = 0; i < kItems; ++i) {
        uint32_t r, g, n, m;
        if (!place(i, r, g, n, m) || m + 8 > p.m) continue;
        if (p.e.times) f[i].times = load16_stream((const uint16_t*)p.e.times + n * p.e.times_stride + m);
        if (p.e.residual) f[i].residual = load16_stream((const uint16_t*)p.e.residual + n * p.e.residual_stride + m);
      }
    }
    if (j0) __syncthreads();
    // group c (4 values) of a row lies at place c ^ (n & 15)
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const uint32_t n = (wave % T::WN) * (kAtOnce * 16) + j * 16 + (lane & 15);
#pragma unroll
      for (int i = 0; i < T::FM; ++i) {
        const uint32_t c = T::m_of(i, lane, wave) >> 2;
        *(f32x4_t*)(lds + n * (T::BM * 4) + ((c ^ (n & 15)) << 4)) = acc[i][j0 + j];
      }
    }
    __syncthreads();
    auto finish = [&](uint32_t i, const Fetched& o, auto fetched) {
      uint32_t r, g, n, m;
      if (!place(i, r, g, n, m)) return;
      const f32x4_t lo = *(const f32x4_t*)(lds + r * (T::BM * 4) + (((2 * g) ^ (r & 15)) << 4));
      const f32x4_t hi = *(const f32x4_t*)(lds + r * (T::BM * 4) + (((2 * g + 1) ^ (r & 15)) << 4));
      float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      if constexpr (ACT == kPlain)
        store_eight(p.out, n * p.out_ld + m, true, p.wide, p.stream, p.m - m, v);
      else
        finish_eight<decltype(fetched)::value>(p, o, ACT, v, n, m);
    };
    if (fetch) {
#pragma unroll
      for (uint32_t i = 0; i < kItems; ++i) finish(i, f[i], std::true_type{});
    } else {
#pragma unroll 2
      for (uint32_t i = 0; i < kItems; ++i) finish(i, f[0], std::false_type{});
    }
  };
  // (a loop of this size the compiler would not unroll, as the sums' registers need)
  pass(std::integral_constant<int, 0>{});
  if constexpr (T::FN > kAtOnce) pass(std::integral_constant<int, kAtOnce>{});
}

template <typename T, bool AK, bool BK, int ACT, bool PAIRS>
__global__ __launch_bounds__(T::kThreads) void product_kernel(ProductParams p) {
  __shared__ alignas(1024) char lds[T::kLds];
  product_block<T, AK, BK, ACT, PAIRS>(p, lds, p.first_tile + blockIdx.x, blockIdx.y);
}

// dx's and dW's products in one launch: dx's blocks, whose sums are the longer ones, first.
template <typename TX, typename TW, bool PAIRS>
__global__ __launch_bounds__(TX::kThreads) void both_kernel(ProductParams x, ProductParams w) {
  static_assert(TX::kThreads == TW::kThreads && TX::kLds == TW::kLds, "blocks of one shape");
  __shared__ alignas(1024) char lds[TX::kLds];
  const uint32_t first = x.tiles_m * x.tiles_n;
  if (blockIdx.x < first) product_block<TX, true, false, kPlain, PAIRS>(x, lds, blockIdx.x, 0);
  else product_block<TW, true, true, kPlain, PAIRS>(w, lds, blockIdx.x - first, 0);
}

// The splits' sums, added in order, and the epilogue: a thread an eight of a row.
__global__ __launch_bounds__(256) void join_kernel(ProductParams p, uint32_t splits) {
  const uint32_t eights = (p.m + 7) / 8;
  const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x, n = id / eights;
  if (n >= p.n) return;
  const uint32_t m = (uint32_t)(id % eights) * 8;
  const bool second = m + 4 < p.m_ld;
  f32x4_t lo = {0.0f, 0.0f, 0.0f, 0.0f}, hi = lo;
#pragma unroll 4
  for (uint32_t s = 0; s < splits; ++s) {
    const float* const from = p.sums + ((uint64_t)s * p.n + n) * p.m_ld + m;
    lo += *(const f32x4_t*)from;
    if (second) hi += *(const f32x4_t*)(from + 4);
  }
  float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  finish_eight<false>(p, Fetched{}, p.e.act, v, n, m);
}

// ---------------------------------------------------------------- what goes before the products

// Rows to be padded with zeros from `cols` to `ld`; rows 0: none.
struct PadJob {
  const uint16_t* from;
  uint64_t from_ld, rows;
  uint32_t cols, ld;
  uint16_t* to;
};

__device__ __forceinline__ void pad_rows(const PadJob& j, uint32_t block, uint32_t blocks) {
  const uint64_t groups = j.ld / 8, all = j.rows * groups;
  for (uint64_t i = (uint64_t)block * blockDim.x + threadIdx.x; i < all; i += (uint64_t)blocks * blockDim.x) {
    const uint64_t r = i / groups;
    const uint32_t c = (uint32_t)(i % groups) * 8;
    const uint16_t* const row = j.from + r * j.from_ld;
    uint4 v;
    if (c + 8 <= j.cols) {
      v = load16_any(row + c);
    } else {
      uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e)
        if (c + e < j.cols) w[e >> 1] |= (uint32_t)row[c + e] << (16 * (e & 1));
      v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    store16(j.to + r * j.ld + c, v);
  }
}

// d as two BF16 values of one sign: `v` becomes its upper half, and what that leaves is
// given back, whose rounding is off by 2^-16 of d at most.  Cut, not rounded, so that no
// finite d becomes infinite, and never 0 but for d = 0: an infinite weight or token makes
// of the second product the infinity that it makes of the first, not a NaN (where nothing
// is left 2^-126 stands there, FP32's smallest, which is more than 2^-16 of a d below 2^-110).
__device__ __forceinline__ float take_upper(float& v) {
  v = __builtin_canonicalizef(v);  // a NaN's upper half is one then
  const float all = __builtin_fabsf(v);
  v = __uint_as_float(__float_as_uint(v) & 0xFFFF0000u);
  return __builtin_copysignf(__builtin_fmaxf(all - __builtin_fabsf(v), __builtin_fminf(all, 0x1p-126f)), v);
}

struct SlopeParams {
  const void* dy;
  uint64_t dy_stride;
  const void* pre;  // null: neither activation nor multiplier
  uint64_t pre_stride;
  const void* times;
  uint64_t times_stride;
  void* dtimes;
  uint64_t dtimes_stride;
  uint16_t* d;  // null: dy serves; rows of d_ld, zeros past the last feature
  uint32_t d_ld;
  uint64_t low;  // elements from d's upper parts to its lower ones; 0: d is BF16 as it is
  float* partial;  // null: no bias; [chunks][rows] (one chunk: dbias itself)
  uint32_t tokens, rows, chunk;
  int act, bf16;
  bool wide;
};

// d, dtimes and sums of d: a block takes 64 W features, W a lane, of `chunk` tokens, its
// waves the tokens in turn, two or four at a time.
template <int W, int WAVES>
__device__ __forceinline__ void slope_rows(const SlopeParams& p, uint32_t strip, uint32_t chunk) {
  constexpr int kAtOnce = W == 8 ? 2 : 4;
  __shared__ float s_sum[WAVES - 1][64 * W];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t row = (strip * 64 + lane) * W, left = row < p.rows ? p.rows - row : 0;
  const uint32_t end = p.tokens - chunk * p.chunk < p.chunk ? p.tokens : (chunk + 1) * p.chunk;
  auto load = [&](const void* from, uint64_t at, float(&v)[W]) {
    if constexpr (W == 8) load_eight(from, at, p.bf16, p.wide, left, v);
    else v[0] = left ? load_f32(from, at, p.bf16) : 0.0f;
  };
  float sum[W] = {};
  if (row < p.d_ld)
    for (uint64_t t0 = chunk * p.chunk + wave; t0 < end; t0 += WAVES * kAtOnce) {
      float v[kAtOnce][W], pre[kAtOnce][W], times[kAtOnce][W];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const uint64_t t = t0 + k * WAVES < end ? t0 + k * WAVES : t0;
        load(p.dy, t * p.dy_stride + row, v[k]);
        if (p.pre) load(p.pre, t * p.pre_stride + row, pre[k]);
        if (p.times) load(p.times, t * p.times_stride + row, times[k]);
      }
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const uint64_t t = t0 + k * WAVES;
        if (t >= end) break;
        if (p.pre) {
          float g[W];
#pragma unroll
          for (int i = 0; i < W; ++i) {
            const float2 a = activate2(p.act, pre[k][i]);
            g[i] = v[k][i] * a.x;
            v[k][i] *= p.times ? a.y * times[k][i] : a.y;
            if ((uint32_t)i >= left) v[k][i] = 0.0f;
          }
          if (p.dtimes) {
            const uint64_t at = t * p.dtimes_stride + row;
            if constexpr (W == 8) {
              store_eight(p.dtimes, at, p.bf16, p.wide, true, left, g);
            } else if (left) {
              if (p.bf16) ((uint16_t*)p.dtimes)[at] = (uint16_t)bf16x2_rne(__float_as_uint(g[0]), 0u);
              else ((float*)p.dtimes)[at] = g[0];
            }
          }
        }
#pragma unroll
        for (int i = 0; i < W; ++i) sum[i] += v[k][i];
        if (p.d) {
          uint16_t* const d = p.d + t * p.d_ld + row;
          if (p.low) {
            float rest[W];
#pragma unroll
            for (int i = 0; i < W; ++i) rest[i] = take_upper(v[k][i]);
            if constexpr (W == 8) store16(d + p.low, pack_eight(rest));
            else d[p.low] = (uint16_t)bf16x2_rne(__float_as_uint(rest[0]), 0u);
          }
          if constexpr (W == 8) store16(d, pack_eight(v[k]));
          else *d = (uint16_t)bf16x2_rne(__float_as_uint(v[k][0]), 0u);
        }
      }
    }
  if (!p.partial) return;
  if (wave) {
#pragma unroll
    for (int i = 0; i < W; ++i) s_sum[wave - 1][i * 64 + lane] = sum[i];
  }
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int i = 0; i < W; ++i) {
#pragma unroll
    for (int w = 0; w < WAVES - 1; ++w) sum[i] += s_sum[w][i * 64 + lane];
    if ((uint32_t)i < left) p.partial[(uint64_t)chunk * p.rows + row + i] = sum[i];
  }
}

// One launch for the copies and the gradient's elementwise part: `pad_w` and `pad_x`
// blocks, then strips * chunks.
template <int W, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void prepare_kernel(PadJob w, PadJob x, SlopeParams s, uint32_t pad_w,
                                                             uint32_t pad_x, uint32_t strips) {
  if (blockIdx.x < pad_w) return pad_rows(w, blockIdx.x, pad_w);
  if (blockIdx.x < pad_w + pad_x) return pad_rows(x, blockIdx.x - pad_w, pad_x);
  const uint32_t block = blockIdx.x - pad_w - pad_x;
  slope_rows<W, WAVES>(s, block % strips, block / strips);
}

// dbias from the chunks' sums: 64 features a block, its 4 waves a slice of the chunks each.
__global__ __launch_bounds__(256) void dbias_kernel(const float* partial, uint32_t chunks, uint32_t rows, float* dbias) {
  __shared__ float s[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t row = blockIdx.x * 64 + lane;
  float v = 0.0f;
  if (row < rows) {
#pragma unroll 4
    for (uint32_t c = wave; c < chunks; c += 4) v += partial[(uint64_t)c * rows + row];
  }
  s[wave][lane] = v;
  __syncthreads();
  if (wave == 0 && row < rows) dbias[row] = (s[0][lane] + s[1][lane]) + (s[2][lane] + s[3][lane]);
}

// ---------------------------------------------------------------- shapes

uint32_t up(uint32_t v, uint32_t to) { return (v + to - 1) / to * to; }
uint32_t parts(uint64_t v, uint32_t of) { return (uint32_t)((v + of - 1) / of); }

constexpr uint64_t kMaxStride = 1u << 20;    // a tile's byte offsets stay in 32 bits
constexpr uint32_t kTilesAtOnce = 1u << 22;  // of up to 512 threads; a multiple of 8, the XCDs
constexpr uint64_t kSumBytes = 32ull << 20;  // the most that splits' sums take
constexpr uint32_t kMinSplit = 256;          // of k
constexpr uint32_t kFewTokens = kLinearFewTokens;
constexpr uint64_t kStreamBytes = 64ull << 20;  // results of more are written past the caches

// Few values before the gradient's products: a feature a lane, all tokens in one block's 16
// waves and dbias summed there.  Else eight features a lane, chunks of tokens and a launch
// that adds their sums.  us of a gradient with a weight of 64 columns, so and the other way,
// BF16 silu and multiplier / FP32 gelu and bias: 17 tokens, 1,003 rows 21 and 32 / 21 and 34;
// 128, 4,864 29.5 and 28.9 / 29.5 and 33.9; 17, 27,648 44 and 45 / 43 and 50; 64, 18,944 48 and 46 /
// 47 and 51; 128, 27,648 66 and 53 / 58 and 58; 200, 200 22 and 16 / 20 and 21; 512, 1,003 44 and 34.
bool few_values(uint64_t tokens, uint64_t rows) { return tokens <= 128 && tokens * rows <= 1u << 20; }

// Time of a product in thousands of cycles: rounds of blocks, each with a fixed part and
// one per 64 of k (which grows with the CUs that share the L2s), and, with splits, their
// sums' way and a launch.  The tiles' figures are those measured for the cross entropy's,
// whose epilogue is another.  us as chosen, and by 256 x 256, 256 x 128 and 128 x 64 without
// splits, BF16 with silu and multiplier, forward (pre-activation too) / gradient:
//      64 tokens, 18,944 x 3,584    31, 68, 41, 30        106, 699, 432, 346
//   1,024 tokens,  4,864 x   896    22, 41, 23, 33         75, 226, 138, 127
//   2,048 tokens, 18,944 x 3,584   279, 281, 266, 510   1,003, 1,249, 1,036, 2,062
//   4,096 tokens,  4,864 x   896    84, 85, 68, 104       250, 363, 232, 347
struct TileCost {
  uint32_t bm, bn;
  float fixed, step, shared;
};
constexpr TileCost kCosts[3] = {{256, 256, 18.0f, 2.2f, 0.0f}, {256, 128, 11.0f, 1.2f, 1.1f}, {128, 64, 6.0f, 0.9f, 0.6f}};

struct Shape {
  int tile;
  uint32_t splits;
};

// each: steps of 64 k, two for pairs.
Shape shape_of(uint32_t m, uint32_t n, uint32_t k, uint32_t each) {
  constexpr float kCus = 256.0f;
  Shape best = {2, 1};
  float least = 0.0f;
  const uint64_t bytes = (uint64_t)n * up(m, 4) * 4;
  for (int i = 0; i < 3; ++i) {
    const TileCost& c = kCosts[i];
    const float tiles = (float)parts(m, c.bm) * (float)parts(n, c.bn);
    for (uint32_t splits = 1; splits <= 64; ++splits) {
      if (splits > 1 && (splits * bytes > kSumBytes || k < splits * kMinSplit || tiles * splits > 2 * kCus)) break;
      const float blocks = tiles * splits;
      const float rounds = (float)(uint64_t)((blocks + kCus - 1) / kCus), busy = blocks < kCus ? blocks / kCus : 1.0f;
      const float steps = (float)(parts(parts(k, splits), kGemmK) * each);
      float cost = rounds * (c.fixed + (c.step + c.shared * busy) * steps);
      if (splits > 1) cost += 8.0f + (float)((splits + 1) * bytes) / 2e6f;
      if (least == 0.0f || cost < least) {
        least = cost;
        best = {i, splits};
      }
    }
  }
  return best;
}

template <typename T>
void set_tiles(ProductParams& p) {
  p.tiles_m = parts(p.m, T::BM);
  p.tiles_n = parts(p.n, T::BN);
}

template <bool AK, bool BK>
using TileL = Gemm<256, 256, 2, 4, 2, AK, BK>;
template <bool AK, bool BK>
using TileM = Gemm<256, 128, 4, 2, 3, AK, BK>;
template <bool AK, bool BK>
using TileS = Gemm<128, 64, 4, 1, 4, AK, BK>;

template <bool AK, bool BK, int ACT, bool PAIRS>
void run_product(ProductParams p, float* sums, hipStream_t stream) {
  const Shape s = shape_of(p.m, p.n, p.k, PAIRS ? 2 : 1);
  p.stream = (uint64_t)p.m * p.n * (p.e.out_bf16 ? 2 : 4) >= kStreamBytes;
  p.m_ld = up(p.m, 4);
  p.sums = s.splits > 1 ? sums : nullptr;
  p.k_split = up(parts(p.k, s.splits), kGemmK);
  auto launch = [&](auto tile) {
    typedef decltype(tile) T;
    set_tiles<T>(p);
    const uint64_t tiles = (uint64_t)p.tiles_m * p.tiles_n;
    for (uint64_t first = 0; first < tiles; first += kTilesAtOnce) {
      p.first_tile = (uint32_t)first;
      const uint64_t left = tiles - first;
      hipLaunchKernelGGL((product_kernel<T, AK, BK, ACT, PAIRS>), dim3(left < kTilesAtOnce ? (uint32_t)left : kTilesAtOnce, s.splits),
                         dim3(T::kThreads), 0, stream, p);
    }
  };
  if (s.tile == 0) launch(TileL<AK, BK>{});
  else if (s.tile == 1) launch(TileM<AK, BK>{});
  else launch(TileS<AK, BK>{});
  if (s.splits > 1) {
    const uint64_t threads = (uint64_t)p.n * parts(p.m, 8);
    hipLaunchKernelGGL(join_kernel, dim3(parts(threads, 256)), dim3(256), 0, stream, p, s.splits);
  }
}

// dx and dW: where the smallest tiles of both are fewer than CUs, and the sums short, one
// launch instead of two to four (each costs 3 us on the host and as much on the GPU), whose
// blocks take a tile's steps one after the other.  us in one launch and in several, d of one
// part: k up to 512 9.7 and 13.0 (128 x 512 x 512), 1,024 10.4 and 16.1, 2,048 17.4 and 16.2 to
// 16.9 and 17.6 (2,048 x 128 x 128, 300 x 2,040 x 520); of two parts: 512 18.4 and 23.0, 1,024 25.3
// and 26.2, 2,048 41.9 and 26.2.
template <bool PAIRS>
void run_gradients(ProductParams x, ProductParams w, float* sums, hipStream_t stream) {
  typedef TileS<true, false> TX;
  typedef TileS<true, true> TW;
  set_tiles<TX>(x);
  set_tiles<TW>(w);
  const uint64_t tiles = (uint64_t)x.tiles_m * x.tiles_n + (uint64_t)w.tiles_m * w.tiles_n;
  constexpr uint32_t kMost = PAIRS ? 1024 : 2048;  // of k
  if (tiles <= 256 && x.k <= kMost && w.k <= kMost) {
    hipLaunchKernelGGL((both_kernel<TX, TW, PAIRS>), dim3((uint32_t)tiles), dim3(TX::kThreads), 0, stream, x, w);
    return;
  }
  run_product<true, false, kPlain, PAIRS>(x, sums, stream);
  run_product<true, true, kPlain, PAIRS>(w, sums, stream);
}

struct Plan {
  uint32_t ld, d_ld, chunk, chunks;
  uint64_t w, x, d, partial, sums;
  uint64_t low;  // d's lower parts: the forward pass's workspace ends here
  uint64_t total;
};

Plan plan_of(uint32_t tokens, uint32_t rows, uint32_t cols) {
  Plan q;
  q.ld = up(cols, 8);
  q.d_ld = up(rows, 8);
  // chunks of tokens for some eight blocks a CU; few tokens in one
  const uint32_t strips = parts(rows, 512), wanted = strips < 2048 ? 2048 / strips : 1;
  q.chunk = few_values(tokens, rows) ? tokens : up(parts(tokens, wanted), 16);
  q.chunks = parts(tokens, q.chunk);
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) {
    const uint64_t here = at;
    at += (bytes + 255) & ~255ull;
    return here;
  };
  q.w = take(cols % 8 ? (uint64_t)rows * q.ld * 2 : 0);
  q.x = take((uint64_t)tokens * q.ld * 2);
  q.d = take((uint64_t)tokens * q.d_ld * 2);
  q.partial = take((uint64_t)q.chunks * rows * 4);
  auto sums = [&](uint32_t m, uint32_t n, uint32_t k, uint32_t each) -> uint64_t {
    const Shape s = shape_of(m, n, k, each);
    return s.splits > 1 ? (uint64_t)s.splits * n * up(m, 4) * 4 : 0;
  };
  uint64_t most = sums(rows, tokens, q.ld, 1);
  for (uint32_t each : {1u, 2u})
    for (uint64_t v : {sums(cols, tokens, rows, each), sums(cols, rows, tokens, each)})
      if (v > most) most = v;
  q.sums = take(most);
  q.low = take((uint64_t)tokens * q.d_ld * 2);
  q.total = at;
  return q;
}

// A matrix as the products take it, rows of 16-byte groups and not too far apart: itself,
// or a copy in `to`.
struct Tidy {
  const uint16_t* p;
  uint64_t ld;
  PadJob job;
  uint32_t blocks;
};

Tidy tidy(const uint16_t* from, uint64_t stride, uint64_t rows, uint32_t cols, uint16_t* to, uint32_t ld,
          uint32_t threads) {
  if (cols % 8 == 0 && stride % 8 == 0 && stride <= kMaxStride) return {from, stride, {}, 0};
  const uint64_t blocks = (rows * (ld / 8) + threads - 1) / threads;
  return {to, ld, {from, stride, rows, cols, ld, to}, blocks < 8192 ? (uint32_t)blocks : 8192};
}

}  // namespace

uint64_t linear_needs(bool forward, uint32_t tokens, uint32_t rows, uint32_t cols) {
  if (forward && tokens <= kFewTokens) return 0;
  const Plan q = plan_of(tokens, rows, cols);
  return forward ? q.low : q.total;
}

// A call of fewer tokens may take more splits, and shorter chunks: bounds on those parts.
uint64_t linear_bytes(uint32_t tokens, uint32_t rows, uint32_t cols) {
  const Plan q = plan_of(tokens, rows, cols);
  const uint32_t strips = parts(rows, 512);
  const uint64_t chunks = strips < 2048 ? 2048 / strips : 1;
  uint64_t sums = 0;  // at most k / kMinSplit splits
  auto product = [&](uint64_t m, uint64_t n, uint64_t k) {
    const uint64_t bytes = k / kMinSplit * n * (m + 3) * 4;
    if (bytes > sums) sums = bytes;
  };
  product(rows, tokens, q.ld);
  product(cols, tokens, rows);
  product(cols, rows, tokens);
  if (sums > kSumBytes) sums = kSumBytes;
  return q.partial + ((chunks * rows * 4 + 255) & ~255ull) + ((sums + 255) & ~255ull) + q.total - q.low;
}

hipError_t launch_linear(const LinearParams& c, char* ws, hipStream_t stream) {
  if (c.tokens <= kFewTokens) {
    const uint64_t n = (uint64_t)c.rows * c.cols;
    LowpMatmulParams p = {(const uint8_t*)c.weight, nullptr, 1.0f, c.rows, c.cols, 2 * n, 0, c.x, c.x_stride, c.tokens,
                          c.y, c.y_stride, c.e.out_bf16, c.e};
    return launch_lowp_matmul(kWeightBf16, true, p, stream);
  }
  const Plan q = plan_of(c.tokens, c.rows, c.cols);
  const Tidy w = tidy(c.weight, c.cols, c.rows, c.cols, (uint16_t*)(ws + q.w), q.ld, 256);
  const Tidy x = tidy(c.x, c.x_stride, c.tokens, c.cols, (uint16_t*)(ws + q.x), q.ld, 256);
  if (w.blocks + x.blocks)
    hipLaunchKernelGGL((prepare_kernel<8, 4>), dim3(w.blocks + x.blocks), dim3(256), 0, stream, w.job, x.job,
                       SlopeParams{}, w.blocks, x.blocks, 1u);
  ProductParams p = {};
  p.a = {w.p, w.ld, c.rows};
  p.b = {x.p, x.ld, c.tokens};
  p.m = c.rows;
  p.n = c.tokens;
  p.k = q.ld;
  p.out = c.y;
  p.out_ld = c.y_stride;
  p.e = c.e;
  const uint64_t unit = c.e.out_bf16 ? 8 : 4;
  p.wide = c.y_stride % unit == 0 && (!c.e.pre || c.e.pre_stride % unit == 0) &&
           (!c.e.times || c.e.times_stride % unit == 0) && (!c.e.residual || c.e.residual_stride % unit == 0);
  float* const sums = (float*)(ws + q.sums);
  switch (c.e.act) {
    case kActRelu: run_product<false, false, kActRelu, false>(p, sums, stream); break;
    case kActSilu: run_product<false, false, kActSilu, false>(p, sums, stream); break;
    case kActGelu: run_product<false, false, kActGelu, false>(p, sums, stream); break;
    case kActGeluTanh: run_product<false, false, kActGeluTanh, false>(p, sums, stream); break;
    default: run_product<false, false, kActNone, false>(p, sums, stream);
  }
  return hipGetLastError();
}

hipError_t launch_linear_grad(const LinearGradParams& c, char* ws, hipStream_t stream) {
  const Plan q = plan_of(c.tokens, c.rows, c.cols);
  const bool few = few_values(c.tokens, c.rows);
  const uint32_t threads = few ? 1024 : 256;
  const Tidy w = tidy(c.weight, c.cols, c.rows, c.cols, (uint16_t*)(ws + q.w), q.ld, threads);
  const Tidy x = tidy(c.x, c.x_stride, c.tokens, c.cols, (uint16_t*)(ws + q.x), q.ld, threads);
  // d, dtimes and dbias
  const bool exact = c.bf16 && !c.times && (c.act == kActNone || c.act == kActRelu);  // d is dy or 0
  const bool serves = exact && !c.act && c.rows % 8 == 0 && c.dy_stride % 8 == 0 && c.dy_stride <= kMaxStride;
  SlopeParams s = {};
  s.dy = c.dy;
  s.dy_stride = c.dy_stride;
  s.pre = c.act || c.times ? c.pre : nullptr;
  s.pre_stride = c.pre_stride;
  s.times = c.times;
  s.times_stride = c.times_stride;
  s.dtimes = c.dtimes;
  s.dtimes_stride = c.dtimes_stride;
  s.d = serves ? nullptr : (uint16_t*)(ws + q.d);
  s.d_ld = q.d_ld;
  s.low = exact ? 0 : (q.low - q.d) / 2;
  s.partial = !c.dbias ? nullptr : q.chunks == 1 ? c.dbias : (float*)(ws + q.partial);
  s.tokens = c.tokens;
  s.rows = c.rows;
  s.chunk = q.chunk;
  s.act = c.act;
  s.bf16 = c.bf16;
  const uint64_t unit = c.bf16 ? 8 : 4;
  s.wide = c.dy_stride % unit == 0 && (!s.pre || c.pre_stride % unit == 0) &&
           (!c.times || (c.times_stride % unit == 0 && (!c.dtimes || c.dtimes_stride % unit == 0)));
  // few tokens: a feature a lane and 16 waves, for more blocks and fewer turns
  const uint32_t strips = parts(c.rows, few ? 64 : 512);
  const uint32_t blocks = w.blocks + x.blocks + (s.d || s.partial ? strips * q.chunks : 0);
  if (blocks && few)
    hipLaunchKernelGGL((prepare_kernel<1, 16>), dim3(blocks), dim3(1024), 0, stream, w.job, x.job, s, w.blocks, x.blocks,
                       strips);
  else if (blocks)
    hipLaunchKernelGGL((prepare_kernel<8, 4>), dim3(blocks), dim3(256), 0, stream, w.job, x.job, s, w.blocks, x.blocks,
                       strips);
  if (c.dbias && q.chunks > 1)
    hipLaunchKernelGGL(dbias_kernel, dim3(parts(c.rows, 64)), dim3(256), 0, stream, s.partial, q.chunks, c.rows, c.dbias);
  const uint16_t* const d = serves ? (const uint16_t*)c.dy : s.d;
  const uint64_t d_ld = serves ? c.dy_stride : q.d_ld;
  ProductParams p = {};
  p.e.out_bf16 = 1;
  p.a = {w.p, w.ld, q.ld};
  p.b = {d, d_ld, c.tokens};
  p.m = c.cols;
  p.n = c.tokens;
  p.k = c.rows;
  p.out = c.dx;
  p.out_ld = c.dx_stride;
  p.low = s.low * 2;
  p.wide = c.dx_stride % 8 == 0;
  ProductParams g = p;
  g.a = {x.p, x.ld, q.ld};
  g.b = {d, d_ld, q.d_ld};
  g.n = c.rows;
  g.k = c.tokens;
  g.out = c.dweight;
  g.out_ld = c.cols;
  g.wide = c.cols % 8 == 0;
  if (exact) run_gradients<false>(p, g, (float*)(ws + q.sums), stream);
  else run_gradients<true>(p, g, (float*)(ws + q.sums), stream);
  return hipGetLastError();
}

}  // namespace pulse
