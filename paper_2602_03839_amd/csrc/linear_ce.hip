// linear_ce.hip -- softmax cross entropy of z = s x W^T over a large vocabulary,
// forward and backward, with the logits in registers only.
//
// Forward: a block computes a tile of 256 (128 for few) vocabulary entries by its tokens
// (gemm_tile.hpp), reduces it per token to the largest logit and the sum of
// exponentials below it, and writes those two numbers; a second kernel joins a
// token's pairs.  The logit of the target is written by the lane that has it.
//
// Backward: the vocabulary is taken in pieces.  For a piece, the logits are
// computed again and turned into G[t][v] = g_t s (e^(z - lse) - [v = y_t]) in
// BF16, and two products follow: dx += G W (FP32 sums, kept across pieces) and
// dw = G^T X.  G of one piece is all that is ever stored, in BF16 since the
// products need a BF16 operand.  What the rounding takes is added back:
//   to dx, what the target's entry lost (`rest`, FP32) times W[y]; the same for every
//     other entry that lost kLargeLoss of the token's dloss or more (at most 16, which
//     have a sixteenth of the probability or more each); and what the others lost
//     together times the mean of 64 rows of W.  The exact row of G sums to zero, so
//     a direction that the rows of W share cancels in dx, but the rounded row does
//     not: with rows 10 times as long as what they differ by and half the probability on
//     one entry beside the target, dx was 0.009 off in the 2-norm, a token's 0.026
//     (0.0017 and 0.0020 now, which is the rounding of dx itself);
//   to dw, rest x in row y.  The other entries' roundings are relative to each and
//     independent, and average out over many tokens; for few, what they lose is kept
//     as a second BF16 matrix.  A row that one token's entry dominates, not its
//     target, is left with the rounding of that entry beside its own (0.0024).
//
// The three products of the backward pass and the one of the forward pass are
// bound by the matrix cores for many tokens (4,096 at 152,064 x 3,584, 4.46 TFLOP
// each: forward 3.5 ms, G 3.8, dx 3.5, dw 4.0), by the weight's bytes for few (61 at
// 152,064 x 5,120, 1.56 GB: 288, 305 and 278 us to read it, 294 to write dw).
#include "device_common.hpp"
#include "gemm_tile.hpp"
#include "head.hpp"

namespace pulse {

namespace {

constexpr uint32_t kBand = 8;  // tiles in m of a band: 32 CUs then work on 8 by 4
constexpr float kLog2e = 1.4426950408889634f;

// An entry of G that loses this share of |dloss| or more in the rounding is kept by itself:
// BF16 takes at most 2^-8 of a value, so it has p >= 1/16, and a token has 16 at most.
constexpr float kLargeLoss = 0x1p-12f;
constexpr uint32_t kLargeLosses = 16;
constexpr uint32_t kMeanRows = 64;  // of W, evenly spread, for the mean row: an eighth of a row off
constexpr uint32_t kLostTile = 128;  // entries to a sum of losses: the smallest tile's

// An entry of a token that is not its target, and what it lost in the rounding.
struct LargeLoss {
  int32_t v;
  float lost;
};

// 2^x (v_exp_f32, 1 ulp).
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A pair (largest logit, sum of exponentials below it) as a sum below `top`.  Where the
// largest is infinite the exponentials are taken as they are: the sum is 0 or
// infinite.  A NaN stays one.
__device__ __forceinline__ float below(float2 q, float top) {
  return q.y * (q.x == top ? 1.0f : exp2_fast((q.x - top) * kLog2e));
}

// Where target y lies among a lane's entries first + 16 i + e (e < 4), as 16 i + e;
// -1 where it does not.
__device__ __forceinline__ int32_t entry_of(int64_t y, uint32_t first, int rows) {
  const int64_t d = y - (int64_t)first;
  return d >= 0 && d < rows * 16 && (d & 15) < 4 ? (int32_t)d : -1;
}

// ---------------------------------------------------------------- logits

struct LogitParams {
  const uint16_t* w;
  uint64_t w_ld;
  const uint16_t* x;
  uint64_t x_ld;
  const int64_t* targets;
  uint32_t tokens, hidden;
  uint32_t v_begin, v_end;  // the piece; forward: the whole vocabulary
  uint32_t tiles_m, tiles_n;
  uint32_t first_tile;  // of this launch
  float scale;
  // forward
  float2* part;  // [tokens][tiles_m]: largest logit, sum of exponentials below it
  float* hit;    // [tokens]: the target's logit
  // backward
  const float* lse;
  const float* dloss;
  uint32_t vocab;
  uint16_t* g;  // [tokens][g_ld]
  uint64_t g_ld;
  float* rest;  // [tokens]: what the target's entry lost in the rounding
  float* lost;  // [tokens][lost_ld]: what the other entries lost, by kLostTile of the vocabulary
  uint32_t lost_ld;
  uint32_t* large_count;  // [tokens]: of `large`, zero before the first piece; above
                          // kLargeLosses, with an lse that is not the forward's, none count
  LargeLoss* large;       // [tokens][kLargeLosses], in any order
  bool rest_rows;  // what every entry lost follows G, as as many rows again
};

template <typename T>
__global__ __launch_bounds__(T::kThreads) void ce_forward_kernel(LogitParams p) {
  __shared__ alignas(1024) char lds[T::kLds];
  uint32_t tm, tn;
  gemm_tile_of(p.first_tile + blockIdx.x, p.tiles_m, p.tiles_n, kBand, tm, tn);
  const uint32_t m0 = p.v_begin + tm * T::BM, n0 = tn * T::BN;
  typename T::Acc acc;
  const GemmOperand a = {p.w + (uint64_t)m0 * p.w_ld, p.w_ld, p.v_end - m0};
  const GemmOperand b = {p.x + (uint64_t)n0 * p.x_ld, p.x_ld, p.tokens - n0};
  T::run(lds, a, b, 0, p.hidden, acc);

  // The work per entry is kept to a scaling, a maximum, a difference, a factor, an
  // exponential and a sum: with a short hidden size this is a third of the time.
  // The end of the vocabulary and the target are looked at where they occur.
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float2(*s_part)[T::BN] = (float2(*)[T::BN])lds;  // [WM][BN]
  const uint32_t mine = m0 + T::m_of(0, lane, wave);  // the lane's entries: + 16 i + e
#pragma unroll
  for (int j = 0; j < T::FN; ++j) {
    const uint32_t n = T::n_of(j, lane, wave), t = n0 + n;
#pragma unroll
    for (int i = 0; i < T::FM; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][j][e] *= p.scale;
    if (m0 + T::BM > p.v_end) {
#pragma unroll
      for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (mine + i * 16 + e >= p.v_end) acc[i][j][e] = -INFINITY;
    }
    const int32_t at = entry_of(t < p.tokens ? p.targets[t] : -1, mine, T::FM);
    if (__builtin_amdgcn_ballot_w64(at >= 0)) {
      float z = 0.0f;
#pragma unroll
      for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) z = at == i * 16 + e ? acc[i][j][e] : z;
      if (at >= 0) p.hit[t] = z;
    }
    // a NaN is passed over here and comes out of the sum
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < T::FM; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) top = __builtin_fmaxf(top, acc[i][j][e]);
    top = __builtin_fmaxf(top, __shfl_xor(top, 16));
    top = __builtin_fmaxf(top, __shfl_xor(top, 32));
    const float from = __builtin_fabsf(top) == INFINITY ? 0.0f : top;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < T::FM; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += exp2_fast((acc[i][j][e] - from) * kLog2e);
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (lane < 16) s_part[wave / T::WN][n] = make_float2(top, sum);
  }
  __syncthreads();
  for (uint32_t n = threadIdx.x; n < T::BN; n += T::kThreads) {
    float top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int w = 0; w < T::WM; ++w) top = __builtin_fmaxf(top, s_part[w][n].x);
#pragma unroll
    for (int w = 0; w < T::WM; ++w) sum += below(s_part[w][n], top);
    if (n0 + n < p.tokens) p.part[(uint64_t)(n0 + n) * p.tiles_m + tm] = make_float2(top, sum);
  }
}

template <typename T>
__global__ __launch_bounds__(T::kThreads) void ce_grad_kernel(LogitParams p) {
  constexpr int kRows = T::BM * T::BN * 2, kSums = T::WM * T::BN * 4;  // of the results' way out
  __shared__ alignas(1024) char lds[T::kLds > kRows + kSums ? T::kLds : kRows + kSums];
  float(*const s_lost)[T::BN] = (float(*)[T::BN])(lds + kRows);  // [WM][BN]
  uint32_t tm, tn;
  gemm_tile_of(p.first_tile + blockIdx.x, p.tiles_m, p.tiles_n, kBand, tm, tn);
  const uint32_t m0 = p.v_begin + tm * T::BM, n0 = tn * T::BN;
  typename T::Acc acc;
  const GemmOperand a = {p.w + (uint64_t)m0 * p.w_ld, p.w_ld, p.v_end - m0};
  const GemmOperand b = {p.x + (uint64_t)n0 * p.x_ld, p.x_ld, p.tokens - n0};
  T::run(lds, a, b, 0, p.hidden, acc);

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t y[T::FN];
  float by[T::FN], lse[T::FN];
#pragma unroll
  for (int j = 0; j < T::FN; ++j) {
    const uint32_t t = n0 + T::n_of(j, lane, wave);
    y[j] = t < p.tokens ? p.targets[t] : -1;
    const bool kept = y[j] >= 0 && y[j] < (int64_t)p.vocab;
    if (!kept) y[j] = -1;
    by[j] = kept ? p.dloss[t] * p.scale : 0.0f;
    lse[j] = kept ? p.lse[t] : 0.0f;
  }
  const uint32_t mine = m0 + T::m_of(0, lane, wave);  // the lane's entries: + 16 i + e
  int32_t at[T::FN];                                  // which of them is the target
  auto rounded = [&](int i, int j) {
    uint2 o;
    o.x = bf16x2_rne(__float_as_uint(acc[i][j][0]), __float_as_uint(acc[i][j][1]));
    o.y = bf16x2_rne(__float_as_uint(acc[i][j][2]), __float_as_uint(acc[i][j][3]));
    return o;
  };
  auto losses = [&](int i, int j) {  // exact
    const uint2 o = rounded(i, j);
    return acc[i][j] - f32x4_t{__uint_as_float(o.x << 16), __uint_as_float(o.x & 0xFFFF0000u),
                               __uint_as_float(o.y << 16), __uint_as_float(o.y & 0xFFFF0000u)};
  };
#pragma unroll
  for (int j = 0; j < T::FN; ++j) {
    at[j] = entry_of(y[j], mine, T::FM);
    const bool any = __builtin_amdgcn_ballot_w64(at[j] >= 0) != 0;
#pragma unroll
    for (int i = 0; i < T::FM; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        // z rounded as in the forward pass and the difference before the factor:
        // exact where z is near lse, so a large logit costs a likely target no digits
        acc[i][j][e] = exp2_fast((acc[i][j][e] * p.scale - lse[j]) * kLog2e);
    if (any) {
#pragma unroll
      for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = at[j] == i * 16 + e ? acc[i][j][e] - 1.0f : acc[i][j][e];
    }
#pragma unroll
    for (int i = 0; i < T::FM; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][j][e] = y[j] >= 0 ? acc[i][j][e] * by[j] : 0.0f;
    if (m0 + T::BM > p.v_end) {
#pragma unroll
      for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (mine + i * 16 + e >= p.v_end) acc[i][j][e] = 0.0f;
    }
    const uint32_t n = T::n_of(j, lane, wave);
    float lost = 0.0f, most = 0.0f;
#pragma unroll
    for (int i = 0; i < T::FM; ++i) {
      const f32x4_t r = losses(i, j);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        lost += r[e];
        most = __builtin_fmaxf(most, __builtin_fabsf(r[e]));
      }
    }
    if (any) {
      float rest = 0.0f;
#pragma unroll
      for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) rest = at[j] == i * 16 + e ? acc[i][j][e] : rest;
      rest -= __uint_as_float(bf16x2_rne(__float_as_uint(rest), 0u) << 16);
      if (at[j] >= 0) {
        p.rest[n0 + n] = rest;
        lost -= rest;
      }
    }
    const float large = kLargeLoss * __builtin_fabsf(by[j]);
    if (__builtin_amdgcn_ballot_w64(most >= large && most > 0.0f)) {
      uint32_t which = 0;
#pragma unroll
      for (int i = 0; i < T::FM; ++i) {
        const f32x4_t r = losses(i, j);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float size = __builtin_fabsf(r[e]);
          which |= (uint32_t)(size >= large && size > 0.0f && at[j] != i * 16 + e) << (i * 4 + e);
        }
      }
      uint32_t slot = which ? atomicAdd(p.large_count + n0 + n, (uint32_t)__builtin_popcount(which)) : 0;
      for (; which && slot < kLargeLosses; ++slot) {
        const int k = __builtin_ctz(which);
        which &= which - 1;
        float r = 0.0f;
#pragma unroll
        for (int i = 0; i < T::FM; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) r = k == i * 4 + e ? acc[i][j][e] : r;
        r -= __uint_as_float(bf16x2_rne(__float_as_uint(r), 0u) << 16);
        p.large[(uint64_t)(n0 + n) * kLargeLosses + slot] = {(int32_t)(mine + (k >> 2) * 16 + (k & 3)), r};
      }
    }
    lost += __shfl_xor(lost, 16);
    lost += __shfl_xor(lost, 32);
    if (lane < 16) s_lost[wave / T::WN][n] = lost;
  }
  uint16_t* const out = p.g + n0 * p.g_ld + (m0 - p.v_begin);
  T::template store_rows<false, true>(lds, out, p.g_ld, T::BM, p.tokens - n0, rounded);  // meets between
  for (uint32_t n = threadIdx.x; n < T::BN; n += T::kThreads) {
    float lost = 0.0f;
#pragma unroll
    for (int w = 0; w < T::WM; ++w) lost += s_lost[w][n];
    if (n0 + n >= p.tokens) continue;
    const uint32_t slot = m0 / kLostTile;
    float* const to = p.lost + (uint64_t)(n0 + n) * p.lost_ld + slot;
    to[0] = lost;
    if (T::BM > kLostTile && slot + 1 < p.lost_ld) to[1] = 0.0f;  // the tile's other half
  }
  if (p.rest_rows) {  // few tokens: the rests of all entries, as rows of their own
    __syncthreads();
    T::template store_rows<false, true>(lds, out + (uint64_t)p.tokens * p.g_ld, p.g_ld, T::BM, p.tokens - n0,
                                  [&](int i, int j) {
                                    acc[i][j] = losses(i, j);
                                    return rounded(i, j);
                                  });
  }
}

// A token's pairs joined, one wave each, from token `first` on.
__global__ __launch_bounds__(256) void ce_join_kernel(const float2* part, const float* hit,
                                                      const int64_t* targets, uint32_t first,
                                                      uint32_t tokens, uint32_t vocab, uint32_t tiles,
                                                      float* loss, float* lse) {
  const uint32_t t = first + blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= tokens) return;
  const int lane = threadIdx.x & 63;
  const float2* mine = part + (uint64_t)t * tiles;
  float top = -INFINITY, sum = 0.0f;
  for (uint32_t i = lane; i < tiles; i += 64) top = __builtin_fmaxf(top, mine[i].x);
#pragma unroll
  for (int x = 1; x < 64; x *= 2) top = __builtin_fmaxf(top, __shfl_xor(top, x));
  for (uint32_t i = lane; i < tiles; i += 64) sum += below(mine[i], top);
  sum = wave_sum(sum);
  if (lane == 0) {
    const float rest = logf(sum);
    const int64_t y = targets[t];
    lse[t] = top + rest;
    // the difference first: a target that is the largest logit leaves log(sum)
    loss[t] = y >= 0 && y < (int64_t)vocab ? (top - hit[t]) + rest : 0.0f;
  }
}

// ---------------------------------------------------------------- products of the gradient

struct GradParams {
  GemmOperand a, b;  // at the first tile
  uint32_t m, n, k;  // sizes
  uint32_t tiles_m, tiles_n, band;
  uint32_t k_split;  // k per blockIdx.y, a multiple of 64
  float* sums;       // dx: [splits][n][m]
  int add;           // dx: onto what is there
  uint16_t* out;     // dw: [n][out_ld]
  uint64_t out_ld;
  const int32_t* y;  // dw: [k] targets, -1 for none
  uint32_t v_begin;  // the piece's first entry
  const float* rest;
};

template <typename T, bool AK, bool BK>
__device__ __forceinline__ void grad_tile(const GradParams& p, char* lds, uint32_t id, uint32_t split,
                                          uint32_t& m0, uint32_t& n0, typename T::Acc& acc) {
  uint32_t tm, tn;
  gemm_tile_of(id, p.tiles_m, p.tiles_n, p.band, tm, tn);
  m0 = tm * T::BM;
  n0 = tn * T::BN;
  const GemmOperand a = {p.a.p + (AK ? (uint64_t)m0 : m0 * p.a.ld), p.a.ld, p.a.limit - m0};
  const GemmOperand b = {p.b.p + (BK ? (uint64_t)n0 : n0 * p.b.ld), p.b.ld, p.b.limit - n0};
  const uint32_t k0 = split * p.k_split;
  // a split past the end has no k and gives zeros
  const uint32_t k1 = k0 >= p.k ? k0 : p.k - k0 < p.k_split ? p.k : k0 + p.k_split;
  T::run(lds, a, b, k0, k1, acc);
}

// Block `id` of dx: its split's part of a tile of the sums.
template <typename T>
__device__ void dx_block(const GradParams& p, char* lds, uint32_t id) {
  const uint32_t tiles = p.tiles_m * p.tiles_n, split = id / tiles;
  uint32_t m0, n0;
  typename T::Acc acc;
  grad_tile<T, true, false>(p, lds, id % tiles, split, m0, n0, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float* sums = p.sums + (uint64_t)split * p.n * p.m;
#pragma unroll
  for (int j = 0; j < T::FN; ++j) {
    const uint32_t n = n0 + T::n_of(j, lane, wave);
    if (n >= p.n) continue;
#pragma unroll
    for (int i = 0; i < T::FM; ++i) {
      const uint32_t m = m0 + T::m_of(i, lane, wave);
      if (m >= p.m) continue;  // p.m is a multiple of 8
      f32x4_t* at = (f32x4_t*)(sums + (uint64_t)n * p.m + m);
      *at = p.add ? *at + acc[i][j] : acc[i][j];
    }
  }
}

// Adds rest[t] x[t] to the row of the tile that is token t's target: more steps of the
// product, of 64 such tokens each.  The block looks through the targets and collects
// those of its rows in LDS in a fixed order; their rows of x are one operand, and
// the other is zeros but for each token's rest (BF16 of a number that is itself
// what BF16 dropped) in the column of its target.
template <typename T>
__device__ void add_rests(const GradParams& p, char* lds, uint32_t m0, uint32_t n0, typename T::Acc& acc) {
  int lane = threadIdx.x & 63;
  // opaque, so that no address below is worked out before the product and kept
  // in registers through it
  asm volatile("" : "+v"(lane));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr uint32_t kSeen = 4 * T::kThreads;                // tokens looked at at a time
  uint32_t* const s_list = (uint32_t*)(lds + T::kStage);      // [kSeen], past the first step's tiles
  uint32_t* const s_count = s_list + kSeen;                  // [kWaves]
  static_assert(T::kStage >= 4 * kSeen + 4 * T::kWaves, "the list fits the second buffer");
  char* const tile_b = lds + T::A::kBytes;
  const GemmOperand a = {p.a.p + m0, p.a.ld, p.a.limit - m0};
  for (uint32_t base = 0; base < p.k; base += kSeen) {
    uint64_t hits[4];
    uint32_t count = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t t = base + q * T::kThreads + threadIdx.x;
      const uint32_t at = (t < p.k ? (uint32_t)p.y[t] : ~0u) - p.v_begin - n0;  // none: not below BN
      hits[q] = __builtin_amdgcn_ballot_w64(at < T::BN);
      count += (uint32_t)__popcll(hits[q]);
    }
    if (lane == 0) s_count[wave] = count;
    __syncthreads();
    uint32_t all = 0, before = 0;
#pragma unroll
    for (int w = 0; w < T::kWaves; ++w) {
      if (w == wave) before = all;
      all += s_count[w];
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (hits[q] >> lane & 1)
        s_list[before + __popcll(hits[q] & ((1ull << lane) - 1))] = base + q * T::kThreads + threadIdx.x;
      before += (uint32_t)__popcll(hits[q]);
    }
    __syncthreads();
    for (uint32_t h = 0; h < all; h += kGemmK) {
      const uint32_t left = all - h;
      T::A::gather(a, lds, wave, lane, [&](uint32_t k) { return k < left ? (int32_t)s_list[h + k] : -1; });
      for (uint32_t i = threadIdx.x; i < T::B::kBytes / 16; i += T::kThreads)
        *(uint4*)(tile_b + i * 16) = make_uint4(0, 0, 0, 0);
      __syncthreads();
      if (threadIdx.x < kGemmK && threadIdx.x < left) {
        const uint32_t t = s_list[h + threadIdx.x];
        *(uint16_t*)(tile_b + T::B::place(threadIdx.x, (uint32_t)p.y[t] - p.v_begin - n0)) =
            (uint16_t)bf16x2_rne(__float_as_uint(p.rest[t]), 0u);
      }
      wait_and_meet<0>();
      T::add_step(lds, acc);
      __syncthreads();  // the tiles are free again
    }
  }
  __syncthreads();
}

// (The 256 by 256 tile's rests and way out keep 60 registers in scratch memory; the
// product's loop does not.)
template <typename T, bool RESTS>
__device__ void dw_block(const GradParams& p, char* lds, uint32_t id) {
  uint32_t m0, n0;
  typename T::Acc acc;
  grad_tile<T, true, true>(p, lds, id, 0, m0, n0, acc);
  if constexpr (RESTS) add_rests<T>(p, lds, m0, n0, acc);
  auto value = [&](int i, int j) {
    uint2 o;
    o.x = bf16x2_rne(__float_as_uint(acc[i][j][0]), __float_as_uint(acc[i][j][1]));
    o.y = bf16x2_rne(__float_as_uint(acc[i][j][2]), __float_as_uint(acc[i][j][3]));
    return o;
  };
  uint16_t* const out = p.out + n0 * p.out_ld + m0;
  if (p.out_ld % 8 == 0) T::template store_rows<true, true>(lds, out, p.out_ld, p.m - m0, p.n - n0, value);
  else T::template store_rows<false, false>(lds, out, p.out_ld, p.m - m0, p.n - n0, value);
}

template <typename T>
__global__ __launch_bounds__(T::kThreads) void ce_dx_kernel(GradParams p) {
  __shared__ alignas(1024) char lds[T::kLds];
  dx_block<T>(p, lds, blockIdx.x);
}

template <typename T, bool RESTS>
__global__ __launch_bounds__(T::kThreads) void ce_dw_kernel(GradParams p) {
  __shared__ alignas(1024) char lds[T::kLds];
  dw_block<T, RESTS>(p, lds, blockIdx.x);
}

// Both products in one launch: dx's blocks first, whose sums are the longer ones.
template <typename TX, typename TW, bool RESTS>
__global__ __launch_bounds__(TX::kThreads) void ce_both_kernel(GradParams x, GradParams w, uint32_t dx_blocks) {
  static_assert(TX::kThreads == TW::kThreads, "blocks of one size");
  __shared__ alignas(1024) char lds[TX::kLds > TW::kLds ? TX::kLds : TW::kLds];
  if (blockIdx.x < dx_blocks) dx_block<TX>(x, lds, blockIdx.x);
  else dw_block<TW, RESTS>(w, lds, blockIdx.x - dx_blocks);
}

// dw for up to 64 tokens, where writing it bounds the time: a block keeps its 256
// hidden columns of x in registers, for all k (the tokens twice, for G and its rests),
// and runs on over the vocabulary, 64 entries at a time: the next tiles of G are on
// their way while one is multiplied, turned into rows in LDS and stored.
// 61 tokens, 152,064 x 5,120: 303 us (5.1 TB/s of writes); 406 with a block a tile.
// With a ring of 3 and two blocks a CU, forward and backward together took 1,181 us
// to 1,154.
constexpr int kRunN = 64, kRunRing = 4;

__global__ __launch_bounds__(512) void ce_dw_run_kernel(GradParams p, uint32_t runs) {
  typedef GemmTile<256, 8, true> A;  // of 64 k each
  typedef GemmTile<kRunN, 8, true> B;
  constexpr int kSlot = 2 * B::kBytes, kRowBytes = 256 * 2;
  constexpr int kLoads = 2, kStores = kRunN * kRowBytes / 16 / 512;  // of a thread and tile
  static_assert(B::kLoads == 1 && 2 * A::kBytes <= kRunRing * kSlot, "x passes through the ring");
  __shared__ alignas(1024) char ring[kRunRing * kSlot];
  __shared__ alignas(1024) char rows[kRunN * kRowBytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t tm, run;  // every column tile of a run side by side: whole rows of dw at a time
  gemm_tile_of(blockIdx.x, p.tiles_m, runs, p.tiles_m, tm, run);
  const uint32_t m0 = tm * 256, m_left = p.m - m0;
  const uint32_t tiles = (p.n + kRunN - 1) / kRunN, each = (tiles + runs - 1) / runs;
  const uint32_t first = run * each, count = first >= tiles ? 0 : tiles - first < each ? tiles - first : each;
  if (count == 0) return;

  // the wave's 32 columns of x: fragments of all four halves of k
  bf16x8_t fa[4][2];
  {
    const GemmOperand x = {p.a.p + m0, p.a.ld, p.a.limit - m0};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int32_t left = (int32_t)p.k - 64 * h;
      A::gather(x, ring + h * A::kBytes, wave, lane, [&](uint32_t k) { return (int32_t)k < left ? (int32_t)(64 * h + k) : -1; });
    }
    wait_and_meet<0>();
    const uint32_t at = lds_address(ring) + A::lane_place(wave * 32, lane);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int i = 0; i < 2; ++i) fa[2 * h + ks][i] = A::fragment(at + h * A::kBytes, i, ks);
    __syncthreads();
  }

  // rows of G past the last token meet zeros of x: any row will do
  uint32_t off[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t k = B::k_of(0, wave, lane), g = lane % (kRunN / 8);
    const uint32_t row = 64 * h + k < p.k ? 64 * h + k : p.k - 1;
    off[h] = (uint32_t)(row * p.b.ld * 2 + ((((g >> 1) ^ B::mix(k)) << 1 | (g & 1)) * 16));
  }
  auto load = [&](uint32_t tile) {  // the run's tile
    char* const to = ring + tile % kRunRing * kSlot + wave * 1024;
    const u32x4_t from = buffer_at(p.b.p + (uint64_t)(first + tile) * kRunN);
#pragma unroll
    for (int h = 0; h < 2; ++h) load_to_lds<false>(to + h * B::kBytes, off[h], from);
  };
  for (uint32_t i = 0; i < kRunRing - 1 && i < count; ++i) load(i);
  const uint32_t at_b = lds_address(ring) + B::lane_place(0, lane);
  for (uint32_t i = 0; i < count; ++i) {
    // tile i has landed.  After its loads came the stores of three tiles and the loads
    // of two; near the ends there were fewer, so everything is waited for
    if (i >= kRunRing - 1 && i + kRunRing - 1 < count) wait_and_meet<(kRunRing - 1) * kStores + (kRunRing - 2) * kLoads>();
    else wait_and_meet<0>();
    if (i + kRunRing - 1 < count) load(i + kRunRing - 1);  // where tile i - 1 was
    f32x4_t acc[2][4];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[m][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t at = at_b + i % kRunRing * kSlot;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (q * 32 >= (int)p.k) break;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bf16x8_t b = B::fragment(at + q / 2 * B::kBytes, j, q % 2);
#pragma unroll
        for (int m = 0; m < 2; ++m)
          acc[m][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[q][m], b, acc[m][j], 0, 0, 0);
      }
    }
    // group c of row n lies at place c ^ (n & 15)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t n = j * 16 + (lane & 15);
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const uint32_t c = wave * 32 + m * 16 + (lane >> 4) * 4;
        uint2 o;
        o.x = bf16x2_rne(__float_as_uint(acc[m][j][0]), __float_as_uint(acc[m][j][1]));
        o.y = bf16x2_rne(__float_as_uint(acc[m][j][2]), __float_as_uint(acc[m][j][3]));
        *(uint2*)(rows + n * kRowBytes + (((c >> 3) ^ (n & 15)) << 4) + (c & 4) * 2) = o;
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const uint32_t n0 = (first + i) * kRunN;
    uint16_t* const out = p.out + (uint64_t)n0 * p.out_ld + m0;
#pragma unroll
    for (int r = 0; r < kStores; ++r) {
      const uint32_t q = threadIdx.x + r * 512, n = q / 32, c = q % 32;
      const uint4 v = *(const uint4*)(rows + n * kRowBytes + ((c ^ (n & 15)) << 4));
      // a wave always has a lane that stores, but for the vocabulary's last tile, after
      // which nothing is counted
      if (n0 + n < p.n && c * 8 < m_left) store16_stream(out + n * p.out_ld + c * 8, v);
    }
  }
}

struct DxJoinParams {
  uint32_t first;     // token of this launch
  const float* sums;  // [splits][tokens][ld]
  uint32_t splits, tokens, ld, hidden;
  const int64_t* targets;
  uint32_t vocab;
  const uint16_t* w;
  uint64_t w_ld;
  const float* rest;
  const float* lost;
  uint32_t lost_ld;
  const uint32_t* large_count;
  const LargeLoss* large;
  const float* mean;  // [ld]: W's mean row
  uint16_t* dx;
  uint64_t dx_ld;
};

// dx from the splits' sums and what G's rounding took; a token without a target gets zeros.
__global__ __launch_bounds__(256) void ce_dx_join_kernel(DxJoinParams p) {
  __shared__ float s_lost[4];
  __shared__ LargeLoss s_large[kLargeLosses];
  const uint32_t t = p.first + blockIdx.x;
  const uint32_t c = (blockIdx.y * 256 + threadIdx.x) * 4;
  const int64_t y = p.targets[t];
  f32x4_t a = {0.0f, 0.0f, 0.0f, 0.0f};
  if (y >= 0 && y < (int64_t)p.vocab) {  // the whole block
    float lost = 0.0f;
    for (uint32_t i = threadIdx.x; i < p.lost_ld; i += 256) lost += p.lost[(uint64_t)t * p.lost_ld + i];
    lost = wave_sum(lost);
    if ((threadIdx.x & 63) == 0) s_lost[threadIdx.x >> 6] = lost;
    const uint32_t listed = p.large_count[t], count = listed > kLargeLosses ? 0 : listed;
    if (threadIdx.x < 64) {  // in the order of the vocabulary, whatever order they were written in
      const LargeLoss mine = threadIdx.x < count ? p.large[(uint64_t)t * kLargeLosses + threadIdx.x]
                                                 : LargeLoss{0x7FFFFFFF, 0.0f};
      uint32_t place = 0;
#pragma unroll
      for (uint32_t i = 0; i < kLargeLosses; ++i) place += __builtin_amdgcn_readlane(mine.v, i) < mine.v;
      if (threadIdx.x < count) s_large[place] = mine;
    }
    __syncthreads();
    lost = (s_lost[0] + s_lost[1]) + (s_lost[2] + s_lost[3]);
    if (c >= p.ld) return;
    auto add = [&](float by, const uint16_t* row) {
      const uint2 v = *(const uint2*)(row + c);
      a[0] = __builtin_fmaf(by, __uint_as_float(v.x << 16), a[0]);
      a[1] = __builtin_fmaf(by, __uint_as_float(v.x & 0xFFFF0000u), a[1]);
      a[2] = __builtin_fmaf(by, __uint_as_float(v.y << 16), a[2]);
      a[3] = __builtin_fmaf(by, __uint_as_float(v.y & 0xFFFF0000u), a[3]);
    };
#pragma unroll 8
    for (uint32_t s = 0; s < p.splits; ++s)
      a += *(const f32x4_t*)(p.sums + ((uint64_t)s * p.tokens + t) * p.ld + c);
    add(p.rest[t], p.w + y * p.w_ld);
#pragma unroll 4
    for (uint32_t k = 0; k < count; ++k) {
      lost -= s_large[k].lost;
      add(s_large[k].lost, p.w + (uint64_t)s_large[k].v * p.w_ld);
    }
    const f32x4_t mean = *(const f32x4_t*)(p.mean + c);
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] = __builtin_fmaf(lost, mean[e], a[e]);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (c + e < p.hidden) p.dx[t * p.dx_ld + c + e] = (uint16_t)bf16x2_rne(__float_as_uint(a[e]), 0u);
}

// ---------------------------------------------------------------- copies

// Rows to be padded with zeros to `ld`, `times` over.
struct CopyJob {
  const uint16_t* from;  // null: no such job
  uint64_t from_ld;
  uint16_t* to;
  uint64_t rows;
  uint32_t times;
};

struct PrepareParams {
  CopyJob w, x;
  uint32_t cols, ld;
  const int64_t* targets;  // null, or: rows of x without a target become zeros, as
  uint32_t vocab;          // what is in them must not reach the other rows' sums;
  int32_t* y;              // and the targets as 32 bits, -1 for none
  uint32_t* zero;          // with targets: [rows of x], set to zero
  float* mean;             // null, or: [ld] to take the mean row of `mean_of`
  const uint16_t* mean_of;  // [vocab] rows, mean_ld apart
  uint64_t mean_ld;
  uint32_t mean_blocks;  // the first ones: 64 columns each
};

// 8 elements of a row from its column c on, zeros past its end.
__device__ __forceinline__ uint4 load_group(const uint16_t* row, uint32_t c, uint32_t cols) {
  if (c + 8 <= cols) return load16_any(row + c);
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (c + e < cols) w[e >> 1] |= (uint32_t)row[c + e] << (16 * (e & 1));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// The mean of kMeanRows rows (all, if there are fewer), 64 columns a block; zero in a
// column where it is not finite.
__device__ __forceinline__ void mean_row(const PrepareParams& p) {
  __shared__ float s[32][64];
  const uint32_t group = threadIdx.x & 7, first = threadIdx.x >> 3, c = blockIdx.x * 64 + group * 8;
  const uint32_t rows = p.vocab < kMeanRows ? p.vocab : kMeanRows;
  float sum[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (uint32_t i = 0; i < kMeanRows / 32; ++i) {
    const uint32_t r = first + i * 32;
    const uint64_t row = rows < kMeanRows ? r : (uint64_t)r * p.vocab / kMeanRows;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (r < rows) v = load_group(p.mean_of + row * p.mean_ld, c, p.cols);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sum[2 * e] += __uint_as_float(get_u32(v, e) << 16);
      sum[2 * e + 1] += __uint_as_float(get_u32(v, e) & 0xFFFF0000u);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) s[first][group * 8 + e] = sum[e];
  __syncthreads();
  const uint32_t at = blockIdx.x * 64 + threadIdx.x;
  if (threadIdx.x >= 64 || at >= p.ld) return;
  float mean = 0.0f;
#pragma unroll
  for (int i = 0; i < 32; ++i) mean += s[i][threadIdx.x];
  mean /= (float)rows;
  p.mean[at] = mean - mean == 0.0f ? mean : 0.0f;
}

__device__ __forceinline__ void copy_group(const CopyJob& j, uint32_t cols, uint32_t ld, uint64_t r, uint32_t c,
                                           bool kept) {
  uint4 v = make_uint4(0, 0, 0, 0);
  if (kept) v = load_group(j.from + r * j.from_ld, c, cols);
  for (uint32_t k = 0; k < j.times; ++k) store16(j.to + (k * j.rows + r) * ld + c, v);
}

__global__ __launch_bounds__(256) void ce_prepare_kernel(PrepareParams p) {
  if (blockIdx.x < p.mean_blocks) return mean_row(p);
  const uint32_t block = blockIdx.x - p.mean_blocks, blocks = gridDim.x - p.mean_blocks;
  const uint64_t groups = p.ld / 8;  // of 8 elements, in a row
  const uint64_t nx = p.x.from ? p.x.rows * groups : 0, all = nx + (p.w.from ? p.w.rows * groups : 0);
  for (uint64_t i = (uint64_t)block * 256 + threadIdx.x; i < all; i += (uint64_t)blocks * 256) {
    if (i >= nx) {
      copy_group(p.w, p.cols, p.ld, (i - nx) / groups, (uint32_t)((i - nx) % groups) * 8, true);
      continue;
    }
    const uint64_t r = i / groups;
    const uint32_t c = (uint32_t)(i % groups) * 8;
    bool kept = true;
    if (p.targets) {
      const int64_t y = p.targets[r];
      kept = y >= 0 && y < (int64_t)p.vocab;
      if (c == 0) {
        p.y[r] = kept ? (int32_t)y : -1;
        p.zero[r] = 0;
      }
    }
    copy_group(p.x, p.cols, p.ld, r, c, kept);
  }
}

void prepare(PrepareParams p, hipStream_t stream) {
  const uint64_t rows = (p.x.from ? p.x.rows : 0) + (p.w.from ? p.w.rows : 0);
  if (rows == 0) return;
  uint64_t blocks = (rows * (p.ld / 8) + 255) / 256;
  if (blocks > 8192) blocks = 8192;
  p.mean_blocks = p.mean ? (p.ld + 63) / 64 : 0;
  hipLaunchKernelGGL(ce_prepare_kernel, dim3((uint32_t)blocks + p.mean_blocks), dim3(256), 0, stream, p);
}

// ---------------------------------------------------------------- shapes

uint32_t up(uint32_t v, uint32_t to) { return (v + to - 1) / to * to; }
uint32_t parts(uint64_t v, uint32_t of) { return (uint32_t)((v + of - 1) / of); }

constexpr uint32_t kVocabTile = 256;
constexpr uint32_t kBothBlocks = 512;
// A launch has fewer than 2^32 threads: more tiles or tokens than these take several.
constexpr uint32_t kTilesAtOnce = 1u << 22;  // of up to 512 threads; a multiple of 8, the XCDs
constexpr uint32_t kTokensAtOnce = 1u << 22;  // of up to 256 threads in x
constexpr uint64_t kRunElements = 1ull << 26;  // of dw: 16 tiles of 64 entries for every CU
constexpr uint32_t kSmallTokens = 512;  // up to here the gradient's products take the smaller tiles
constexpr uint32_t kWantedTiles = 192;
constexpr uint32_t kFewTokens = 128;  // up to here G's rests are kept for all entries

// Tiles: vocabulary (or hidden) by tokens (or vocabulary).  The large ones reach the
// matrix cores' rate where there are tiles enough for all CUs; the smaller ones fill
// the chip with fewer and overlap one block's epilogue with another's loads.
typedef Gemm<256, 256, 2, 4, 2, false, false> LogitsL;
typedef Gemm<256, 128, 4, 2, 3, false, false> LogitsM;
typedef Gemm<256, 64, 4, 1, 4, false, false> LogitsS;
typedef Gemm<256, 64, 4, 1, 4, false, false, true> LogitsW;  // past the caches, for a weight larger than they are
typedef Gemm<128, 64, 4, 1, 4, false, false> LogitsT;
typedef Gemm<256, 256, 2, 4, 2, true, false> DxL;
typedef Gemm<256, 128, 4, 2, 3, true, false> DxM;
typedef Gemm<128, 64, 4, 1, 2, true, false, true> DxS;
typedef Gemm<256, 256, 2, 4, 2, true, true> DwL;
typedef Gemm<128, 128, 4, 2, 2, true, true> DwM;
typedef Gemm<128, 128, 2, 2, 2, true, true> DwS;

constexpr uint64_t kCacheBytes = 256ull << 20;  // of the last level
constexpr uint64_t kMaxStride = 1u << 20;  // a tile's byte offsets stay in 32 bits
constexpr uint64_t kPieceBytes = 256ull << 20;  // of G

struct Plan {
  uint32_t ld;      // of the padded copies and of dx's sums: hidden to a multiple of 8
  bool copy_w;
  uint32_t piece;   // vocabulary entries a piece, a multiple of the tile
  uint32_t splits;  // of dx's k
  bool small;       // the products in the smaller tiles
  // byte offsets in the workspace
  uint64_t w, x, part, hit, g, y, rest, sums, lost, large_count, large, mean, forward, total;
};

Plan plan_of(uint32_t tokens, uint32_t vocab, uint32_t hidden) {
  Plan q;
  q.ld = up(hidden, 8);
  q.copy_w = hidden % 8 != 0;
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) {
    const uint64_t here = at;
    at += (bytes + 255) & ~255ull;
    return here;
  };
  q.w = take(q.copy_w ? (uint64_t)vocab * q.ld * 2 : 0);
  const uint32_t times = tokens <= kFewTokens ? 2 : 1;
  q.x = take((uint64_t)times * tokens * q.ld * 2);
  const uint64_t both = at;
  q.part = take((uint64_t)tokens * parts(vocab, LogitsT::BM) * sizeof(float2));
  q.hit = take((uint64_t)tokens * sizeof(float));
  q.forward = at;
  at = both;
  uint64_t piece = kPieceBytes / 2 / tokens;
  piece = piece / kVocabTile * kVocabTile;
  if (piece < kVocabTile) piece = kVocabTile;
  const uint32_t pieces = parts(vocab, (uint32_t)(piece > vocab ? up(vocab, kVocabTile) : piece));
  q.piece = up(parts(vocab, pieces), kVocabTile);
  // few tokens: split dx's k until the blocks fill the chip
  q.small = tokens <= kSmallTokens || parts(q.ld, 256) * parts(q.piece, 256) < 256;
  const uint32_t bm = tokens <= 64 ? DxS::BM : 256, bn = tokens <= 64 ? 64 : q.small ? 128 : 256;
  const uint32_t tiles = parts(q.ld, bm) * parts(tokens, bn);
  // (three of the small tiles fit a CU, one of the others)
  const uint32_t wanted = tokens <= 64 ? 768 : kWantedTiles;
  q.splits = tiles < wanted ? wanted / tiles : 1;
  if (q.splits > q.piece / 256) q.splits = q.piece / 256;
  q.g = take((uint64_t)times * tokens * q.piece * 2);
  q.y = take((uint64_t)tokens * sizeof(int32_t));
  q.rest = take((uint64_t)tokens * sizeof(float));
  q.sums = take((uint64_t)q.splits * tokens * q.ld * 4);
  q.lost = take((uint64_t)tokens * parts(vocab, kLostTile) * sizeof(float));
  q.large_count = take((uint64_t)tokens * sizeof(uint32_t));
  q.large = take((uint64_t)tokens * kLargeLosses * sizeof(LargeLoss));
  q.mean = take((uint64_t)q.ld * sizeof(float));
  q.total = at > q.forward ? at : q.forward;
  return q;
}

template <typename T>
uint32_t run_logits(LogitParams p, bool forward, hipStream_t stream) {
  p.tiles_m = parts(p.v_end - p.v_begin, T::BM);
  p.tiles_n = parts(p.tokens, T::BN);
  const uint32_t tiles = p.tiles_m * p.tiles_n;
  for (p.first_tile = 0; p.first_tile < tiles; p.first_tile += kTilesAtOnce) {
    const uint32_t left = tiles - p.first_tile;
    const dim3 grid(left < kTilesAtOnce ? left : kTilesAtOnce), block(T::kThreads);
    if (forward) hipLaunchKernelGGL(ce_forward_kernel<T>, grid, block, 0, stream, p);
    else hipLaunchKernelGGL(ce_grad_kernel<T>, grid, block, 0, stream, p);
    if (left <= kTilesAtOnce) break;
  }
  return T::BM;
}

// A block's time in thousands of cycles, for the choice of a tile: a fixed part (the first
// loads and the epilogue) and one per step of 64 k, which grows as more CUs share
// the L2s (the smaller a tile, the more it loads for its products).  Measured, one
// launch of forward, us, L / M / S (T for the last):
//   tokens 2048, 151936 x 896:  498 / 628 / 657     752, 3060 x 3008:  60 / 38 / 41
//   589, 54805 x 5069 (padded): 250 / 568 / -       160, 310 x 1728:   40 / 28 / 23
//   1024, 8192 x 4096:           86 /  60 / 67      926, 120888 x 64:  65 / 80 / 78
struct TileCost {
  uint32_t bm, bn;
  float fixed, step, shared;
};

float cost_of(const TileCost& c, uint32_t entries, uint32_t tokens, uint32_t k) {
  constexpr float kCus = 256.0f;
  const float blocks = (float)parts(entries, c.bm) * (float)parts(tokens, c.bn);
  const float rounds = (float)(uint32_t)((blocks + kCus - 1) / kCus);
  const float busy = blocks < kCus ? blocks / kCus : 1.0f;
  return rounds * (c.fixed + (c.step + c.shared * busy) * (float)parts(k, kGemmK));
}

constexpr TileCost kCostL = {256, 256, 18.0f, 2.2f, 0.0f}, kCostM = {256, 128, 11.0f, 1.2f, 1.1f},
                   kCostS = {256, 64, 8.0f, 1.5f, 0.7f}, kCostT = {128, 64, 6.0f, 0.9f, 0.6f};

// Returns the tile's entries.
uint32_t run_logits(const LogitParams& p, bool forward, hipStream_t stream) {
  const uint32_t entries = p.v_end - p.v_begin;
  const float s = cost_of(kCostS, entries, p.tokens, p.hidden), t = cost_of(kCostT, entries, p.tokens, p.hidden);
  if (p.tokens > 64) {
    const float l = cost_of(kCostL, entries, p.tokens, p.hidden), m = cost_of(kCostM, entries, p.tokens, p.hidden);
    if (l <= m && l <= s && l <= t) return run_logits<LogitsL>(p, forward, stream);
    if (m <= s && m <= t) return run_logits<LogitsM>(p, forward, stream);
  }
  if (t < s) return run_logits<LogitsT>(p, forward, stream);
  // a weight larger than the caches streams past them, if it is read once
  if (p.tokens <= 64 && (uint64_t)p.vocab * p.w_ld * 2 > kCacheBytes) return run_logits<LogitsW>(p, forward, stream);
  return run_logits<LogitsS>(p, forward, stream);
}

// dx's and dw's products of a piece.  One launch where both fit the chip at once
// (each launch costs 3 us on the host and 2 to 4 of latency on the GPU); for more blocks
// each product keeps the registers and LDS, hence the occupancy, of its own kernel.
template <typename TX, typename TW, bool RESTS>
void run_products(GradParams x, uint32_t splits, GradParams w, hipStream_t stream) {
  x.tiles_m = parts(x.m, TX::BM);
  x.tiles_n = parts(x.n, TX::BN);
  x.band = kBand;
  w.tiles_m = parts(w.m, TW::BM);
  w.tiles_n = parts(w.n, TW::BN);
  // few tokens: bound by writing dw, so whole rows of it at a time
  w.band = RESTS ? kBand : w.tiles_m;
  const uint32_t nx = x.tiles_m * x.tiles_n * splits, nw = w.tiles_m * w.tiles_n;
  if (w.k <= 128 && w.out_ld % 8 == 0 && (uint64_t)w.m * w.n >= kRunElements) {
    w.tiles_m = parts(w.m, 256);
    const uint32_t runs = w.tiles_m < 256 ? 256 / w.tiles_m : 1;
    hipLaunchKernelGGL(ce_dx_kernel<TX>, dim3(nx), dim3(TX::kThreads), 0, stream, x);
    hipLaunchKernelGGL(ce_dw_run_kernel, dim3(w.tiles_m * runs), dim3(512), 0, stream, w, runs);
    return;
  }
  if (nx + nw <= kBothBlocks) {
    hipLaunchKernelGGL((ce_both_kernel<TX, TW, RESTS>), dim3(nx + nw), dim3(TX::kThreads), 0, stream, x, w, nx);
    return;
  }
  hipLaunchKernelGGL(ce_dx_kernel<TX>, dim3(nx), dim3(TX::kThreads), 0, stream, x);
  hipLaunchKernelGGL((ce_dw_kernel<TW, RESTS>), dim3(nw), dim3(TW::kThreads), 0, stream, w);
}

}  // namespace

__global__ __launch_bounds__(256) void zero_bytes_kernel(uint16_t* p, uint64_t n) {
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) p[i] = 0;
}

hipError_t launch_zero_bytes(void* p, uint64_t bytes, hipStream_t stream) {
  hipLaunchKernelGGL(zero_bytes_kernel, dim3(4096), dim3(256), 0, stream, (uint16_t*)p, bytes / 2);
  return hipGetLastError();
}

uint64_t linear_ce_needs(uint32_t tokens, uint32_t vocab, uint32_t hidden) {
  return plan_of(tokens, vocab, hidden).total;
}

// What a plan needs does not grow with the tokens alone (its tiles, splits and
// pieces change with them), so: the largest of every plan up to 512 tokens, and past
// those a bound on each part.
uint64_t linear_ce_bytes(uint32_t tokens, uint32_t vocab, uint32_t hidden) {
  uint64_t most = 0;
  for (uint32_t t = 1; t <= tokens && t <= kSmallTokens; ++t) {
    const uint64_t total = plan_of(t, vocab, hidden).total;
    if (total > most) most = total;
  }
  if (tokens <= kSmallTokens) return most;
  const uint64_t t = tokens, ld = up(hidden, 8), entries = up(vocab, kVocabTile);
  const uint64_t g = t * entries * 2 < kPieceBytes ? t * entries * 2 : kPieceBytes + t * kVocabTile * 2;
  // splits * tokens is at most the tokens, or the tiles wanted times a tile's tokens
  const uint64_t sums = (t + (uint64_t)kWantedTiles * 256 / parts(ld, 256)) * ld * 4;
  const uint64_t both = (hidden % 8 ? (uint64_t)vocab * ld * 2 : 0) + t * ld * 2;
  const uint64_t forward = t * parts(vocab, LogitsT::BM) * sizeof(float2) + t * sizeof(float);
  const uint64_t lost = t * (parts(vocab, kLostTile) * sizeof(float) + 4 + kLargeLosses * sizeof(LargeLoss)) + ld * 4;
  const uint64_t backward = g + t * 8 + sums + lost;
  const uint64_t bound = both + (backward > forward ? backward : forward) + 16 * 256;
  return bound > most ? bound : most;
}

hipError_t launch_linear_ce(const LinearCeParams& c, char* ws, hipStream_t stream) {
  const Plan q = plan_of(c.tokens, c.vocab, c.hidden);
  LogitParams p = {};
  PrepareParams r = {};
  r.cols = c.hidden;
  r.ld = q.ld;
  p.w = c.weight;
  p.w_ld = c.hidden;
  if (q.copy_w) {
    r.w = {c.weight, c.hidden, (uint16_t*)(ws + q.w), c.vocab, 1};
    p.w = r.w.to;
    p.w_ld = q.ld;
  }
  p.x = c.x;
  p.x_ld = c.x_stride;
  if (c.hidden % 8 || c.x_stride % 8 || c.x_stride > kMaxStride) {
    r.x = {c.x, c.x_stride, (uint16_t*)(ws + q.x), c.tokens, 1};
    p.x = r.x.to;
    p.x_ld = q.ld;
  }
  prepare(r, stream);
  p.targets = c.targets;
  p.tokens = c.tokens;
  p.hidden = q.ld;
  p.v_begin = 0;
  p.v_end = p.vocab = c.vocab;
  p.scale = c.logit_scale;
  p.part = (float2*)(ws + q.part);
  p.hit = (float*)(ws + q.hit);
  const uint32_t tile = run_logits(p, true, stream);
  for (uint32_t first = 0; first < c.tokens; first += kTokensAtOnce) {
    const uint32_t left = c.tokens - first, now = left < kTokensAtOnce ? left : kTokensAtOnce;
    hipLaunchKernelGGL(ce_join_kernel, dim3(parts(now, 4)), dim3(256), 0, stream, p.part, p.hit, c.targets, first,
                       c.tokens, c.vocab, parts(c.vocab, tile), c.loss, c.lse);
  }
  return hipGetLastError();
}

hipError_t launch_linear_ce_grad(const LinearCeGradParams& c, char* ws, hipStream_t stream) {
  const Plan q = plan_of(c.tokens, c.vocab, c.hidden);
  LogitParams p = {};
  PrepareParams r = {};
  r.cols = c.hidden;
  r.ld = q.ld;
  p.w = c.weight;
  p.w_ld = c.hidden;
  if (q.copy_w) {
    r.w = {c.weight, c.hidden, (uint16_t*)(ws + q.w), c.vocab, 1};
    p.w = r.w.to;
    p.w_ld = q.ld;
  }
  // few tokens: G's rests are 128 more rows at most of k for dw, which then meet x
  // again; more tokens add the targets' rests alone
  const bool few = c.tokens <= kFewTokens;
  int32_t* y = (int32_t*)(ws + q.y);
  r.x = {c.x, c.x_stride, (uint16_t*)(ws + q.x), c.tokens, few ? 2u : 1u};
  r.targets = c.targets;
  r.vocab = c.vocab;
  r.y = y;
  r.zero = (uint32_t*)(ws + q.large_count);
  r.mean = (float*)(ws + q.mean);
  r.mean_of = c.weight;
  r.mean_ld = c.hidden;
  prepare(r, stream);
  p.x = r.x.to;
  p.x_ld = q.ld;
  p.targets = c.targets;
  p.tokens = c.tokens;
  p.hidden = q.ld;
  p.vocab = c.vocab;
  p.scale = c.logit_scale;
  p.lse = c.lse;
  p.dloss = c.dloss;
  p.g = (uint16_t*)(ws + q.g);
  p.g_ld = q.piece;
  p.rest = (float*)(ws + q.rest);
  p.lost = (float*)(ws + q.lost);
  p.lost_ld = parts(c.vocab, kLostTile);
  p.large_count = r.zero;
  p.large = (LargeLoss*)(ws + q.large);
  p.rest_rows = few;
  float* sums = (float*)(ws + q.sums);
  for (uint32_t v = 0; v < c.vocab; v += q.piece) {
    const uint32_t n = c.vocab - v < q.piece ? c.vocab - v : q.piece;
    p.v_begin = v;
    p.v_end = v + n;
    run_logits(p, false, stream);
    GradParams d = {};
    d.a = {p.w + (uint64_t)v * p.w_ld, p.w_ld, q.ld};
    d.b = {p.g, q.piece, c.tokens};
    d.m = q.ld;
    d.n = c.tokens;
    d.k = n;
    d.k_split = up(parts(q.piece, q.splits), kGemmK);
    d.sums = sums;
    d.add = v > 0;
    // a short last piece leaves the last splits without k: their sums stay
    const uint32_t splits = v > 0 ? parts(n, d.k_split) : q.splits;
    GradParams e = {};
    e.a = {p.x, q.ld, q.ld};
    e.b = {p.g, q.piece, q.piece};
    e.m = c.hidden;
    e.n = n;
    e.k = e.k_split = few ? 2 * c.tokens : c.tokens;
    e.y = y;
    e.rest = p.rest;
    e.v_begin = v;
    e.out = c.dweight + (uint64_t)v * c.hidden;
    e.out_ld = c.hidden;
    if (c.tokens <= 64) run_products<DxS, DwS, false>(d, splits, e, stream);
    else if (few) run_products<DxM, DwM, false>(d, splits, e, stream);
    else if (q.small) run_products<DxM, DwM, true>(d, splits, e, stream);
    else run_products<DxL, DwL, true>(d, splits, e, stream);
  }
  DxJoinParams j = {0, sums, q.splits, c.tokens, q.ld, c.hidden, c.targets, c.vocab, p.w, p.w_ld, p.rest, p.lost,
                          p.lost_ld, p.large_count, p.large, r.mean, c.dx, c.dx_stride};
  for (; j.first < c.tokens; j.first += kTokensAtOnce) {
    const uint32_t left = c.tokens - j.first;
    hipLaunchKernelGGL(ce_dx_join_kernel, dim3(left < kTokensAtOnce ? left : kTokensAtOnce, parts(q.ld, 1024)), dim3(256), 0,
                       stream, j);
  }
  return hipGetLastError();
}

}  // namespace pulse
