// verify_drafts.hip -- drafted tokens held against the target's probabilities.
//
//   p = softmax(scale z), q = softmax(draft_scale zd) (or 1 at the draft)
//   drafts are taken while u_k q(x_k) < p(x_k); then one token is drawn, from
//   max(p - q, 0) at the first draft that is not taken, else from p.
//
// Every logit is read once, which bounds the first kernel (HBM; its second cost is
// an exponential a logit); of each sequence one row, or a target's and a draft's,
// is read a second time, mostly from a cache.
//
// Probabilities are FP64.  The draw is the first entry whose cumulated probability
// exceeds u times the total: in FP32 each of some 150,000 borders would be off by 1e-7
// of the total, so that one draw in 30 gave another token than the definition's.  With
// borders off by 1e-12 it is one in a million.  An exponential is 9 FMAs and a handful
// of other FP64 instructions, which issue as fast as FP32's here.
//
// Three kernels: per row and tile of the vocabulary the largest logit and the sum of
// exponentials below it; per sequence and tile the decisions (each block joins its
// sequence's sums again: some KB from the L2) and a refused row's sum of max(p - q, 0);
// per sequence the tile that holds the draw, then the entry in it.
#include "device_common.hpp"
#include "head.hpp"

namespace pulse {

namespace {

constexpr double kNoEntry = -1100.0;  // 2^x is 0

// 2^x for x <= 0, or a little above, off by 1.1e-12: x to the nearest integer and a
// polynomial for the rest, interpolated at the 9 Chebyshev nodes of [-1/2, 1/2].
__device__ __forceinline__ double exp2_64(double x) {
  x = __builtin_fmax(x, kNoEntry);
  const double k = __builtin_rint(x), f = x - k;
  double v = 1.3255224878668817e-06;
  v = __builtin_fma(v, f, 1.5310079402249296e-05);
  v = __builtin_fma(v, f, 0.00015403455852453838);
  v = __builtin_fma(v, f, 0.0013333450568000645);
  v = __builtin_fma(v, f, 0.009618129159402558);
  v = __builtin_fma(v, f, 0.05550410941205933);
  v = __builtin_fma(v, f, 0.2402265069581299);
  v = __builtin_fma(v, f, 0.6931471805459335);
  v = __builtin_fma(v, f, 1.0);
  return __builtin_ldexp(v, (int)k);
}

__device__ __forceinline__ float logit_of(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float logit_of(float v) { return v; }

// Entries c to c + 7 of a row, -inf past its end.
__device__ __forceinline__ void load_logits(const uint16_t* row, uint32_t c, uint32_t vocab, float (&z)[8]) {
  if (c + 8 <= vocab) {
    const uint4 v = load16_any(row + c);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      z[e] = __uint_as_float(e & 1 ? get_u32(v, e >> 1) & 0xFFFF0000u : get_u32(v, e >> 1) << 16);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = c < vocab && e < vocab - c ? logit_of(row[c + e]) : -INFINITY;
  }
}
__device__ __forceinline__ void load_logits(const float* row, uint32_t c, uint32_t vocab, float (&z)[8]) {
  if (c + 8 <= vocab) {
    const uint4 a = load16_any(row + c), b = load16_any(row + c + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      z[e] = __uint_as_float(get_u32(a, e));
      z[4 + e] = __uint_as_float(get_u32(b, e));
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = c < vocab && e < vocab - c ? row[c + e] : -INFINITY;
  }
}

__device__ __forceinline__ double shuffle_xor(double v, int mask) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __shfl_xor((uint32_t)b, mask), hi = __shfl_xor((uint32_t)(b >> 32), mask);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int x = 1; x < 64; x *= 2) v += shuffle_xor(v, x);
  return v;
}

// The sum over lanes 0 to this one.
__device__ __forceinline__ double wave_scan64(double v) {
  const int lane = lane_id();
#pragma unroll
  for (int x = 1; x < 64; x *= 2) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __shfl_up((uint32_t)b, x), hi = __shfl_up((uint32_t)(b >> 32), x);
    if (lane >= x) v += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  }
  return v;
}

__device__ __forceinline__ uint32_t length_of(const VerifyParams& p, uint32_t b) {
  if (!p.lengths) return p.drafts;
  const int32_t n = p.lengths[b];
  return n < 0 ? 0 : (uint32_t)n < p.drafts ? (uint32_t)n : p.drafts;
}

// Rows in the order of the workspace: of a sequence its drafts + 1 target rows, then its
// draft rows.
__device__ __forceinline__ const char* row_at(const VerifyParams& p, uint32_t b, uint32_t r, uint64_t size) {
  return r <= p.drafts ? (const char*)p.target + ((uint64_t)b * (p.drafts + 1) + r) * p.target_stride * size
                       : (const char*)p.draft + ((uint64_t)b * p.drafts + (r - p.drafts - 1)) * p.draft_stride * size;
}

__device__ __forceinline__ double probability(const VerifyRow& d, float z) {
  // the largest logit is infinite where the row is empty: no difference is taken then
  return d.inv == 0.0 ? 0.0 : exp2_64(((double)z - (double)d.top) * d.by) * d.inv;
}

// A tile of a row: the largest logit, and the sum of exponentials below it (NaN where a
// logit is NaN or the largest is infinite; 0 where every one is -inf).
template <typename T, int TILE>
__global__ __launch_bounds__(256) void verify_sums_kernel(VerifyParams p, uint64_t first) {
  constexpr int kGroups = TILE / 2048;
  const uint64_t block = first + blockIdx.x;
  const uint64_t id = block / p.tiles;
  const uint32_t tile = (uint32_t)(block % p.tiles), b = (uint32_t)(id / p.rows), r = (uint32_t)(id % p.rows);
  const uint32_t length = length_of(p, b);
  if (r <= p.drafts ? r > length : r - p.drafts - 1 >= length) return;  // nobody asks
  const T* const row = (const T*)row_at(p, b, r, sizeof(T));
  const uint32_t c0 = tile * TILE + threadIdx.x * 8;
  float z[kGroups][8];
#pragma unroll
  for (int j = 0; j < kGroups; ++j) load_logits(row, c0 + j * 2048, p.vocab, z[j]);
  float top = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int j = 0; j < kGroups; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      top = __builtin_fmaxf(top, z[j][e]);
      nan |= z[j][e] != z[j][e];
    }
  __shared__ float s_top[4];
  __shared__ double s_sum[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
  for (int x = 1; x < 64; x *= 2) top = __builtin_fmaxf(top, __shfl_xor(top, x));
  if (lane == 0) s_top[wave] = top;
  __syncthreads();
  top = __builtin_fmaxf(__builtin_fmaxf(s_top[0], s_top[1]), __builtin_fmaxf(s_top[2], s_top[3]));
  const double by = r <= p.drafts ? p.by : p.draft_by;
  const double from = top == -INFINITY ? 0.0 : (double)top;
  double sum[2] = {nan || top == INFINITY ? (double)NAN : 0.0, 0.0};
#pragma unroll
  for (int j = 0; j < kGroups; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e & 1] += exp2_64(((double)z[j][e] - from) * by);
  const double all = wave_sum64(sum[0] + sum[1]);
  if (lane == 0) s_sum[wave] = all;
  __syncthreads();
  if (threadIdx.x == 0)
    p.parts[id * p.tiles + tile] = {(s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]), top};
}

// A row from its tiles' sums, in every lane of the wave.
__device__ __forceinline__ VerifyRow join_row(const VerifyParams& p, uint32_t b, uint32_t r) {
  const VerifyPart* const parts = p.parts + ((uint64_t)b * p.rows + r) * p.tiles;
  const int lane = threadIdx.x & 63;
  float top = -INFINITY;
  for (uint32_t i = lane; i < p.tiles; i += 64) top = __builtin_fmaxf(top, parts[i].top);
#pragma unroll
  for (int x = 1; x < 64; x *= 2) top = __builtin_fmaxf(top, __shfl_xor(top, x));
  VerifyRow d = {r <= p.drafts ? p.by : p.draft_by, 0.0, top};
  double sum = 0.0;
  if (top > -INFINITY)
    for (uint32_t i = lane; i < p.tiles; i += 64) {
      const VerifyPart q = parts[i];
      sum += q.sum * (q.top == top ? 1.0 : exp2_64(((double)q.top - (double)top) * d.by));
    }
  sum = wave_sum64(sum);
  if (sum > 0.0 && sum < (double)INFINITY) d.inv = 1.0 / sum;  // not where it is NaN
  return d;
}

// The entry's share of what a token is drawn from after a refusal: max(p - q, 0).
__device__ __forceinline__ double rest_of(const VerifyParams& v, const VerifyDecision& d, int64_t draft, float z, float zd,
                                          uint32_t c) {
  const double p = probability(d.p, z);
  const double q = v.draft ? probability(d.q, zd) : (int64_t)c == draft ? 1.0 : 0.0;
  return p > q ? p - q : 0.0;
}

template <typename T, int TILE>
__global__ __launch_bounds__(256) void verify_decide_kernel(VerifyParams p, uint64_t first) {
  constexpr uint32_t kMost = kVerifyMaxDrafts;
  __shared__ VerifyRow s_row[2 * kMost + 1];
  __shared__ uint32_t s_taken;
  __shared__ double s_sum[4];
  const uint64_t block = first + blockIdx.x;
  const uint32_t b = (uint32_t)(block / p.tiles), tile = (uint32_t)(block % p.tiles);
  const uint32_t length = length_of(p, b);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (threadIdx.x == 0) s_taken = length;
  for (uint32_t r = wave; r <= length; r += 4) {
    const VerifyRow d = join_row(p, b, r);
    if (lane == 0) s_row[r] = d;
  }
  if (p.draft)
    for (uint32_t r = wave; r < length; r += 4) {
      const VerifyRow d = join_row(p, b, p.drafts + 1 + r);
      if (lane == 0) s_row[kMost + 1 + r] = d;
    }
  __syncthreads();
  for (uint32_t k = threadIdx.x; k < length; k += 256) {
    const int64_t x = p.tokens[(uint64_t)b * p.drafts + k];
    bool taken = false;
    if (x >= 0 && x < (int64_t)p.vocab) {
      const double at = probability(s_row[k], logit_of(((const T*)row_at(p, b, k, sizeof(T)))[x]));
      const double of = p.draft ? probability(s_row[kMost + 1 + k],
                                              logit_of(((const T*)row_at(p, b, p.drafts + 1 + k, sizeof(T)))[x]))
                                : 1.0;
      taken = (double)p.uniform[(uint64_t)b * (p.drafts + 1) + k] * of < at;
    }
    if (!taken) atomicMin(&s_taken, k);
  }
  __syncthreads();
  const uint32_t taken = s_taken;
  const VerifyDecision d = {s_row[taken], taken < length && p.draft ? s_row[kMost + 1 + taken] : VerifyRow{}, taken, length};
  if (tile == 0) {
    if (threadIdx.x == 0) {
      p.count[b] = (int32_t)taken;
      p.decisions[b] = d;
    }
    // the tokens that are taken, and what follows the one that will be drawn
    for (uint32_t k = threadIdx.x; k <= p.drafts; k += 256) {
      if (k == taken) continue;
      int64_t x = -1;
      float logp = 0.0f;
      if (k < taken) {
        x = p.tokens[(uint64_t)b * p.drafts + k];
        const float z = logit_of(((const T*)row_at(p, b, k, sizeof(T)))[x]);
        logp = (float)(((double)z - (double)s_row[k].top) * p.scale + log(s_row[k].inv));
      }
      p.out[(uint64_t)b * (p.drafts + 1) + k] = x;
      p.logprob[(uint64_t)b * (p.drafts + 1) + k] = logp;
    }
  }
  if (taken == length) return;  // drawn from p, whose tiles' sums are there
  const T* const row = (const T*)row_at(p, b, taken, sizeof(T));
  const T* const draft_row = p.draft ? (const T*)row_at(p, b, p.drafts + 1 + taken, sizeof(T)) : nullptr;
  const int64_t draft = p.tokens[(uint64_t)b * p.drafts + taken];
  const uint32_t c0 = tile * TILE + threadIdx.x * 8;
  float z[TILE / 2048][8], zd[TILE / 2048][8];
#pragma unroll
  for (int j = 0; j < TILE / 2048; ++j) {
    load_logits(row, c0 + j * 2048, p.vocab, z[j]);
    if (draft_row) load_logits(draft_row, c0 + j * 2048, p.vocab, zd[j]);
  }
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < TILE / 2048; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += rest_of(p, d, draft, z[j][e], zd[j][e], c0 + j * 2048 + e);
  sum = wave_sum64(sum);
  if (lane == 0) s_sum[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) p.rests[block] = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
}

// One block a sequence, 8 entries of the tile a thread.
template <typename T, int TILE>
__global__ __launch_bounds__(TILE / 8) void verify_draw_kernel(VerifyParams p, uint32_t first) {
  __shared__ double s_wave[16];
  __shared__ double s_from, s_left;
  __shared__ uint32_t s_tile, s_first, s_last;
  __shared__ float s_z;
  const uint32_t b = first + blockIdx.x;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const VerifyDecision d = p.decisions[b];
  const VerifyPart* const parts = p.parts + ((uint64_t)b * p.rows + d.taken) * p.tiles;
  const double* const rests = p.rests + (uint64_t)b * p.tiles;
  const double u = (double)p.uniform[(uint64_t)b * (p.drafts + 1) + p.drafts];
  if (threadIdx.x == 0) {
    s_first = ~0u;
    s_last = 0;
    s_tile = ~0u;
  }
  __syncthreads();
  // what is drawn from: the rests, or p (where nothing was refused, and where by the
  // roundings nothing is left)
  bool rest = d.taken < d.length;
  if (wave == 0) {
    auto mass = [&](uint32_t i) {
      if (i >= p.tiles) return 0.0;
      if (rest) return rests[i];
      if (d.p.inv == 0.0) return 0.0;
      const VerifyPart q = parts[i];
      return q.sum * (q.top == d.p.top ? 1.0 : exp2_64(((double)q.top - (double)d.p.top) * d.p.by)) * d.p.inv;
    };
    auto total_of = [&] {
      double total = 0.0;
      for (uint32_t i = 0; i < p.tiles; i += 64) total += wave_sum64(mass(i + lane));
      return total;
    };
    double total = total_of();
    if (rest && !(total > 0.0)) {
      rest = false;
      total = total_of();
    }
    // the first tile whose cumulated sum exceeds u total; else the last that has any
    const double goal = u * total;
    double before = 0.0;
    bool found = false;
    for (uint32_t i = 0; i < p.tiles && !found; i += 64) {
      const double m = mass(i + lane), upto = before + wave_scan64(m);
      const uint64_t over = __builtin_amdgcn_ballot_w64(m > 0.0 && upto > goal);
      const uint64_t any = __builtin_amdgcn_ballot_w64(m > 0.0);
      found = over != 0;
      const int at = over ? __builtin_ctzll(over) : any ? 63 - __builtin_clzll(any) : -1;
      if (lane == at) {
        s_tile = i + lane;
        s_from = upto - m;
      }
      before = before + wave_sum64(m);
    }
    if (lane == 0) {
      s_left = rest ? 1.0 : 0.0;
      s_wave[0] = goal;
    }
  }
  __syncthreads();
  const uint32_t tile = s_tile;
  const uint64_t at = (uint64_t)b * (p.drafts + 1) + d.taken;
  if (tile == ~0u) {  // an empty row: the whole block
    if (threadIdx.x == 0) {
      p.out[at] = -1;
      p.logprob[at] = -INFINITY;
    }
    return;
  }
  rest = s_left != 0.0;
  const double goal = s_wave[0] - s_from;
  __syncthreads();
  const T* const row = (const T*)row_at(p, b, d.taken, sizeof(T));
  const uint32_t c0 = tile * TILE + threadIdx.x * 8;
  float z[8], zd[8];
  load_logits(row, c0, p.vocab, z);
  if (rest && p.draft) load_logits((const T*)row_at(p, b, p.drafts + 1 + d.taken, sizeof(T)), c0, p.vocab, zd);
  const int64_t draft = rest ? p.tokens[(uint64_t)b * p.drafts + d.taken] : -1;
  double m[8], mine = 0.0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    m[e] = rest ? rest_of(p, d, draft, z[e], zd[e], c0 + e) : probability(d.p, z[e]);
    mine += m[e];
  }
  const double upto = wave_scan64(mine);
  if (lane == 63) s_wave[wave] = upto;
  __syncthreads();
  double sum = upto - mine;
  for (int w = 0; w < wave; ++w) sum += s_wave[w];
  uint32_t hit = ~0u, last = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    sum += m[e];
    if (m[e] > 0.0) {
      if (hit == ~0u && sum > goal) hit = threadIdx.x * 8 + e;
      last = threadIdx.x * 8 + e + 1;
    }
  }
  if (hit != ~0u) atomicMin(&s_first, hit);
  if (last) atomicMax(&s_last, last);
  __syncthreads();
  // where the roundings leave the tile's sum below the goal: its last entry that has any
  const uint32_t v = s_first != ~0u ? s_first : s_last ? s_last - 1 : 0;
  if (v / 8 == threadIdx.x) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (v % 8 == (uint32_t)e) s_z = z[e];
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    p.out[at] = (int64_t)tile * TILE + v;
    p.logprob[at] = (float)(((double)s_z - (double)d.p.top) * p.scale + log(d.p.inv));
  }
}

constexpr uint32_t kTileL = 8192, kTileS = 2048;
// the larger tile where that still gives every CU eight blocks
constexpr uint64_t kEnoughTiles = 2048;
// A launch has fewer than 2^32 threads.
constexpr uint64_t kBlocksAtOnce = 1u << 21;  // of up to 1,024

uint32_t tiles_of(uint32_t vocab, uint32_t tile) { return (vocab - 1) / tile + 1; }

uint64_t up256(uint64_t v) { return (v + 255) & ~255ull; }

template <typename T, int TILE>
void run_verify(VerifyParams p, hipStream_t stream) {
  const uint64_t sums = (uint64_t)p.batch * p.rows * p.tiles, decide = (uint64_t)p.batch * p.tiles;
  auto in_parts = [&](uint64_t blocks, auto launch) {
    for (uint64_t first = 0; first < blocks; first += kBlocksAtOnce)
      launch(first, dim3((uint32_t)(blocks - first < kBlocksAtOnce ? blocks - first : kBlocksAtOnce)));
  };
  in_parts(sums, [&](uint64_t first, dim3 grid) {
    hipLaunchKernelGGL((verify_sums_kernel<T, TILE>), grid, dim3(256), 0, stream, p, first);
  });
  in_parts(decide, [&](uint64_t first, dim3 grid) {
    hipLaunchKernelGGL((verify_decide_kernel<T, TILE>), grid, dim3(256), 0, stream, p, first);
  });
  in_parts(p.batch, [&](uint64_t first, dim3 grid) {
    hipLaunchKernelGGL((verify_draw_kernel<T, TILE>), grid, dim3(TILE / 8), 0, stream, p, (uint32_t)first);
  });
}

}  // namespace

uint64_t verify_workspace(uint32_t batch, uint32_t drafts, uint32_t vocab) {
  const uint64_t tiles = tiles_of(vocab, kTileS), rows = (uint64_t)batch * (2 * drafts + 1);
  return up256(rows * tiles * sizeof(VerifyPart)) + up256(batch * tiles * sizeof(double)) +
         up256(batch * sizeof(VerifyDecision));
}

hipError_t launch_verify(bool bf16, const VerifyParams& c, char* ws, hipStream_t stream) {
  VerifyParams p = c;
  p.rows = p.drafts + 1 + (p.draft ? p.drafts : 0);
  const bool large = (uint64_t)p.batch * p.rows * tiles_of(p.vocab, kTileL) >= kEnoughTiles;
  p.tiles = tiles_of(p.vocab, large ? kTileL : kTileS);
  const uint64_t tiles = tiles_of(p.vocab, kTileS), rows = (uint64_t)p.batch * (2 * p.drafts + 1);
  p.parts = (VerifyPart*)ws;
  p.rests = (double*)(ws + up256(rows * tiles * sizeof(VerifyPart)));
  p.decisions = (VerifyDecision*)((char*)p.rests + up256(p.batch * tiles * sizeof(double)));
  if (bf16) large ? run_verify<uint16_t, kTileL>(p, stream) : run_verify<uint16_t, kTileS>(p, stream);
  else large ? run_verify<float, kTileL>(p, stream) : run_verify<float, kTileS>(p, stream);
  return hipGetLastError();
}

}  // namespace pulse
