// verify_drafts.hip -- drafted tokens held against the target's probabilities.
//
//   p = softmax(scale z), q = softmax(draft_scale zd) (or 1 at the draft)
//   drafts are taken while u_k q(x_k) < p(x_k); then one token is drawn, from
//   max(p - q, 0) at the first draft that is not taken, else from p.
//
// Every logit is read once; of each sequence one row, or a target's and a draft's, is read
// a second time, mostly from a cache.
//
// Probabilities are FP64.  The draw is the first entry whose cumulated probability
// exceeds u times the total: in FP32 each of some 150,000 borders would be off by 1e-7
// of the total, so that one draw in 30 gave another token than the definition's.  With
// borders off by 1e-12 it is one in a million.  An exponential is 16 FP64 instructions,
// which issue as fast as FP32's here; they bound the first kernel (HBM would take half as
// long for BF16 logits).
//
// A wave takes a segment of a row by itself: 1,024 adjacent entries, or 512 where that
// would leave CUs without work.  Four kernels: per segment the largest logit and the sum
// of exponentials below it; per sequence the decisions; per segment of a refused draft's
// rows the sums of max(p - q, 0), of 512 entries each; per sequence the segment that
// holds the draw, then the entry in it.  Without drafts the first and the last.  64
// sequences of up to 7 drafts, 152,064 BF16 logits: 84 us; one sequence sampled from
// 151,936: 3 and 6.5 us, and the host's way.
#include "device_common.hpp"
#include "head.hpp"

namespace pulse {

namespace {

// 2^(d by) for d <= 0 and d by >= -1000, off by 1.1e-12 and 1 at d = 0, so that no
// probability is above 1: a polynomial for what d by is from the nearest integer,
// interpolated at the 9 Chebyshev nodes of [-1/2, 1/2].  The integer is in the low bits of
// d by + 1.5 * 2^52, and goes into the exponent by an addition.  d is a difference of logits:
// of products with `by` first it would hold their roundings, all of it for logits of 1e20.
__device__ __forceinline__ double exp2_64(double d, double by) {
  const double shifted = __builtin_fma(d, by, 0x1.8p52), f = __builtin_fma(d, by, -(shifted - 0x1.8p52));
  double v = __builtin_fma(1.3255224878668817e-06, f, 1.5310079402249296e-05);
  v = __builtin_fma(v, f, 0.00015403455852453838);
  v = __builtin_fma(v, f, 0.0013333450568000645);
  v = __builtin_fma(v, f, 0.009618129159402558);
  v = __builtin_fma(v, f, 0.05550410941205933);
  v = __builtin_fma(v, f, 0.2402265069581299);
  v = __builtin_fma(v, f, 0.6931471805459335);
  v = __builtin_fma(v, f, 1.0);
  return __hiloint2double(__double2hiint(v) + (__double2loint(shifted) << 20), __double2loint(v));
}

// The same for every d <= 0: below 2^-1000 it is 0.
__device__ __forceinline__ double exp2_or_0(double d, double by) { return d * by > -1000.0 ? exp2_64(d, by) : 0.0; }

// A segment's sum, of exponentials below its own largest logit, as a part of its row's.
__device__ __forceinline__ double part_of(const VerifyPart& q, float top, double by) {
  return q.sum * (q.top == top ? 1.0 : exp2_or_0((double)q.top - (double)top, by));
}

__device__ __forceinline__ float logit_of(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float logit_of(float v) { return v; }

// Entries c to c + 7 of a row as they lie in memory, -inf past its end.
template <typename T>
struct RawLogits {
  uint4 v[sizeof(T) / 2];
};

template <typename T>
__device__ __forceinline__ void load_raw(const T* row, uint32_t c, uint32_t vocab, RawLogits<T>& r) {
  constexpr int kPer = 16 / sizeof(T);
  if (c + 8 <= vocab) {
#pragma unroll
    for (int i = 0; i < 8 / kPer; ++i) r.v[i] = load16_any(row + c + i * kPer);
    return;
  }
  uint32_t w[8];
#pragma unroll
  for (int e = 0; e < 8; ++e)
    w[e] = __float_as_uint(c < vocab && e < vocab - c ? logit_of(row[c + e]) : -INFINITY);
  if constexpr (sizeof(T) == 2) {
    r.v[0] = make_uint4(w[0] >> 16 | w[1], w[2] >> 16 | w[3], w[4] >> 16 | w[5], w[6] >> 16 | w[7]);
  } else {
    r.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
    r.v[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

template <typename T>
__device__ __forceinline__ void unpack(const RawLogits<T>& r, float (&z)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (sizeof(T) == 2) {
      const uint32_t w = get_u32(r.v[0], e >> 1);
      z[e] = __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16);
    } else {
      z[e] = __uint_as_float(get_u32(r.v[e >> 2], e & 3));
    }
  }
}

template <typename T>
__device__ __forceinline__ void load_logits(const T* row, uint32_t c, uint32_t vocab, float (&z)[8]) {
  RawLogits<T> r;
  load_raw(row, c, vocab, r);
  unpack(r, z);
}

// A lane's value (the same lane for all) in every lane.
__device__ __forceinline__ double lane_value(double v, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane),
                          __builtin_amdgcn_readlane(__double2loint(v), lane));
}

template <int CTRL>
__device__ __forceinline__ double dpp64(double v) {
  return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xF, 0xF, true),
                          __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xF, 0xF, true));
}

// The wave's sum and maximum in every lane, as wave_sum.
__device__ __forceinline__ double wave_sum64(double v) {
  v += dpp64<0xB1>(v);   // quad_perm 1,0,3,2
  v += dpp64<0x4E>(v);   // quad_perm 2,3,0,1
  v += dpp64<0x141>(v);  // row_half_mirror
  v += dpp64<0x140>(v);  // row_mirror
  return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}

__device__ __forceinline__ float wave_max(float v) {
  auto with = [&](auto ctrl) {
    v = __builtin_fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xF,
                                                                      0xF, true)));
  };
  with(std::integral_constant<int, 0xB1>{});
  with(std::integral_constant<int, 0x4E>{});
  with(std::integral_constant<int, 0x141>{});
  with(std::integral_constant<int, 0x140>{});
  auto row = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };
  return __builtin_fmaxf(__builtin_fmaxf(row(0), row(16)), __builtin_fmaxf(row(32), row(48)));
}

// The sum over lanes 0 to this one.
__device__ __forceinline__ double wave_scan64(double v) {
  const int lane = lane_id();
#pragma unroll
  for (int x = 1; x < 64; x *= 2) {
    const double up = __hiloint2double(__shfl_up(__double2hiint(v), x), __shfl_up(__double2loint(v), x));
    if (lane >= x) v += up;
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
  return d.inv == 0.0 ? 0.0 : exp2_or_0((double)z - (double)d.top, d.by) * d.inv;
}

// Where a wave's entries lie: eight a lane and 512 at a time, from its segment's first on.
template <int SEG>
__device__ __forceinline__ uint32_t entry_at(uint32_t segment, int j) {
  return segment * SEG + j * 512 + (threadIdx.x & 63) * 8;
}

// A segment of a row, a wave each: the largest logit, and the sum of exponentials below
// it (NaN where a logit is NaN or the largest is +inf; 0 where every one is -inf).
template <typename T, int SEG>
__global__ __launch_bounds__(256) void verify_sums_kernel(VerifyParams p, uint32_t first_row) {
  constexpr int kGroups = SEG / 512;
  const uint32_t blocks = (p.segments + 3) / 4, id = first_row + blockIdx.x / blocks;
  const uint32_t segment = blockIdx.x % blocks * 4 + (threadIdx.x >> 6), b = id / p.rows, r = id % p.rows;
  const uint32_t length = length_of(p, b);
  if (segment >= p.segments || (r <= p.drafts ? r > length : r - p.drafts - 1 >= length)) return;  // nobody asks
  const T* const row = (const T*)row_at(p, b, r, sizeof(T));
  float z[kGroups][8];
#pragma unroll
  for (int j = 0; j < kGroups; ++j) load_logits(row, entry_at<SEG>(segment, j), p.vocab, z[j]);
  // the largest value; the largest bits as whole numbers with and without a sign, which
  // are a NaN's where there is one, and the latter's else the most negative value's
  float top = -INFINITY;
  int32_t bits = 0;
  uint32_t ubits = 0;
#pragma unroll
  for (int j = 0; j < kGroups; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      top = __builtin_fmaxf(top, z[j][e]);
      const int32_t v = __float_as_int(z[j][e]);
      bits = v > bits ? v : bits;
      ubits = (uint32_t)v > ubits ? (uint32_t)v : ubits;
    }
  top = wave_max(top);
  const bool nan = bits > 0x7F800000 || ubits > 0xFF800000u;
  const double by = r <= p.drafts ? p.by : p.draft_by;
  const double least = (double)(ubits >> 31 ? __uint_as_float(ubits) : 0.0f) - (double)top;
  const double floor = r <= p.drafts ? p.floor : p.draft_floor;  // there 2^-1000 stands for 0
  double sum[2] = {0.0, 0.0};
  auto add = [&](auto clamp) {
#pragma unroll
    for (int j = 0; j < kGroups; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        double d = (double)z[j][e] - (double)top;
        if constexpr (decltype(clamp)::value) d = __builtin_fmax(d, floor);
        sum[e & 1] += exp2_64(d, by);
      }
  };
  // the same for the whole wave
  if (!__builtin_amdgcn_ballot_w64(!(least > floor))) add(std::false_type{});
  else if (top > -INFINITY) add(std::true_type{});
  if (nan || top == INFINITY) sum[0] = (double)NAN;
  const double all = wave_sum64(sum[0] + sum[1]);
  if ((threadIdx.x & 63) == 0) p.parts[(uint64_t)id * p.segments + segment] = {all, top};
}

// A row from its segments' sums, in every lane of the wave.
__device__ __forceinline__ VerifyRow join_row(const VerifyParams& p, uint32_t b, uint32_t r) {
  const VerifyPart* const parts = p.parts + ((uint64_t)b * p.rows + r) * p.segments;
  const int lane = threadIdx.x & 63;
  float top = -INFINITY;
#pragma unroll 4
  for (uint32_t i = lane; i < p.segments; i += 64) top = __builtin_fmaxf(top, parts[i].top);
  top = wave_max(top);
  VerifyRow d = {r <= p.drafts ? p.by : p.draft_by, 0.0, top};
  double sum = 0.0;
  if (top > -INFINITY)
#pragma unroll 4
    for (uint32_t i = lane; i < p.segments; i += 64) {
      const VerifyPart q = parts[i];
      sum += part_of(q, top, d.by);
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

// One block a sequence: its rows joined, a wave each, then its drafts looked at, a thread
// each, and what is known written.
template <typename T>
__global__ __launch_bounds__(512) void verify_decide_kernel(VerifyParams p, uint32_t first) {
  constexpr uint32_t kMost = kVerifyMaxDrafts;
  __shared__ VerifyRow s_row[2 * kMost + 1];
  __shared__ uint32_t s_taken;
  const uint32_t b = first + blockIdx.x;
  const uint32_t length = length_of(p, b);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (threadIdx.x == 0) s_taken = length;
  // the drafts' logits are on their way meanwhile
  const uint32_t k = threadIdx.x;
  int64_t x = -1;
  float z = -INFINITY, zd = -INFINITY, u = 0.0f;
  if (k < length) {
    x = p.tokens[(uint64_t)b * p.drafts + k];
    u = p.uniform[(uint64_t)b * (p.drafts + 1) + k];
    if (x >= 0 && x < (int64_t)p.vocab) {
      z = logit_of(((const T*)row_at(p, b, k, sizeof(T)))[x]);
      if (p.draft) zd = logit_of(((const T*)row_at(p, b, p.drafts + 1 + k, sizeof(T)))[x]);
    }
  }
  const uint32_t rows = p.draft ? 2 * length + 1 : length + 1;
  for (uint32_t i = wave; i < rows; i += 8) {
    const VerifyRow d = join_row(p, b, i <= length ? i : p.drafts + i - length);
    if (lane == 0) s_row[i] = d;
  }
  __syncthreads();
  if (k < length) {
    const double at = probability(s_row[k], z), of = p.draft ? probability(s_row[length + 1 + k], zd) : 1.0;
    if (!(x >= 0 && x < (int64_t)p.vocab && (double)u * of < at)) atomicMin(&s_taken, k);
  }
  __syncthreads();
  const uint32_t taken = s_taken;
  if (threadIdx.x == 0) {
    p.count[b] = (int32_t)taken;
    VerifyRow q = {};
    if (taken < length && p.draft) q = s_row[length + 1 + taken];
    p.decisions[b] = {s_row[taken], q, taken, length};
  }
  // the tokens that are taken, and what follows the one that will be drawn
  if (k <= p.drafts && k != taken) {
    const uint64_t at = (uint64_t)b * (p.drafts + 1) + k;
    p.out[at] = k < taken ? x : -1;
    p.logprob[at] =
        k < taken ? (float)(((double)z - (double)s_row[k].top) * p.scale + log(s_row[k].inv)) : 0.0f;
  }
}

// The rests of refused sequences, by 512 entries, a wave each.
template <typename T>
__global__ __launch_bounds__(256) void verify_rests_kernel(VerifyParams p, uint32_t first) {
  const uint32_t blocks = (p.rest_count + 3) / 4, b = first + blockIdx.x / blocks;
  const uint32_t at = blockIdx.x % blocks * 4 + (threadIdx.x >> 6), c = entry_at<512>(at, 0);
  const VerifyDecision d = p.decisions[b];
  if (at >= p.rest_count || d.taken == d.length) return;
  const int64_t draft = p.tokens[(uint64_t)b * p.drafts + d.taken];
  float z[8], zd[8];
  load_logits((const T*)row_at(p, b, d.taken, sizeof(T)), c, p.vocab, z);
  if (p.draft) load_logits((const T*)row_at(p, b, p.drafts + 1 + d.taken, sizeof(T)), c, p.vocab, zd);
  double sum = 0.0;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum += rest_of(p, d, draft, z[e], zd[e], c + e);
  sum = wave_sum64(sum);
  if ((threadIdx.x & 63) == 0) p.rests[(uint64_t)b * p.rest_count + at] = sum;
}

// One wave a sequence.  ALONE: there are no drafts, so nothing was decided before, and
// the row's sums are joined here.
template <typename T, int SEG, bool ALONE>
__global__ __launch_bounds__(64) void verify_draw_kernel(VerifyParams p, uint32_t first) {
  constexpr uint32_t kKept = 5;  // of 64 sums each, in registers
  const uint32_t b = first + blockIdx.x;
  const int lane = threadIdx.x;
  const double u = (double)p.uniform[(uint64_t)b * (p.drafts + 1) + p.drafts];
  VerifyDecision d;
  if constexpr (ALONE) d = {join_row(p, b, 0), {}, 0, 0};
  else d = p.decisions[b];
  const VerifyPart* const parts = p.parts + ((uint64_t)b * p.rows + d.taken) * p.segments;
  const double* const rests = p.rests + (uint64_t)b * p.rest_count;
  // what is drawn from: the rests, or p (where nothing was refused, and where by the
  // roundings nothing is left)
  bool rest = !ALONE && d.taken < d.length;
  uint32_t count = rest ? p.rest_count : p.segments;
  double kept[kKept];
  auto mass = [&](uint32_t i) {
    if (i >= count) return 0.0;
    if (rest) return rests[i];
    if (d.p.inv == 0.0) return 0.0;
    const VerifyPart q = parts[i];
    return part_of(q, d.p.top, d.p.by) * d.p.inv;
  };
  auto total_of = [&] {
    double mine = 0.0;
#pragma unroll
    for (uint32_t c = 0; c < kKept; ++c) mine += kept[c] = mass(c * 64 + lane);
    for (uint32_t i = kKept * 64; i < count; i += 64) mine += mass(i + lane);
    return wave_sum64(mine);
  };
  double total = total_of();
  if (rest && !(total > 0.0)) {
    rest = false;
    count = p.segments;
    total = total_of();
  }
  // the first whose cumulated sum exceeds u total; else the last that has any
  const double goal = u * total;
  double before = 0.0, from = 0.0;
  int64_t where = -1;
  bool found = false;
  auto look = [&](uint32_t i, double m) {
    const double upto = before + wave_scan64(m);
    const uint64_t over = __builtin_amdgcn_ballot_w64(m > 0.0 && upto > goal);
    const uint64_t any = __builtin_amdgcn_ballot_w64(m > 0.0);
    found = over != 0;
    if (any) {
      const int at = over ? __builtin_ctzll(over) : 63 - __builtin_clzll(any);
      where = i + at;
      from = lane_value(upto - m, at);
    }
    before = lane_value(upto, 63);
  };
#pragma unroll
  for (uint32_t c = 0; c < kKept; ++c)
    if (!found && c * 64 < count) look(c * 64, kept[c]);
  for (uint32_t i = kKept * 64; i < count && !found; i += 64) look(i, mass(i + lane));
  const uint64_t at = (uint64_t)b * (p.drafts + 1) + d.taken;
  if (ALONE && lane == 0) p.count[b] = 0;
  if (where < 0) {  // an empty row
    if (lane == 0) {
      p.out[at] = -1;
      p.logprob[at] = -INFINITY;
    }
    return;
  }
  const T* const row = (const T*)row_at(p, b, d.taken, sizeof(T));
  const T* const draft_row =
      rest && p.draft ? (const T*)row_at(p, b, p.drafts + 1 + d.taken, sizeof(T)) : nullptr;
  const int64_t draft = rest ? p.tokens[(uint64_t)b * p.drafts + d.taken] : -1;
  // the entry, 512 at a time; where the roundings leave the sum below the goal, the last
  // that has any
  const uint32_t begin = rest ? (uint32_t)where * 512 : (uint32_t)where * SEG;
  const int steps = rest ? 1 : SEG / 512;
  uint32_t entry = begin;
  float logit = 0.0f;
  before = from;
  found = false;
  for (int j = 0; j < steps && !found; ++j) {
    const uint32_t c = begin + j * 512 + lane * 8;
    float z[8], zd[8];
    load_logits(row, c, p.vocab, z);
    if (draft_row) load_logits(draft_row, c, p.vocab, zd);
    double m[8], mine = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      m[e] = rest ? rest_of(p, d, draft, z[e], zd[e], c + e) : probability(d.p, z[e]);
      mine += m[e];
    }
    const double upto = before + wave_scan64(mine);
    double sum = upto - mine;
    int hit = -1, last = -1;
    float z_hit = 0.0f, z_last = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sum += m[e];
      if (m[e] > 0.0) {
        if (hit < 0 && sum > goal) {
          hit = e;
          z_hit = z[e];
        }
        last = e;
        z_last = z[e];
      }
    }
    const uint64_t over = __builtin_amdgcn_ballot_w64(hit >= 0), any = __builtin_amdgcn_ballot_w64(last >= 0);
    found = over != 0;
    if (any) {
      const int l = over ? __builtin_ctzll(over) : 63 - __builtin_clzll(any);
      entry = begin + j * 512 + l * 8 + __builtin_amdgcn_readlane(over ? hit : last, l);
      logit = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(over ? z_hit : z_last), l));
    }
    before = lane_value(upto, 63);
  }
  if (lane == 0) {
    p.out[at] = (int64_t)entry;
    p.logprob[at] = (float)(((double)logit - (double)d.p.top) * p.scale + log(d.p.inv));
  }
}

constexpr uint32_t kSegL = 1024, kSegS = 512;
// the longer segments where they still give every SIMD eight waves (64 x 7 drafts of
// 152,064, us by entries: 1,024 81, 2,048 85, 4,096 91)
constexpr uint64_t kEnoughSegments = 8192;
// A launch has fewer than 2^32 threads.
constexpr uint32_t kUnitsAtOnce = 1u << 22;  // of up to 512

uint32_t parts_of(uint32_t n, uint32_t of) { return (n - 1) / of + 1; }

uint64_t up256(uint64_t v) { return (v + 255) & ~255ull; }

template <typename T, int SEG>
void run_verify(const VerifyParams& p, hipStream_t stream) {
  // `count` rows, or sequences, of `each` units
  auto in_parts = [&](uint64_t count, uint32_t each, auto launch) {
    const uint32_t most = kUnitsAtOnce / each;
    for (uint64_t first = 0; first < count; first += most)
      launch((uint32_t)first, (uint32_t)(count - first < most ? count - first : most) * each);
  };
  in_parts((uint64_t)p.batch * p.rows, parts_of(p.segments, 4), [&](uint32_t first, uint32_t all) {
    hipLaunchKernelGGL((verify_sums_kernel<T, SEG>), dim3(all), dim3(256), 0, stream, p, first);
  });
  if (p.drafts) {
    in_parts(p.batch, 1, [&](uint32_t first, uint32_t all) {
      hipLaunchKernelGGL(verify_decide_kernel<T>, dim3(all), dim3(512), 0, stream, p, first);
    });
    in_parts(p.batch, parts_of(p.rest_count, 4), [&](uint32_t first, uint32_t all) {
      hipLaunchKernelGGL(verify_rests_kernel<T>, dim3(all), dim3(256), 0, stream, p, first);
    });
  }
  in_parts(p.batch, 1, [&](uint32_t first, uint32_t all) {
    if (p.drafts) hipLaunchKernelGGL((verify_draw_kernel<T, SEG, false>), dim3(all), dim3(64), 0, stream, p, first);
    else hipLaunchKernelGGL((verify_draw_kernel<T, SEG, true>), dim3(all), dim3(64), 0, stream, p, first);
  });
}

}  // namespace

uint64_t verify_workspace(uint32_t batch, uint32_t drafts, uint32_t vocab) {
  const uint64_t segments = parts_of(vocab, kSegS), rows = (uint64_t)batch * (2 * drafts + 1);
  return up256(rows * segments * sizeof(VerifyPart)) + up256(batch * segments * sizeof(double)) +
         up256(batch * sizeof(VerifyDecision));
}

hipError_t launch_verify(bool bf16, const VerifyParams& c, char* ws, hipStream_t stream) {
  VerifyParams p = c;
  p.rows = p.drafts + 1 + (p.draft ? p.drafts : 0);
  const bool large = (uint64_t)p.batch * p.rows * parts_of(p.vocab, kSegL) >= kEnoughSegments;
  p.segments = parts_of(p.vocab, large ? kSegL : kSegS);
  p.rest_count = parts_of(p.vocab, kSegS);
  const uint64_t rows = (uint64_t)p.batch * (2 * p.drafts + 1);
  p.parts = (VerifyPart*)ws;
  p.rests = (double*)(ws + up256(rows * p.rest_count * sizeof(VerifyPart)));
  p.decisions = (VerifyDecision*)((char*)p.rests + up256((uint64_t)p.batch * p.rest_count * sizeof(double)));
  if (bf16) large ? run_verify<uint16_t, kSegL>(p, stream) : run_verify<uint16_t, kSegS>(p, stream);
  else large ? run_verify<float, kSegL>(p, stream) : run_verify<float, kSegS>(p, stream);
  return hipGetLastError();
}

}  // namespace pulse
