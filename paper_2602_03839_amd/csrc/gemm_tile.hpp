// gemm_tile.hpp -- one block's tile of out[m][n] = sum_k A[m][k] B[n][k] on BF16
// operands with FP32 sums, for the products of the cross entropy.
//
// Each operand is either k-contiguous (row m or n holds adjacent k) or k-major
// (row k holds adjacent m or n), so that no operand has to be transposed in
// memory first.  64 k at a time go straight from global memory to LDS
// (16 bytes a lane, no registers), into one of NST buffers, while the matrix
// cores work on an earlier one: with one step ahead a step takes at least the way to
// memory (some 2,000 cycles), which the 256 by 256 tile's products fill; smaller
// tiles have more steps ahead, or several blocks on a CU.
//
// LDS layout.  Such a load writes a wave's 64 groups of 16 bytes side by side, so
// any permutation has to be made on the global side: which lane loads
// which group.
//   k-contiguous: rows of 128 bytes (8 groups).  Group c of row r lies at
//     place c ^ ((r >> 1) & 7): the 16 rows that a fragment read touches at
//     one c then cover all 64 banks once.
//   k-major: rows of all the tile's m (or n).  Pairs of groups (16 elements, one
//     fragment's width) are permuted by k: the transposing read takes 4
//     rows of 32 bytes for each of its lane groups, 8 rows apart, which then
//     lie in different banks.
//
// A fragment of v_mfma_f32_16x16x32_bf16 is 8 adjacent k of one m (or n) per lane:
// lane l has m = l & 15 and k = 8 (l >> 4) + 0..7.  From a k-major tile two
// ds_read_b64_tr_b16 give 4 of those k each.
#pragma once

#include "device_common.hpp"
#include "head.hpp"
#include "lds_load.hpp"

namespace pulse {

// One operand as the block sees it: `p` points to its first row (m or n) at
// k = 0, or, k-major, to its first column at k = 0.  `limit` counts the rows (or
// columns, a multiple of 8) from there to the matrix's end: what lies past it is
// read from the last one and dropped by the epilogue.
struct GemmOperand {
  const uint16_t* p;
  uint64_t ld;  // elements from row to row
  uint32_t limit;
};

namespace {
__device__ __align__(16) uint32_t gemm_zeros[4];  // what k past the end is read from
}

// Waits until at most N of the wave's loads into LDS are on their way and its LDS
// reads are done, then for the block's other waves.
template <int N>
__device__ __forceinline__ void wait_and_meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

constexpr int kGemmK = 64;  // k per buffer

template <int ROWS, int WAVES, bool KMAJOR>
struct GemmTile {
  static constexpr int kBytes = ROWS * kGemmK * 2;
  static constexpr int kLoads = kBytes / 1024 / WAVES;  // per wave and buffer
  static_assert(kBytes % (1024 * WAVES) == 0, "whole wave loads");

  static __device__ __forceinline__ uint32_t mix(uint32_t k) {
    return ROWS >= 128 ? (k & 3) | ((k >> 3) & 1) << 2 : ((k >> 1) & 1) | ((k >> 3) & 1) << 1;
  }

  uint32_t off[kLoads];  // byte offset from the operand's k position
  const char* at;
  uint64_t step;

  // k (of the 64) that the lane's i-th load starts at
  static __device__ __forceinline__ int32_t k_of(int i, int wave, int lane) {
    if constexpr (!KMAJOR) return (((lane & 7) ^ (((lane >> 4) & 3) | (((i * WAVES + wave) & 1) << 2))) * 8);
    else return (i * WAVES + wave) * (512 / ROWS) + lane / (ROWS / 8);
  }

  __device__ __forceinline__ void init(const GemmOperand& o, uint32_t k0, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      if constexpr (!KMAJOR) {
        uint32_t r = (i * WAVES + wave) * 8 + (lane >> 3);
        if (r >= o.limit) r = o.limit - 1;
        off[i] = (uint32_t)(r * o.ld * 2 + k_of(i, wave, lane) * 2);
      } else {
        const uint32_t k = k_of(i, wave, lane), g = lane % (ROWS / 8);
        uint32_t c = (((g >> 1) ^ mix(k)) << 1 | (g & 1)) * 8;
        if (c >= o.limit) c = o.limit - 8;
        off[i] = (uint32_t)(k * o.ld * 2 + c * 2);
      }
    }
    at = (const char*)o.p + (KMAJOR ? k0 * o.ld * 2 : (uint64_t)k0 * 2);
    step = KMAJOR ? kGemmK * o.ld * 2 : kGemmK * 2;
  }

  // The i-th load of the next 64 k, all in the matrix, into `lds`; then next().
  template <bool STREAM>
  __device__ __forceinline__ void load(char* lds, int i, int wave) const {
    load_to_lds<STREAM>(lds + (i * WAVES + wave) * 1024, off[i], buffer_at(at));
  }
  __device__ __forceinline__ void next() { at += step; }

  // The same where only `left` of the 64 k may lie in the matrix.
  __device__ __forceinline__ void load_end(char* lds, int32_t left, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const char* from = k_of(i, wave, lane) < left ? at + off[i] : (const char*)gemm_zeros;
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)from,
          (__attribute__((address_space(3))) void*)(lds + (i * WAVES + wave) * 1024), 16, 0, 0);
    }
  }

  // k-major: rows of the operand picked by `row(k)` (negative: zeros) as the 64 k.
  template <typename F>
  static __device__ __forceinline__ void gather(const GemmOperand& o, char* lds, int wave, int lane, F row) {
    static_assert(KMAJOR, "");
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint32_t k = k_of(i, wave, lane), g = lane % (ROWS / 8);
      uint32_t c = (((g >> 1) ^ mix(k)) << 1 | (g & 1)) * 8;
      if (c >= o.limit) c = o.limit - 8;
      const int32_t r = row(k);
      const uint16_t* from = r >= 0 ? o.p + (uint64_t)(uint32_t)r * o.ld + c : (const uint16_t*)gemm_zeros;
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)from,
          (__attribute__((address_space(3))) void*)(lds + (i * WAVES + wave) * 1024), 16, 0, 0);
    }
  }
  // k-major: where element (k, row) lies.
  static __device__ __forceinline__ uint32_t place(uint32_t k, uint32_t row) {
    return k * (ROWS * 2) + (((row >> 4) ^ mix(k)) << 5) + (row & 15) * 2;
  }

  // The lane's part of a fragment's place, for the rows from `first` (the wave's; a
  // multiple of 16 fragments' rows): fragment i and half ks of the step are told by
  // constants, so one register serves all of a wave's reads.
  static __device__ __forceinline__ uint32_t lane_place(uint32_t first, int lane) {
    const uint32_t r = lane & 15, g = lane >> 4;
    if constexpr (!KMAJOR) return (first + r) * 128 + ((g ^ ((r >> 1) & 7)) << 4);
    const uint32_t k = g * 8 + (r >> 2);
    return k * (ROWS * 2) + ((first * 2) ^ (mix(k) << 5)) + (r & 3) * 8;
  }

  // The lane's fragment of rows 16 i ..., k = 32 ks ..., `at`: its place and the tile's.
  static __device__ __forceinline__ bf16x8_t fragment(uint32_t at, int i, int ks) {
    if constexpr (!KMAJOR) {
      return *(const __attribute__((address_space(3))) bf16x8_t*)((at ^ (ks << 6)) + i * 2048);
    } else {
      const uint32_t to = (at ^ (i << 5)) + ks * 32 * ROWS * 2;
      s16x4_t v[2];
      v[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)to);
      v[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(to + 4 * ROWS * 2));
      return __builtin_bit_cast(bf16x8_t, *(const uint4*)v);
    }
  }
};

template <int BM_, int BN_, int WM_, int WN_, int NST_, bool AK_, bool BK_, bool STREAM_ = false>
struct Gemm {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NST = NST_;
  static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
  static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;  // fragments of a wave
  typedef GemmTile<BM, kWaves, AK_> A;
  typedef GemmTile<BN, kWaves, BK_> B;
  static constexpr int kStage = A::kBytes + B::kBytes;
  static constexpr int kLds = NST * kStage;
  static constexpr int kLoads = A::kLoads + B::kLoads;  // of a wave and step
  typedef f32x4_t Acc[FM][FN];

  // acc[i][j][e] of lane (l & 15, l >> 4): m = wave's m + 16 i + 4 (l >> 4) + e,
  // n = wave's n + 16 j + (l & 15).
  static __device__ __forceinline__ uint32_t m_of(int i, int lane, int wave) {
    return (wave / WN) * (FM * 16) + i * 16 + (lane >> 4) * 4;
  }
  static __device__ __forceinline__ uint32_t n_of(int j, int lane, int wave) {
    return (wave % WN) * (FN * 16) + j * 16 + (lane & 15);
  }

  // The tile as BF16 rows out[n][m], 16 bytes a lane and whole lines at a time: a
  // lane's own four values of 16 rows would be written in pieces of 32 bytes.
  // `value(i, j)` gives them as two packed pairs; only n < n_left and m < m_left are
  // written.  Group c of row n lies at place c ^ (n & 15).  ALIGNED: rows start at 16
  // bytes and m_left is a multiple of 8.  STREAM: written past the caches.
  template <bool STREAM, bool ALIGNED, typename F>
  static __device__ __forceinline__ void store_rows(char* lds, uint16_t* out, uint64_t ld, uint32_t m_left,
                                                    uint32_t n_left, F value) {
    static_assert(BM >= 128 && BM * BN * 2 <= kLds, "the tile fits, with 16 groups a row");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const uint32_t n = n_of(j, lane, wave);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const uint32_t m = m_of(i, lane, wave);
        *(uint2*)(lds + n * (BM * 2) + (((m >> 3) ^ (n & 15)) << 4) + (m & 4) * 2) = value(i, j);
      }
    }
    __syncthreads();
#pragma unroll 4
    for (uint32_t q = threadIdx.x; q < BN * (BM / 8); q += kThreads) {
      const uint32_t n = q / (BM / 8), c = q % (BM / 8);
      const uint4 v = *(const uint4*)(lds + n * (BM * 2) + ((c ^ (n & 15)) << 4));
      uint16_t* const to = out + n * ld + c * 8;
      if (n >= n_left || c * 8 >= m_left) continue;
      if constexpr (!ALIGNED) {
        if (c * 8 + 8 <= m_left) {
          store16_any(to, v);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (c * 8 + e < m_left) to[e] = (uint16_t)(get_u32(v, e >> 1) >> (16 * (e & 1)));
        }
      } else if constexpr (STREAM) {
        store16_stream(to, v);
      } else {
        store16(to, v);
      }
    }
  }

  // One more step of up to 64 k on `lds` (a step's two tiles, landed for every wave).
  static __device__ __forceinline__ void add_step(const char* lds, Acc& acc) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t at_a = lds_address(lds) + A::lane_place((wave / WN) * (FM * 16), lane);
    const uint32_t at_b = lds_address(lds) + A::kBytes + B::lane_place((wave % WN) * (FN * 16), lane);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      bf16x8_t b[FN];
#pragma unroll
      for (int j = 0; j < FN; ++j) b[j] = B::fragment(at_b, j, ks);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const bf16x8_t a = A::fragment(at_a, i, ks);
#pragma unroll
        for (int j = 0; j < FN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b[j], acc[i][j], 0, 0, 0);
      }
    }
  }

  // Sums over k0 <= k < k1 (k0 a multiple of 64).  Every wave calls it; ends with
  // a barrier, after which `lds` is free.  PAIRS: B's values are pairs of BF16 whose sums
  // are meant, the second ones `low` bytes behind the first; each 64 k of A are then
  // two steps.
  template <bool PAIRS = false>
  static __device__ __forceinline__ void run(char* lds, const GemmOperand& a, const GemmOperand& b, uint32_t k0,
                                             uint32_t k1, Acc& acc, uint64_t low = 0) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    A la;
    B lb;
    la.init(a, k0, wave, lane);
    lb.init(b, k0, wave, lane);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int32_t kEach = PAIRS ? 2 : 1;
    const int32_t full = (int32_t)((k1 - k0) / kGemmK) * kEach;
    const int32_t steps = (int32_t)((k1 - k0 + kGemmK - 1) / kGemmK) * kEach;
    if (steps == 0) return;
    const int32_t rest = (int32_t)((k1 - k0) % kGemmK);
    const uint32_t at_a = lds_address(lds) + A::lane_place((wave / WN) * (FM * 16), lane);
    const uint32_t at_b = lds_address(lds) + A::kBytes + B::lane_place((wave % WN) * (FN * 16), lane);

    struct Frags {
      bf16x8_t a[FM], b[FN];
    };
    // the buffers of the step that is worked on and of the one after it
    uint32_t here = 0, after = kStage;
    auto advance = [&] {
      here = after;
      after = after + kStage == kLds ? 0 : after + kStage;
    };
    bool second = false;  // the next step is the second of its 64 k
    auto next = [&] {
      if constexpr (PAIRS) {
        la.at += second ? la.step : 0;
        lb.at += second ? lb.step - low : low;
        second = !second;
      } else {
        la.next();
        lb.next();
      }
    };
    auto load = [&](uint32_t buffer, int i) {  // the i-th load of the next step, which is whole
      char* to = lds + buffer;
      if (i < A::kLoads) la.template load<STREAM_>(to, i, wave);
      else lb.template load<false>(to + A::kBytes, i - A::kLoads, wave);
    };
    auto load_step = [&](uint32_t buffer, int32_t s) {  // step s, any
      char* to = lds + buffer;
      if (s < full) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load(buffer, i);
      } else {
        la.load_end(to, rest, wave, lane);
        lb.load_end(to + A::kBytes, rest, wave, lane);
      }
      next();
    };
    auto read = [&](Frags& f, uint32_t from, int ks, int i) {  // fragment i of that half of a buffer
      if (i < FN) f.b[i] = B::fragment(from + at_b, i, ks);
      else f.a[i - FN] = A::fragment(from + at_a, i - FN, ks);
    };
    auto multiply = [&](const Frags& f, int i) {
#pragma unroll
      for (int j = 0; j < FN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.a[i], f.b[j], acc[i][j], 0, 0, 0);
    };

    // Half a step ahead: while the matrix cores work on one half of a buffer the
    // other half's fragments are read.  Between the halves the next buffer has
    // landed and this one is done with, so the step NST ahead goes there.
    // Loads, reads and products are issued in turn, in this order; the last
    // turn has no reads, so that they are back when the next half starts.
    constexpr int kTurns = FM - 1;
    Frags f0, f1;
    auto half = [&](Frags& to, uint32_t from, int ks, const Frags& by, bool loads, uint32_t buffer) {
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        if (loads) {
#pragma unroll
          for (int l = i * kLoads / FM; l < (i + 1) * kLoads / FM; ++l) load(buffer, l);
        }
#pragma unroll
        for (int r = i * (FM + FN) / kTurns; r < (i + 1) * (FM + FN) / kTurns && r < FM + FN; ++r)
          read(to, from, ks, r);
        multiply(by, i);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
#pragma unroll
    for (int i = 0; i < NST; ++i)
      if (i < steps) load_step(i * kStage, i);
    // step 0 has landed, where NST are on their way
    if (steps >= NST) wait_and_meet<(NST - 1) * kLoads>();
    else wait_and_meet<0>();
#pragma unroll
    for (int i = 0; i < FM + FN; ++i) read(f0, 0, 0, i);
    int32_t s = 0;
    for (; s + NST < full; ++s) {
      half(f1, here, 1, f0, false, 0);
      wait_and_meet<(NST - 2) * kLoads>();
      half(f0, after, 0, f1, true, here);
      next();
      advance();
    }
    // the last steps (and short sums), one half after the other
    for (; s < steps; ++s) {
#pragma unroll
      for (int i = 0; i < FM; ++i) multiply(f0, i);
#pragma unroll
      for (int i = 0; i < FM + FN; ++i) read(f0, here, 1, i);
#pragma unroll
      for (int i = 0; i < FM; ++i) multiply(f0, i);
      if (s + 1 == steps) break;
      wait_and_meet<0>();
      if (s + NST < steps) load_step(here, s + NST);
#pragma unroll
      for (int i = 0; i < FM + FN; ++i) read(f0, after, 0, i);
      advance();
    }
    __syncthreads();
  }
};

// Tile (m, n) of block `id`: each of the 8 XCDs, to which blocks go in turn, gets
// a run of adjacent tiles, `band` of them in m, then on in n, so that its L2 serves
// each operand row several times.
__device__ __forceinline__ void gemm_tile_of(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, uint32_t band,
                                             uint32_t& m, uint32_t& n) {
  const uint32_t all = tiles_m * tiles_n, per = all / 8, rest = all % 8;
  const uint32_t x = id % 8, at = id / 8;
  const uint32_t t = x * per + (x < rest ? x : rest) + at;
  const uint32_t b = t / (band * tiles_n), in = t % (band * tiles_n);
  const uint32_t high = tiles_m - b * band < band ? tiles_m - b * band : band;
  m = b * band + in % high;
  n = in / high;
}

}  // namespace pulse
