// lowp_matmul.hip -- y = x W^T for a few BF16 tokens x and a weight W that a
// receiver holds as MXFP4 or FP8 codes.
//
// The codes' way from HBM bounds the kernels: half a byte and a thirty-second of a byte
// of scale a value (MXFP4), or a byte (FP8).  They are read once for every 32 tokens, or
// 16 (rows that start inside a unit, tokens in LDS, fewer blocks than CUs), after the
// first time from the last level cache if they fit there.  A wave
// takes 16 rows and converts 16 bytes of each lane's codes to BF16 in registers:
// exact, since a code has at most 3 (FP8: 4) significant bits and a power-of-two
// scale moves only the exponent.  v_mfma_f32_16x16x32_bf16 multiplies them with 16
// tokens; its columns past the last token are computed and dropped, which costs
// nothing here.  Products are exact in FP32 and summed in FP32.
//
// Two kernels: the slab kernel below for rows of whole chunks (FP8: units), up to 64 tokens, whose
// values fit LDS or registers (152,064 x 5,120 MXFP4, 1 and 16 tokens: 65 and 79 us,
// 6.4 and 5.3 TB/s); and lowp_matmul_kernel for every other call.
//
// Any order of k serves a dot product as long as both operands use the same:
// lane (row r, group g) holds one block of 32 values (FP8: 16) with one scale,
// and reads the tokens' values of that block, so each scale is needed by the
// lane that has it and every load is 16 bytes wide.
//
// A row whose length is no multiple of the unit (32 values, FP8 16) starts
// inside a unit.  Rows that are `unit` apart start at the same place in theirs,
// so a tile then takes 16 such rows: with the tokens shifted by that place the
// products are the same as before, and only the row's first and last chunk are
// masked.
#include "device_common.hpp"
#include "head.hpp"
#include "lds_load.hpp"

namespace pulse {

namespace {

constexpr uint32_t kLpGroups = 4;  // lane groups of a wave: units side by side in a chunk

template <bool MX>
struct Unit {
  static constexpr uint32_t kValues = MX ? 32 : 16;  // in 16 bytes of codes
  static constexpr uint32_t kFrags = kValues / 8;    // MFMA operands of 8 values
  static constexpr uint32_t kChunk = kValues * kLpGroups;
};

template <bool MX>
__device__ __forceinline__ bf16x8_t decode8(const uint4& c, int f, float scale) {
  typedef __bf16 pair_t __attribute__((ext_vector_type(2)));
  pair_t v[4];
  if constexpr (MX) {
    const uint32_t w = get_u32(c, f);
    v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
    v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
    v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  } else {
    const uint32_t a = get_u32(c, 2 * f), b = get_u32(c, 2 * f + 1);
    v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false);
    v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
    v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false);
    v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
  }
  return __builtin_bit_cast(bf16x8_t, *(const uint4*)v);
}

// Codes of a unit, of which only the values [lo, hi) count; the others become
// code 0, which is zero in both types.
template <bool MX>
__device__ __forceinline__ uint4 mask_codes(uint4 c, int lo, int hi) {
  constexpr int kBits = MX ? 4 : 8, kPer = 32 / kBits;
  uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    int l = lo - j * kPer, h = hi - j * kPer;
    l = l < 0 ? 0 : l;
    h = h > kPer ? kPer : h;
    const uint32_t below = h >= kPer ? ~0u : h <= 0 ? 0u : (1u << (h * kBits)) - 1;
    const uint32_t skip = l >= kPer ? ~0u : (1u << (l * kBits)) - 1;
    w[j] &= below & ~skip;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// What a lane holds of one chunk: its unit's codes and scale byte for RT row
// tiles, its unit's values of one token in each of NT token tiles.
template <bool MX, int RT, int NT>
struct Held {
  uint4 codes[RT];
  uint32_t scale[RT];
  uint4 x[NT][Unit<MX>::kFrags];
};

// A wave's chunks are w, w + nwk, ...; `base` holds each row tile's first unit
// (a byte offset of its codes), `shift` where in that unit the row starts.
template <bool MX, int RT, int NT, bool SHIFT>
__device__ __forceinline__ void load_chunk(const LowpMatmulParams& p, const uint64_t (&unit)[RT],
                                           const uint16_t* const (&xrow)[NT], uint32_t chunk, int g,
                                           uint32_t shift, Held<MX, RT, NT>& h) {
  typedef Unit<MX> U;
  const uint32_t u = chunk * kLpGroups + g;                        // the lane's unit in its row
  const int64_t k = (int64_t)u * U::kValues - (SHIFT ? shift : 0);  // its first value's column
  const int64_t k0 = (int64_t)chunk * U::kChunk - (SHIFT ? shift : 0);
  if (k0 >= 0 && k0 + U::kChunk <= p.cols) {  // the whole chunk lies in the row
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      h.codes[r] = load16_any(p.codes + (unit[r] + u) * 16);
      if constexpr (MX) h.scale[r] = p.scales[unit[r] + u];
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (uint32_t f = 0; f < U::kFrags; ++f) h.x[n][f] = load16_any(xrow[n] + k + 8 * f);
    return;
  }
  const int lo = k < 0 ? (int)-k : 0;
  const int64_t left = (int64_t)p.cols - k;
  const int hi = left > (int)U::kValues ? (int)U::kValues : left < 0 ? 0 : (int)left;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const uint64_t at = (unit[r] + u) * 16;
    uint4 c = make_uint4(0, 0, 0, 0);
    h.scale[r] = 127;
    if (lo < hi) {
      if (at + 16 <= p.code_bytes) {
        c = load16_any(p.codes + at);
      } else {
        uint32_t w[4] = {0, 0, 0, 0};
        for (uint32_t b = 0; b < 16; ++b)
          if (at + b < p.code_bytes) w[b >> 2] |= (uint32_t)p.codes[at + b] << (8 * (b & 3));
        c = make_uint4(w[0], w[1], w[2], w[3]);
      }
      if constexpr (MX) h.scale[r] = p.scales[unit[r] + u];
      c = mask_codes<MX>(c, lo, hi);
    }
    h.codes[r] = c;
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (uint32_t f = 0; f < U::kFrags; ++f) {
      uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int v = (int)f * 8 + e;
        if (v >= lo && v < hi) w[e >> 1] |= (uint32_t)xrow[n][k + v] << (16 * (e & 1));
      }
      h.x[n][f] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <bool MX, int RT, int NT>
__device__ __forceinline__ void multiply_chunk(const Held<MX, RT, NT>& h, f32x4_t (&acc)[RT][NT]) {
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    // the scale byte is the exponent field of its FP32 value; the conversion
    // takes 0 as 2^-127 and 255 as NaN
    const float scale = MX ? __uint_as_float(h.scale[r] << 23) : 1.0f;
#pragma unroll
    for (uint32_t f = 0; f < Unit<MX>::kFrags; ++f) {
      const bf16x8_t a = decode8<MX>(h.codes[r], f, scale);
#pragma unroll
      for (int n = 0; n < NT; ++n)
        acc[r][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            a, __builtin_bit_cast(bf16x8_t, h.x[n][f]), acc[r][n], 0, 0, 0);
    }
  }
}

// grid.x: groups of RT row tiles from `first` on; grid.y: groups of NT token tiles.  The
// block's waves share the chunks of one group and add their sums at the end.
template <bool MX, int RT, int NT, bool SHIFT>
__global__ __launch_bounds__(1024) void lowp_matmul_kernel(LowpMatmulParams p, uint32_t classes, uint32_t first) {
  typedef Unit<MX> U;
  extern __shared__ f32x4_t s_part[];  // [waves - 1][RT * NT][64]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int r16 = lane & 15, g = lane >> 4;
  // tile t of class c holds the rows c + classes * (16 t + i): one class and
  // adjacent rows where every row starts a unit
  const uint32_t block = first + blockIdx.x;
  const uint32_t cls = SHIFT ? block % classes : 0;
  const uint32_t group = SHIFT ? block / classes : block;
  if (cls >= p.rows) return;  // fewer rows than classes: the whole block
  const uint32_t shift = SHIFT ? (uint32_t)(((uint64_t)cls * p.cols) % U::kValues) : 0;
  auto row_of = [&](int r, uint32_t i) -> uint64_t {
    const uint64_t in = ((uint64_t)group * RT + r) * 16 + i;
    return SHIFT ? cls + in * classes : in;
  };
  uint64_t unit[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    uint64_t row = row_of(r, r16);
    if (row >= p.rows) row = cls;  // some row of the class: its sums are dropped
    unit[r] = (row * p.cols - shift) / U::kValues;
  }
  const uint16_t* xrow[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    uint32_t t = (blockIdx.y * NT + n) * 16 + r16;
    if (t >= p.tokens) t = p.tokens - 1;
    xrow[n] = p.x + t * p.x_stride;
  }
  f32x4_t acc[RT][NT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[r][n] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

  const uint32_t chunks = (uint32_t)(((uint64_t)p.cols + shift + U::kChunk - 1) / U::kChunk);
  uint32_t c = wave;
  if (c < chunks) {
    Held<MX, RT, NT> h;
    load_chunk<MX, RT, NT, SHIFT>(p, unit, xrow, c, g, shift, h);
    for (c += waves; c < chunks; c += waves) {
      Held<MX, RT, NT> next;
      load_chunk<MX, RT, NT, SHIFT>(p, unit, xrow, c, g, shift, next);
      multiply_chunk<MX, RT, NT>(h, acc);
      h = next;
    }
    multiply_chunk<MX, RT, NT>(h, acc);
  }

  if (waves > 1) {
    if (wave > 0) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) s_part[((wave - 1) * RT * NT + r * NT + n) * 64 + lane] = acc[r][n];
    }
    __syncthreads();
    if (wave > 0) return;
    for (int w = 0; w < waves - 1; ++w)
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[r][n] += s_part[(w * RT * NT + r * NT + n) * 64 + lane];
  }
  // lane (token r16, group g) has the rows 4 g + i of each tile
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const uint32_t t = (blockIdx.y * NT + n) * 16 + r16;
    if (t >= p.tokens) continue;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint64_t row = row_of(r, 4 * g + i);
        if (row >= p.rows) continue;
        const float v = MX ? acc[r][n][i] : acc[r][n][i] / p.inv_scale;
        if (p.y_bf16) ((uint16_t*)p.y)[t * p.y_stride + row] = (uint16_t)bf16x2_rne(__float_as_uint(v), 0u);
        else ((float*)p.y)[t * p.y_stride + row] = v;
      }
  }
}

// The sum of a tile's parts and its rows' results: lane (token r16, group g) has
// the rows row0 + 4 g + i.
__device__ __forceinline__ void store_result(const LowpMatmulParams& p, bool mx, f32x4_t v, uint32_t t,
                                             uint64_t row) {
  if (t >= p.tokens) return;
  if (!mx) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] /= p.inv_scale;
  }
  const uint64_t at = t * p.y_stride + row;
  if (p.y_bf16) {
    uint16_t* y = (uint16_t*)p.y + at;
    const uint2 o = make_uint2(bf16x2_rne(__float_as_uint(v[0]), __float_as_uint(v[1])),
                               bf16x2_rne(__float_as_uint(v[2]), __float_as_uint(v[3])));
    if (at % 4 == 0 && row + 4 <= p.rows) {
      *(uint2*)y = o;
    } else {
      const uint32_t w[2] = {o.x, o.y};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (row + i < p.rows) y[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
  } else {
    float* y = (float*)p.y + at;
    if (at % 4 == 0 && row + 4 <= p.rows) {
      *(f32x4_t*)y = v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (row + i < p.rows) y[i] = v[i];
    }
  }
}

struct __attribute__((packed)) Bytes4 {
  uint32_t w;
};

// ---------------------------------------------------------------- slabs
//
// Codes through LDS.  A lane of the matrix instruction has its own row, so loading
// codes where they are used reads 16 rows, 64 bytes of each, at a time: 4.4 to
// 5.4 TB/s here.  Read as pieces of 256 bytes and marked as read once, the same
// weight streams at 6.8 to 6.9.  So a wave loads a slab, 16 rows by 256 bytes,
// into LDS of its own and reads it back by rows.  No barrier is needed for that:
// each wave waits for its own loads and has up to `depth` slabs on their way, over
// the ends of tiles.
//
// In a slab, unit 4 g + s of a row (16 bytes of codes) belongs to lane group g,
// so that a lane's four scales are adjacent too.  Unit u of row r lies at place
// u ^ r: the 16 rows that are read at one u are then in different banks.
constexpr uint32_t kSlabUnits = 16;
constexpr uint32_t kSlabBytes = 16 * kSlabUnits * 16 + 256;  // codes, then scales

struct SlabShape {
  uint32_t tiles, slabs;   // of 16 rows; of a row
  uint32_t wk, wr, depth;  // waves side by side in k, in rows; slabs ahead
  uint32_t run;            // groups of wr tiles that a block takes in a row
};

// TIGHT: places are computed where they are used, since no registers are left to keep them in.
template <bool TIGHT>
__device__ __forceinline__ uint32_t afresh(uint32_t lane) {
  if constexpr (TIGHT) asm volatile("" : "+v"(lane));
  return lane;
}

template <bool MX, bool TIGHT>
struct SlabStream {
  const LowpMatmulParams& p;
  const SlabShape& z;
  char* ring;
  uint32_t units, kw, rw, lane;
  uint32_t group, slab, slot = 0;  // of the next load
  int flying = 0;

  // The block's next group of tiles: `run` adjacent ones, so that their results'
  // lines are completed in one L2, then the next blocks' runs are passed over.
  __device__ __forceinline__ uint32_t after(uint32_t at) const {
    return (at + 1) % z.run ? at + 1 : at + 1 + (gridDim.x - 1) * z.run;
  }

  __device__ __forceinline__ void load() {
    const uint32_t tile = group * z.wr + rw < z.tiles ? group * z.wr + rw : z.tiles - 1;
    const uint32_t row0 = tile * 16, u0 = slab * kSlabUnits;
    const uint32_t rows = p.rows - row0 < 16 ? p.rows - row0 : 16;
    const uint32_t left = units - u0 < kSlabUnits ? units - u0 : kSlabUnits;
    const uint64_t first = (uint64_t)row0 * units + u0;
    char* const to = ring + slot * kSlabBytes;
    const u32x4_t codes = buffer_at(p.codes + first * 16);
    const uint32_t lane = afresh<TIGHT>(this->lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // what lies past the last row or the row's end is read from before it
      uint32_t r = i * 4 + (lane >> 4), u = (lane & 15) ^ r;
      r = r < rows ? r : rows - 1;
      u = u < left ? u : left - 1;
      load_to_lds<true>(to + i * 1024, (r * units + u) * 16, codes);
    }
    if constexpr (MX) {
      uint32_t r = lane >> 2, u = (lane & 3) * 4;
      r = r < rows ? r : rows - 1;
      u = u < left ? u : left - 4;
      load4_to_lds(to + 4096, r * units + u, buffer_at(p.scales + first));
    }
    slot = slot + 1 == z.depth ? 0 : slot + 1;
    ++flying;
    slab += z.wk;
    if (slab >= z.slabs) {
      slab = kw;
      group = after(group);
    }
  }
  __device__ __forceinline__ bool more() const { return group * z.wr < z.tiles; }

  // Waits until the oldest slab has landed.
  __device__ __forceinline__ void wait() {
    constexpr int kLoads = MX ? 5 : 4;
    if (flying >= 4) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * kLoads) : "memory");
    else if (flying == 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kLoads) : "memory");
    else if (flying == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    --flying;
  }
};

// NS > 0: each wave has up to NS slabs of k for good (slabs <= NS wk) and the tokens'
// values of them in registers; otherwise all tokens' values lie in LDS.  A block
// takes NT tiles of 16 tokens.
template <bool MX, int NS, int NT>
__global__ __launch_bounds__(NS ? 768 : 1024) void lowp_slab_kernel(LowpMatmulParams p, SlabShape z) {
  typedef Unit<MX> U;
  constexpr bool XREG = NS > 0;
  // units of a lane's codes, and parts of a sum, in registers at once
  constexpr int kAtOnce = NT == 1 ? 4 : 2, kAdds = NT == 1 ? 5 : 2;
  static_assert(XREG || NT == 1, "LDS holds one tile of tokens");
  extern __shared__ char s_lds[];  // waves' slabs, [2][waves][NT][64] parts, the tokens' rows
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t waves = z.wk * z.wr, kw = wave % z.wk, rw = wave / z.wk;
  const uint32_t r16 = lane & 15, g = lane >> 4;
  const uint32_t units = p.cols / U::kValues;
  const uint32_t t0 = blockIdx.y * 16 * NT, tokens = p.tokens - t0 < 16 * NT ? p.tokens - t0 : 16 * NT;
  f32x4_t* const s_part = (f32x4_t*)(s_lds + waves * z.depth * kSlabBytes);
  char* const s_x = (char*)(s_part + 2 * waves * NT * 64);
  // bytes of a token's row in LDS, zeros from its end to the slab's; the 16 move each
  // row to other banks
  const uint32_t ld = z.slabs * kSlabUnits * U::kValues * 2 + 16;

  uint4 x[NT][XREG ? 4 * NS : 1][U::kFrags];
  uint32_t t[NT];  // the lane's token of each tile, or some other: its sums are dropped
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    t[n] = n * 16 + r16 < tokens ? n * 16 + r16 : tokens - 1;
    if constexpr (XREG) {
#pragma unroll
      for (int s = 0; s < 4 * NS; ++s) {
        const uint32_t u = (kw + s / 4 * z.wk) * kSlabUnits + g * 4 + s % 4;
#pragma unroll
        for (uint32_t f = 0; f < U::kFrags; ++f)
          x[n][s][f] = u < units ? load16_any(p.x + (t0 + t[n]) * p.x_stride + (uint64_t)u * U::kValues + 8 * f)
                                 : make_uint4(0, 0, 0, 0);
      }
    }
  }
  SlabStream<MX, (NT > 1)> in = {p, z, s_lds + wave * z.depth * kSlabBytes, units, kw, rw, lane, blockIdx.x * z.run, kw};
  for (uint32_t i = 0; i < z.depth && in.more(); ++i) in.load();
  if constexpr (!XREG) {
    const uint32_t pieces = (ld - 16) / 16, filled = p.cols / 8;  // of 16 bytes, in a row
    for (uint32_t i = threadIdx.x; i < tokens * pieces; i += blockDim.x) {
      const uint32_t row = i / pieces, c = i % pieces;
      *(uint4*)(s_x + row * ld + c * 16) =
          c < filled ? load16_any(p.x + (t0 + row) * p.x_stride + c * 8) : make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
  }

  uint32_t slot = 0, turn = 0;
  for (uint32_t group = blockIdx.x * z.run; group * z.wr < z.tiles; group = in.after(group), ++turn) {
    f32x4_t acc[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    auto take = [&](uint32_t slab, int own) {
      in.wait();
      const char* const from = in.ring + slot * kSlabBytes;
      const uint32_t now = afresh<(NT > 1)>(lane), r16 = now & 15, g = now >> 4;
      slot = slot + 1 == z.depth ? 0 : slot + 1;
      uint32_t scales = 0;
      if constexpr (MX) scales = *(const uint32_t*)(from + 4096 + (r16 * 4 + g) * 4);
      // past the row's end the tokens are zeros; the scale has to be finite there
      if (slab * kSlabUnits + g * 4 >= units) scales = 0x7F7F7F7Fu;
      uint4 c[kAtOnce];
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        if (s % kAtOnce == 0) {
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i) c[i] = *(const uint4*)(from + r16 * 256 + (((g * 4 + s + i) ^ r16) << 4));
          if (s + kAtOnce == 4) {
            // the slab is in registers: its place is free for the next load
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (in.more()) in.load();
          }
        }
        const float scale = MX ? __uint_as_float((scales >> (8 * s) & 255u) << 23) : 1.0f;
#pragma unroll
        for (uint32_t f = 0; f < U::kFrags; ++f) {
          const bf16x8_t a = decode8<MX>(c[s % kAtOnce], f, scale);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            uint4 v;
            if constexpr (XREG) v = x[n][own * 4 + s][f];
            else v = *(const uint4*)(s_x + t[n] * ld + (slab * kSlabUnits + g * 4 + s) * (U::kValues * 2) + f * 16);
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8_t, v), acc[n], 0, 0, 0);
          }
        }
      }
    };
    if constexpr (XREG) {
#pragma unroll
      for (int n = 0; n < NS; ++n)
        if (kw + n * z.wk < z.slabs) take(kw + n * z.wk, n);
    } else {
      for (uint32_t slab = kw; slab < z.slabs; slab += z.wk) take(slab, 0);
    }
    const uint32_t tile = group * z.wr + rw;
    const uint32_t lane = afresh<(NT > 1)>(threadIdx.x & 63), r16 = lane & 15, g = lane >> 4;
    if (z.wk > 1) {
      // the parts of a tile are added by one of its waves, in turn; they are free again
      // after the next barrier but one
      f32x4_t* const part = s_part + (turn & 1) * waves * NT * 64;
#pragma unroll
      for (int n = 0; n < NT; ++n) part[(wave * NT + n) * 64 + lane] = acc[n];
      __syncthreads();
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        if ((turn * NT + n) % z.wk != kw) continue;
        acc[n] = part[(rw * z.wk * NT + n) * 64 + lane];
#pragma unroll kAdds
        for (uint32_t w = 1; w < z.wk; ++w) acc[n] += part[((rw * z.wk + w) * NT + n) * 64 + lane];
        if (tile < z.tiles) store_result(p, MX, acc[n], t0 + n * 16 + r16, (uint64_t)tile * 16 + 4 * g);
      }
    } else if (tile < z.tiles) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
        store_result(p, MX, acc[n], t0 + n * 16 + r16, (uint64_t)tile * 16 + 4 * g);
    }
  }
}

// A launch has fewer than 2^32 threads (2^21 groups of up to 1,024) and groups in y.
constexpr uint32_t kGroupsAtOnce = 1u << 21;
constexpr uint32_t kTokensAtOnce = 1u << 15;

template <bool MX, int RT, int NT, bool SHIFT>
void launch_shape(const LowpMatmulParams& p, hipStream_t stream) {
  typedef Unit<MX> U;
  const uint32_t classes = SHIFT ? U::kValues : 1;
  const uint64_t per_class = (p.rows + classes - 1) / classes;
  const uint64_t groups = (per_class + 16 * RT - 1) / (16 * RT) * classes;
  const uint32_t tgroups = (p.tokens + 16 * NT - 1) / (16 * NT);
  const uint32_t chunks = (p.cols + (SHIFT ? U::kValues - 1 : 0) + U::kChunk - 1) / U::kChunk;
  // waves share a row group's chunks until the chip has 16 waves a CU
  uint32_t waves = 1;
  while (waves < 16 && 2 * waves <= chunks && groups * tgroups * waves < 4096) waves *= 2;
  const size_t lds = (size_t)(waves - 1) * RT * NT * 64 * sizeof(f32x4_t);
  for (uint64_t first = 0; first < groups; first += kGroupsAtOnce) {
    const uint64_t left = groups - first;
    hipLaunchKernelGGL((lowp_matmul_kernel<MX, RT, NT, SHIFT>),
                       dim3(left < kGroupsAtOnce ? (uint32_t)left : kGroupsAtOnce, tgroups), dim3(64 * waves), lds,
                       stream, p, classes, (uint32_t)first);
  }
}

constexpr uint32_t kLpCus = 256;
constexpr uint32_t kLpLds = 160 * 1024;

// Up to 64 tokens by slabs, 16 or 32 at a time (the weight is then read again, from the last
// level cache if it fits there); false where that does not fit: rows that are not whole
// units (MXFP4, whose scales are loaded by fours: groups of four), other alignment, or too
// many values of the tokens.  FP8 rows of whole units, 27,648 x 5,136, 1 and 64 tokens: 25
// and 84 us (30 and 96 by the other kernel).
template <bool MX>
bool launch_slabs(const LowpMatmulParams& p, hipStream_t stream) {
  typedef Unit<MX> U;
  if (p.tokens > 64 || p.cols % (MX ? U::kChunk : U::kValues) || ((uintptr_t)p.codes & 15) ||
      (MX && ((uintptr_t)p.scales & 3)))
    return false;
  SlabShape z;
  z.tiles = (p.rows + 15) / 16;
  // a block with one tile or two loads its tokens for little: the other kernel's blocks,
  // which take two tiles of each at once, are one round up to kLpCus tiles.  64 tokens,
  // us by slabs and by the other: MXFP4, 2,048 x 3,584 11 and 12, 2,080 x 3,584 20 and 12,
  // 4,096 x 3,584 22 and 12.5, 8,192 x 3,584 27 and 21, 8,192 x 896 11.5 and 8, 12,288 x 5,120
  // both 44; FP8, 2,080 x 3,584 24 and 14, 4,096 x 5,120 36 and 19, 8,192 x 3,584 34 and 24,
  // 8,192 x 896 13 and 9.  (40 tokens of 2,080 rows: 11 and 12, FP8 12.5 and 14)
  if (p.tokens > 32 && z.tiles > kLpCus / 2 && z.tiles <= 2 * kLpCus) return false;
  z.slabs = (p.cols / U::kValues + kSlabUnits - 1) / kSlabUnits;
  const uint64_t x_bytes = (p.tokens < 16 ? p.tokens : 16) * ((uint64_t)z.slabs * kSlabUnits * U::kValues * 2 + 16);
  // the tokens in registers where a block's waves cover k; then as many rows of waves
  // as make twelve
  constexpr uint32_t kEach = MX ? 1 : 2;  // 64 registers of them
  const bool xreg = z.slabs <= 12 * kEach;
  if (xreg) {
    z.wk = z.slabs <= 12 ? z.slabs : (z.slabs + 1) / 2;
    z.wr = 12 / z.wk;
    while (z.wr > 1 && z.wr * kLpCus > z.tiles) --z.wr;
  } else {
    // as many waves as give each the same number of slabs
    const uint32_t each = (z.slabs + 11) / 12;
    z.wk = (z.slabs + each - 1) / each;
    z.wr = 1;
  }
  const uint32_t waves = z.wk * z.wr;
  // two tiles of tokens where one would leave blocks waiting for a CU: 64 tokens, MXFP4,
  // 152,064 x 5,120: 182 us (311 with one); 512 x 3,584, 128 blocks: 10 (7 with one)
  const uint32_t groups = (z.tiles + z.wr - 1) / z.wr;
  const uint32_t nt = xreg && p.tokens > 16 && groups * ((p.tokens + 15) / 16) > kLpCus ? 2 : 1;
  const uint64_t rest = (uint64_t)2 * waves * nt * 64 * sizeof(f32x4_t) + (xreg ? 0 : x_bytes);
  if (rest + waves * kSlabBytes > kLpLds) return false;
  z.depth = (uint32_t)((kLpLds - rest) / (waves * kSlabBytes));
  if (z.depth > 4) z.depth = 4;
  z.run = groups >= 16 * kLpCus ? 2 : 1;
  const dim3 grid(groups < kLpCus ? groups : kLpCus, (p.tokens + 16 * nt - 1) / (16 * nt)), block(64 * waves);
  const size_t lds = (size_t)(rest + (uint64_t)z.depth * waves * kSlabBytes);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, lds, stream, p, z); };
  if (!xreg) launch(lowp_slab_kernel<MX, 0, 1>);
  else if (z.slabs <= z.wk) launch(nt == 1 ? lowp_slab_kernel<MX, 1, 1> : lowp_slab_kernel<MX, 1, 2>);
  else launch(nt == 1 ? lowp_slab_kernel<MX, kEach, 1> : lowp_slab_kernel<MX, kEach, 2>);
  return true;
}

template <bool MX>
void launch_type(const LowpMatmulParams& p, hipStream_t stream) {
  typedef Unit<MX> U;
  if (p.cols % U::kValues) return launch_shape<MX, 1, 1, true>(p, stream);
  if (launch_slabs<MX>(p, stream)) return;
  // Each group of row tiles reads all tokens' values again, and a round of blocks takes as
  // long as its last: as few groups as fit one round; of many rounds, two tiles each.  16
  // tokens, MXFP4, in us with 1, 2 and 4 tiles: 5,120 x 27,648 (320 tiles) 75 and 51;
  // 12,288 x 16,384 (768) 65 with 2, 52 with 4, 16,384 x 27,648 (1,024) 113 and 88, FP8 70 and
  // 58, 125 and 104 (5 tokens: 48 and 43, FP8 58 and 52; the least gain at 513 tiles, 8,208 x
  // 27,648: 65 and 70, FP8 68 and 79); one token, 40,000 x 5,056 (2,500) 33, 28, 33.
  const uint32_t tiles = (p.rows + 15) / 16;
  if (p.tokens <= 16 && tiles <= kLpCus) launch_shape<MX, 1, 1, false>(p, stream);
  else if (p.tokens <= 16 && tiles > 2 * kLpCus && tiles <= 4 * kLpCus) launch_shape<MX, 4, 1, false>(p, stream);
  else if (p.tokens <= 16) launch_shape<MX, 2, 1, false>(p, stream);
  else launch_shape<MX, 2, 2, false>(p, stream);
}

}  // namespace

hipError_t launch_lowp_matmul(bool mxfp4, const LowpMatmulParams& p, hipStream_t stream) {
  for (uint32_t first = 0; first < p.tokens; first += kTokensAtOnce) {
    LowpMatmulParams q = p;
    q.x = p.x + first * p.x_stride;
    q.y = (char*)p.y + first * p.y_stride * (p.y_bf16 ? 2 : 4);
    q.tokens = p.tokens - first < kTokensAtOnce ? p.tokens - first : kTokensAtOnce;
    if (mxfp4) launch_type<true>(q, stream);
    else launch_type<false>(q, stream);
  }
  return hipGetLastError();
}

}  // namespace pulse
