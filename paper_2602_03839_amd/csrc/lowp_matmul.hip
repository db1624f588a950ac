// lowp_matmul.hip -- y = x W^T for a few BF16 tokens x and a weight W that a
// receiver holds as MXFP4 or FP8 codes.
//
// The codes are read once from HBM, which bounds the kernel: half a byte and a
// thirty-second of a byte of scale a value (MXFP4), or a byte (FP8).  A wave
// takes 16 rows (times RT) and converts 16 bytes of each lane's codes to BF16
// in registers: exact, since a code has at most 3 (FP8: 4) significant bits and
// a power-of-two scale moves only the exponent.  v_mfma_f32_16x16x32_bf16
// multiplies them with 16 tokens (times NT); its columns past the last token
// are computed and dropped, which costs nothing here.  Products are exact in
// FP32 and summed in FP32.
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

namespace pulse {

namespace {

constexpr uint32_t kLpGroups = 4;  // lane groups of a wave: units side by side in a chunk

template <bool MX>
struct Unit {
  static constexpr uint32_t kValues = MX ? 32 : 16;  // in 16 bytes of codes
  static constexpr uint32_t kFrags = kValues / 8;    // MFMA operands of 8 values
  static constexpr uint32_t kChunk = kValues * kLpGroups;
};

struct __attribute__((packed, aligned(2))) Unaligned16 {
  uint32_t w[4];
};

__device__ __forceinline__ uint4 load16_any(const void* p) {
  const Unaligned16 u = *reinterpret_cast<const Unaligned16*>(p);
  return make_uint4(u.w[0], u.w[1], u.w[2], u.w[3]);
}

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

// grid.x: groups of RT row tiles; grid.y: groups of NT token tiles.  The
// block's waves share the chunks of one group and add their sums at the end.
template <bool MX, int RT, int NT, bool SHIFT>
__global__ __launch_bounds__(1024) void lowp_matmul_kernel(LowpMatmulParams p, uint32_t classes) {
  typedef Unit<MX> U;
  extern __shared__ f32x4_t s_part[];  // [waves - 1][RT * NT][64]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int r16 = lane & 15, g = lane >> 4;
  // tile t of class c holds the rows c + classes * (16 t + i): one class and
  // adjacent rows where every row starts a unit
  const uint32_t cls = SHIFT ? blockIdx.x % classes : 0;
  const uint32_t group = SHIFT ? blockIdx.x / classes : blockIdx.x;
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

// A tile's parts added by one wave; the waves take turns.  `part` is free again
// after the next tile's barrier, so callers alternate between two.
__device__ __forceinline__ void join_parts(const LowpMatmulParams& p, bool mx, f32x4_t* part, f32x4_t acc,
                                           uint32_t turn, uint32_t t, uint32_t tile) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  part[wave * 64 + lane] = acc;
  __syncthreads();
  if ((int)(turn % waves) != wave) return;
  f32x4_t v = part[lane];
#pragma unroll 5
  for (int w = 1; w < waves; ++w) v += part[w * 64 + lane];
  store_result(p, mx, v, t, (uint64_t)tile * 16 + 4 * (lane >> 4));
}

// A lane's codes of one chunk of row `row`: its unit, and its scale byte.
template <bool MX>
struct ChunkCodes {
  uint4 c;
  uint32_t scale;
};

// Always a load, so that nothing branches on the way: a row past the last is the
// last, and a unit past the row's end its last unit, with a finite scale; the
// tokens' values there are zeros.
template <bool MX>
__device__ __forceinline__ void load_codes(const LowpMatmulParams& p, uint32_t row, uint32_t units, uint32_t u,
                                           ChunkCodes<MX>& q) {
  if (row >= p.rows) row = p.rows - 1;
  const bool in = u < units;
  const uint64_t unit = (uint64_t)row * units + (in ? u : units - 1);
  q.c = load16_any(p.codes + unit * 16);
  if constexpr (MX) {
    const uint32_t scale = p.scales[unit];
    q.scale = in ? scale : 127u;
  }
}

template <bool MX>
__device__ __forceinline__ f32x4_t multiply_codes(const ChunkCodes<MX>& q, const uint4 (&x)[Unit<MX>::kFrags],
                                                  f32x4_t acc) {
  const float scale = MX ? __uint_as_float(q.scale << 23) : 1.0f;
#pragma unroll
  for (uint32_t f = 0; f < Unit<MX>::kFrags; ++f)
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(decode8<MX>(q.c, f, scale), __builtin_bit_cast(bf16x8_t, x[f]),
                                                  acc, 0, 0, 0);
  return acc;
}

// Up to 16 tokens whose values fit LDS.  The block's waves share a row tile: they take
// pairs of chunks in turn (a pair is 128 bytes of each row, a whole line).  Each wave
// has the codes of its next kAheadPairs pairs on their way, over the ends of tiles,
// and reads the tokens' values of a chunk when it gets there.
constexpr int kAheadPairs = 4;

template <bool MX>
__global__ __launch_bounds__(1024) void lowp_lds_kernel(LowpMatmulParams p, uint32_t tiles, uint32_t pairs) {
  typedef Unit<MX> U;
  extern __shared__ f32x4_t s_part[];  // [2][waves][64], then the tokens' rows
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int r16 = lane & 15, g = lane >> 4;
  const uint32_t units = p.cols / U::kValues;
  // bytes of a token's row, zeros from its end to the pair's; the 16 move each
  // row to other banks
  const uint32_t ld = pairs * U::kChunk * 4 + 16;
  char* const s_x = (char*)(s_part + 2 * waves * 64);

  // where the wave's loads are, ahead of its products
  uint32_t load_tile = blockIdx.x, load_pair = wave;
  ChunkCodes<MX> q[kAheadPairs][2];
  auto fetch = [&](ChunkCodes<MX> (&to)[2]) {
    if (load_tile >= tiles) return;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      load_codes<MX>(p, load_tile * 16 + r16, units, (load_pair * 2 + h) * kLpGroups + g, to[h]);
    load_pair += waves;
    if (load_pair >= pairs) {
      load_pair = wave;
      load_tile += gridDim.x;
    }
  };
#pragma unroll
  for (int i = 0; i < kAheadPairs; ++i) fetch(q[i]);

  const uint32_t pieces = pairs * U::kChunk / 4, filled = p.cols / 8;  // of 16 bytes, in a row
  for (uint32_t i = threadIdx.x; i < p.tokens * pieces; i += blockDim.x) {
    const uint32_t t = i / pieces, c = i % pieces;
    *(uint4*)(s_x + t * ld + c * 16) = c < filled ? load16_any(p.x + t * p.x_stride + c * 8) : make_uint4(0, 0, 0, 0);
  }
  __syncthreads();
  const char* const mine = s_x + (r16 < (int)p.tokens ? r16 : p.tokens - 1) * ld + g * (U::kValues * 2);

  uint32_t tile = blockIdx.x, pair = wave, turn = 0;
  f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (;;) {
#pragma unroll
    for (int i = 0; i < kAheadPairs; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint4 x[U::kFrags];
#pragma unroll
        for (uint32_t f = 0; f < U::kFrags; ++f)
          x[f] = *(const uint4*)(mine + (pair * 2 + h) * (U::kChunk * 2) + f * 16);
        acc = multiply_codes<MX>(q[i][h], x, acc);
      }
      fetch(q[i]);
      pair += waves;
      if (pair >= pairs) {
        join_parts(p, MX, s_part + (turn & 1) * waves * 64, acc, turn, r16, tile);
        acc = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        pair = wave;
        tile += gridDim.x;
        ++turn;
        if (tile >= tiles) return;
      }
    }
  }
}

// Up to 16 tokens, in registers: wave w of a block owns the chunks w S ... w S + S - 1
// of k for as long as it runs, and the block goes through row tiles, the next two
// tiles' codes on their way.  The waves of a block together read whole rows, 16 of
// them adjacent; nothing but codes and scales is loaded in the loop.
template <bool MX, int S, int AHEAD>
__global__ __launch_bounds__(768) void lowp_sweep_kernel(LowpMatmulParams p, uint32_t tiles) {
  typedef Unit<MX> U;
  extern __shared__ f32x4_t s_part[];  // [2][waves][64]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int r16 = lane & 15, g = lane >> 4;
  const uint32_t units = p.cols / U::kValues;  // of a row
  const uint32_t t = blockIdx.y * 16 + r16;
  const uint16_t* const xrow = p.x + (uint64_t)(t < p.tokens ? t : p.tokens - 1) * p.x_stride;

  uint4 x[S][U::kFrags];
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const uint32_t u = (wave * S + s) * kLpGroups + g;
#pragma unroll
    for (uint32_t f = 0; f < U::kFrags; ++f)
      x[s][f] = u < units ? load16_any(xrow + (uint64_t)u * U::kValues + 8 * f) : make_uint4(0, 0, 0, 0);
  }
  ChunkCodes<MX> q[AHEAD + 1][S];
  uint32_t last = blockIdx.x;
  auto fetch = [&](ChunkCodes<MX> (&to)[S], uint32_t tile) {
    if (tile < tiles) last = tile;  // past the last tile: the same again, unused
#pragma unroll
    for (int s = 0; s < S; ++s) load_codes<MX>(p, last * 16 + r16, units, (wave * S + s) * kLpGroups + g, to[s]);
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) fetch(q[i], blockIdx.x + i * gridDim.x);
  uint32_t tile = blockIdx.x, turn = 0;
  while (tile < tiles) {
#pragma unroll
    for (int i = 0; i < AHEAD + 1; ++i) {
      if (tile >= tiles) break;
      fetch(q[(i + AHEAD) % (AHEAD + 1)], tile + AHEAD * gridDim.x);
      f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < S; ++s) acc = multiply_codes<MX>(q[i][s], x[s], acc);
      join_parts(p, MX, s_part + (turn & 1) * waves * 64, acc, turn, t, tile);
      ++turn;
      tile += gridDim.x;
    }
  }
}

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
  hipLaunchKernelGGL((lowp_matmul_kernel<MX, RT, NT, SHIFT>), dim3((uint32_t)groups, tgroups),
                     dim3(64 * waves), lds, stream, p, classes);
}

constexpr uint32_t kLpCus = 256;

// Whether 16 tokens or fewer fit LDS beside the parts of 16 waves.
bool tokens_fit(const LowpMatmulParams& p, uint64_t row_bytes) {
  return p.tokens <= 16 && p.tokens * (row_bytes + 16) <= 128 * 1024;
}

template <bool MX>
void launch_lds(const LowpMatmulParams& p, uint32_t chunks, hipStream_t stream) {
  const uint32_t tiles = (p.rows + 15) / 16, pairs = (chunks + 1) / 2;
  // as many waves as give each the same number of pairs, and blocks the same of tiles
  const uint32_t each = (pairs + 15) / 16, waves = (pairs + each - 1) / each;
  const uint32_t rounds = (tiles + 2 * kLpCus - 1) / (2 * kLpCus), blocks = (tiles + rounds - 1) / rounds;
  const size_t lds = (size_t)2 * waves * 64 * sizeof(f32x4_t) + (size_t)p.tokens * (pairs * Unit<MX>::kChunk * 4 + 16);
  hipLaunchKernelGGL(lowp_lds_kernel<MX>, dim3(blocks), dim3(64 * waves), lds, stream, p, tiles, pairs);
}

template <bool MX, int S, int AHEAD>
void launch_sweep(const LowpMatmulParams& p, uint32_t chunks, hipStream_t stream) {
  const uint32_t tiles = (p.rows + 15) / 16, waves = (chunks + S - 1) / S;
  hipLaunchKernelGGL((lowp_sweep_kernel<MX, S, AHEAD>), dim3(tiles < kLpCus ? tiles : kLpCus, (p.tokens + 15) / 16),
                     dim3(64 * waves), (size_t)2 * waves * 64 * sizeof(f32x4_t), stream, p, tiles);
}

template <bool MX>
void launch_type(const LowpMatmulParams& p, hipStream_t stream) {
  typedef Unit<MX> U;
  if (p.cols % U::kValues) return launch_shape<MX, 1, 1, true>(p, stream);
  const uint32_t chunks = (p.cols + U::kChunk - 1) / U::kChunk;
  if (tokens_fit(p, (uint64_t)(chunks + 1) / 2 * U::kChunk * 4)) return launch_lds<MX>(p, chunks, stream);
  constexpr int kS = MX ? 4 : 8;
  if (p.tokens <= 16 && chunks <= 12 * kS) return launch_sweep<MX, kS, MX ? 2 : 1>(p, chunks, stream);
  if (p.tokens <= 16) launch_shape<MX, 1, 1, false>(p, stream);
  else if (p.tokens <= 32) launch_shape<MX, 2, 2, false>(p, stream);
  else launch_shape<MX, 2, 4, false>(p, stream);
}

}  // namespace

hipError_t launch_lowp_matmul(bool mxfp4, const LowpMatmulParams& p, hipStream_t stream) {
  if (mxfp4) launch_type<true>(p, stream);
  else launch_type<false>(p, stream);
  return hipGetLastError();
}

}  // namespace pulse
