// tvq_rows.hip -- attention of many query rows over the compressed cache (gfx950): several new
// tokens per sequence with a causal mask (prompts, draft tokens), or one token over a list of
// blocks, from the codes, without writing decoded keys or values.
//
// As in tvq_attention.hip the work is done in the rotated domain,
//   s_t = (scale W D q) . y'_K,t     o = D W (sum_t p_t y'_V,t) / sum_t p_t,
// with y' the rebuilt pairs, 1/sqrt(d) folded in: one butterfly per query row and one per output
// row.  With 32 rows and more per KV head the two products are matrix products, and a rebuilt tile
// of keys and values serves all rows of the workgroup.
//
// Arithmetic.  The products run on v_mfma_f32_32x32x16_f16 with fp32 accumulation; scores, softmax
// statistics and accumulators are fp32.  fp16 keeps 11 bits of an operand, three more than bf16, at
// the same rate; its range is made to fit by powers of two that cost nothing:
//   - q^ of a row is scaled by the power of two that brings its largest element near 2^7;
//   - the pairs of the 16 (d = 128) or 32 (d = 64) tokens that a wave rebuilds together are scaled
//     by 2^-E, E the largest multiple of 8 not above the exponent of their largest norm.  The
//     scores' factor 2^E goes with the row's into the multiply-add before the exponential; for
//     the values the accumulators carry the largest E met, and the weights of a group with a
//     smaller one are scaled down to it (groups of one cache nearly always share one E).
// Where o is fp32 each operand is the sum of two fp16 numbers (22 bits) and the products are the
// three that matter: hi hi + hi lo + lo hi.
//
// Layout of the instruction (A 32 x 16, B 16 x 32): lane l gives row (A) or column (B) l % 32 and
// the 8 k's 8 (l / 32) ..; register i of the result is row (i % 4) + 8 (i / 4) + 4 (l / 32), column
// l % 32.
//   scores  A = y'_K (rows: 32 tokens, k: elements) from LDS, B = q^ in registers: a lane holds 16
//           scores of one query row, so maximum and sum are in-lane but for one exchange of the
//           two halves of the wave.
//   values  A = y'_V transposed (rows: 32 elements, k: 16 tokens) by the transposing LDS read, B =
//           the weights: the tokens that a lane holds after the scores are the k's it must give,
//           taken in that order on both sides, so the weights stay where they are.
// The accumulators of a row lie in one lane pair (elements (i % 4) + 8 (i / 4) + 4 (l / 32) + 32 m),
// as does q^ before, so both butterflies are register arithmetic with one exchange.
//
// Tiles.  A wave rebuilds 64 / (d / 32) tokens at once, d / 32 lanes per token, 16 pairs a lane,
// into LDS rows of d fp16 (hi and lo planes), 16-byte chunks permuted by the token so that reads
// by token and the transposing reads meet no bank twice.  The codes of the next tile are requested
// before the current one is worked on.
//
// m of a row is a reference point: it is raised, and sum and accumulators rescaled, only when a
// score exceeds it by more than kLazy (log2 units); weights stay below 2^(kLazy + kBias) and
// those down to 2^-(24 + kBias) of the largest are kept.
#include <float.h>
#include <hip/hip_runtime.h>

#include <type_traits>

#include "tvq_codes.h"
#include "tvq_device.h"
#include "tvq_internal.h"
#include "tvq_lanes.h"
#include "tvq_rows.h"

namespace tvq {
namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float v16f __attribute__((ext_vector_type(16)));

constexpr float kLazy = 8.0f, kBias = 6.0f;
constexpr float kNoScore = -1.0e38f;         // m before the first score
constexpr int kNoExp = -1000;                // E of the accumulators before the first values

__device__ __forceinline__ h2 cvt_h2(float a, float b) {
  return __builtin_convertvector((f2){a, b}, h2);
}
__device__ __forceinline__ uint32_t h2_bits(h2 v) {
  uint32_t u;
  __builtin_memcpy(&u, &v, 4);
  return u;
}

// x of the lower and of the upper half of the wave, on both.
__device__ __forceinline__ void halves(float x, float& lo, float& hi) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  lo = __uint_as_float(r[0]);
  hi = __uint_as_float(r[1]);
}

// 2^e as fp32; 0 below the normal range.
__device__ __forceinline__ float pow2i(int e) {
  return e < -126 ? 0.0f : __uint_as_float((uint32_t)(min(e, 127) + 127) << 23);
}

// One butterfly stage between registers h apart.
template <int N>
__device__ __forceinline__ void stage_regs(float (&x)[N], int h) {
#pragma unroll
  for (int j = 0; j < N; ++j)
    if ((j & h) == 0) {
      const float a = x[j], b = x[j + h];
      x[j] = a + b;
      x[j + h] = a - b;
    }
}

// The stage between the halves of the wave.
template <int N>
__device__ __forceinline__ void stage_halves(float (&x)[N], int half) {
  const float sgn = half ? -1.0f : 1.0f;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    float lo, hi;
    halves(x[j], lo, hi);
    x[j] = __builtin_fmaf(hi, sgn, lo);
  }
}

// The raw codes of one lane's 16 pairs.
struct RawCodes {
  uint32_t ang[4], nrm[4], hdr[2];
};

template <int D, int WAVES, int PARTS>
struct Shape {
  static constexpr int LPV = D / kElemsPerLane;          // lanes per token
  static constexpr int GROUP = kWave / LPV;              // tokens that a wave rebuilds at once
  static constexpr int TILE = WAVES == 1 ? 32 : 64;      // tokens
  static constexpr int NG = TILE / GROUP;
  static constexpr int TASKS = (2 * NG + WAVES - 1) / WAVES;   // (kind, group) tasks of a wave
  static constexpr int ROW = 2 * D;                      // bytes of a token in a plane
  static constexpr int CHUNKS = D / 8;
  static constexpr int PLANE = TILE * ROW;
  static constexpr int KIND = PARTS * PLANE;
  static constexpr int BUFS = WAVES == 1 || (WAVES == 4 && PARTS == 2) ? 1 : 2;
  static constexpr int LUT = 256 * 4 * PARTS;
};

// Place of 16-byte chunk c in the row of token t.  Keys are read 16 bytes a lane, a token per lane,
// the same chunk: 16 tokens next to each other lie in different places of 256 bytes.  Values are read
// by the transposing read, 16 lanes taking two chunks of four tokens: their pairs lie apart.
template <int D>
__device__ __forceinline__ uint32_t key_chunk(uint32_t c, uint32_t t) {
  return D == 128 ? c ^ (t & 15u) : c ^ ((t >> 1) & 7u);
}
template <int D>
__device__ __forceinline__ uint32_t value_swap(uint32_t t) {
  return D == 128 ? ((2u * t) & 14u) | ((t >> 3) & 1u) : (t & 6u) | ((t >> 3) & 1u);
}

// Raw codes of the token at record `slot0` + j (slot0 the same for the wave), slice `sub`.  Angle
// codes: 16 bytes from the lane's first word on; what lies past them is the planes behind.
__device__ __forceinline__ RawCodes load_raw(const RowsArgs& a, int kind, int d, uint32_t slot0,
                                             uint32_t j, uint32_t sub) {
  const uint32_t n = a.n[kind];
  const uint32_t w = n == 64 ? 6u : n == 128 ? 7u : 8u;
  const uint32_t ra = (uint32_t)d * w / 16, rn = a.log_norms[kind] ? d / 4 : d / 2;
  RawCodes r;
  const uint32_t odd = w == 7 ? sub & 1u : 0u;
  load_words<4>((const uint32_t*)(a.plane[kind][0] + (uint64_t)slot0 * ra +
                                  (j * ra + 2 * w * sub - 2 * odd)), r.ang);
  const uint8_t* pn = a.plane[kind][1] + (uint64_t)slot0 * rn;
  if (a.log_norms[kind]) {
    uint32_t v[2];
    load_words<2>((const uint32_t*)(pn + (j * rn + 8 * sub)), v);
    r.nrm[0] = v[0], r.nrm[1] = v[1], r.nrm[2] = r.nrm[3] = 0;
  } else {
    load_words<4>((const uint32_t*)(pn + (j * rn + 16 * sub)), r.nrm);
  }
  const u32x2 h = *(const u32x2*)(a.plane[kind][2] + (uint64_t)slot0 * 8 + j * 8);
  r.hdr[0] = h.x, r.hdr[1] = h.y;
  return r;
}

template <int W>
__device__ __forceinline__ void angle_codes(const RawCodes& r, uint32_t odd, uint32_t (&c)[16]) {
  Chunk<W> o;
  if constexpr (W == 7) {
#pragma unroll
    for (int i = 0; i < 3; ++i) o.w[i] = __builtin_amdgcn_alignbit(r.ang[i + 1], r.ang[i], 16u * odd);
    o.w[3] = r.ang[3] >> (16u * odd);
  } else {
#pragma unroll
    for (int i = 0; i < Chunk<W>::kWords; ++i) o.w[i] = r.ang[i];
  }
  unpack16_index<W>(o, c);
}

// Rebuilds a lane's 16 pairs into the tile at `dst` (its token's row); returns E of the group.
template <int D, int PARTS>
__device__ __forceinline__ int rebuild(const RawCodes& raw, uint32_t n, bool log_norms,
                                       const char* lut, char* dst, int plane, uint32_t sub,
                                       uint32_t swap) {
  const float rmin = __uint_as_float(raw.hdr[0]), rmax = __uint_as_float(raw.hdr[1]);
  // E: the largest norm of the group's tokens (the lanes of a token hold the same)
  int top = (int)raw.hdr[1];
  if constexpr (D == 64) top = max(top, (int)row_ror<2>((uint32_t)top));
  top = max(top, (int)row_ror<4>((uint32_t)top));
  top = max(top, (int)row_ror<8>((uint32_t)top));
  top = max(max(__builtin_amdgcn_readlane(top, 0), __builtin_amdgcn_readlane(top, 16)),
            max(__builtin_amdgcn_readlane(top, 32), __builtin_amdgcn_readlane(top, 48)));
  const int e = min(max(((top >> 23) - 127) & ~7, -120), 120);
  const float down = pow2i(-e);

  uint32_t c[16];
  if (n == 64) angle_codes<6>(raw, 0, c);
  else if (n == 128) angle_codes<7>(raw, sub & 1u, c);
  else angle_codes<8>(raw, 0, c);

  float r[16];
  if (log_norms) {
    const float lo = fmaxf(rmin, FLT_MIN), hi = fmaxf(rmax, FLT_MIN);
    const float l0 = __builtin_amdgcn_logf(lo == hi ? rmin : lo);
    const float step = lo == hi ? 0.0f : (__builtin_amdgcn_logf(hi) - l0) * (1.0f / 15.0f);
    const float base = l0 - (float)e;
    uint32_t nib[4];                             // code 8 j + 2 k + s: byte k of nib[2 j + s]
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      nib[2 * j] = raw.nrm[j] & 0x0F0F0F0Fu;
      nib[2 * j + 1] = (raw.nrm[j] >> 4) & 0x0F0F0F0Fu;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float q = (float)((nib[2 * (i / 8) + i % 2] >> (8 * (i % 8 / 2))) & 255u);
      r[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(q, step, base));
    }
  } else {
    const float step = linear_step255(rmin, rmax) * down, base = rmin * down;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      r[i] = __builtin_fmaf((float)((raw.nrm[i / 4] >> (8 * (i % 4))) & 255u), step, base);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = 4 * j + k;
      if constexpr (PARTS == 1) {
        const h2 cs = ((const h2*)lut)[c[i]];
        const h2 rr = cvt_h2(r[i & ~1], r[i | 1]);
        hi[k] = h2_bits((i % 2 ? (h2){rr.y, rr.y} : (h2){rr.x, rr.x}) * cs);
      } else {
        const float2 cs = ((const float2*)lut)[c[i]];
        const float x = r[i] * cs.x, y = r[i] * cs.y;
        const h2 h = cvt_h2(x, y);
        hi[k] = h2_bits(h);
        lo[k] = h2_bits(cvt_h2(x - (float)h.x, y - (float)h.y));
      }
    }
    char* const at = dst + 16u * ((4u * sub + j) ^ swap);
    *(u32x4a*)at = u32x4a{hi[0], hi[1], hi[2], hi[3]};
    if constexpr (PARTS == 2) *(u32x4a*)(at + plane) = u32x4a{lo[0], lo[1], lo[2], lo[3]};
  }
  return e;
}

__device__ __forceinline__ h8 read_h8(const char* p) { return *(const h8*)p; }

// Four 16-bit values of one column of four rows: the 16 lanes of a group give the 8-byte pieces of
// four rows of 16 columns, lane 4 j + k piece k of row j, and lane i gets column i.
__device__ __forceinline__ s4 read_columns(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)p);
}

// What a unit's rows attend to.
struct Unit {
  uint32_t b, h, rb;
  uint32_t rows;      // rows of the (sequence, KV head)
  uint32_t n_new;     // its new tokens
  int64_t pos0;       // position of its first new token
  uint32_t tokens;    // tokens that the unit's last row sees
};

__device__ __forceinline__ Unit unit_at(const RowsArgs& a, uint32_t unit) {
  Unit u;
  const uint32_t bh = unit % (a.B * a.H);
  u.rb = unit / (a.B * a.H);
  u.b = bh / a.H;
  u.h = bh - u.b * a.H;
  if (a.list) {
    const int32_t len = a.pg.seq[bh];
    u.n_new = 1;
    u.rows = a.G;
    u.tokens = len <= 0 ? 0u : min((uint32_t)len, a.t_end);
    u.pos0 = (int64_t)u.tokens - 1;
    return u;
  }
  int32_t n = (int32_t)a.T;
  if (a.q_lens) n = min(max(a.q_lens[u.b], 0), n);
  uint32_t ctx = a.t_end;
  if (a.pg.seq) {
    const int32_t len = a.pg.seq[u.b];
    ctx = len <= 0 ? 0u : min((uint32_t)len, a.t_end);
  }
  u.n_new = (uint32_t)n;
  u.rows = (uint32_t)n * a.G;
  u.pos0 = (int64_t)ctx - n;
  const uint32_t end = min(u.rows, (u.rb + 1) * a.unit_rows);        // rows [.., end) of the unit
  const int64_t seen = end == 0 ? 0 : u.pos0 + (int64_t)((end - 1) / a.G) + 1;
  u.tokens = seen < 0 ? 0u : (uint32_t)seen;
  return u;
}

// o of one row from its rotated-domain sum: x holds elements (i % 4) + 8 (i / 4) + 4 half + 32 m at
// 16 m + i.
template <int D>
__device__ __forceinline__ void store_row(const RowsArgs& a, uint64_t at, float (&x)[D / 2], int half,
                                          bool on) {
  stage_regs(x, 1);
  stage_regs(x, 2);
  stage_halves(x, half);
  stage_regs(x, 4);
  stage_regs(x, 8);
  stage_regs(x, 16);
  if constexpr (D == 128) stage_regs(x, 32);
#pragma unroll
  for (int m = 0; m < D / 2; m += 4) {
    const int e = 32 * (m / 16) + 8 * ((m % 16) / 4) + 4 * half;
    const uint32_t s0 = a.signs[e / 2], s1 = a.signs[e / 2 + 1];
    const float y[4] = {__uint_as_float(__float_as_uint(x[m]) ^ (s0 << 16 & 0x80000000u)),
                        __uint_as_float(__float_as_uint(x[m + 1]) ^ (s0 & 0x80000000u)),
                        __uint_as_float(__float_as_uint(x[m + 2]) ^ (s1 << 16 & 0x80000000u)),
                        __uint_as_float(__float_as_uint(x[m + 3]) ^ (s1 & 0x80000000u))};
    if (!on) continue;
    if (a.o_f32)
      *(float4*)((float*)a.o + at + e) = make_float4(y[0], y[1], y[2], y[3]);
    else
      *(uint2*)((uint16_t*)a.o + at + e) = make_uint2(bf16x2_rne(y[0], y[1]), bf16x2_rne(y[2], y[3]));
  }
}

// q^ = scale W D q of the lane's row as fp16 parts, elements 16 k + 8 half + i at [k][i]; returns
// the power of two that the scores must be multiplied by.
template <int D, int PARTS>
__device__ __forceinline__ float load_rows(const RowsArgs& a, uint64_t at, int half,
                                           h8 (&q)[PARTS][D / 16]) {
  float x[D / 2];
#pragma unroll
  for (int k = 0; k < D / 16; ++k) {
    const int e = 16 * k + 8 * half;
    const u32x4a s = *(const u32x4a*)(a.signs + e / 2);
    if (a.q_f32) {
      const float* p = (const float*)a.q + at + e;
      const float4 u = *(const float4*)p, v = *(const float4*)(p + 4);
      const float f[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 8; ++i)
        x[8 * k + i] = __uint_as_float(__float_as_uint(f[i]) ^
                                       ((i % 2 ? s[i / 2] : s[i / 2] << 16) & 0x80000000u));
    } else {
      const u32x4a v = *(const u32x4a*)((const uint16_t*)a.q + at + e) ^ s;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[8 * k + 2 * i] = __uint_as_float(v[i] << 16);
        x[8 * k + 2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
      }
    }
  }
  stage_regs(x, 1);
  stage_regs(x, 2);
  stage_regs(x, 4);
  stage_halves(x, half);
  stage_regs(x, 8);
  stage_regs(x, 16);
  if constexpr (D == 128) stage_regs(x, 32);
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < D / 2; ++i) {
    x[i] *= a.qscale;
    top = fmaxf(top, fabsf(x[i]));
  }
  float lo, hi;
  halves(top, lo, hi);
  // largest element in [2^7, 2^8)
  const int e = min(max((int)(__float_as_uint(fmaxf(lo, hi)) >> 23) - 127 - 7, -119), 120);
  const float down = pow2i(-e);
#pragma unroll
  for (int k = 0; k < D / 16; ++k) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = x[8 * k + i] * down;
      q[0][k][i] = (_Float16)v;
      if constexpr (PARTS == 2) q[1][k][i] = (_Float16)(v - (float)q[0][k][i]);
    }
  }
  return pow2i(e);
}

template <int D, int WAVES, int PARTS>
__global__ __launch_bounds__(WAVES * kWave, WAVES == 1 ? 2 : 2) void rows_kernel(RowsArgs a) {
  using S = Shape<D, WAVES, PARTS>;
  __shared__ __attribute__((aligned(16))) char s_lut[2][S::LUT];
  __shared__ __attribute__((aligned(16))) char s_tile[S::BUFS][2][S::KIND];
  __shared__ int s_exp[S::BUFS][2][S::NG];
  const uint32_t wave = WAVES == 1 ? 0u : __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lane = threadIdx.x % kWave, half = lane >> 5;
  // units with the most tokens first (the last rows see the most), a unit's spans together; the
  // (sequence, KV head) goes round the XCDs, so that its units meet in one L2
  const uint32_t heads = a.B * a.H;
  const uint32_t bh = blockIdx.x % heads, rest = blockIdx.x / heads;
  const uint32_t span = rest % a.n_split, rb = a.n_rb - 1 - rest / a.n_split;
  const uint32_t unit = rb * heads + bh;
  const Unit u = unit_at(a, unit);
  const uint32_t row0 = rb * (WAVES * 32);
  if (row0 >= u.rows) return;
  const uint32_t tiles = (u.tokens + S::TILE - 1) / S::TILE;
  const uint32_t spans = row_spans(tiles, a.n_split, a.min_tiles);
  if (span >= spans) return;
  const uint32_t t0 = span_start(tiles, spans, span), t1 = span_start(tiles, spans, span + 1);

  // tables
  for (int kind = 0; kind < 2; ++kind)
    for (uint32_t i = threadIdx.x; i < a.n[kind]; i += WAVES * kWave) {
      const float2 cs = ((const float2*)a.lut[kind])[i];
      if constexpr (PARTS == 1) ((h2*)s_lut[kind])[i] = cvt_h2(cs.x, cs.y);
      else ((float2*)s_lut[kind])[i] = cs;
    }

  // the lane's query row (past the last: the last, not stored)
  const uint32_t row = row0 + wave * 32 + (lane & 31);
  const bool on = row < u.rows;
  const bool busy = row0 + wave * 32 < u.rows;          // the wave has rows
  const uint32_t r = min(row, u.rows - 1);
  const uint32_t j = r / a.G, g = r - j * a.G;
  const uint64_t q_at = (uint64_t)u.b * a.q_stride[0] + (uint64_t)(u.h * a.G + g) * a.q_stride[1] +
                        (uint64_t)j * a.q_stride[2];
  h8 q[PARTS][D / 16];
  const float qf = load_rows<D, PARTS>(a, q_at, half, q);
  const int64_t seen = u.pos0 + j + 1;                   // tokens that the row sees
  const uint32_t lim = seen < 0 ? 0u : (uint32_t)seen;
  // the least and the most of the wave's rows: its first and its last
  const uint32_t lim_lo = (uint32_t)__builtin_amdgcn_readlane((int)lim, 0);
  const uint32_t lim_hi = (uint32_t)__builtin_amdgcn_readlane((int)lim, 31);

  // pool blocks: lane i holds that of the sequence's (or the list's) block blk0 + i
  uint32_t blk0 = 0, blk = 0;
  auto load_blocks = [&](uint32_t first) {
    blk0 = first;
    uint32_t i = first + (uint32_t)lane;
    bool ok = true;
    if (a.list) {
      ok = i < a.n_list;
      i = ok ? (uint32_t)a.list[(size_t)bh * a.n_list + i] : 0u;
    }
    ok = ok && i < a.pg.max_blocks;
    const uint32_t p = ok ? (uint32_t)a.pg.table[(size_t)u.b * a.pg.max_blocks + i] : 0u;
    blk = p < a.pg.n_blocks ? p : 0u;
  };
  const uint32_t sub = (uint32_t)lane % S::LPV, vec = (uint32_t)lane / S::LPV;
  RawCodes raw[S::TASKS];
  auto load_tile = [&](uint32_t tile) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < S::TASKS; ++k) {
      const uint32_t task = wave + WAVES * k;
      if (2 * S::NG % WAVES != 0 && task >= 2 * S::NG) continue;
      const int kind = (int)(task / S::NG);
      // a group past the last token reads the last group's, a token past it the last token's
      uint32_t first = tile * S::TILE + (task % S::NG) * S::GROUP;
      first = min(first, (u.tokens - 1) / S::GROUP * S::GROUP);
      const uint32_t jj = min(vec, u.tokens - 1 - first);
      uint32_t slot0 = (u.b * a.H + u.h) * a.cap + first;
      if (a.pg.table) {
        const uint32_t i = first >> a.pg.block_log2;
        if (i - blk0 >= kWave) load_blocks(i);
        const uint32_t p = (uint32_t)__builtin_amdgcn_readlane((int)blk, (int)(i - blk0));
        slot0 = ((p * a.H + u.h) << a.pg.block_log2) + (first & ((1u << a.pg.block_log2) - 1u));
      }
      raw[k] = load_raw(a, kind, D, slot0, jj, sub);
    }
  };
  auto rebuild_tile = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < S::TASKS; ++k) {
      const uint32_t task = wave + WAVES * k;
      if (2 * S::NG % WAVES != 0 && task >= 2 * S::NG) continue;
      const int kind = (int)(task / S::NG);
      const uint32_t group = task % S::NG, t = group * S::GROUP + vec;
      const uint32_t swap = kind == 0 ? key_chunk<D>(0, t) : value_swap<D>(t);
      const int e = rebuild<D, PARTS>(raw[k], a.n[kind], a.log_norms[kind] != 0, s_lut[kind],
                                      s_tile[buf][kind] + t * S::ROW, S::PLANE, sub, swap);
      if (lane == 0) s_exp[buf][kind][group] = e;
    }
  };

  float m = kNoScore, l = 0.0f;
  int vexp = kNoExp;                                     // E of the accumulators
  v16f acc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc[i] = (v16f)(0.0f);

  // the lane's places in a tile of keys (its token's row, by k) and of values (by element block and
  // half of the 16 tokens)
  uint32_t ka[D / 16], va[D / 32][2];
#pragma unroll
  for (int k = 0; k < D / 16; ++k)
    ka[k] = (lane & 31) * S::ROW + 16u * key_chunk<D>(2 * k + half, lane & 31);
#pragma unroll
  for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const uint32_t tk = 8 * z + 4 * half + (((uint32_t)lane >> 2) & 3u);
      const uint32_t chunk = 4 * mb + 2 * (((uint32_t)lane >> 4) & 1u) + (((uint32_t)lane >> 1) & 1u);
      va[mb][z] = tk * S::ROW + 16u * (chunk ^ value_swap<D>(tk)) + 8u * (lane & 1);
    }

  // 32 tokens from `tb` on, at offset `part` of the tile in `buf`
  auto work32 = [&](auto buf_c, auto part_c, uint32_t tb) __attribute__((always_inline)) {
    constexpr int buf = decltype(buf_c)::value, part = decltype(part_c)::value;
    // ---- scores ----
    const char* const kt = s_tile[buf][0] + 32 * part * S::ROW;
    v16f s = (v16f)(0.0f);
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const h8 kh = read_h8(kt + ka[k]);
      s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kh, q[0][k], s, 0, 0, 0);
      if constexpr (PARTS == 2) {
        const h8 kl = read_h8(kt + ka[k] + S::PLANE);
        s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kh, q[1][k], s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kl, q[0][k], s, 0, 0, 0);
      }
    }
    // registers 0 .. 7 hold the tokens of the first group of 16, 8 .. 15 those of the second
    if (tb + 32 > lim_lo) {
      const uint32_t t = tb + 4 * half;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = t + (i % 4) + 8 * (i / 4) < lim ? s[i] : -INFINITY;
    }
    float f[2], top = -INFINITY;
    int ve[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int group = (32 * part + 16 * p) / S::GROUP;
      f[p] = fmaxf(qf * pow2i(__builtin_amdgcn_readfirstlane(s_exp[buf][0][group])), FLT_MIN);
      ve[p] = __builtin_amdgcn_readfirstlane(s_exp[buf][1][group]);
      float mx = s[8 * p];
#pragma unroll
      for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[8 * p + i]);
      top = fmaxf(top, mx * f[p]);
    }
    if (__builtin_amdgcn_ballot_w64(top > m + (kLazy + kBias)) != 0) {
      float lo, hi;
      halves(top, lo, hi);
      // rows that stay below keep their reference: a row's bits do not depend on its neighbours
      const float most = fmaxf(lo, hi);
      const float mn = most > m + (kLazy + kBias) ? most - kBias : m;
      const float down = __builtin_amdgcn_exp2f(m - mn);
      l *= down;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) acc[i] *= down;
      m = mn;
    }
    const int vmax = max(ve[0], ve[1]);
    if (vmax > vexp) {
      const float down = pow2i(vexp - vmax);
#pragma unroll
      for (int i = 0; i < D / 32; ++i) acc[i] *= down;
      vexp = vmax;
    }
    // ---- weights (their sum is that of the rounded ones) and values, 16 tokens at a time ----
    const char* const vt = s_tile[buf][1] + 32 * part * S::ROW;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      h8 ph, pl;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * p + i], f[p], -m));
        float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * p + i + 1], f[p], -m));
        if constexpr (PARTS == 1) {
          const h2 v = cvt_h2(w0, w1);
          l = __builtin_amdgcn_fdot2(v, (h2){(_Float16)1.0f, (_Float16)1.0f}, l, false);
          ph[i] = v.x, ph[i + 1] = v.y;
        } else {
          l += w0 + w1;
          if (ve[p] != vexp) {
            const float down = pow2i(ve[p] - vexp);
            w0 *= down, w1 *= down;
          }
          const h2 v = cvt_h2(w0, w1), z = cvt_h2(w0 - (float)v.x, w1 - (float)v.y);
          ph[i] = v.x, ph[i + 1] = v.y;
          pl[i] = z.x, pl[i + 1] = z.y;
        }
      }
      if constexpr (PARTS == 1)
        if (ve[p] != vexp) ph *= (_Float16)pow2i(ve[p] - vexp);
#pragma unroll
      for (int mb = 0; mb < D / 32; ++mb) {
        h8 vh, vl;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const char* const at = vt + va[mb][z] + 16 * p * S::ROW;
          const s4 c = read_columns(at);
          __builtin_memcpy((char*)&vh + 8 * z, &c, 8);
          if constexpr (PARTS == 2) {
            const s4 cl = read_columns(at + S::PLANE);
            __builtin_memcpy((char*)&vl + 8 * z, &cl, 8);
          }
        }
        acc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vh, ph, acc[mb], 0, 0, 0);
        if constexpr (PARTS == 2) {
          acc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vh, pl, acc[mb], 0, 0, 0);
          acc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vl, ph, acc[mb], 0, 0, 0);
        }
      }
    }
  };
  auto work = [&](auto buf_c, uint32_t tile) __attribute__((always_inline)) {
    const uint32_t tb = tile * S::TILE;
    if (busy && tb < lim_hi) work32(buf_c, std::integral_constant<int, 0>{}, tb);
    if constexpr (S::TILE > 32)
      if (busy && tb + 32 < lim_hi) work32(buf_c, std::integral_constant<int, 1>{}, tb + 32);
  };

  if (t0 < t1) {
    if (a.pg.table) load_blocks((t0 * S::TILE) >> a.pg.block_log2);
    load_tile(t0);
  }
  if constexpr (S::BUFS == 1) {
    for (uint32_t t = t0; t < t1; ++t) {
      __syncthreads();                                   // the tables; the last tile's reads
      rebuild_tile(0);
      if (t + 1 < t1) load_tile(t + 1);
      __syncthreads();
      work(std::integral_constant<int, 0>{}, t);
    }
  } else {
    // two tiles a round, so that the places in LDS are known when it is compiled
    auto step = [&](auto buf_c, uint32_t t) __attribute__((always_inline)) {
      if (t + 1 < t1) rebuild_tile(decltype(buf_c)::value ^ 1);
      if (t + 2 < t1) load_tile(t + 2);
      work(buf_c, t);
      __syncthreads();
    };
    __syncthreads();
    if (t0 < t1) rebuild_tile(0);
    if (t0 + 1 < t1) load_tile(t0 + 1);
    __syncthreads();
    for (uint32_t t = t0; t < t1; t += 2) {
      step(std::integral_constant<int, 0>{}, t);
      if (t + 1 < t1) step(std::integral_constant<int, 1>{}, t + 1);
    }
  }
  if (!busy) return;

  float lo, hi;
  halves(l, lo, hi);
  l = lo + hi;
  float y[D / 2];
  const bool none = m == kNoScore;                       // no token, or no score that is a number
  const float up = none ? 0.0f : pow2i(vexp);
  if (a.n_split == 1) {
    const float inv = none ? 0.0f : 1.0f / l;
#pragma unroll
    for (int i = 0; i < D / 2; ++i) y[i] = none ? 0.0f : acc[i / 16][i % 16] * inv * up;
    const uint64_t at = (uint64_t)u.b * a.o_stride[0] + (uint64_t)(u.h * a.G + g) * a.o_stride[1] +
                        (uint64_t)j * a.o_stride[2];
    store_row<D>(a, at, y, half, on);
    return;
  }
  if (!on) return;
  const uint64_t part = ((uint64_t)unit * a.n_split + span) * (WAVES * 32) + wave * 32 + (lane & 31);
#pragma unroll
  for (int i = 0; i < D / 2; i += 4) {
    const int e = 32 * (i / 16) + 8 * ((i % 16) / 4) + 4 * half;
    float4 v;
    v.x = acc[i / 16][i % 16] * up;
    v.y = acc[i / 16][i % 16 + 1] * up;
    v.z = acc[i / 16][i % 16 + 2] * up;
    v.w = acc[i / 16][i % 16 + 3] * up;
    *(float4*)(a.ws_acc + part * D + e) = none ? make_float4(0, 0, 0, 0) : v;
  }
  if (half == 0) *(float2*)(a.ws_ml + part * 2) = make_float2(m, none ? 0.0f : l);
}

// The spans of one row, a row per wave, its elements across the lanes: M = max m, then
// o = D W (sum 2^(m - M) acc) / (sum 2^(m - M) l).  The spans' (m, l) are read 64 at a time, one
// per lane, and 8 spans' rows are requested together, the first ones before M is known.
template <int D>
__global__ __launch_bounds__(kBlockThreads) void rows_merge_kernel(RowsArgs a) {
  constexpr int EPL = D / kWave;
  constexpr uint32_t kRows = 8;
  const int lane = threadIdx.x & (kWave - 1);
  const uint32_t i = __builtin_amdgcn_readfirstlane(blockIdx.x * kWavesPerBlock + threadIdx.x / kWave);
  const uint32_t unit = i / a.unit_rows, in_unit = i - unit * a.unit_rows;
  if (unit >= a.B * a.H * a.n_rb) return;
  const Unit u = unit_at(a, unit);
  const uint32_t row = u.rb * a.unit_rows + in_unit;
  if (row >= u.rows) return;
  const uint32_t spans = row_spans((u.tokens + a.tile - 1) / a.tile, a.n_split, a.min_tiles);
  const uint64_t part = (uint64_t)unit * a.n_split * a.unit_rows + in_unit;
  const float* const ml = a.ws_ml + part * 2;
  const float* const acc = a.ws_acc + part * D + EPL * lane;
  const size_t next = (size_t)a.unit_rows;              // partials of the next span
  auto load_ml = [&](uint32_t s) {
    return s < spans ? *(const float2*)(ml + s * next * 2) : make_float2(kNoScore, 0.0f);
  };
  float r[kRows][EPL];
  auto load_acc = [&](uint32_t s0) {
#pragma unroll
    for (uint32_t k = 0; k < kRows; ++k)
#pragma unroll
      for (int e = 0; e < EPL; ++e) r[k][e] = acc[min(s0 + k, spans - 1) * next * D + e];
  };
  float2 v = load_ml(lane);
  load_acc(0);
  const uint32_t smw = a.signs[(EPL * lane) / 2];
  float M = v.x;
  for (uint32_t s = (uint32_t)lane + kWave; s < spans; s += kWave) M = fmaxf(M, load_ml(s).x);
  M = wave_max(M);
  float L = 0.0f, x[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) x[e] = 0.0f;
  for (uint32_t s0 = 0; s0 < spans; s0 += kWave) {
    if (s0 != 0) v = load_ml(s0 + lane);
    const float w = __builtin_amdgcn_exp2f(v.x - M);
    L = __builtin_fmaf(v.y, w, L);
    const uint32_t n = min(spans - s0, (uint32_t)kWave);
    for (uint32_t k0 = 0; k0 < n; k0 += kRows) {
      if (s0 + k0 != 0) load_acc(s0 + k0);
#pragma unroll
      for (uint32_t k = 0; k < kRows; ++k) {
        const float f = s0 + k0 + k < spans ? lane_value(w, (int)(k0 + k)) : 0.0f;
#pragma unroll
        for (int e = 0; e < EPL; ++e) x[e] = __builtin_fmaf(r[k][e], f, x[e]);
      }
    }
  }
  L = wave_sum(L);
  const float inv = 1.0f / L;
#pragma unroll
  for (int e = 0; e < EPL; ++e) x[e] = M == kNoScore ? 0.0f : x[e] * inv;
  fwht_across_lanes<EPL>(x, lane);
  apply_signs<EPL>(x, smw, lane);
  const uint32_t j = row / a.G, g = row - j * a.G;
  const uint64_t at = (uint64_t)u.b * a.o_stride[0] + (uint64_t)(u.h * a.G + g) * a.o_stride[1] +
                      (uint64_t)j * a.o_stride[2] + EPL * lane;
  if constexpr (EPL == 2) {
    if (a.o_f32) *(float2*)((float*)a.o + at) = make_float2(x[0], x[1]);
    else *(uint32_t*)((uint16_t*)a.o + at) = bf16x2_rne(x[0], x[1]);
  } else {
    if (a.o_f32) ((float*)a.o)[at] = x[0];
    else ((uint16_t*)a.o)[at] = (uint16_t)(bf16x2_rne(x[0], 0.0f) & 0xFFFFu);
  }
}

template <int D>
int launch(const RowsArgs& a, unsigned waves, bool wide, hipStream_t s) {
  const uint64_t units = (uint64_t)a.B * a.H * a.n_rb;
  const dim3 grid((unsigned)(units * a.n_split)), block(waves * kWave);
  if (waves == 1) {
    if (wide) hipLaunchKernelGGL((rows_kernel<D, 1, 2>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((rows_kernel<D, 1, 1>), grid, block, 0, s, a);
  } else if (waves == 8) {
    if (wide) hipLaunchKernelGGL((rows_kernel<D, 8, 2>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((rows_kernel<D, 8, 1>), grid, block, 0, s, a);
  } else {
    if (wide) hipLaunchKernelGGL((rows_kernel<D, 4, 2>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((rows_kernel<D, 4, 1>), grid, block, 0, s, a);
  }
  if (hipGetLastError() != hipSuccess) return -2;
  if (a.n_split == 1) return 0;
  const uint64_t rows = units * a.unit_rows;
  hipLaunchKernelGGL((rows_merge_kernel<D>), dim3((unsigned)((rows + kWavesPerBlock - 1) / kWavesPerBlock)),
                     dim3(kBlockThreads), 0, s, a);
  return hipGetLastError() == hipSuccess ? 0 : -2;
}

}  // namespace
}  // namespace tvq

int tvq_launch_rows(const tvq::RowsArgs& a, int d, unsigned waves, bool wide, void* stream) {
  if (d == 128) return tvq::launch<128>(a, waves, wide, (hipStream_t)stream);
  if (d == 64) return tvq::launch<64>(a, waves, wide, (hipStream_t)stream);
  return -1;
}
