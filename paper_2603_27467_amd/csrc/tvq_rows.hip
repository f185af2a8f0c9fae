// tvq_rows.hip -- attention of many query rows over the compressed cache (gfx950): several new
// tokens per sequence with a causal mask (prompts, draft tokens), or one token over a list of
// blocks, from the codes, without writing decoded keys or values.
//
// As in tvq_attention.hip the work is done in the rotated domain,
//   s_t = (scale W D q) . y'_K,t     o = D W (sum_t p_t y'_V,t) / sum_t p_t,
// with y' the rebuilt pairs, 1/sqrt(d) folded in: one butterfly per query row and one per output
// row.  Both products are matrix products over tiles of rebuilt keys and values in LDS, which serve
// all rows of a workgroup.  How a call is cut up, and which kernel it takes, stands in tvq_rows.h:
//   few_rows_kernel    up to 32 query rows per KV head: the waves take tokens of their own
//   rows_kernel        more: the waves take 32 rows each and share the tiles they rebuild together
//   rows_many_kernel   many, bf16 outputs: the same on tiles that rows_tiles_kernel rebuilt once
//   rows_merge_kernel, rows_merge_many_kernel   the partials of spans
// A rebuilt pair costs 6 to 7 vector instructions however many rows use it: few rows are bound by the
// rebuilding, many by the products.
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
// Layout of v_mfma_f32_32x32x16_f16 (A 32 x 16, B 16 x 32): lane l gives row (A) or column (B) l % 32
// and the 8 k's 8 (l / 32) ..; register i of the result is row (i % 4) + 8 (i / 4) + 4 (l / 32), column
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
// by token and the transposing reads meet no bank twice.  (Copies of the tables against conflicts of
// the gathers, 2 to 8 of them, change nothing.)
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

// f over the values of the LPR lanes that hold a row (lane bits 5 and, of four, 4).
template <int LPR, class F>
__device__ __forceinline__ float over_row(float x, F f) {
  if constexpr (LPR == 4) {
    const uint32_t u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  float lo, hi;
  halves(x, lo, hi);
  return f(lo, hi);
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
  static constexpr int TILE = 64;                        // tokens
  static constexpr int NG = TILE / GROUP;
  static constexpr int TASKS = (2 * NG + WAVES - 1) / WAVES;   // (kind, group) tasks of a wave
  static constexpr int ROW = 2 * D;                      // bytes of a token in a plane
  static constexpr int CHUNKS = D / 8;
  static constexpr int PLANE = TILE * ROW;
  static constexpr int KIND = PARTS * PLANE;
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

// Rebuilds a lane's 16 pairs into the tile at `dst` (its token's row); returns E of the group.  The
// table reads go out first and return while the norms are computed.
template <int D, int PARTS>
__device__ __forceinline__ int rebuild(const RawCodes& raw, uint32_t n, bool log_norms,
                                       const char* lut, char* dst, uint32_t plane, uint32_t sub,
                                       uint32_t swap) {
  using Entry = std::conditional_t<PARTS == 1, h2, float2>;        // cos, sin
  Entry cs[16];
  uint32_t c[16];
  if (n == 64) angle_codes<6>(raw, 0, c);
  else if (n == 128) angle_codes<7>(raw, sub & 1u, c);
  else angle_codes<8>(raw, 0, c);
#pragma unroll
  for (int i = 0; i < 16; ++i) cs[i] = ((const Entry*)lut)[c[i]];
  // E: the largest norm of the group's tokens (the lanes of a token hold the same)
  const float rmin = __uint_as_float(raw.hdr[0]), rmax = __uint_as_float(raw.hdr[1]);
  int top = (int)raw.hdr[1];
  if constexpr (D == 64) top = max(top, (int)row_ror<2>((uint32_t)top));
  top = max(top, (int)row_ror<4>((uint32_t)top));
  top = max(top, (int)row_ror<8>((uint32_t)top));
  top = max(max(__builtin_amdgcn_readlane(top, 0), __builtin_amdgcn_readlane(top, 16)),
            max(__builtin_amdgcn_readlane(top, 32), __builtin_amdgcn_readlane(top, 48)));
  const int e = min(max(((top >> 23) - 127) & ~7, -120), 120);
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
    const float down = pow2i(-e);
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
        const h2 rr = cvt_h2(r[i & ~1], r[i | 1]);
        hi[k] = h2_bits((i % 2 ? (h2){rr.y, rr.y} : (h2){rr.x, rr.x}) * cs[i]);
      } else {
        const float x = r[i] * cs[i].x, y = r[i] * cs[i].y;
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

// q^ = scale W D q of the lane's row as fp16 parts; the lanes l and l + 32 hold a row, elements 16 k +
// 8 half + i at [k][i].  Returns the power of two that the scores must be multiplied by.
template <int D, int PARTS>
__device__ __forceinline__ float load_row(const RowsArgs& a, uint64_t at, int lane,
                                          h8 (&q)[PARTS][D / 16]) {
  constexpr int N = D / 2;
  const int half = lane >> 5;
  float x[N];
#pragma unroll
  for (int k = 0; k < N / 8; ++k) {
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
#pragma unroll
  for (int h = 1; h < N; h <<= 1) stage_regs(x, h);
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = fwht_stage<32>(x[i], lane) * a.qscale;
    top = fmaxf(top, fabsf(x[i]));
  }
  top = over_row<2>(top, [](float u, float v) { return fmaxf(u, v); });
  // largest element in [2^7, 2^8)
  const int e = min(max((int)(__float_as_uint(top) >> 23) - 127 - 7, -119), 120);
  const float down = pow2i(-e);
#pragma unroll
  for (int k = 0; k < N / 8; ++k) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = x[8 * k + i] * down;
      q[0][k][i] = (_Float16)v;
      if constexpr (PARTS == 2) q[1][k][i] = (_Float16)(v - (float)q[0][k][i]);
    }
  }
  return pow2i(e);
}

// What the 32 tokens' groups of 16 are scaled by: exponents of the keys and of the values.
struct Scales {
  int ke[2], ve[2];
};

// 32 query rows, one on each pair of lanes l and l + 32: queries, statistics, accumulators, and the
// steps of the softmax.
template <int D, int PARTS>
struct Rows {
  uint32_t j, g;                                // token and query head of the lane's row
  uint32_t in_unit;                             // its place in the unit
  bool on, busy;                                // the row, and any of the 32, is one
  uint32_t lim, lim_lo, lim_hi;                 // tokens that the row sees; fewest and most of the 32
  h8 q[PARTS][D / 16];
  float qf;
  float m, l;
  int vexp;                                     // E of the accumulators
  v16f acc[D / 32];

  // Rows from `first` of the unit on (past the sequence's last: that one, not stored).
  __device__ __forceinline__ void start(const RowsArgs& a, const Unit& u, uint32_t first, int lane) {
    const uint32_t row0 = u.rb * a.unit_rows + first;
    in_unit = first + (lane & 31);
    on = row0 + (lane & 31) < u.rows;
    busy = row0 < u.rows;
    const uint32_t r = min(row0 + (lane & 31), u.rows - 1);
    j = r / a.G;
    g = r - j * a.G;
    const int64_t seen = u.pos0 + j + 1;
    lim = seen < 0 ? 0u : (uint32_t)seen;
    lim_lo = (uint32_t)__builtin_amdgcn_readlane((int)lim, 0);     // rows in order of their tokens
    lim_hi = (uint32_t)__builtin_amdgcn_readlane((int)lim, 31);
    const uint64_t at = (uint64_t)u.b * a.q_stride[0] + (uint64_t)(u.h * a.G + g) * a.q_stride[1] +
                        (uint64_t)j * a.q_stride[2];
    qf = load_row<D, PARTS>(a, at, lane, q);
    m = kNoScore;
    l = 0.0f;
    vexp = kNoExp;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) acc[i] = (v16f)(0.0f);
  }

  __device__ __forceinline__ float factor(const Scales& c, int p) const {
    return fmaxf(qf * pow2i(c.ke[p]), FLT_MIN);
  }

  __device__ __forceinline__ void lower(float by) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) acc[i] *= by;
  }

  // Before the weights of 32 tokens from tb on: scores that a row does not see, the reference point,
  // the accumulators' exponent.  Registers 0 .. 7 of s hold the first 16 tokens, 8 .. 15 the second.
  __device__ __forceinline__ void settle(v16f& s, const Scales& c, uint32_t tb, int half) {
    if (tb + 32 > lim_lo) {
      const uint32_t t = tb + 4 * half;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = t + (i % 4) + 8 * (i / 4) < lim ? s[i] : -INFINITY;
    }
    float top = -INFINITY;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      float mx = s[8 * p];
#pragma unroll
      for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[8 * p + i]);
      top = fmaxf(top, mx * factor(c, p));
    }
    if (__builtin_amdgcn_ballot_w64(top > m + (kLazy + kBias)) != 0) {
      float lo, hi;
      halves(top, lo, hi);
      // rows that stay below keep their reference: a row's bits do not depend on its neighbours
      const float most = fmaxf(lo, hi);
      const float mn = most > m + (kLazy + kBias) ? most - kBias : m;
      const float down = __builtin_amdgcn_exp2f(m - mn);
      l *= down;
      lower(down);
      m = mn;
    }
    const int vmax = max(c.ve[0], c.ve[1]);
    if (vmax > vexp) {
      lower(pow2i(vexp - vmax));
      vexp = vmax;
    }
  }

  // The weights as operands; bf16 outputs take the sum of the rounded ones.
  __device__ __forceinline__ void weigh(const v16f& s, const Scales& c, h8 (&w)[PARTS][2]) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const float f = factor(c, p);
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * p + i], f, -m));
        float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * p + i + 1], f, -m));
        if constexpr (PARTS == 1) {
          const h2 v = cvt_h2(w0, w1);
          l = __builtin_amdgcn_fdot2(v, (h2){(_Float16)1.0f, (_Float16)1.0f}, l, false);
          w[0][p][i] = v.x, w[0][p][i + 1] = v.y;
        } else {
          l += w0 + w1;
          const float down = pow2i(c.ve[p] - vexp);
          w0 *= down, w1 *= down;
          const h2 v = cvt_h2(w0, w1), z = cvt_h2(w0 - (float)v.x, w1 - (float)v.y);
          w[0][p][i] = v.x, w[0][p][i + 1] = v.y;
          w[PARTS - 1][p][i] = z.x, w[PARTS - 1][p][i + 1] = z.y;
        }
      }
    }
  }
  // (fp16 weights only) those of a group whose values are scaled less than the accumulators
  __device__ __forceinline__ void weights_down(const Scales& c, h8 (&w)[PARTS][2]) const {
    if constexpr (PARTS == 1) {
      if (__builtin_expect(min(c.ve[0], c.ve[1]) != vexp, 0)) {      // vexp is the larger of the two, or more
        w[0][0] *= (_Float16)pow2i(c.ve[0] - vexp);
        w[0][1] *= (_Float16)pow2i(c.ve[1] - vexp);
      }
    }
  }

  // Outputs, or the partial of span `span` of unit `unit`.
  __device__ __forceinline__ void finish(const RowsArgs& a, const Unit& u, uint32_t unit, uint32_t span,
                                         int half) {
    if (!busy) return;
    float lo, hi;
    halves(l, lo, hi);
    l = lo + hi;
    const bool none = m == kNoScore;                     // no token, or no score that is a number
    const float up = none ? 0.0f : pow2i(vexp);
    if (a.n_split == 1) {
      const float inv = none ? 0.0f : 1.0f / l;
      float y[D / 2];
#pragma unroll
      for (int i = 0; i < D / 2; ++i) y[i] = none ? 0.0f : acc[i / 16][i % 16] * inv * up;
      const uint64_t at = (uint64_t)u.b * a.o_stride[0] + (uint64_t)(u.h * a.G + g) * a.o_stride[1] +
                          (uint64_t)j * a.o_stride[2];
      store_row<D>(a, at, y, half, on);
      return;
    }
    if (!on) return;
    const uint64_t part = ((uint64_t)unit * a.n_split + span) * a.unit_rows + in_unit;
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
};

// A wave's place in the call, the codes under way, and where its lanes find operands in a tile.
template <int D, int WAVES, int PARTS>
struct RowsWave {
  using S = Shape<D, WAVES, PARTS>;
  const RowsArgs& a;
  Unit u;
  uint32_t wave, bh, unit, span, t0, t1;        // the span's tiles [t0, t1)
  int lane, half;
  uint32_t blk0 = 0, blk = 0;                   // lane i: the pool block of block blk0 + i
  RawCodes raw[S::TASKS];
  uint32_t ka, va;                              // places of chunk 0 in a tile of keys and of values

  __device__ __forceinline__ RowsWave(const RowsArgs& args) : a(args) {
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    lane = threadIdx.x % kWave;
    half = lane >> 5;
  }

  // Finds the workgroup's unit and span; false where it has none.
  __device__ __forceinline__ bool start() {
    // units with the most tokens first (the last rows see the most), a unit's spans together; the
    // (sequence, KV head) goes round the XCDs, so that its units meet in one L2
    const uint32_t heads = a.B * a.H;
    bh = blockIdx.x % heads;
    const uint32_t rest = blockIdx.x / heads;
    span = rest % a.n_split;
    unit = (a.n_rb - 1 - rest / a.n_split) * heads + bh;
    u = unit_at(a, unit);
    if (u.rb * a.unit_rows >= u.rows) return false;
    const uint32_t tiles = (u.tokens + a.tile - 1) / a.tile;
    const uint32_t spans = row_spans(tiles, a.n_split, a.min_tiles);
    if (span >= spans) return false;
    t0 = span_start(tiles, spans, span);
    t1 = span_start(tiles, spans, span + 1);
    // Chunk 2 k + half of a key's row lies at ka ^ 32 k, and column piece (lane's) of element block mb
    // of values at va ^ 64 mb, for tokens 8 on at (va ^ 16 ^ 64 mb) + 8 rows.
    ka = (lane & 31) * S::ROW + 16u * key_chunk<D>(half, lane & 31);
    const uint32_t tk = 4 * half + (((uint32_t)lane >> 2) & 3u);
    const uint32_t chunk = 2 * (((uint32_t)lane >> 4) & 1u) + (((uint32_t)lane >> 1) & 1u);
    va = tk * S::ROW + 16u * (chunk ^ value_swap<D>(tk)) + 8u * (lane & 1);
    return true;
  }

  __device__ __forceinline__ void load_blocks(uint32_t first) {
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
  }

  // Codes of the group of tokens from `first` on: past the last token those of the last group, in it
  // those of the last token.
  __device__ __forceinline__ RawCodes load_group(int kind, uint32_t first) {
    first = min(first, (u.tokens - 1) / S::GROUP * S::GROUP);
    const uint32_t jj = min((uint32_t)lane / S::LPV, u.tokens - 1 - first);
    uint32_t slot0 = (u.b * a.H + u.h) * a.cap + first;
    if (a.pg.table) {
      const uint32_t i = first >> a.pg.block_log2;
      if (i - blk0 >= kWave) load_blocks(i);
      const uint32_t p = (uint32_t)__builtin_amdgcn_readlane((int)blk, (int)(i - blk0));
      slot0 = ((p * a.H + u.h) << a.pg.block_log2) + (first & ((1u << a.pg.block_log2) - 1u));
    }
    return load_raw(a, kind, D, slot0, jj, (uint32_t)lane % S::LPV);
  }

  __device__ __forceinline__ void load_tile(uint32_t tile) {
#pragma unroll
    for (int k = 0; k < S::TASKS; ++k) {
      const uint32_t task = wave + WAVES * k;
      if (2 * S::NG % WAVES != 0 && task >= 2 * S::NG) continue;
      raw[k] = load_group((int)(task / S::NG), tile * S::TILE + (task % S::NG) * S::GROUP);
    }
  }

  // The codes under way into the tile at `tile` (keys, then values), their E's into `exps`.
  __device__ __forceinline__ void rebuild_tile(const char* lut, char* tile, int* exps) {
#pragma unroll
    for (int k = 0; k < S::TASKS; ++k) {
      const uint32_t task = wave + WAVES * k;
      if (2 * S::NG % WAVES != 0 && task >= 2 * S::NG) continue;
      const int kind = (int)(task / S::NG);
      const uint32_t t = task % S::NG * S::GROUP + (uint32_t)lane / S::LPV;
      const uint32_t swap = kind == 0 ? key_chunk<D>(0, t) : value_swap<D>(t);
      const int e = rebuild<D, PARTS>(raw[k], a.n[kind], a.log_norms[kind] != 0, lut + kind * S::LUT,
                                      tile + kind * S::KIND + t * S::ROW, S::PLANE,
                                      (uint32_t)lane % S::LPV, swap);
      if (lane == 0) exps[kind * S::NG + task % S::NG] = e;
    }
  }

  __device__ __forceinline__ void load_tables(char* lut) {
    for (int kind = 0; kind < 2; ++kind)
      for (uint32_t i = threadIdx.x; i < a.n[kind]; i += WAVES * kWave) {
        const float2 cs = ((const float2*)a.lut[kind])[i];
        if constexpr (PARTS == 1) ((h2*)(lut + kind * S::LUT))[i] = cvt_h2(cs.x, cs.y);
        else ((float2*)(lut + kind * S::LUT))[i] = cs;
      }
  }

  // Operands of 32 tokens whose keys or values begin at `at`.
  __device__ __forceinline__ h8 key(const char* at, int k) const {
    return read_h8(at + (ka ^ (32u * k)));
  }
  __device__ __forceinline__ h8 value(const char* at, int mb) const {
    h8 v;
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const s4 c = read_columns(at + ((va ^ (16u * z) ^ (64u * mb)) + 8u * z * S::ROW));
      __builtin_memcpy((char*)&v + 8 * z, &c, 8);
    }
    return v;
  }
  __device__ __forceinline__ static Scales scales(const int* exps, int part) {
    Scales c;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int group = (32 * part + 16 * p) / S::GROUP;
      c.ke[p] = __builtin_amdgcn_readfirstlane(exps[group]);
      c.ve[p] = __builtin_amdgcn_readfirstlane(exps[S::NG + group]);
    }
    return c;
  }
};

// Every workgroup rebuilds its own tiles; 32 rows a wave.  Eight waves have two tiles in LDS and
// rebuild the next before they use the current one, one wait a tile; fewer waves, several of whose
// workgroups share a compute unit, rebuild a tile and then use it.
// 8 sequences, 4,100 tokens, 8 KV heads, d = 128: 64 rows each 50 us, 128 rows 55 (196 TFLOP/s), 256
// rows 70 (304); two prompts of 2,047 tokens, 4 KV heads, d = 64, fp32 107 us, 17 GFLOP of scores and
// sums at three products each (480 TFLOP/s), the last units' 32 tiles one after another.
template <int D, int WAVES, int PARTS>
__global__ __launch_bounds__(WAVES * kWave, 2) void rows_kernel(RowsArgs a) {
  using S = Shape<D, WAVES, PARTS>;
  constexpr int BUFS = WAVES == 8 ? 2 : 1;
  __shared__ __attribute__((aligned(16))) char s_lut[2 * S::LUT];
  __shared__ __attribute__((aligned(1024))) char s_tile[BUFS][2 * S::KIND];
  __shared__ int s_exp[BUFS][2 * S::NG];
  RowsWave<D, WAVES, PARTS> w(a);
  if (!w.start()) return;
  w.load_tables(s_lut);
  Rows<D, PARTS> r;
  r.start(a, w.u, 32 * w.wave, w.lane);
  if (w.t0 < w.t1) {
    if (a.pg.table) w.load_blocks((w.t0 * S::TILE) >> a.pg.block_log2);
    w.load_tile(w.t0);
  }
  auto work = [&](auto buf_c, uint32_t t) __attribute__((always_inline)) {
    constexpr int buf = decltype(buf_c)::value;
#pragma unroll
    for (int part = 0; part < S::TILE / 32; ++part) {
      const uint32_t tb = t * S::TILE + 32 * part;
      if (!r.busy || tb >= r.lim_hi) continue;
      const char* const kt = s_tile[buf] + 32 * part * S::ROW;
      const char* const vt = kt + S::KIND;
      v16f s = (v16f)(0.0f);
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const h8 h = w.key(kt, k);
        s = __builtin_amdgcn_mfma_f32_32x32x16_f16(h, r.q[0][k], s, 0, 0, 0);
        if constexpr (PARTS == 2) {
          s = __builtin_amdgcn_mfma_f32_32x32x16_f16(h, r.q[1][k], s, 0, 0, 0);
          s = __builtin_amdgcn_mfma_f32_32x32x16_f16(w.key(kt + S::PLANE, k), r.q[0][k], s, 0, 0, 0);
        }
      }
      const Scales c = w.scales(s_exp[buf], part);
      r.settle(s, c, tb, w.half);
      h8 p[PARTS][2];
      r.weigh(s, c, p);
      r.weights_down(c, p);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int mb = 0; mb < D / 32; ++mb) {
          const h8 h = w.value(vt + 16 * i * S::ROW, mb);
          r.acc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(h, p[0][i], r.acc[mb], 0, 0, 0);
          if constexpr (PARTS == 2) {
            const h8 g = w.value(vt + 16 * i * S::ROW + S::PLANE, mb);
            r.acc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(h, p[1][i], r.acc[mb], 0, 0, 0);
            r.acc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(g, p[0][i], r.acc[mb], 0, 0, 0);
          }
        }
    }
  };
  const std::integral_constant<int, 0> c0;
  if constexpr (BUFS == 1) {
    for (uint32_t t = w.t0; t < w.t1; ++t) {
      __syncthreads();                                   // the tables; the last tile's reads
      w.rebuild_tile(s_lut, s_tile[0], s_exp[0]);
      if (t + 1 < w.t1) w.load_tile(t + 1);
      __syncthreads();
      work(c0, t);
    }
  } else {
    const std::integral_constant<int, 1> c1;
    auto step = [&](auto buf_c, uint32_t t) __attribute__((always_inline)) {
      constexpr int other = 1 - decltype(buf_c)::value;
      if (t + 1 < w.t1) w.rebuild_tile(s_lut, s_tile[other], s_exp[other]);
      if (t + 2 < w.t1) w.load_tile(t + 2);
      work(buf_c, t);
      __syncthreads();
    };
    __syncthreads();
    if (w.t0 < w.t1) w.rebuild_tile(s_lut, s_tile[0], s_exp[0]);
    if (w.t0 + 1 < w.t1) w.load_tile(w.t0 + 1);
    __syncthreads();
    for (uint32_t t = w.t0; t < w.t1; t += 2) {          // so that the places in LDS are constants
      step(c0, t);
      if (t + 1 < w.t1) step(c1, t + 1);
    }
  }
  r.finish(a, w.u, w.unit, w.span, w.half);
}

// The tiles of a call's tokens, rebuilt once into the workspace as rows_many_kernel holds them in LDS,
// with their E's: a tile per workgroup, by way of LDS so that whole cache lines are stored.  Bound by
// the stores: 32,700 tokens, 8 heads, d = 128, 134 MB in 42 us (3.2 TB/s).
template <int D>
__global__ __launch_bounds__(kBlockThreads) void rows_tiles_kernel(RowsArgs a) {
  using S = Shape<D, 4, 1>;
  __shared__ __attribute__((aligned(16))) char s_lut[2 * S::LUT];
  __shared__ __attribute__((aligned(1024))) char s_tile[2 * S::KIND];
  __shared__ int s_exp[2 * S::NG];
  RowsWave<D, 4, 1> w(a);
  const uint32_t heads = a.B * a.H;
  w.bh = blockIdx.x % heads;
  const uint32_t tile = blockIdx.x / heads;
  w.u = unit_at(a, (a.n_rb - 1) * heads + w.bh);         // the last rows see the most
  if (tile * S::TILE >= w.u.tokens) return;
  if (a.pg.table) w.load_blocks((tile * S::TILE) >> a.pg.block_log2);
  w.load_tile(tile);
  w.load_tables(s_lut);
  __syncthreads();
  w.rebuild_tile(s_lut, s_tile, s_exp);
  __syncthreads();
  const uint64_t at = (uint64_t)w.bh * a.n_tiles + tile;
  char* const out = a.ws_tiles + at * (2 * S::KIND);
#pragma unroll
  for (uint32_t i = threadIdx.x * 16; i < 2 * S::KIND; i += kBlockThreads * 16)
    *(u32x4a*)(out + i) = *(const u32x4a*)(s_tile + i);
  if (threadIdx.x < 2 * S::NG) a.ws_exps[at * (2 * S::NG) + threadIdx.x] = s_exp[threadIdx.x];
}

// Eight waves on rebuilt tiles, three of them in LDS.  The steps of 32 tokens i overlap: the score
// products of i + 1 are issued between the exponentials of i (beside an MFMA of 32 cycles five or six
// vector instructions run, of the same wave too), and every operand is read from LDS a phase before
// its products: the keys of i + 2 before the value products of i, the values of i + 1 after them.
// In the middle of tile t the waves meet: tile t + 1 is then complete and tile t - 1 read, and its
// place is taken by t + 2, which was requested a tile before.
// 1,025 tokens behind 31,675, 8 KV heads of 4, d = 128: 540 GFLOP in 690 to 740 us (730 to 780
// TFLOP/s; the library's product of 8192 reaches 1,187).  The clock falls to 2.04 GHz under it: power
// bounds it, and neither earlier reads, 64 rows a wave nor other orders of the phases gain.
template <int D>
__global__ __launch_bounds__(8 * kWave, 2) void rows_many_kernel(RowsArgs a) {
  using S = Shape<D, 8, 1>;
  constexpr uint32_t SLOT = 2 * S::KIND, THREADS = 8 * kWave, EACH = SLOT / (THREADS * 16);
  __shared__ __attribute__((aligned(1024))) char s_tile[3 * SLOT];
  __shared__ int s_exp[3][2 * S::NG];
  RowsWave<D, 8, 1> w(a);
  if (!w.start()) return;
  Rows<D, 1> r;
  r.start(a, w.u, 32 * w.wave, w.lane);
  const uint64_t tile0 = (uint64_t)w.bh * a.n_tiles;
  u32x4a moved[EACH];
  int moved_exp = 0;
  const bool has_exp = threadIdx.x < 2 * S::NG;
  auto fetch = [&](uint32_t tile) __attribute__((always_inline)) {
    const char* const src = a.ws_tiles + (tile0 + tile) * SLOT + threadIdx.x * 16;
#pragma unroll
    for (uint32_t i = 0; i < EACH; ++i) moved[i] = *(const u32x4a*)(src + i * (THREADS * 16));
    if (has_exp) moved_exp = a.ws_exps[(tile0 + tile) * (2 * S::NG) + threadIdx.x];
  };
  auto place = [&](uint32_t slot) __attribute__((always_inline)) {
    char* const dst = s_tile + slot * SLOT + threadIdx.x * 16;
#pragma unroll
    for (uint32_t i = 0; i < EACH; ++i) *(u32x4a*)(dst + i * (THREADS * 16)) = moved[i];
    if (has_exp) s_exp[slot][threadIdx.x] = moved_exp;
  };
  if (w.t0 < w.t1) {
    fetch(w.t0);
    place(0);
  }
  if (w.t0 + 1 < w.t1) {
    fetch(w.t0 + 1);
    place(1);
  }
  if (w.t0 + 2 < w.t1) fetch(w.t0 + 2);
  __syncthreads();

  h8 kh[D / 16], p[1][2];
  auto read_keys = [&](const char* at) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < D / 16; ++k) kh[k] = w.key(at, k);
  };
  auto scores = [&]() __attribute__((always_inline)) {
    v16f x = (v16f)(0.0f);
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
      x = __builtin_amdgcn_mfma_f32_32x32x16_f16(kh[k], r.q[0][k], x, 0, 0, 0);
    return x;
  };

  read_keys(s_tile);
  v16f s = scores();
  read_keys(s_tile + 32 * S::ROW);
  uint32_t slot = 0;                                     // of tile t
  for (uint32_t t = w.t0; t < w.t1; ++t) {
    const uint32_t next = slot == 2 ? 0u : slot + 1, after = next == 2 ? 0u : next + 1;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      const char* const vt = s_tile + slot * SLOT + S::KIND + 32 * part * S::ROW;
      const Scales c = w.scales(s_exp[slot], part);
      r.settle(s, c, t * S::TILE + 32 * part, w.half);
      const v16f s1 = scores();                          // past the last tile: of what lies there, unused
      r.weigh(s, c, p);
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);             // an MFMA,
        __builtin_amdgcn_sched_group_barrier(0x2, 768 / D, 0);       // vector instructions
      }
      r.weights_down(c, p);
      s = s1;
      if (part == 0) {
        __syncthreads();
        if (t + 2 < w.t1) place(after);
        if (t + 3 < w.t1) fetch(t + 3);
      }
      h8 vh[2][D / 32];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int mb = 0; mb < D / 32; ++mb) vh[i][mb] = w.value(vt + 16 * i * S::ROW, mb);
      read_keys(s_tile + next * SLOT + 32 * part * S::ROW);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int mb = 0; mb < D / 32; ++mb)
          r.acc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vh[i][mb], p[0][i], r.acc[mb], 0, 0, 0);
    }
    slot = next;
  }
  r.finish(a, w.u, w.unit, w.span, w.half);
}

// o of a row whose rotated-domain sum lies across the lanes of the wave, elements EPL lane ...
template <int D>
__device__ __forceinline__ void store_across(const RowsArgs& a, const Unit& u, uint32_t row,
                                             float (&x)[D / kWave], int lane) {
  constexpr int EPL = D / kWave;
  fwht_across_lanes<EPL>(x, lane);
  apply_signs<EPL>(x, a.signs[(EPL * lane) / 2], lane);
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

// 16 query rows, a row on the lanes l, l + 16, l + 32 and l + 48, for calls with few rows: as Rows on
// v_mfma_f32_16x16x32_f16 (A 16 x 32, B 32 x 16: lane l gives row or column l % 16 and the k's
// 8 (l / 16) ..; register i of the result is row 4 (l / 16) + i).  The scores of 32 tokens are two
// results, tokens 4 (l / 16) + i and 16 more, which in this order are the 8 k's that the lane gives
// to the value products.
template <int D, int PARTS>
struct FewRows {
  typedef float v4f __attribute__((ext_vector_type(4)));
  uint32_t lim, lim_lo;                         // tokens that the row sees; the fewest of the 16
  h8 q[PARTS][D / 32];
  float qf, m, l;
  int vexp;
  v4f acc[D / 16];

  __device__ __forceinline__ void start(const RowsArgs& a, const Unit& u, uint32_t first, int lane) {
    const uint32_t r = min(u.rb * a.unit_rows + first + (lane & 15), u.rows - 1);
    const int64_t seen = u.pos0 + r / a.G + 1;
    lim = seen < 0 ? 0u : (uint32_t)seen;
    lim_lo = (uint32_t)__builtin_amdgcn_readlane((int)lim, 0);
    m = kNoScore;
    l = 0.0f;
    vexp = kNoExp;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) acc[i] = (v4f)(0.0f);
  }

  __device__ __forceinline__ void lower(float by) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i) acc[i] *= by;
  }

  // The weights of 32 tokens from tb on, as operand, with what the state needs before (Rows::settle).
  __device__ __forceinline__ void weigh(v4f (&s)[2], const Scales& c, uint32_t tb, int lane,
                                        h8 (&w)[PARTS]) {
    if (tb + 32 > lim_lo) {
      const uint32_t t = tb + 4 * (lane >> 4);
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[p][i] = t + 16 * p + i < lim ? s[p][i] : -INFINITY;
    }
    float f[2], top = -INFINITY;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      f[p] = fmaxf(qf * pow2i(c.ke[p]), FLT_MIN);
      top = fmaxf(top, fmaxf(fmaxf(s[p][0], s[p][1]), fmaxf(s[p][2], s[p][3])) * f[p]);
    }
    if (__builtin_amdgcn_ballot_w64(top > m + (kLazy + kBias)) != 0) {
      const float most = over_row<4>(top, [](float x, float y) { return fmaxf(x, y); });
      const float mn = most > m + (kLazy + kBias) ? most - kBias : m;
      const float down = __builtin_amdgcn_exp2f(m - mn);
      l *= down;
      lower(down);
      m = mn;
    }
    const int vmax = max(c.ve[0], c.ve[1]);
    if (vmax > vexp) {
      lower(pow2i(vexp - vmax));
      vexp = vmax;
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[p][i], f[p], -m));
        float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[p][i + 1], f[p], -m));
        h2 v = cvt_h2(w0, w1);
        if constexpr (PARTS == 1) {
          l = __builtin_amdgcn_fdot2(v, (h2){(_Float16)1.0f, (_Float16)1.0f}, l, false);
        } else {
          l += w0 + w1;
          const float down = pow2i(c.ve[p] - vexp);
          w0 *= down, w1 *= down;
          v = cvt_h2(w0, w1);
          const h2 z = cvt_h2(w0 - (float)v.x, w1 - (float)v.y);
          w[PARTS - 1][4 * p + i] = z.x, w[PARTS - 1][4 * p + i + 1] = z.y;
        }
        w[0][4 * p + i] = v.x, w[0][4 * p + i + 1] = v.y;
      }
    if constexpr (PARTS == 1)
      if (__builtin_expect(min(c.ve[0], c.ve[1]) != vexp, 0)) {
        const _Float16 d0 = (_Float16)pow2i(c.ve[0] - vexp), d1 = (_Float16)pow2i(c.ve[1] - vexp);
        w[0] *= (h8){d0, d0, d0, d0, d1, d1, d1, d1};
      }
  }
};

// A query row on 16 lanes, d / 16 elements each: four rows a wave.  As requested, and transformed.
template <int D>
struct QueryPiece {
  static constexpr int N = D / 16;
  uint32_t raw[N], signs[N / 2];

  __device__ __forceinline__ void request(const RowsArgs& a, const Unit& u, uint32_t row, int lane) {
    const uint32_t r = min(row, u.rows - 1), j = r / a.G, g = r - j * a.G;
    const uint32_t e = N * (lane & 15);
    const uint64_t at = (uint64_t)u.b * a.q_stride[0] + (uint64_t)(u.h * a.G + g) * a.q_stride[1] +
                        (uint64_t)j * a.q_stride[2] + e;
    load_words<N / 2>(a.signs + e / 2, signs);
    if (a.q_f32) load_words<N>((const uint32_t*)a.q + at, raw);
    else load_words<N / 2>((const uint32_t*)((const uint16_t*)a.q + at), raw);
  }

  // scale W D q, scaled so that the largest element of the row is in [2^7, 2^8), into x; the exponent
  // taken out.
  __device__ __forceinline__ int transform(const RowsArgs& a, int lane, float (&x)[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t v = a.q_f32 ? raw[i] : i % 2 ? raw[i / 2] & 0xFFFF0000u : raw[i / 2] << 16;
      x[i] = __uint_as_float(v ^ ((i % 2 ? signs[i / 2] : signs[i / 2] << 16) & 0x80000000u));
    }
#pragma unroll
    for (int h = 1; h < N; h <<= 1) stage_regs(x, h);
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = fwht_stage<8>(fwht_stage<4>(fwht_stage<2>(fwht_stage<1>(x[i], lane), lane), lane), lane);
      x[i] *= a.qscale;
      top = fmaxf(top, fabsf(x[i]));
    }
    top = fmaxf(top, row_ror<8>(top));
    top = fmaxf(top, row_ror<4>(top));
    top = fmaxf(top, row_ror<2>(top));
    top = fmaxf(top, row_ror<1>(top));
    const int e = min(max((int)(__float_as_uint(top) >> 23) - 127 - 7, -119), 120);
    const float down = pow2i(-e);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] *= down;
    return e;
  }
};

// Up to 16 NR query rows per KV head: four waves, each on tokens of its own in a tile of 32 of its own,
// which holds the keys and then, once the scores are there, the values.  No waits between the waves;
// their sums meet in LDS at the end, and a row is finished by one wave.
// 16 sequences, 64 blocks of 64 tokens for each of 8 KV heads of 4, d = 128: 112 MB of codes in 38 us
// (2.9 TB/s); five draft tokens (20 rows, NR = 2) behind 4,100 tokens of 8 sequences 31 us.  Of a
// wave's time 40 % are vector instructions, nearly all of them the rebuilding, and 40 % waits for LDS
// and memory with two or three waves on a SIMD; requesting the codes a whole tile ahead, q^ in LDS
// for a third wave and four waves a SIMD were each slower (their registers do not fit).
template <int D, int PARTS, int NR>
__global__ __launch_bounds__(kBlockThreads, PARTS * NR == 1 ? 3 : PARTS * NR == 4 ? 1 : 2)
void few_rows_kernel(RowsArgs a) {
  using S = Shape<D, 4, PARTS>;
  typedef float v4f __attribute__((ext_vector_type(4)));
  constexpr int TILE = 32, NG = TILE / S::GROUP, PLANE = TILE * S::ROW, PITCH = D + 4;
  constexpr int BYTES = PARTS * PLANE > 16 * PITCH * 4 ? PARTS * PLANE : (16 * PITCH * 4 + 1023) / 1024 * 1024;
  __shared__ __attribute__((aligned(16))) char s_lut[2 * S::LUT];
  __shared__ __attribute__((aligned(1024))) char s_wave[kWavesPerBlock][BYTES];
  __shared__ float2 s_ml[kWavesPerBlock][16];
  RowsWave<D, 4, PARTS> w(a);
  if (!w.start()) return;
  const uint32_t n_tiles = w.t1 - w.t0;
  const uint32_t t0 = w.t0 + span_start(n_tiles, 4, w.wave), t1 = w.t0 + span_start(n_tiles, 4, w.wave + 1);
  const int lane = w.lane, part = lane >> 4;
  RawCodes raw[NG];                                      // the codes under way: keys, values, keys ...
  auto load = [&](int kind, uint32_t t) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < NG; ++g) raw[g] = w.load_group(kind, t * TILE + g * S::GROUP);
  };
  // Everything the start needs is requested before any of it is used: a table entry a thread, 4 NR
  // query rows a wave, the first codes.
  float2 entry[2];
#pragma unroll
  for (int kind = 0; kind < 2; ++kind)
    entry[kind] = ((const float2*)a.lut[kind])[min(threadIdx.x, a.n[kind] - 1)];
  QueryPiece<D> piece[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n)
    piece[n].request(a, w.u, w.u.rb * a.unit_rows + 16 * n + 4 * w.wave + part, lane);
  if (t0 < t1) {
    if (a.pg.table) w.load_blocks((t0 * TILE) >> a.pg.block_log2);
    load(0, t0);
  }
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    char* const at = s_lut + kind * S::LUT;
    if constexpr (PARTS == 1) ((h2*)at)[threadIdx.x] = cvt_h2(entry[kind].x, entry[kind].y);
    else ((float2*)at)[threadIdx.x] = entry[kind];
  }
  // q^ of all rows by way of LDS (where the tiles will be), chunks in the places of a tile of keys
  char* const s_q = s_wave[0];
  constexpr int Q_PLANE = 16 * NR * S::ROW;
  static_assert(PARTS * Q_PLANE <= kWavesPerBlock * BYTES, "q^ fits the tiles' places");
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    constexpr int N = D / 16;
    float x[N];
    const int e = piece[n].transform(a, lane, x);
    const uint32_t i = 4 * w.wave + part, at = N * (lane & 15) * 2;          // row of the 16, byte in it
    char* const dst = s_q + (16 * n + i) * S::ROW + 16u * key_chunk<D>(at / 16, i) + at % 16;
    uint32_t hi[N / 2], lo[N / 2];
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
      const h2 h = cvt_h2(x[2 * k], x[2 * k + 1]);
      hi[k] = h2_bits(h);
      lo[k] = h2_bits(cvt_h2(x[2 * k] - (float)h.x, x[2 * k + 1] - (float)h.y));
    }
    store_words<N / 2>((uint32_t*)dst, hi);
    if constexpr (PARTS == 2) store_words<N / 2>((uint32_t*)(dst + Q_PLANE), lo);
    if ((lane & 15) == 0) s_ml[n][i].x = pow2i(e);
  }
  static_assert(NR <= kWavesPerBlock, "a factor per row");
  __syncthreads();
  FewRows<D, PARTS> r[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    r[n].start(a, w.u, 16 * n, lane);
    r[n].qf = s_ml[n][lane & 15].x;
#pragma unroll
    for (int k = 0; k < D / 32; ++k)
#pragma unroll
      for (int q = 0; q < PARTS; ++q)
        r[n].q[q][k] = read_h8(s_q + q * Q_PLANE + (16 * n + (lane & 15)) * S::ROW +
                               16u * key_chunk<D>(4 * k + part, lane & 15));
  }
  __syncthreads();                                       // q^ is read, the tables are there

  char* const tile = s_wave[w.wave];
  // (the swaps of tokens GROUP apart are the same)
  auto rebuild_kind = [&](int kind, int (&e)[2]) __attribute__((always_inline)) {
    const uint32_t t = (uint32_t)lane / S::LPV;
#pragma unroll
    for (int g = 0; g < NG; ++g)
      e[g] = rebuild<D, PARTS>(raw[g], a.n[kind], a.log_norms[kind] != 0, s_lut + kind * S::LUT,
                               tile + (t + g * S::GROUP) * S::ROW, PLANE, (uint32_t)lane % S::LPV,
                               kind == 0 ? key_chunk<D>(0, t) : value_swap<D>(t));
    if constexpr (NG == 1) e[1] = e[0];
  };
  // Chunk 4 k + part of the key of token lane % 16 lies at ka ^ 64 k, 16 tokens on 16 rows further;
  // the lane's column piece of element block mb of values at va ^ 32 mb, likewise.
  const uint32_t ka = (lane & 15) * S::ROW + 16u * key_chunk<D>(part, lane & 15);
  const uint32_t tk = 4 * part + (((uint32_t)lane >> 2) & 3u);
  const uint32_t va = tk * S::ROW + 16u * ((((uint32_t)lane >> 1) & 1u) ^ value_swap<D>(tk)) + 8u * (lane & 1);
  for (uint32_t t = t0; t < t1; ++t) {
    Scales c;
    rebuild_kind(0, c.ke);
    load(1, t);
    wave_lds_sync();
    v4f s[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) s[n][0] = s[n][1] = (v4f)(0.0f);
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int k = 0; k < D / 32; ++k) {
        const char* const at = tile + (ka ^ (64u * k)) + 16 * p * S::ROW;
        const h8 h = read_h8(at);
        h8 lo;
        if constexpr (PARTS == 2) lo = read_h8(at + PLANE);
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          s[n][p] = __builtin_amdgcn_mfma_f32_16x16x32_f16(h, r[n].q[0][k], s[n][p], 0, 0, 0);
          if constexpr (PARTS == 2) {
            s[n][p] = __builtin_amdgcn_mfma_f32_16x16x32_f16(h, r[n].q[1][k], s[n][p], 0, 0, 0);
            s[n][p] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, r[n].q[0][k], s[n][p], 0, 0, 0);
          }
        }
      }
    wave_lds_sync();                                     // the keys are read
    rebuild_kind(1, c.ve);
    if (t + 1 < t1) load(0, t + 1);
    h8 p[NR][PARTS];
#pragma unroll
    for (int n = 0; n < NR; ++n) r[n].weigh(s[n], c, t * TILE, lane, p[n]);
    wave_lds_sync();
#pragma unroll
    for (int mb = 0; mb < D / 16; ++mb) {
      h8 v[PARTS];
#pragma unroll
      for (int z = 0; z < 2; ++z)
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
          const s4 x = read_columns(tile + (va ^ (32u * mb)) + 16 * z * S::ROW + q * PLANE);
          __builtin_memcpy((char*)&v[q] + 8 * z, &x, 8);
        }
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        r[n].acc[mb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[0], p[n][0], r[n].acc[mb], 0, 0, 0);
        if constexpr (PARTS == 2) {
          r[n].acc[mb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[0], p[n][PARTS - 1], r[n].acc[mb], 0, 0, 0);
          r[n].acc[mb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[PARTS - 1], p[n][0], r[n].acc[mb], 0, 0, 0);
        }
      }
    }
    wave_lds_sync();                                     // the values are read
  }

  // the waves' sums: row lane % 16, elements 16 mb + 4 part + i
  constexpr int EPL = D / kWave;
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const bool none = r[n].m == kNoScore;
    const float up = none ? 0.0f : pow2i(r[n].vexp);
    const float sum = over_row<4>(r[n].l, [](float x, float y) { return x + y; });
#pragma unroll
    for (int mb = 0; mb < D / 16; ++mb) {
      v4f x = r[n].acc[mb] * up;
      if (none) x = (v4f)(0.0f);
      *(v4f*)((float*)tile + (lane & 15) * PITCH + 16 * mb + 4 * part) = x;
    }
    if (lane < 16) s_ml[w.wave][lane] = make_float2(r[n].m, none ? 0.0f : sum);
    __syncthreads();
    for (uint32_t i = w.wave; i < 16; i += kWavesPerBlock) {
      const uint32_t in_unit = 16 * n + i, row = w.u.rb * a.unit_rows + in_unit;
      if (row >= w.u.rows) break;
      float M = kNoScore, L = 0.0f, x[EPL];
#pragma unroll
      for (int v = 0; v < kWavesPerBlock; ++v) M = fmaxf(M, s_ml[v][i].x);
#pragma unroll
      for (int e = 0; e < EPL; ++e) x[e] = 0.0f;
#pragma unroll
      for (int v = 0; v < kWavesPerBlock; ++v) {
        const float2 ml = s_ml[v][i];
        const float f = __builtin_amdgcn_exp2f(ml.x - M);
        L = __builtin_fmaf(ml.y, f, L);
#pragma unroll
        for (int e = 0; e < EPL; ++e)
          x[e] = __builtin_fmaf(((const float*)s_wave[v])[i * PITCH + EPL * lane + e], f, x[e]);
      }
      if (a.n_split == 1) {
        const float inv = 1.0f / L;
#pragma unroll
        for (int e = 0; e < EPL; ++e) x[e] = M == kNoScore ? 0.0f : x[e] * inv;
        store_across<D>(a, w.u, row, x, lane);
        continue;
      }
      const uint64_t at = ((uint64_t)w.unit * a.n_split + w.span) * a.unit_rows + in_unit;
#pragma unroll
      for (int e = 0; e < EPL; ++e) a.ws_acc[at * D + EPL * lane + e] = x[e];
      if (lane == 0) *(float2*)(a.ws_ml + at * 2) = make_float2(M, L);
    }
    if (n + 1 < NR) __syncthreads();
  }
}

// The spans of one row, a row per wave, its elements across the lanes: M = max m, then
// o = D W (sum 2^(m - M) acc) / (sum 2^(m - M) l).  The spans' (m, l) are read 64 at a time, one
// per lane, and 8 spans' rows are requested together, the first ones before M is known.  Bound by the
// launch: 4 us.
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
  store_across<D>(a, u, row, x, lane);
}

// The same for units of 256 rows: kMergeRows rows a wave, four at a time, a row on 16 lanes, d / 16
// elements each, and 8 of its spans requested together.  A launch has so many rows then that what
// each wave finds out first is most of a row per wave: 32,000 rows of 4 spans took 18.8 us, so 11.6.
// Units of fewer rows are merged faster by a wave per row (8 heads of 80 rows of 63 spans: 8 us, so
// 16).
constexpr uint32_t kMergeRows = 8;

template <int D>
__global__ __launch_bounds__(kBlockThreads) void rows_merge_many_kernel(RowsArgs a) {
  constexpr int N = D / 16;
  constexpr uint32_t AT_ONCE = 8;
  const int lane = threadIdx.x & (kWave - 1);
  const uint32_t sub = lane & 15;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * kWavesPerBlock + threadIdx.x / kWave);
  const uint32_t waves = a.unit_rows / kMergeRows, unit = wave / waves;
  if (unit >= a.B * a.H * a.n_rb) return;
  const Unit u = unit_at(a, unit);
  const uint32_t row0 = u.rb * a.unit_rows, first = (wave - unit * waves) * kMergeRows;
  if (row0 + first >= u.rows) return;
  const uint32_t spans = row_spans((u.tokens + a.tile - 1) / a.tile, a.n_split, a.min_tiles);
  uint32_t signs[N / 2];
  load_words<N / 2>(a.signs + N * sub / 2, signs);
  for (uint32_t step = 0; step < kMergeRows && row0 + first + step < u.rows; step += 4) {
    const uint32_t row = row0 + first + step + (lane >> 4), in_unit = min(row, u.rows - 1) - row0;
    auto part = [&](uint32_t s) {
      return ((uint64_t)unit * a.n_split + min(s, spans - 1)) * a.unit_rows + in_unit;
    };
    float M = kNoScore, L = 0.0f, x[N];
    for (uint32_t s = sub; s < spans; s += 16) M = fmaxf(M, a.ws_ml[part(s) * 2]);
    M = fmaxf(M, row_ror<8>(M));
    M = fmaxf(M, row_ror<4>(M));
    M = fmaxf(M, row_ror<2>(M));
    M = fmaxf(M, row_ror<1>(M));
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = 0.0f;
    for (uint32_t s0 = 0; s0 < spans; s0 += AT_ONCE) {
      float2 ml[AT_ONCE];
      float4 y[AT_ONCE][N / 4];
#pragma unroll
      for (uint32_t k = 0; k < AT_ONCE; ++k) {
        const uint64_t at = part(s0 + k);
        ml[k] = *(const float2*)(a.ws_ml + at * 2);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) y[k][i] = *(const float4*)(a.ws_acc + at * D + N * sub + 4 * i);
      }
#pragma unroll
      for (uint32_t k = 0; k < AT_ONCE; ++k) {
        const float f = s0 + k < spans ? __builtin_amdgcn_exp2f(ml[k].x - M) : 0.0f;
        L = __builtin_fmaf(ml[k].y, f, L);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
          x[4 * i] = __builtin_fmaf(y[k][i].x, f, x[4 * i]);
          x[4 * i + 1] = __builtin_fmaf(y[k][i].y, f, x[4 * i + 1]);
          x[4 * i + 2] = __builtin_fmaf(y[k][i].z, f, x[4 * i + 2]);
          x[4 * i + 3] = __builtin_fmaf(y[k][i].w, f, x[4 * i + 3]);
        }
      }
    }
    const float inv = 1.0f / L;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = M == kNoScore ? 0.0f : x[i] * inv;
#pragma unroll
    for (int h = 1; h < N; h <<= 1) stage_regs(x, h);
    uint32_t o[N], v[N / 2];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = fwht_stage<8>(fwht_stage<4>(fwht_stage<2>(fwht_stage<1>(x[i], lane), lane), lane), lane);
      o[i] = __float_as_uint(x[i]) ^ ((i % 2 ? signs[i / 2] : signs[i / 2] << 16) & 0x80000000u);
    }
    if (row >= u.rows) continue;
    const uint32_t j = row / a.G, g = row - j * a.G;
    const uint64_t at = (uint64_t)u.b * a.o_stride[0] + (uint64_t)(u.h * a.G + g) * a.o_stride[1] +
                        (uint64_t)j * a.o_stride[2] + N * sub;
    if (a.o_f32) {
      store_words<N>((uint32_t*)a.o + at, o);
      continue;
    }
#pragma unroll
    for (int i = 0; i < N / 2; ++i)
      v[i] = bf16x2_rne(__uint_as_float(o[2 * i]), __uint_as_float(o[2 * i + 1]));
    store_words<N / 2>((uint32_t*)((uint16_t*)a.o + at), v);
  }
}

template <int D>
int launch(const RowsArgs& a, unsigned waves, bool wide, hipStream_t s) {
  const uint64_t units = (uint64_t)a.B * a.H * a.n_rb;
  const dim3 grid((unsigned)(units * a.n_split)), block(waves * kWave);
  if (a.ws_tiles) {
    hipLaunchKernelGGL((rows_tiles_kernel<D>), dim3(a.B * a.H * a.n_tiles), dim3(4 * kWave), 0, s, a);
    if (hipGetLastError() != hipSuccess) return -2;
  }
  if (a.unit_rows == 16) {
    if (wide) hipLaunchKernelGGL((few_rows_kernel<D, 2, 1>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((few_rows_kernel<D, 1, 1>), grid, block, 0, s, a);
  } else if (a.unit_rows == 32) {
    if (wide) hipLaunchKernelGGL((few_rows_kernel<D, 2, 2>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((few_rows_kernel<D, 1, 2>), grid, block, 0, s, a);
  } else if (waves == 8) {
    if (wide) hipLaunchKernelGGL((rows_kernel<D, 8, 2>), grid, block, 0, s, a);
    else if (a.ws_tiles) hipLaunchKernelGGL((rows_many_kernel<D>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((rows_kernel<D, 8, 1>), grid, block, 0, s, a);
  } else {
    if (wide) hipLaunchKernelGGL((rows_kernel<D, 4, 2>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((rows_kernel<D, 4, 1>), grid, block, 0, s, a);
  }
  if (hipGetLastError() != hipSuccess) return -2;
  if (a.n_split == 1) return 0;
  const uint64_t rows = units * a.unit_rows;                             // four waves a workgroup
  if (a.unit_rows == 256)
    hipLaunchKernelGGL((rows_merge_many_kernel<D>), dim3((unsigned)((rows / kMergeRows + 3) / 4)),
                       dim3(kBlockThreads), 0, s, a);
  else
    hipLaunchKernelGGL((rows_merge_kernel<D>), dim3((unsigned)((rows + 3) / 4)), dim3(kBlockThreads), 0, s, a);
  return hipGetLastError() == hipSuccess ? 0 : -2;
}

}  // namespace
}  // namespace tvq

int tvq_launch_rows(const tvq::RowsArgs& a, int d, unsigned waves, bool wide, void* stream) {
  if (d == 128) return tvq::launch<128>(a, waves, wide, (hipStream_t)stream);
  if (d == 64) return tvq::launch<64>(a, waves, wide, (hipStream_t)stream);
  return -1;
}
