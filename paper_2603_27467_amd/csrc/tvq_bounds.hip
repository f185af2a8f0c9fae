// tvq_bounds.hip -- bounds of the keys of every pool block, and the choice of blocks by them
// (gfx950): what an attention over part of a long cache needs.
//
// Bounds.  For a pool block, layer and KV head, lo_c and hi_c are the smallest and largest value of
// channel c over the keys written to the block, [L][n_blocks][H][2][d] bf16, fp32 keys rounded
// outward, so that lo_c <= k_c <= hi_c holds for every key as it was given.  Minimum and maximum
// have no order, so a block may be filled by any sequence of calls.
//
// Choice.  For every key of a block q . k = sum_c q_c k_c <= sum_c max(q_c lo_c, q_c hi_c): the
// score of the block, one pass over 4 d bytes in place of its keys.  With q+ = max(q, 0) and
// q- = min(q, 0) it is q+ . hi + q- . lo, and with c = lo + hi and w = hi - lo
//   2 score = q . c + |q| . w,
// two multiply-adds per channel, the absolute value an operand modifier.  It is summed in fp64 (on
// gfx950 as fast as fp32) and rounded to fp32 once: lists made from it are compared by index, and a
// fp32 sum would leave the order of near scores to its own order of addition.
#include <hip/hip_runtime.h>

#include "tvq_bounds.h"
#include "tvq_device.h"
#include "tvq_internal.h"
#include "tvq_lanes.h"

namespace tvq {
namespace {

constexpr float kBf16Max = 3.38953139e38f;       // largest finite bf16, 0x7F7F

// x rounded to bf16 toward +infinity (UP) or -infinity: the bit pattern's high half, one more where
// the cut moved the value to the wrong side.
template <bool UP>
__device__ __forceinline__ uint16_t bf16_outward(float x) {
  const uint32_t u = __float_as_uint(x);
  const bool away = (u & 0xFFFFu) != 0 && (UP ? (u >> 31) == 0 : (u >> 31) != 0);
  return (uint16_t)((u >> 16) + (away ? 1u : 0u));
}

__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// The 8 channels of a lane: running bounds inside the finite range of bf16, which a NaN leaves as
// they are.
struct Bounds8 {
  float lo[8], hi[8];
  __device__ __forceinline__ void none() {
#pragma unroll
    for (int i = 0; i < 8; ++i) lo[i] = kBf16Max, hi[i] = -kBf16Max;
  }
  __device__ __forceinline__ void add(int i, float x) {
    lo[i] = fminf(lo[i], x);
    hi[i] = fmaxf(hi[i], x);
  }
};

template <bool F32>
__device__ __forceinline__ void add_key(Bounds8& m, const void* k, uint64_t elem) {
  if constexpr (F32) {
    const float* p = (const float*)k + elem;
    const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
    const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) m.add(i, x[i]);
  } else {
    const u32x4a v = *(const u32x4a*)((const uint16_t*)k + elem);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m.add(2 * i, __uint_as_float(v[i] << 16));
      m.add(2 * i + 1, __uint_as_float(v[i] & 0xFFFF0000u));
    }
  }
}

// f over the values of the lanes that hold the same channels: a value every LPT lanes.
template <int LPT, class F>
__device__ __forceinline__ float over_tokens(float x, F f) {
  if constexpr (LPT == 8) x = f(x, row_ror<8>(x));
  uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  u = __float_as_uint(f(__uint_as_float(r[0]), __uint_as_float(r[1])));
  const auto h = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return f(__uint_as_float(h[0]), __uint_as_float(h[1]));
}

// The tokens of a call that fall into one pool block of one (layer, sequence, KV head): d / 8 lanes
// hold the channels of a token, 8 a lane (16 bytes of bf16).  SLOTS groups of such lanes share the
// tokens of a block: one where a block gets few tokens, a wave else.  The order of blocks follows the
// heads, which a projection leaves beside each other in memory and which the bounds hold beside each
// other too.
template <int D, bool F32, int SLOTS>
__global__ __launch_bounds__(kBlockThreads) void key_bounds_kernel(KeyBoundsArgs a) {
  constexpr int LPT = D / 8;                       // lanes of a token
  constexpr int GROUPS = kBlockThreads / LPT;      // of a workgroup
  constexpr int TASKS = GROUPS / SLOTS;            // blocks of a workgroup
  static_assert(SLOTS == 1 || SLOTS == kWave / LPT, "a group or a wave per block");
  const uint32_t sub = threadIdx.x % LPT, group = threadIdx.x / LPT;
  const uint32_t slot = group % SLOTS;
  const uint64_t task = (uint64_t)blockIdx.x * TASKS + group / SLOTS;
  uint32_t x = (uint32_t)task;                     // the host keeps the count below 2^31
  const uint32_t h = x % a.H;
  x /= a.H;
  const uint32_t j = x % a.n_touch;
  x /= a.n_touch;
  const uint32_t b = x % a.B, l = x / a.B;
  bool work = l < a.L;
  int32_t p0 = -1;
  if (work) p0 = a.pg.seq[b];
  work = work && p0 >= 0;
  const uint32_t lg = a.pg.block_log2;
  const uint64_t end = (uint64_t)(work ? p0 : 0) + a.T;              // positions [p0, end)
  const uint64_t i = ((uint64_t)(work ? p0 : 0) >> lg) + j;          // block of the sequence
  const uint64_t first = max((uint64_t)(work ? p0 : 0), i << lg), last = min(end, (i + 1) << lg);
  work = work && first < last && i < a.pg.max_blocks;
  uint32_t blk = 0;
  if (work) blk = (uint32_t)a.pg.table[(size_t)b * a.pg.max_blocks + i];
  work = work && blk < a.pg.n_blocks;

  Bounds8 m;
  m.none();
  if (work) {
    const uint64_t base = (uint64_t)l * a.stride_l + (uint64_t)b * a.stride_b +
                          (uint64_t)h * a.stride_h + 8 * sub;
    const uint32_t t0 = (uint32_t)(first - (uint64_t)p0), n = (uint32_t)(last - first);
#pragma unroll 4
    for (uint32_t t = slot; t < n; t += SLOTS)
      add_key<F32>(m, a.k, base + (uint64_t)(t0 + t) * a.stride_t);
  }
  if constexpr (SLOTS > 1) {
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      m.lo[c] = over_tokens<LPT>(m.lo[c], [](float x, float y) { return fminf(x, y); });
      m.hi[c] = over_tokens<LPT>(m.hi[c], [](float x, float y) { return fmaxf(x, y); });
    }
    if (slot != 0) return;
  }
  if (!work) return;
  uint16_t* out = a.bounds + ((((uint64_t)l * a.pg.n_blocks + blk) * a.H + h) * 2) * D + 8 * sub;
  uint16_t lo[8], hi[8];
  const bool goes_on = (first & ((1ull << lg) - 1)) != 0;            // row 0 is an earlier call's
  if (goes_on) {
    *(u32x4a*)lo = *(const u32x4a*)out;
    *(u32x4a*)hi = *(const u32x4a*)(out + D);
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      m.lo[c] = fminf(m.lo[c], widen(lo[c]));
      m.hi[c] = fmaxf(m.hi[c], widen(hi[c]));
    }
  }
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    lo[c] = bf16_outward<false>(fmaxf(m.lo[c], -kBf16Max));
    hi[c] = bf16_outward<true>(fminf(m.hi[c], kBf16Max));
  }
  *(u32x4a*)out = *(const u32x4a*)lo;
  *(u32x4a*)(out + D) = *(const u32x4a*)hi;
}

// Blocks of sequence b's context.
__device__ __forceinline__ uint32_t context_blocks(const SelectArgs& a, uint32_t b, uint32_t& ctx) {
  const int32_t len = a.pg.seq[b];
  ctx = len <= 0 ? 0u : min((uint32_t)len, a.max_ctx);
  return (ctx + (1u << a.pg.block_log2) - 1u) >> a.pg.block_log2;
}

// fp32 scores as unsigned integers in the same order; NaN comes first, the two zeros are one.
__device__ __forceinline__ uint32_t score_key(float s) {
  const uint32_t u = __float_as_uint(s + 0.0f);
  if (s != s) return 0u;
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// Set bits of a ballot below the lane's own.
__device__ __forceinline__ uint32_t lanes_below(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}

// A fp64 value of lane ^ B.
template <int B>
__device__ __forceinline__ double lane_xor_f64(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = __float_as_uint(lane_xor<B>(__uint_as_float((uint32_t)u)));
  const uint32_t hi = __float_as_uint(lane_xor<B>(__uint_as_float((uint32_t)(u >> 32))));
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}

constexpr uint32_t kHeadRounds = 2;

// The part of a wave in the scores: d / 8 lanes per block, 8 channels a lane, so that a wave reads
// whole rows of bounds, 4 (d = 128) or 8 blocks at a time.  Four query heads at a time: their sums
// over the lanes meet by exchanges that halve the heads a lane looks after twice, then add.
template <int D, bool F32>
struct Scorer {
  static constexpr uint32_t LPB = D / 8, BPW = kWave / LPB;            // lanes of a block, blocks of a wave
  const SelectArgs& a;
  const uint32_t row, b, h, lane, sub;
  double q[4][8];

  __device__ __forceinline__ Scorer(const SelectArgs& args, uint32_t r, uint32_t l)
      : a(args), row(r), b(r / args.H), h(r - r / args.H * args.H), lane(l), sub(l % LPB) {}

  __device__ __forceinline__ void load_bounds(uint32_t i, u32x4a& lo, u32x4a& hi) const {
    uint32_t blk = (uint32_t)a.pg.table[(size_t)b * a.pg.max_blocks + i];
    if (blk >= a.pg.n_blocks) blk = 0;
    const uint16_t* p = a.bounds + (((uint64_t)blk * a.H + h) * 2) * D + 8 * sub;
    lo = *(const u32x4a*)p;
    hi = *(const u32x4a*)(p + D);
  }

  // query heads g0 .. g0 + 3 (past the last: that one)
  __device__ __forceinline__ void load_heads(uint32_t g0) {
#pragma unroll
    for (uint32_t g = 0; g < 4; ++g) {
      const uint64_t at = ((uint64_t)row * a.G + min(g0 + g, a.G - 1)) * D + 8 * sub;
      float x[8];
      if constexpr (F32) {
        const float4 u = *(const float4*)((const float*)a.q + at);
        const float4 v = *(const float4*)((const float*)a.q + at + 4);
        x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
      } else {
        const u32x4a u = *(const u32x4a*)((const uint16_t*)a.q + at);
#pragma unroll
        for (int k = 0; k < 8; ++k)
          x[k] = __uint_as_float(k % 2 ? u[k / 2] & 0xFFFF0000u : u[k / 2] << 16);
      }
      // not finite: NaN, which both products of the sum then are
#pragma unroll
      for (int k = 0; k < 8; ++k) q[g][k] = (double)__builtin_fmaf(x[k], 0.0f, x[k]);
    }
  }

  // the largest of the four heads' scores, as key
  __device__ __forceinline__ uint32_t score(const u32x4a& lo, const u32x4a& hi) const {
    double acc[4] = {};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t wl = lo[k / 2], wh = hi[k / 2];
      const double x = (double)__uint_as_float(k % 2 ? wl & 0xFFFF0000u : wl << 16);
      const double y = (double)__uint_as_float(k % 2 ? wh & 0xFFFF0000u : wh << 16);
      const double mid = x + y, wide = y - x;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        acc[g] = __builtin_fma(q[g][k], mid, acc[g]);
        acc[g] = __builtin_fma(__builtin_fabs(q[g][k]), wide, acc[g]);
      }
    }
    // lanes with bit 0 of sub clear keep heads 0 and 1, then bit 1 picks one of the two
    const bool b0 = (lane & 1) != 0, b1 = (lane & 2) != 0;
    const double k0 = b0 ? acc[2] : acc[0], s0 = b0 ? acc[0] : acc[2];
    const double k1 = b0 ? acc[3] : acc[1], s1 = b0 ? acc[1] : acc[3];
    const double t0 = k0 + lane_xor_f64<1>(s0), t1 = k1 + lane_xor_f64<1>(s1);
    double s = (b1 ? t1 : t0) + lane_xor_f64<2>(b1 ? t0 : t1);
    s += lane_xor_f64<4>(s);
    if constexpr (LPB == 16) s += lane_xor_f64<8>(s);
    // the heads' scores lie on the lanes of a quad
    uint32_t key = score_key((float)(0.5 * s));
    key = max(key, (uint32_t)__builtin_amdgcn_mov_dpp((int)key, 0xB1, 0xF, 0xF, true));
    return max(key, (uint32_t)__builtin_amdgcn_mov_dpp((int)key, 0x4E, 0xF, 0xF, true));
  }
};

// Scores of the blocks of one (sequence, KV head) of up to 4 query heads: `rounds` times 4 or 8 blocks a
// wave, the next ones requested before the present ones are worked on.  Bound by the bounds' bytes:
// 64 sequences of 2,032 blocks, d = 128, 533 MB in 110 us (4.8 TB/s); a few blocks by the start, 3.6 us.
template <int D, bool F32>
__global__ __launch_bounds__(kBlockThreads) void block_score_kernel(SelectArgs a, uint32_t rounds) {
  constexpr uint32_t LPB = D / 8, BPW = kWave / LPB, STEP = BPW * kWavesPerBlock;
  const uint32_t per = STEP * rounds, per_row = (a.n_keys + per - 1) / per;    // blocks, workgroups of a row
  const uint32_t row = blockIdx.x / per_row;
  const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  Scorer<D, F32> s(a, row, lane);
  const uint32_t first = (blockIdx.x - row * per_row) * per + wave * BPW;
  uint32_t ctx;
  const uint32_t n = min(context_blocks(a, s.b, ctx), (blockIdx.x - row * per_row + 1) * per);
  if (first >= n) return;
  uint32_t* const keys = a.keys + (uint64_t)row * a.n_keys;
  uint32_t i = first + lane / LPB;
  u32x4a lo, hi;
  s.load_bounds(min(i, n - 1), lo, hi);
  s.load_heads(0);
  for (; i - lane / LPB < n; i += STEP) {
    const u32x4a l = lo, u = hi;
    s.load_bounds(min(i + STEP, n - 1), lo, hi);
    const uint32_t key = s.score(l, u);
    if (s.sub == 0 && i < n) keys[i] = key;
  }
}

// The same of more query heads: two rounds of blocks a wave, which stay in registers while the heads
// pass by.  (By the loop above, a pass over the blocks for every 4 heads: 16,375 blocks of 8 heads 16 us
// in place of 12.8.)
template <int D, bool F32>
__global__ __launch_bounds__(kBlockThreads) void block_score_heads_kernel(SelectArgs a) {
  constexpr uint32_t LPB = D / 8, BPW = kWave / LPB;
  constexpr uint32_t PER = BPW * kHeadRounds * kWavesPerBlock;
  const uint32_t per_row = (a.n_keys + PER - 1) / PER;
  const uint32_t row = blockIdx.x / per_row;
  const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  Scorer<D, F32> s(a, row, lane);
  const uint32_t i0 = (blockIdx.x - row * per_row) * PER + wave * BPW * kHeadRounds + lane / LPB;
  uint32_t ctx;
  const uint32_t n = context_blocks(a, s.b, ctx);
  if (i0 - lane / LPB >= n) return;
  u32x4a lo[kHeadRounds], hi[kHeadRounds];
#pragma unroll
  for (uint32_t r = 0; r < kHeadRounds; ++r) s.load_bounds(min(i0 + r * BPW, n - 1), lo[r], hi[r]);
  uint32_t best[kHeadRounds] = {};
  for (uint32_t g0 = 0; g0 < a.G; g0 += 4) {
    s.load_heads(g0);
#pragma unroll
    for (uint32_t r = 0; r < kHeadRounds; ++r) best[r] = max(best[r], s.score(lo[r], hi[r]));
  }
#pragma unroll
  for (uint32_t r = 0; r < kHeadRounds; ++r)
    if (s.sub == 0 && i0 + r * BPW < n) a.keys[(uint64_t)row * a.n_keys + i0 + r * BPW] = best[r];
}

// What a list holds without a comparison: its length, the first and last blocks.  False where that is
// all of it.
template <int THREADS>
__device__ __forceinline__ bool begin_list(const SelectArgs& a, uint32_t row, uint32_t n, uint32_t ctx) {
  const uint32_t t = threadIdx.x, keep = min(n, a.n_sel);
  int32_t* const out = a.blocks + (uint64_t)row * a.n_sel;
  // the last block of the context is always kept, and it alone may be short
  if (t == 0)
    a.lens[row] = n == 0 ? 0 : (int32_t)(((keep - 1) << a.pg.block_log2) + ctx -
                                         ((n - 1) << a.pg.block_log2));
  if (n <= a.n_sel) {
    for (uint32_t i = t; i < a.n_sel; i += THREADS) out[i] = i < n ? (int32_t)i : -1;
    return false;
  }
  const uint32_t ends = a.n_first + a.n_last;
  for (uint32_t i = t; i < ends; i += THREADS)
    out[i < a.n_first ? i : a.n_sel - ends + i] = (int32_t)(i < a.n_first ? i : n - ends + i);
  return a.n_sel > ends;
}

// The rest of the list: the largest of the keys of the blocks between the ends (keys: from n_first
// on), the lower block first among equals.  The key of the last kept block is found from its
// top down, 8 bits a step, by counting the keys of the range that is left by their next 8 bits (most
// steps end early: as soon as all of a bin are kept).  A wave looks after KPT x 64 consecutive keys
// (KPT = 0: of any number, read again in every step), 64 at a time in ascending order, so that places
// among the kept come from counted ballots.  Bound by the vector instructions of its one workgroup,
// six passes over the keys.
template <int THREADS, int KPT>
__device__ __forceinline__ void choose(const SelectArgs& a, uint32_t row, uint32_t n,
                                       const uint32_t* keys) {
  constexpr uint32_t WAVES = THREADS / kWave;
  __shared__ __attribute__((aligned(16))) uint32_t s_hist[256];
  __shared__ uint32_t s_wave[2][WAVES], s_pick[3];
  const uint32_t t = threadIdx.x, lane = t % kWave, wave = t / kWave;
  int32_t* const out = a.blocks + (uint64_t)row * a.n_sel;
  const uint32_t want = a.n_sel - a.n_first - a.n_last;              // kept between the ends
  const uint32_t m = n - a.n_first - a.n_last;                       // blocks between them
  const uint32_t per = KPT > 0 ? (uint32_t)KPT : (m + THREADS - 1) / THREADS;
  const uint32_t first = wave * per * kWave + lane;
  uint32_t k[KPT > 0 ? KPT : 1];
  if constexpr (KPT > 0) {
#pragma unroll
    for (int c = 0; c < KPT; ++c) k[c] = keys[min(first + c * kWave, m - 1)];
  }
  // f(place, key, whether there is one) for the thread's keys, by all threads
  auto each = [&](auto&& f) {
    if constexpr (KPT > 0) {
#pragma unroll
      for (int c = 0; c < KPT; ++c) f(first + c * kWave, k[c], first + c * kWave < m);
    } else {
      constexpr uint32_t AT_ONCE = 8;
      for (uint32_t c = 0, i = first; c < per; c += AT_ONCE, i += AT_ONCE * kWave) {
        uint32_t x[AT_ONCE];
#pragma unroll
        for (uint32_t j = 0; j < AT_ONCE; ++j) x[j] = keys[min(i + j * kWave, m - 1)];
#pragma unroll
        for (uint32_t j = 0; j < AT_ONCE; ++j) f(i + j * kWave, x[j], c + j < per && i + j * kWave < m);
      }
    }
  };
  uint32_t base = 0xFFFFFFFFu, top = 0;
  each([&](uint32_t, uint32_t x, bool there) {
    if (there) base = min(base, x), top = max(top, x);
  });
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    base = min(base, (uint32_t)__shfl_xor((int)base, s));
    top = max(top, (uint32_t)__shfl_xor((int)top, s));
  }
  if (lane == 0) s_wave[0][wave] = base, s_wave[1][wave] = top;
  __syncthreads();
  for (uint32_t w = 0; w < WAVES; ++w) base = min(base, s_wave[0][w]), top = max(top, s_wave[1][w]);
  // the range [base, base + span] that holds the key, inside [.., top], so that one comparison tells
  uint32_t span = top - base, need = want;         // need: kept among the keys of the range
  uint32_t left = span == 0 ? 0u : 32u - (uint32_t)__builtin_clz(span);             // bits to find
  while (left > 0) {
    const uint32_t sh = left - min(left, 8u);
    __syncthreads();                               // s_wave and s_pick are read
    for (uint32_t i = t; i < 256; i += THREADS) s_hist[i] = 0;
    __syncthreads();
    each([&](uint32_t, uint32_t x, bool there) {
      if (there && x - base <= span) atomicAdd(&s_hist[(x - base) >> sh], 1u);
    });
    __syncthreads();
    if (wave == 0) {                               // lane l: bins 255 - 4 l down to 252 - 4 l
      const uint4 v = *(const uint4*)(s_hist + 252 - 4 * lane);
      const uint32_t sum = v.x + v.y + v.z + v.w;
      const uint32_t end = wave_scan(sum);
      uint32_t before = end - sum;
      if (before < need && end >= need) {
        const uint32_t c[4] = {v.w, v.z, v.y, v.x};
        uint32_t i = 0;
        while (before + c[i] < need) before += c[i++];
        s_pick[0] = 255 - 4 * lane - i, s_pick[1] = before, s_pick[2] = c[i];
      }
    }
    __syncthreads();
    base += s_pick[0] << sh;
    span = min((1u << sh) - 1u, top - base);
    need -= s_pick[1];
    left = sh;
    if (s_pick[2] == need) break;                  // all of the bin are kept
  }
  // kept: the keys above the range, and the first `need` in it
  auto above = [&](uint32_t x, bool there) { return there && x > base + span; };
  auto equal = [&](uint32_t x, bool there) { return there && x - base <= span; };
  uint32_t na = 0, ne = 0;
  each([&](uint32_t, uint32_t x, bool there) {
    na += __popcll(__builtin_amdgcn_ballot_w64(above(x, there)));
    ne += __popcll(__builtin_amdgcn_ballot_w64(equal(x, there)));
  });
  __syncthreads();
  if (lane == 0) s_wave[0][wave] = na, s_wave[1][wave] = ne;
  __syncthreads();
  na = ne = 0;
  for (uint32_t w = 0; w < wave; ++w) na += s_wave[0][w], ne += s_wave[1][w];
  each([&](uint32_t i, uint32_t x, bool there) {
    const bool is_above = above(x, there), is_equal = equal(x, there);
    const uint64_t ma = __builtin_amdgcn_ballot_w64(is_above), me = __builtin_amdgcn_ballot_w64(is_equal);
    const uint32_t ea = na + lanes_below(ma), ee = ne + lanes_below(me);
    if (is_above || (is_equal && ee < need)) out[a.n_first + ea + min(ee, need)] = (int32_t)(a.n_first + i);
    na += __popcll(ma);
    ne += __popcll(me);
  });
}

template <int THREADS, int KPT>
__global__ __launch_bounds__(THREADS) void block_select_kernel(SelectArgs a) {
  const uint32_t row = blockIdx.x;
  uint32_t ctx;
  const uint32_t n = context_blocks(a, row / a.H, ctx);
  if (begin_list<THREADS>(a, row, n, ctx))
    choose<THREADS, KPT>(a, row, n, a.keys + (uint64_t)row * a.n_keys + a.n_first);
}

// Scores and choice of a short list in one workgroup, the keys in LDS: a launch less.
constexpr uint32_t kShortThreads = 512;

template <int D, bool F32>
__global__ __launch_bounds__(kShortThreads) void block_short_kernel(SelectArgs a) {
  constexpr uint32_t LPB = D / 8, BPW = kWave / LPB, STEP = BPW * kShortThreads / kWave;
  __shared__ uint32_t s_keys[kShortThreads];
  const uint32_t row = blockIdx.x, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  Scorer<D, F32> s(a, row, lane);
  uint32_t ctx;
  const uint32_t n = context_blocks(a, s.b, ctx);
  if (!begin_list<kShortThreads>(a, row, n, ctx)) return;
  for (uint32_t g0 = 0; g0 < a.G; g0 += 4) {
    uint32_t i = wave * BPW + lane / LPB;
    u32x4a lo, hi;
    s.load_bounds(min(i, n - 1), lo, hi);
    s.load_heads(g0);
    for (; i - lane / LPB < n; i += STEP) {
      const u32x4a l = lo, u = hi;
      s.load_bounds(min(i + STEP, n - 1), lo, hi);
      const uint32_t key = s.score(l, u);
      if (s.sub == 0 && i < n) s_keys[i] = g0 == 0 ? key : max(key, s_keys[i]);
    }
  }
  __syncthreads();
  choose<kShortThreads, 1>(a, row, n, s_keys + a.n_first);
}

// Tokens of a block up to which a group takes it.  32 layers, 16 sequences, 8 heads of d = 128, us by
// a group and by a wave: 1 token 4.8 and 6.4, 8 tokens 5.2 and 11.5, 16 tokens 7.2 and 11.2; 4,099
// tokens of one sequence 58 and 53, of which the copy rate of the device (5.15 TB/s) would need 54.
constexpr uint32_t kGroupTokens = 16;

template <int D, bool F32>
void launch_bounds(const KeyBoundsArgs& a, hipStream_t s) {
  constexpr uint32_t GROUPS = kBlockThreads / (D / 8);
  const uint64_t tasks = (uint64_t)a.L * a.B * a.n_touch * a.H;
  const uint64_t per = (uint64_t)min(a.T, 1u << a.pg.block_log2);    // tokens of a block at most
  if (per > kGroupTokens)
    hipLaunchKernelGGL((key_bounds_kernel<D, F32, kWave / (D / 8)>),
                       dim3((unsigned)((tasks + kWavesPerBlock - 1) / kWavesPerBlock)),
                       dim3(kBlockThreads), 0, s, a);
  else
    hipLaunchKernelGGL((key_bounds_kernel<D, F32, 1>), dim3((unsigned)((tasks + GROUPS - 1) / GROUPS)),
                       dim3(kBlockThreads), 0, s, a);
}

// Rounds of a wave: the device full with 4 workgroups a compute unit, 16 at most.  us a call, 4 / 8
// workgroups: 513 blocks of 16 sequences 13.6 / 14.7, 2,032 blocks 31.7 / 29.3, of 64 sequences 120 / 119.
constexpr uint32_t kScorePlaces = 4, kScoreRounds = 16;

template <int D, bool F32>
void launch_scores(const SelectArgs& a, hipStream_t s) {
  constexpr uint32_t STEP = kBlockThreads / (D / 8);
  if (a.G > 4) {
    const uint32_t per_row = (a.n_keys + STEP * kHeadRounds - 1) / (STEP * kHeadRounds);
    hipLaunchKernelGGL((block_score_heads_kernel<D, F32>), dim3(per_row * a.B * a.H), dim3(kBlockThreads), 0, s, a);
    return;
  }
  const uint64_t steps = (uint64_t)a.B * a.H * ((a.n_keys + STEP - 1) / STEP);
  const uint32_t rounds = (uint32_t)min(max(steps / (kScorePlaces * a.cus), (uint64_t)1), (uint64_t)kScoreRounds);
  const uint32_t per_row = (a.n_keys + STEP * rounds - 1) / (STEP * rounds);
  hipLaunchKernelGGL((block_score_kernel<D, F32>), dim3(per_row * a.B * a.H), dim3(kBlockThreads), 0, s, a,
                     rounds);
}

// Lists up to which one workgroup scores and chooses; the second, where there are as many lists as
// compute units.  us on the device, by one launch and by two: one sequence (8 lists) of 129 blocks 7.4
// and 7.1 (a call of the host 9 and 13), of 250 blocks 9.6 and 7.1; 64 sequences of 129 blocks 10.7 and
// 14.7, of 511 blocks 24 and 41.
constexpr uint32_t kShortKeys = 160, kManyShortKeys = 512;

template <int D, bool F32>
void launch_short(const SelectArgs& a, hipStream_t s) {
  static_assert(kManyShortKeys <= kShortThreads, "a key a thread");
  hipLaunchKernelGGL((block_short_kernel<D, F32>), dim3(a.B * a.H), dim3(kShortThreads), 0, s, a);
}

// The keys of a list stay in registers where 1024 threads can hold them, of the fewest that do: a list
// of 129 keys takes 3.8 us on 256 threads of 4, 4.9 on 1024 of 4 and 7.7 on 1024 of 16; 3,125 keys 5.4
// on 1024 of 4, 8.7 on 1024 of 16; 16,375 keys 9.5 on 1024 of 16 and 13.2 read again in every step.
void launch_select(const SelectArgs& a, hipStream_t s) {
  const dim3 grid(a.B * a.H);
  if (a.n_keys <= 256 * 4)
    hipLaunchKernelGGL((block_select_kernel<256, 4>), grid, dim3(256), 0, s, a);
  else if (a.n_keys <= 1024 * 4)
    hipLaunchKernelGGL((block_select_kernel<1024, 4>), grid, dim3(1024), 0, s, a);
  else if (a.n_keys <= 1024 * 16)
    hipLaunchKernelGGL((block_select_kernel<1024, 16>), grid, dim3(1024), 0, s, a);
  else
    hipLaunchKernelGGL((block_select_kernel<1024, 0>), grid, dim3(1024), 0, s, a);
}

}  // namespace
}  // namespace tvq

int tvq_launch_key_bounds(const tvq::KeyBoundsArgs& a, int d, bool f32, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (d == 128) f32 ? tvq::launch_bounds<128, true>(a, s) : tvq::launch_bounds<128, false>(a, s);
  else if (d == 64) f32 ? tvq::launch_bounds<64, true>(a, s) : tvq::launch_bounds<64, false>(a, s);
  else return -1;
  return hipGetLastError() == hipSuccess ? 0 : -2;
}

int tvq_launch_select(const tvq::SelectArgs& a, int d, bool f32, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  const bool apart = a.n_keys > (a.B * a.H >= a.cus ? tvq::kManyShortKeys : tvq::kShortKeys);
  if (d == 128 && apart) f32 ? tvq::launch_scores<128, true>(a, s) : tvq::launch_scores<128, false>(a, s);
  else if (d == 64 && apart) f32 ? tvq::launch_scores<64, true>(a, s) : tvq::launch_scores<64, false>(a, s);
  else if (d == 128) f32 ? tvq::launch_short<128, true>(a, s) : tvq::launch_short<128, false>(a, s);
  else if (d == 64) f32 ? tvq::launch_short<64, true>(a, s) : tvq::launch_short<64, false>(a, s);
  else return -1;
  if (!apart) return hipGetLastError() == hipSuccess ? 0 : -2;
  if (hipGetLastError() != hipSuccess) return -2;
  tvq::launch_select(a, s);
  return hipGetLastError() == hipSuccess ? 0 : -2;
}
