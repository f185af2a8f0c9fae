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

// The tokens of a call that fall into one pool block of one (layer, sequence, KV head): d / 8 lanes
// hold the channels of a token, 8 a lane (16 bytes of bf16).  SLOTS groups of such lanes share the
// tokens of a block and are summed up in LDS; the order of blocks follows the heads, which a
// projection leaves beside each other in memory and which the bounds hold beside each other too.
template <int D, bool F32, int SLOTS>
__global__ __launch_bounds__(kBlockThreads) void key_bounds_kernel(KeyBoundsArgs a) {
  constexpr int LPT = D / 8;                       // lanes of a token
  constexpr int GROUPS = kBlockThreads / LPT;      // of a workgroup
  constexpr int TASKS = GROUPS / SLOTS;            // blocks of a workgroup
  static_assert(SLOTS == 1 || SLOTS == GROUPS, "a group or a workgroup per block");
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
    __shared__ float s_lo[SLOTS][D + 4], s_hi[SLOTS][D + 4];
#pragma unroll
    for (int c = 0; c < 8; ++c) s_lo[slot][8 * sub + c] = m.lo[c], s_hi[slot][8 * sub + c] = m.hi[c];
    __syncthreads();
    if (slot != 0) return;
    for (int s = 1; s < SLOTS; ++s)
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        m.lo[c] = fminf(m.lo[c], s_lo[s][8 * sub + c]);
        m.hi[c] = fmaxf(m.hi[c], s_hi[s][8 * sub + c]);
      }
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

// Scores of the blocks of one (sequence, KV head), a block per lane.
template <int D, bool F32>
__global__ __launch_bounds__(kBlockThreads) void block_score_kernel(SelectArgs a) {
  constexpr uint32_t PASS = 4;                     // query heads at a time
  extern __shared__ float s_q[];                   // [G][D]
  const uint32_t per_row = (a.n_keys + kBlockThreads - 1) / kBlockThreads;
  const uint32_t row = blockIdx.x / per_row, i0 = (blockIdx.x - row * per_row) * kBlockThreads;
  const uint32_t b = row / a.H, h = row - b * a.H;
  uint32_t ctx;
  const uint32_t n = context_blocks(a, b, ctx);
  if (i0 >= n) return;
  const uint64_t q0 = (uint64_t)row * a.G * D;
  for (uint32_t e = threadIdx.x; e < a.G * D; e += kBlockThreads) {
    const float v = F32 ? ((const float*)a.q)[q0 + e] : widen(((const uint16_t*)a.q)[q0 + e]);
    s_q[e] = __builtin_isfinite(v) ? v : NAN;          // both products of the sum are then NaN
  }
  __syncthreads();
  const uint32_t i = i0 + threadIdx.x;
  if (i >= n) return;
  uint32_t blk = (uint32_t)a.pg.table[(size_t)b * a.pg.max_blocks + i];
  if (blk >= a.pg.n_blocks) blk = 0;
  const uint16_t* lo = a.bounds + (((uint64_t)blk * a.H + h) * 2) * D;
  uint32_t best = 0;
  for (uint32_t g0 = 0; g0 < a.G; g0 += PASS) {
    double acc[PASS] = {};
    for (int c = 0; c < D; c += 8) {
      const u32x4a vl = *(const u32x4a*)(lo + c), vh = *(const u32x4a*)(lo + D + c);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t wl = vl[k / 2], wh = vh[k / 2];
        const double x = (double)__uint_as_float(k % 2 ? wl & 0xFFFF0000u : wl << 16);
        const double y = (double)__uint_as_float(k % 2 ? wh & 0xFFFF0000u : wh << 16);
        const double mid = x + y, wide = y - x;
#pragma unroll
        for (uint32_t g = 0; g < PASS; ++g) {
          const double q = (double)s_q[min(g0 + g, a.G - 1) * D + c + k];
          acc[g] = __builtin_fma(q, mid, acc[g]);
          acc[g] = __builtin_fma(__builtin_fabs(q), wide, acc[g]);
        }
      }
    }
#pragma unroll
    for (uint32_t g = 0; g < PASS; ++g) best = max(best, score_key((float)(0.5 * acc[g])));
  }
  a.keys[(uint64_t)row * a.n_keys + i] = best;
}

// Exclusive prefix count of `on` over the workgroup, and the total.
__device__ __forceinline__ uint32_t count_before(bool on, uint32_t* s_wave, uint32_t& total) {
  const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const uint64_t m = __builtin_amdgcn_ballot_w64(on);
  if (lane == 0) s_wave[wave] = (uint32_t)__builtin_popcountll(m);
  __syncthreads();
  uint32_t before = __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32),
                                              __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
  total = 0;
  for (uint32_t w = 0; w < kWavesPerBlock; ++w) {
    before += w < wave ? s_wave[w] : 0u;
    total += s_wave[w];
  }
  __syncthreads();
  return before;
}

// The n_sel largest keys of one (sequence, KV head), the lower block first among equals: the
// smallest kept key by its bytes from the top (histograms of the keys that share the bytes found so
// far), then one pass in block order that writes the kept blocks.
__global__ __launch_bounds__(kBlockThreads) void block_select_kernel(SelectArgs a) {
  __shared__ uint32_t s_hist[256], s_wave[kWavesPerBlock], s_pick[2];
  const uint32_t row = blockIdx.x, b = row / a.H, t = threadIdx.x;
  uint32_t ctx;
  const uint32_t n = context_blocks(a, b, ctx);
  const uint32_t keep = min(n, a.n_sel);
  const uint32_t* const keys = a.keys + (uint64_t)row * a.n_keys;
  int32_t* const out = a.blocks + (uint64_t)row * a.n_sel;
  auto key = [&](uint32_t i) {
    return i < a.n_first || i + a.n_last >= n ? 0xFFFFFFFFu : keys[i];
  };
  uint32_t floor_key = 0, equal = n;               // kept: key > floor_key, or the first `equal` of it
  if (n > a.n_sel) {
    uint32_t want = a.n_sel;                       // rank of the smallest kept key among the rest
    for (int shift = 24; shift >= 0; shift -= 8) {
      s_hist[t] = 0;
      __syncthreads();
      const uint32_t done = shift == 24 ? 0u : 0xFFFFFFFFu << (shift + 8);
      for (uint32_t i = t; i < n; i += kBlockThreads) {
        const uint32_t k = key(i);
        if ((k & done) == (floor_key & done)) atomicAdd(&s_hist[(k >> shift) & 255u], 1u);
      }
      __syncthreads();
      uint32_t above = 0;
      for (uint32_t v = t + 1; v < 256; ++v) above += s_hist[v];
      if (above < want && above + s_hist[t] >= want) s_pick[0] = t, s_pick[1] = above;
      __syncthreads();
      floor_key |= s_pick[0] << shift;
      want -= s_pick[1];
      __syncthreads();
    }
    equal = want;
  }
  uint32_t kept = 0, same = 0;
  for (uint32_t i0 = 0; i0 < n; i0 += kBlockThreads) {
    const uint32_t i = i0 + t;
    const uint32_t k = i < n ? key(i) : 0u;
    uint32_t more;
    const bool eq = i < n && k == floor_key;
    const uint32_t rank = same + count_before(eq, s_wave, more);
    same += more;
    const bool on = i < n && (k > floor_key || (eq && rank < equal));
    const uint32_t at = kept + count_before(on, s_wave, more);
    kept += more;
    if (on && at < keep) out[at] = (int32_t)i;
  }
  for (uint32_t i = keep + t; i < a.n_sel; i += kBlockThreads) out[i] = -1;
  // the last block of the context is always kept, and it alone may be short
  if (t == 0)
    a.lens[row] = n == 0 ? 0 : (int32_t)(((keep - 1) << a.pg.block_log2) + ctx -
                                         ((n - 1) << a.pg.block_log2));
}

template <int D, bool F32>
void launch_bounds(const KeyBoundsArgs& a, hipStream_t s) {
  constexpr uint32_t GROUPS = kBlockThreads / (D / 8);
  const uint64_t tasks = (uint64_t)a.L * a.B * a.n_touch * a.H;
  const uint64_t per = (uint64_t)min(a.T, 1u << a.pg.block_log2);    // tokens of a block at most
  if (per > 4)
    hipLaunchKernelGGL((key_bounds_kernel<D, F32, GROUPS>), dim3((unsigned)tasks),
                       dim3(kBlockThreads), 0, s, a);
  else
    hipLaunchKernelGGL((key_bounds_kernel<D, F32, 1>), dim3((unsigned)((tasks + GROUPS - 1) / GROUPS)),
                       dim3(kBlockThreads), 0, s, a);
}

template <int D, bool F32>
void launch_scores(const SelectArgs& a, hipStream_t s) {
  const uint32_t per_row = (a.n_keys + kBlockThreads - 1) / kBlockThreads;
  hipLaunchKernelGGL((block_score_kernel<D, F32>), dim3(per_row * a.B * a.H), dim3(kBlockThreads), a.G * D * 4, s, a);
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
  if (d == 128) f32 ? tvq::launch_scores<128, true>(a, s) : tvq::launch_scores<128, false>(a, s);
  else if (d == 64) f32 ? tvq::launch_scores<64, true>(a, s) : tvq::launch_scores<64, false>(a, s);
  else return -1;
  if (hipGetLastError() != hipSuccess) return -2;
  hipLaunchKernelGGL(tvq::block_select_kernel, dim3(a.B * a.H), dim3(tvq::kBlockThreads), 0, s, a);
  return hipGetLastError() == hipSuccess ? 0 : -2;
}
