// tvq_lanes.h -- a vector spread over the lanes of a wave: exchanges, reductions and the
// Walsh-Hadamard butterfly of the attention kernels (gfx950).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tvq_device.h"

namespace tvq {

// Rotation inside each row of 16 lanes (DPP row_ror: a register operation, no LDS traffic).
template <int N>
__device__ __forceinline__ uint32_t row_ror(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x120 + N, 0xF, 0xF, true);
}
template <int N>
__device__ __forceinline__ float row_ror(float v) {
  return __uint_as_float(row_ror<N>(__float_as_uint(v)));
}

// The value of lane ^ B, by register moves (B = 4: the mirror of each half row is lane ^ 7).
template <int B>
__device__ __forceinline__ float lane_xor(float v) {
  static_assert(B == 1 || B == 2 || B == 4 || B == 8, "inside a row of 16 lanes");
  if constexpr (B == 1) return quad_perm<0xB1>(v);
  else if constexpr (B == 2) return quad_perm<0x4E>(v);
  else if constexpr (B == 4) return quad_perm<0x1B>(quad_perm<0x141>(v));
  else return row_ror<8>(v);
}

// Maximum and sum over the wave, uniform: the rows by rotations, then their four values.
__device__ __forceinline__ float lane_value(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, row_ror<8>(v));
  v = fmaxf(v, row_ror<4>(v));
  v = fmaxf(v, row_ror<2>(v));
  v = fmaxf(v, row_ror<1>(v));
  return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)),
               fmaxf(lane_value(v, 32), lane_value(v, 48)));
}
__device__ __forceinline__ float wave_sum(float v) {
  v += row_ror<8>(v);
  v += row_ror<4>(v);
  v += row_ror<2>(v);
  v += row_ror<1>(v);
  return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}

// Inclusive prefix sum over the wave's lanes (row shifts inside the rows of 16, then the last
// lane of each row or half broadcast to the next; lanes without a source add 0).
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false);
  return v;
}

// The Sylvester butterfly of a vector held EPL = D / 64 consecutive elements per lane, stages in
// ascending order: element bit 0 inside the lane at d = 128, then the stages over the lane's
// bits, where the lane with the bit clear keeps a + b and its partner a - b.
// Bits 4 and 5: the swap of odd rows (upper half) of one copy with even rows (lower half) of the
// other leaves a in one register and b in the other on both lanes of a pair.
template <int B>
__device__ __forceinline__ float fwht_stage(float x, int lane) {
  const float sgn = (lane & B) ? -1.0f : 1.0f;
  if constexpr (B < 16) {
    return __builtin_fmaf(x, sgn, lane_xor<B>(x));
  } else {
    const uint32_t u = __float_as_uint(x);
    const auto ab = [u] {
      if constexpr (B == 16) return __builtin_amdgcn_permlane16_swap(u, u, false, false);
      else return __builtin_amdgcn_permlane32_swap(u, u, false, false);
    }();
    return __builtin_fmaf(__uint_as_float(ab[1]), sgn, __uint_as_float(ab[0]));
  }
}

template <int EPL>
__device__ __forceinline__ void fwht_across_lanes(float (&x)[EPL], int lane) {
  if constexpr (EPL == 2) {
    const float p = x[0], q = x[1];
    x[0] = p + q;
    x[1] = p - q;
  }
#pragma unroll
  for (int e = 0; e < EPL; ++e) {
    float v = fwht_stage<1>(x[e], lane);
    v = fwht_stage<2>(v, lane);
    v = fwht_stage<4>(v, lane);
    v = fwht_stage<8>(v, lane);
    v = fwht_stage<16>(v, lane);
    x[e] = fwht_stage<32>(v, lane);
  }
}

// The sign bits of a lane's EPL elements from their word of the layer's masks (bit 15: even
// elements, bit 31: odd ones).
template <int EPL>
__device__ __forceinline__ void apply_signs(float (&x)[EPL], uint32_t smw, int lane) {
  const uint32_t lo = (smw << 16) & 0x80000000u, hi = smw & 0x80000000u;
  if constexpr (EPL == 2) {
    x[0] = __uint_as_float(__float_as_uint(x[0]) ^ lo);
    x[1] = __uint_as_float(__float_as_uint(x[1]) ^ hi);
  } else {
    x[0] = __uint_as_float(__float_as_uint(x[0]) ^ ((lane & 1) ? hi : lo));
  }
}

}  // namespace tvq
