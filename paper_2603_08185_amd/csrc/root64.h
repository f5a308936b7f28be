// Sums of squares and their roots in 64 bits: what the norms share (rmsnorm.hip, kv_append.hip).  Squares of 16-bit numbers are exact there and sums of
// them as good as, whatever their order.
#pragma once

#include <float.h>

#include "serq_device.h"

namespace serq {

__device__ __forceinline__ double join64(uint32_t lo, uint32_t hi) { return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo); }
template <int CTRL>
__device__ __forceinline__ double dpp_add(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const int lo = (int)(uint32_t)b, hi = (int)(uint32_t)(b >> 32);
  return v + join64((uint32_t)__builtin_amdgcn_update_dpp(lo, lo, CTRL, 0xf, 0xf, false),
                     (uint32_t)__builtin_amdgcn_update_dpp(hi, hi, CTRL, 0xf, 0xf, false));
}
// the sum over the lanes of a wave, in all of them (wave_reduce for 64 bits)
__device__ __forceinline__ double wave_sum(double v) {
  v = dpp_add<kDpp1>(v);
  v = dpp_add<kDpp2>(v);
  v = dpp_add<kDppMirror8>(v);
  v = dpp_add<kDppMirror16>(v);
  uint64_t b = __builtin_bit_cast(uint64_t, v);
  auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)b, (uint32_t)b, false, false);
  auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(b >> 32), (uint32_t)(b >> 32), false, false);
  v = join64(lo[0], hi[0]) + join64(lo[1], hi[1]);
  b = __builtin_bit_cast(uint64_t, v);
  lo = __builtin_amdgcn_permlane32_swap((uint32_t)b, (uint32_t)b, false, false);
  hi = __builtin_amdgcn_permlane32_swap((uint32_t)(b >> 32), (uint32_t)(b >> 32), false, false);
  return join64(lo[0], hi[0]) + join64(lo[1], hi[1]);
}

// 1 / sqrt(a) to within some 2^-50 (the instruction's own is good to about half of 64 bits' digits, a step of Newton's iteration doubles
// them, the second is for its rounding), rounded to fp32 and kept finite; 0 for 0 and for infinity (whose first step would multiply infinity by 0), NaN for NaN
__device__ __forceinline__ float inv_root(double a) {
  if (!(a > 0.0 && a < __builtin_inf())) return a != a ? __builtin_nanf("") : 0.0f;
  double y = __builtin_amdgcn_rsq(a);
#pragma unroll
  for (int i = 0; i < 2; ++i) y = __builtin_fma(0.5 * y, __builtin_fma(-a * y, y, 1.0), y);
  return fminf((float)y, FLT_MAX);
}

}  // namespace serq
