// From values to codes: what the quantisers of a token's row share, whatever makes the row (quantize_act.hip, grouped.hip, mx.hip, rmsnorm.hip).
#pragma once

#include "serq_device.h"

namespace serq {

// ---- symmetric integer codes --------------------------------------------------------------------------
__device__ __forceinline__ float absmax8(const float v[8], float m) {
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));
  return m;
}

// Codes of 8 flattened values, bit-identical to clip(rne(v / sc)) in IEEE fp32, at the price of
// a multiplication per value.  t = v * rcp(sc) is within 2^-22 |t| of the correctly rounded
// quotient (one ulp from the reciprocal, half an ulp from the product, half an ulp from the
// quotient's own rounding), so the two round to the same integer unless t lies within that distance
// of a half-integer; only then (the ties of synthetic inputs, and about one piece in a hundred
// otherwise) are the divisions carried out.  The margin used is 1.25 * 2^-22 max(|t|, 1) over the piece.
// A token whose scale is tiny (below 1e-30, a wave-uniform test: the reciprocal of a subnormal scale is
// not finite, and neither estimate above holds near the bottom of the exponent range) always takes the
// divisions.
// (The bookkeeping of this check -- four VALU operations per value -- costs about a tenth of the
// kernel's time; the fallback itself is too rare to show.)
// Clamping before rounding equals rounding before clamping for integer bounds, and adding
// 1.5 * 2^23 rounds to nearest-even and leaves the two's-complement code in the low mantissa bits.
template <int ABITS>
__device__ __forceinline__ void codes8(const float v[8], float sc, float rsc, uint32_t u[8]) {
  constexpr float q = (float)((1 << (ABITS - 1)) - 1);
  constexpr float kMagic = 12582912.0f;
  float maxd = 0.0f, maxt = 1.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float tc = __builtin_amdgcn_fmed3f(v[i] * rsc, -q, q);
    const float uf = tc + kMagic;
    u[i] = __float_as_uint(uf);
    maxd = fmaxf(maxd, fabsf(tc - (uf - kMagic)));
    maxt = fmaxf(maxt, fabsf(tc));
  }
  if (sc < 1e-30f || 0.5f - maxd < 2.98023223876953125e-07f * maxt) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float t = rintf(v[i] / sc);          // IEEE division, then round-half-to-even
      t = fminf(fmaxf(t, -q), q);
      u[i] = __float_as_uint(t + kMagic);
    }
  }
}

template <int ABITS>
__device__ __forceinline__ void quant_store8(const float v[8], float sc, void* xq_row, int chunk) {
  const float rsc = __builtin_amdgcn_rcpf(sc);
  uint32_t u[8];
  codes8<ABITS>(v, sc, rsc, u);
  if constexpr (ABITS == 8) {
    // low bytes of u[0..3] and u[4..7]
    const uint32_t d0 = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u) | __builtin_amdgcn_perm(u[3], u[2], 0x04000c0cu);
    const uint32_t d1 = __builtin_amdgcn_perm(u[5], u[4], 0x0c0c0400u) | __builtin_amdgcn_perm(u[7], u[6], 0x04000c0cu);
    ((uint2*)xq_row)[chunk] = make_uint2(d0, d1);
  } else {
    // byte j = code j in the low nibble, code 4+j in the high nibble
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (u[4 + j] << 4) | (u[j] & 0xfu);
    ((uint32_t*)xq_row)[chunk] =
        __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u) | __builtin_amdgcn_perm(w[3], w[2], 0x04000c0cu);
  }
}

// ---- asymmetric integer codes -------------------------------------------------------------------------
// codes of 8 values: rne(v / sc) + z, clamped to [0, top], re-centred.  t = v * rcp(sc) decides unless it
// lies within 1.25 * 2^-22 max(|t|, 1) of a half-integer (then, and for tiny scales, the divisions are done).
template <int ABITS>
__device__ __forceinline__ void asym_codes8(const float v[8], float sc, float rsc, float z, int c[8]) {
  constexpr float top = (float)((1 << ABITS) - 1);
  constexpr float kMagic = 12582912.0f;
  float r[8], maxd = 0.0f, maxt = 1.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = v[i] * rsc;
    r[i] = (t + kMagic) - kMagic;                       // round-half-to-even for |t| < 2^22
    maxd = fmaxf(maxd, fabsf(t - r[i]));
    maxt = fmaxf(maxt, fabsf(t));
  }
  if (sc < 1e-30f || !(maxt < 4194304.0f) || 0.5f - maxd < 2.98023223876953125e-07f * maxt) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = rintf(v[i] / sc);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = (int)fminf(fmaxf(r[i] + z, 0.0f), top) - (1 << (ABITS - 1));
}

template <int ABITS>
__device__ __forceinline__ void store_codes8(const int c[8], void* xq_row, int chunk) {
  if constexpr (ABITS == 8) {
    const uint32_t d0 = (c[0] & 0xff) | ((c[1] & 0xff) << 8) | ((c[2] & 0xff) << 16) | ((uint32_t)(c[3] & 0xff) << 24);
    const uint32_t d1 = (c[4] & 0xff) | ((c[5] & 0xff) << 8) | ((c[6] & 0xff) << 16) | ((uint32_t)(c[7] & 0xff) << 24);
    ((uint2*)xq_row)[chunk] = make_uint2(d0, d1);
  } else {
    uint32_t o = 0;                                     // byte j: code j (low nibble), code 4+j (high nibble)
#pragma unroll
    for (int j = 0; j < 4; ++j) o |= ((uint32_t)(c[j] & 0xf) | ((uint32_t)(c[4 + j] & 0xf) << 4)) << (8 * j);
    ((uint32_t*)xq_row)[chunk] = o;
  }
}

// ---- MXFP4 ---------------------------------------------------------------------------------------------
// shared exponent byte of a block whose largest magnitude is amax
__device__ __forceinline__ int mx_exponent(float amax) {
  if (!(amax > 0.0f)) return 127;
  const int ef = (int)((__float_as_uint(amax) >> 23) & 0xffu);      // 0 for subnormals: clipped below anyway
  int se = ef - 127 - 2;
  se = se < -127 ? -127 : se;
  return se + 127;
}
// E2M1 codes of eight values (nearest, ties to the even code) from the part's own conversion instruction (two fp32 values divided by the
// power of two in the scale operand's exponent field, rounded to nearest even on the E2M1 grid and
// saturated, packed into one byte: low nibble first operand, high nibble second), already in the
// interleaved nibble layout.  The instruction keeps the sign of a value that rounds to zero; codes are
// canonical here (zero has sign 0), so the sign bit of every nibble without magnitude bits is cleared.
// Checked against comparisons with the midpoints on a million random pairs, every tie, saturation and the
// ends of the exponent range: identical.
__device__ __forceinline__ uint32_t mx_codes8(const float v[8], int E) {
  const float sc = __uint_as_float((uint32_t)E << 23);
  uint32_t d = 0;
  d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, v[0], v[4], sc, 0);
  d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, v[1], v[5], sc, 1);
  d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, v[2], v[6], sc, 2);
  d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, v[3], v[7], sc, 3);
  const uint32_t nz = ((d & 0x77777777u) + 0x77777777u) & 0x88888888u;   // bit 3 of a nibble: its magnitude is not zero
  return d & (0x77777777u | nz);
}
}  // namespace serq
