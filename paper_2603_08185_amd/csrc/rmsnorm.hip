// Residual sum, root-mean-square norm, flattening and quantisation of a token's row in one pass (serq_rmsnorm_quantize_act and its forms):
//   h = X + residual, rounded to the stream's type;  rstd = 1 / sqrt(mean h^2 + eps);  u = h gain.
// Integer codes are those of u: the norm's factor is one number a token, which symmetric and asymmetric scales carry along
// (scale = su rstd), so the sum of squares and the largest |u| are found in one round of the workgroup and no code waits
// for the square root.  MXFP4's block scales are powers of two: there v = u rstd is what is quantised.
// The sum of squares is taken in 64 bits: squares of 16-bit numbers are exact there and sums of them as good as, so rstd is good to some 2^-50 before its one
// rounding to fp32 however the row is split: the correctly rounded one but where that lies as close to a border, and with it every code and scale.
//
// A workgroup a token, the row in registers between the two steps.  Bound by memory: stream, residual and sum in 16 bits and 8-bit codes are 7 bytes
// a channel, 16384 tokens of 4096 channels 470 MB in 81.2 us (5.8 TB/s; a copy of 1 GiB reaches 5.1 to 5.3); few tokens by the trip to
// memory and the workgroup's one meeting (one token of 4096 channels 2.55 us a launch, of which an empty one takes most).
#include <float.h>

#include <type_traits>

#include "quant_codes.h"
#include "root64.h"

namespace serq {
namespace {

enum Form { kSym8, kSym4, kAsym8, kAsym4, kMx };

struct NormParams {
  const char* x; const char* res; const float* gain; char* h; char* xq; void* scale; int32_t* zero;
  int64_t ldx, ldr, ldh;  // bytes
  double inv_k, eps;
  int64_t M, m0;          // rows of the call, the launch's first
  int K;
};

template <int XDT>
__device__ __forceinline__ Raw8<XDT> rounded8(const float v[8]) {
  Raw8<XDT> r;
  if constexpr (XDT == SERQ_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r.a[i] = __float_as_uint(v[i]);
      r.b[i] = __float_as_uint(v[4 + i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r.a[i] = XDT == SERQ_BF16 ? f32x2_to_bf16x2(v[2 * i], v[2 * i + 1]) : f32x2_to_f16x2(v[2 * i], v[2 * i + 1]);
  }
  return r;
}
// The sum is not read again before the next layer adds to it: it goes past the caches (us, with / without: 1000 tokens of 4096 channels 6.56 / 6.97, 1000 of 8192
// 13.4 / 14.3, 16384 of 4096 81.2 / 83.0; loads past them too 80.3, but 7.6 for the 1000).
template <int XDT>
__device__ __forceinline__ void store8(void* row, int chunk, const Raw8<XDT>& r) {
  if constexpr (XDT == SERQ_F32) {
    __builtin_nontemporal_store(r.a, (u4*)row + 2 * (size_t)chunk);
    __builtin_nontemporal_store(r.b, (u4*)row + 2 * (size_t)chunk + 1);
  } else {
    __builtin_nontemporal_store(r.a, (u4*)row + chunk);
  }
}

// What a row's threads find out together: the sum of squares, and the range of u (symmetric: lo is unused, hi the largest |u|).
struct Found { double sum; float lo, hi; };
template <int FORM, int KT>
__device__ __forceinline__ Found meet(Found f, Found* red) {
  constexpr bool ASYM = FORM == kAsym8 || FORM == kAsym4;
  f.sum = wave_sum(f.sum);
  if constexpr (FORM != kMx) f.hi = wave_max(f.hi);
  if constexpr (ASYM) f.lo = wave_reduce(f.lo, [](float a, float b) { return fminf(a, b); });
  if constexpr (KT == 64) return f;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = f;
  __syncthreads();
  f = red[0];
#pragma unroll
  for (int i = 1; i < KT / 64; ++i) {
    f.sum += red[i].sum;
    if constexpr (FORM != kMx) f.hi = fmaxf(f.hi, red[i].hi);
    if constexpr (ASYM) f.lo = fminf(f.lo, red[i].lo);
  }
  return f;
}

// KT: threads of a row; NC: pieces of 8 channels that a thread keeps in registers, 0: the row is walked twice, four pieces a time (the second time
// it is read where the first left the sum).  X, residual and h may be the same memory: a thread reads its pieces before it writes them.
template <int XDT, int FORM, int KT, int NC, bool RES>
__global__ __launch_bounds__(KT) void rmsnorm_quantize_kernel(NormParams p) {
  constexpr bool ASYM = FORM == kAsym8 || FORM == kAsym4;
  constexpr int ABITS = FORM == kSym8 || FORM == kAsym8 ? 8 : 4;
  constexpr int NB = NC > 0 ? NC : 4;
  __shared__ Found red[KT / 64];
  const int64_t m = p.m0 + blockIdx.x;
  const int nchunk = p.K >> 3, tid = threadIdx.x;
  const char* row = p.x + m * p.ldx;
  const char* rrow = RES ? p.res + m * p.ldr : nullptr;
  char* hrow = RES ? p.h + m * p.ldh : nullptr;
  float u[NB][8];
  Found f{0.0, 0.0f, 0.0f};

  // the pieces chunk0, chunk0 + KT, ... as u; FIRST: summed, stored and looked at
  const auto fetch = [&](int chunk0, auto first) {
    constexpr bool FIRST = decltype(first)::value;
    Raw8<XDT> x[NB], r[NB];
    v4f ga[NB], gb[NB];
    const char* from = RES && !FIRST ? hrow : row;
    const bool flat = p.gain != nullptr;
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      const int at = min(chunk0 + c * KT, nchunk - 1);        // (past the row: its last piece again)
      x[c] = fetch8<XDT>(from, at);
      if constexpr (RES && FIRST) r[c] = fetch8<XDT>(rrow, at);
      if (flat) {
        ga[c] = ((const v4f*)p.gain)[2 * (size_t)at];
        gb[c] = ((const v4f*)p.gain)[2 * (size_t)at + 1];
      }
    }
    __builtin_amdgcn_sched_barrier(0);                        // (all loads under way before the first value is used)
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      const bool in = chunk0 + c * KT < nchunk;
      values8<XDT>(x[c], u[c]);
      if constexpr (RES && FIRST) {
        float t[8];
        values8<XDT>(r[c], t);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[c][i] += t[i];
        x[c] = rounded8<XDT>(u[c]);
        if (in) store8<XDT>(hrow, chunk0 + c * KT, x[c]);
        values8<XDT>(x[c], u[c]);
      }
      if constexpr (FIRST) {
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = __builtin_fma((double)u[c][i], (double)u[c][i], s);
        f.sum += in ? s : 0.0;
      }
      if (flat) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u[c][i] *= ga[c][i];
          u[c][4 + i] *= gb[c][i];
        }
      }
      // (a piece past the row counts for nothing: where h is X, the last piece may have been written meanwhile)
      if constexpr (FIRST && ASYM) {
        float lo = f.lo, hi = f.hi;
#pragma unroll
        for (int i = 0; i < 8; ++i) { lo = fminf(lo, u[c][i]); hi = fmaxf(hi, u[c][i]); }
        f.lo = in ? lo : f.lo;
        f.hi = in ? hi : f.hi;
      } else if constexpr (FIRST && FORM != kMx) {
        f.hi = in ? absmax8(u[c], f.hi) : f.hi;
      }
    }
  };
  if constexpr (NC > 0) {
    fetch(tid, std::true_type{});
  } else {
    for (int chunk = tid; chunk < nchunk; chunk += NB * KT) fetch(chunk, std::true_type{});
  }
  f = meet<FORM, KT>(f, red);
  const double ms = __builtin_fma(f.sum, p.inv_k, p.eps);

  constexpr float top = ASYM ? (float)((1 << ABITS) - 1) : (float)((1 << (ABITS - 1)) - 1);
  // (a product with the rounded reciprocal: within an ulp of the quotient, and every code waits for it)
  const float unit = (ASYM ? f.hi - f.lo : f.hi) * (1.0f / top);
  const float sc = unit > 0.0f ? unit : 1.0f, rsc = __builtin_amdgcn_rcpf(sc);
  const float z = ASYM ? rintf(-f.lo / sc) : 0.0f;
  const float rstd = FORM == kMx ? inv_root(ms) : 0.0f;
  const size_t Mp = (size_t)((p.M + 1) & ~(int64_t)1);
  uint8_t* xsc = (uint8_t*)p.scale;                           // MXFP4: [ceil(K / 256)][Mp][8]
  const auto store = [&](int chunk0) {
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      const int chunk = chunk0 + c * KT;
      char* xq_row = p.xq + (size_t)m * ((size_t)p.K * ABITS / 8);
      if constexpr (FORM == kMx) {
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) u[c][i] *= rstd;
        amax = absmax8(u[c], amax);
        amax = fmaxf(amax, dpp<kDpp1>(amax));                 // (a row is a multiple of 8 pieces: a block's four are all in it or none)
        amax = fmaxf(amax, dpp<kDpp2>(amax));
        const int E = mx_exponent(amax);
        if (chunk < nchunk) {
          ((uint32_t*)xq_row)[chunk] = mx_codes8(u[c], E);
          if ((chunk & 3) == 0) {
            const int blk = chunk >> 2;
            xsc[((size_t)(blk >> 3) * Mp + (size_t)m) * 8 + (blk & 7)] = (uint8_t)E;
          }
        }
      } else if (chunk < nchunk) {
        if constexpr (ASYM) {
          int c8[8];
          asym_codes8<ABITS>(u[c], sc, rsc, z, c8);
          store_codes8<ABITS>(c8, xq_row, chunk);
        } else {
          quant_store8<ABITS>(u[c], sc, xq_row, chunk);
        }
      }
    }
  };
  if constexpr (NC > 0) {
    store(tid);
  } else {
    for (int chunk = tid; chunk < nchunk; chunk += NB * KT) {
      fetch(chunk, std::false_type{});
      store(chunk);
    }
  }

  if constexpr (FORM == kMx) {
    // scale bytes of the blocks that the last 256-channel tile does not have, and the padding row of an odd M
    const int nblk = p.K >> 5, nblk8 = (nblk + 7) & ~7;
    if (tid < nblk8 - nblk) xsc[((size_t)((nblk + tid) >> 3) * Mp + (size_t)m) * 8 + ((nblk + tid) & 7)] = 127;
    if (m == p.M - 1 && (size_t)p.M < Mp)
      for (int blk = tid; blk < nblk8; blk += KT) xsc[((size_t)(blk >> 3) * Mp + (size_t)p.M) * 8 + (blk & 7)] = 127;
  } else if (tid == 0) {
    // (a sum that is not finite makes the token NaN, whatever the largest finite |u| is)
    ((float*)p.scale)[m] = !(ms < __builtin_inf()) ? __builtin_nanf("") : unit > 0.0f ? sc * inv_root(ms) : 1.0f;
    if constexpr (ASYM) p.zero[m] = (int)z - (1 << (ABITS - 1));
  }
}

// Threads of a row and pieces of each: a row's own latency counts where rows are few and the rate at which waves start where they are many, and both want
// a piece a thread up to 512 of them, but for many rows without a residual, which have little to load; beyond, registers.  Measured
// (symmetric 8-bit codes, bf16, us; threads x pieces):
//   K = 1024  128 x 1 / 64 x 2 / 256 x 1: M = 1 2.16 / 2.35 / 2.17, M = 4096 7.04 / 7.80 / 8.37
//   K = 2624  384 x 1 / 192 x 2 / 512 x 1: M = 1 2.39 / 2.59 / 2.54, M = 1000 5.98 / 6.30 / 6.22, M = 4096 13.9 / 13.7 / 14.4, no residual 10.7 / 9.3 / 11.4
//   K = 4096  512 x 1 / 256 x 2: M = 1 2.55 / 2.72, M = 1000 7.05 / 7.49, M = 16384 82.8 / 83.3, M = 4096 without a residual 12.4 / 11.4
//   K = 5120  320 x 2 / 256 x 3 / 768 x 1: M = 1 2.95 / 3.08 / 2.95, M = 4096 24.9 / 25.4 / 26.8
//   K = 8192  512 x 2 / 1024 x 1 / 256 x 4: M = 1 3.23 / 3.40 / 3.56, M = 4096 35.5 / 36.5 / 36.1
//   K = 11008 512 x 3 / 768 x 2: M = 1 3.78 / 3.74, M = 4096 59.3 / 59.3;  K = 16384 512 x 4 / 1024 x 2: M = 1 4.42 / 4.40, M = 4096 89.6 / 101
//   K = 20480 512 x 6 / 1024 x 3: M = 1 5.66 / 5.29, M = 2000 54.4 / 63.7;  K = 32768 1024 x 4 / 512 x 8: M = 1 6.63 / 7.14, M = 2000 102 / 102
//   K = 65536, walked twice by 1024 / 512: M = 1 12.5 / 13.4, M = 300 42.7 / 45.5
template <int XDT, int FORM, bool RES>
int launch(const NormParams& p, int64_t rows, hipStream_t st) {
  const int nchunk = p.K >> 3;
  const dim3 grid((unsigned)rows);
#define SERQ_NORM(KT, NC) hipLaunchKernelGGL((rmsnorm_quantize_kernel<XDT, FORM, KT, NC, RES>), grid, dim3(KT), 0, st, p)
  if constexpr (!RES) {
    if (rows > 1000 && nchunk > 256 && nchunk <= 512) {
      if (nchunk <= 384) SERQ_NORM(192, 2);
      else SERQ_NORM(256, 2);
      return hipGetLastError() == hipSuccess ? SERQ_OK : SERQ_EHIP;
    }
  }
  if (nchunk <= 64) SERQ_NORM(64, 1);
  else if (nchunk <= 128) SERQ_NORM(128, 1);
  else if (nchunk <= 192) SERQ_NORM(192, 1);
  else if (nchunk <= 256) SERQ_NORM(256, 1);
  else if (nchunk <= 384) SERQ_NORM(384, 1);
  else if (nchunk <= 512) SERQ_NORM(512, 1);
  else if (nchunk <= 640) SERQ_NORM(320, 2);
  else if (nchunk <= 768) SERQ_NORM(384, 2);
  else if (nchunk <= 1024) SERQ_NORM(512, 2);
  else if (nchunk <= 1536) SERQ_NORM(512, 3);
  else if (nchunk <= 2048) SERQ_NORM(512, 4);
  else if (nchunk <= 512 * 6) SERQ_NORM(512, 6);
  else if (nchunk <= 4096) SERQ_NORM(1024, 4);
  else SERQ_NORM(1024, 0);
#undef SERQ_NORM
  return hipGetLastError() == hipSuccess ? SERQ_OK : SERQ_EHIP;
}

template <int FORM>
int launch_form(int x_dtype, const NormParams& p, int64_t rows, hipStream_t st) {
  if (x_dtype == SERQ_F32) return p.res ? launch<SERQ_F32, FORM, true>(p, rows, st) : launch<SERQ_F32, FORM, false>(p, rows, st);
  if (x_dtype == SERQ_F16) return p.res ? launch<SERQ_F16, FORM, true>(p, rows, st) : launch<SERQ_F16, FORM, false>(p, rows, st);
  return p.res ? launch<SERQ_BF16, FORM, true>(p, rows, st) : launch<SERQ_BF16, FORM, false>(p, rows, st);
}

inline bool aligned(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

int rmsnorm_quantize(const void* X, const void* residual, int x_dtype, const float* gain, float eps, int64_t M, int64_t K, int64_t ldx,
                     int64_t ldr, void* h_out, int64_t ldh, int form, void* Xq_out, void* scale_out, int32_t* zero_out, void* stream) {
  if (x_dtype != SERQ_F32 && x_dtype != SERQ_F16 && x_dtype != SERQ_BF16) return SERQ_EDTYPE;
  if (M < 0 || M > (1 << 30) || K < 64 || K > 131072 || (K % 64) != 0) return SERQ_ESHAPE;
  if (!(eps >= 0.0f) || !(eps <= FLT_MAX)) return SERQ_ESHAPE;
  if (!residual && h_out) return SERQ_ESHAPE;                 // (h is X then)
  if (ldx < K || (residual && (ldr < K || ldh < K))) return SERQ_ESHAPE;
  if ((ldx % 8) != 0 || (residual && ((ldr % 8) != 0 || (ldh % 8) != 0))) return SERQ_EALIGN;
  if (M == 0) return SERQ_OK;
  const bool asym = form == kAsym8 || form == kAsym4;
  if (!X || !Xq_out || !scale_out || (residual && !h_out) || (asym && !zero_out)) return SERQ_ENULL;
  if (residual && ((h_out == X && ldh != ldx) || (h_out == residual && ldh != ldr))) return SERQ_ESHAPE;
  if (!aligned(X, 16) || !aligned(residual, 16) || !aligned(gain, 16) || !aligned(h_out, 16) || !aligned(Xq_out, 16) ||
      !aligned(scale_out, form == kMx ? 16 : 4) || !aligned(zero_out, 4))
    return SERQ_EALIGN;
  const int64_t es = x_dtype == SERQ_F32 ? 4 : 2;
  NormParams p{};
  p.x = (const char*)X; p.res = (const char*)residual; p.gain = gain; p.h = (char*)h_out;
  p.xq = (char*)Xq_out; p.scale = scale_out; p.zero = zero_out;
  p.ldx = ldx * es; p.ldr = ldr * es; p.ldh = ldh * es;
  p.inv_k = 1.0 / (double)K; p.eps = (double)eps;
  p.M = M; p.K = (int)K;
  for (p.m0 = 0; p.m0 < M; p.m0 += kLaunchRows) {
    const int64_t rows = M - p.m0 < kLaunchRows ? M - p.m0 : kLaunchRows;
    hipStream_t st = (hipStream_t)stream;
    const int rc = form == kSym8    ? launch_form<kSym8>(x_dtype, p, rows, st)
                   : form == kSym4  ? launch_form<kSym4>(x_dtype, p, rows, st)
                   : form == kAsym8 ? launch_form<kAsym8>(x_dtype, p, rows, st)
                   : form == kAsym4 ? launch_form<kAsym4>(x_dtype, p, rows, st)
                                    : launch_form<kMx>(x_dtype, p, rows, st);
    if (rc != SERQ_OK) return rc;
  }
  return SERQ_OK;
}

}  // namespace
}  // namespace serq

using namespace serq;

extern "C" {

int serq_rmsnorm_quantize_act(const void* X, const void* residual, int x_dtype, const float* gain, float eps, int64_t M, int64_t K, int64_t ldx,
                              int64_t ldr, void* h_out, int64_t ldh, int abits, void* Xq_out, float* scale_out, void* stream) {
  if (abits != 4 && abits != 8) return SERQ_EDTYPE;
  return rmsnorm_quantize(X, residual, x_dtype, gain, eps, M, K, ldx, ldr, h_out, ldh, abits == 8 ? kSym8 : kSym4, Xq_out, scale_out, nullptr, stream);
}

int serq_rmsnorm_quantize_act_asym(const void* X, const void* residual, int x_dtype, const float* gain, float eps, int64_t M, int64_t K,
                                   int64_t ldx, int64_t ldr, void* h_out, int64_t ldh, int abits, void* Xq_out, float* scale_out,
                                   int32_t* zero_out, void* stream) {
  if (abits != 4 && abits != 8) return SERQ_EDTYPE;
  return rmsnorm_quantize(X, residual, x_dtype, gain, eps, M, K, ldx, ldr, h_out, ldh, abits == 8 ? kAsym8 : kAsym4, Xq_out, scale_out, zero_out,
                          stream);
}

int serq_mx_rmsnorm_quantize_act(const void* X, const void* residual, int x_dtype, const float* gain, float eps, int64_t M, int64_t K,
                                 int64_t ldx, int64_t ldr, void* h_out, int64_t ldh, void* Xq_out, uint8_t* xscale_out, void* stream) {
  return rmsnorm_quantize(X, residual, x_dtype, gain, eps, M, K, ldx, ldr, h_out, ldh, kMx, Xq_out, xscale_out, nullptr, stream);
}

}  // extern "C"
