// Shared by the kernels of serq_paged_attn: the parameters, and the places of rows, keys and pages.
//
// A key head's queries form a matrix of rows: row r = i G + g of sequence b is new token i's query head h G + g (G query heads share key
// head h).  A workgroup takes a block of such rows, so that every key it fetches serves all G heads.
#pragma once

#include <float.h>

#include "kv_cache.h"

namespace serq {

struct AttnParams {
  const char* q; char* out; float* lse;                       // strides in bytes
  int64_t ldq, ldqh, ldo, ldoh;
  int q_heads, group, window;
  float scale;
  int direct;             // every sequence fits one block of rows: block = sequence
  int rows_from, rows_to; // sequences with rows_from <= n G < rows_to are this kernel's
  int slices, slice_keys; // most slices of a sequence's keys, keys of one (a multiple of 256)
  uint32_t* tickets;      // [row blocks][key heads]: slices done, zero between calls
  float* part;            // [row blocks][key heads][slices]: rows x D sums, then rows x 2 statistics
  KvView c;
};

// Row blocks of BM rows: sequence b has the blocks from floor(cu[b] G / BM) + b on, up to where sequence b + 1's begin: at least as many as it
// needs, in a place that no sum over the sequences before it is needed for.
struct RowBlock {
  int b, r0, n, L;        // sequence, first row, new tokens, keys
  int rows;               // rows of the block (<= 0: none)
  int begin, end;         // keys that any of its rows sees: begin <= j < end
};
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
template <int BM>
__device__ __forceinline__ RowBlock row_block(const AttnParams& p, int block, int lane) {
  RowBlock k;
  const int G = p.group;
  k.rows = 0;
  k.b = p.direct ? block : sequences_before(block, p.c.seqs, lane, [&](int i) { return p.c.cu[i + 1] * G / BM + i + 1; });
  if (k.b >= p.c.seqs) return k;
  const int c0 = uniform(p.c.cu[k.b]), c1 = uniform(p.c.cu[k.b + 1]);
  k.n = c1 - c0;
  k.L = uniform(p.c.len[k.b]);
  k.r0 = p.direct ? 0 : (block - (c0 * G / BM + k.b)) * BM;
  if (k.n <= 0 || k.n * G < p.rows_from || k.n * G >= p.rows_to || c0 < 0 || c1 > p.c.tokens) return k;
  k.rows = min(k.n * G - k.r0, BM);
  if (k.rows <= 0) return k;
  const int first = k.L - k.n + k.r0 / G, last = k.L - k.n + (k.r0 + k.rows - 1) / G;
  k.end = min(last + 1, p.c.width << p.c.page_shift);
  k.begin = p.window > 0 ? max(0, first - p.window + 1) : 0;
  return k;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }   // an ulp; below 2^-126 to zero

// over the four lanes that hold the same row: l, l ^ 16, l ^ 32, l ^ 48
template <class Op>
__device__ __forceinline__ float quads_reduce(float v, const Op& op) {
  uint32_t i = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane16_swap(i, i, false, false);
  v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
  i = __float_as_uint(v);
  const auto b = __builtin_amdgcn_permlane32_swap(i, i, false, false);
  return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// 16 E4M3 codes as 16-bit floats (exact in both types)
template <int DT>
__device__ __forceinline__ void widen_e4m3(const u4& w, u4& lo, u4& hi) {
  uint32_t o[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == SERQ_BF16) {
      o[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, false));
      o[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, true));
    } else {
      o[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, false));
      o[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, true));
    }
  }
  lo = (u4){o[0], o[1], o[2], o[3]};
  hi = (u4){o[4], o[5], o[6], o[7]};
}

// 4 keys (rows of 16-bit values in LDS) of one channel a lane: 16 lanes give the addresses of 4 x 4 pieces of 4 channels and get a column each
typedef short v4s __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u2 lds_column4(const char* p) {
  return __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)p));
}

template <int DT>
__device__ __forceinline__ uint32_t pack16(float a, float b) { return DT == SERQ_BF16 ? f32x2_to_bf16x2(a, b) : f32x2_to_f16x2(a, b); }

// what is written for a row whose weighted sum is o and whose weights sum to l
__device__ __forceinline__ float row_factor(float l, float v_scale) { return l == 0.0f ? 0.0f : v_scale / l; }
// logarithm of the softmax' sum: m is the running reference in the exponent of 2
__device__ __forceinline__ float row_lse(float m, float l) {
  return l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.693147180559945309f;
}

constexpr int kMaxSlices = 128;
constexpr float kLog2e = 1.44269504088896341f;

size_t paged_attn_few_slot_floats(int nb, int D);
int launch_paged_attn_few(const AttnParams& p, int dtype, bool f8, int D, int nb, int blocks, hipStream_t st);

}  // namespace serq
