// Shared by the kernels of serq_paged_attn: the parameters, and the places of rows, keys and pages.
//
// A key head's queries form a matrix of rows: row r = i G + g of sequence b is new token i's query head h G + g (G query heads share key
// head h).  A workgroup takes a block of such rows, so that every key it fetches serves all G heads.
#pragma once

#include <float.h>

#include <type_traits>

#include "kv_cache.h"

namespace serq {

struct AttnParams {
  const char* q; char* out; float* lse;                       // strides in bytes
  int64_t ldq, ldqh, ldo, ldoh;
  int q_heads, group, window;
  float scale;
  int rows_from, rows_to; // sequences with rows_from <= n G < rows_to are this kernel's
  int slices, slice_keys; // tile kernel: most slices of a sequence's keys, keys of one (a multiple of 64); few: 1, or more, and keys of a share at least
  uint32_t* tickets;      // slices done, zero between calls: [row blocks][key heads]; few: [workgroups]
  float* part;            // the slots where slices meet: [row blocks][key heads][slices]; few: [workgroups][2]
  KvView c;
};

// What may stand between the scores and the softmax: rows that see a range of keys of their own; scores capped by a tanh; scores less a slope times the
// distance (both with such ranges too, or without).
enum Mod { kPlain, kRanges, kCapped, kBiased };
struct AttnModParams : AttnParams {
  const int32_t* from;    // by row of q: the first key that it sees, and the one past its last; or null
  const int32_t* to;
  const float* slopes;    // kBiased: by query head
  float cap;              // kCapped
};
template <int MOD> using ParamsOf = std::conditional_t<MOD == kPlain, AttnParams, AttnModParams>;

struct RowBlock {
  int b, tok0, r0, n, L;  // sequence, its first row of q, the block's first row, new tokens, keys
  int rows;               // rows of the block (<= 0: none)
  int begin, end;         // keys that any of its rows sees: begin <= j < end
  int all_from, all_to;   // keys that all of its rows see
};
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
// The block of BM rows from r0 on of sequence b, whose new tokens are rows c0 .. c0+n-1 of q and which has L keys.
template <int BM>
__device__ __forceinline__ RowBlock row_block(const AttnParams& p, int b, int c0, int n, int L, int r0) {
  RowBlock k;
  const int G = p.group;
  k.b = b;
  k.tok0 = c0;
  k.n = n;
  k.L = L;
  k.r0 = r0;
  k.rows = min(n * G - r0, BM);
  const int first = L - n + r0 / G, last = L - n + (r0 + k.rows - 1) / G;
  k.end = min(last + 1, p.c.width << p.c.page_shift);
  k.begin = p.window > 0 ? max(0, first - p.window + 1) : 0;
  k.all_from = p.window > 0 ? max(0, last - p.window + 1) : 0;
  k.all_to = min(first + 1, k.end);
  return k;
}
// The keys that the row of q at position pos of a sequence of L keys sees: lo <= j < hi (both 0: none).
struct Range { int lo, hi; };
__device__ __forceinline__ Range row_range(const AttnModParams& p, int row, int pos, int L) {
  Range x;
  x.hi = min(p.to ? p.to[row] : pos + 1, min(L, p.c.width << p.c.page_shift));
  x.lo = max(p.from ? p.from[row] : 0, 0);
  if (p.window > 0) x.lo = max(x.lo, pos - p.window + 1);
  return x.hi > x.lo ? x : Range{0, 0};
}
// What rows see together: [begin, end) holds all of it, [all_from, all_to) is seen by each (empty where a row sees nothing).
struct Seen {
  int begin = 0x7fffffff, end = 0, all_from = 0, all_to = 0x7fffffff;
  __device__ __forceinline__ void add(const Range& x) {
    if (x.hi > 0) begin = min(begin, x.lo);
    end = max(end, x.hi);
    all_from = max(all_from, x.lo);
    all_to = min(all_to, x.hi);
  }
};
// op over the 64 lanes of a wave, the result in all of them (as wave_reduce, for whole numbers)
template <class Op>
__device__ __forceinline__ int wave_reduce_int(int v, const Op& op) {
  v = op(v, __builtin_amdgcn_update_dpp(v, v, kDpp1, 0xf, 0xf, false));
  v = op(v, __builtin_amdgcn_update_dpp(v, v, kDpp2, 0xf, 0xf, false));
  v = op(v, __builtin_amdgcn_update_dpp(v, v, kDppMirror8, 0xf, 0xf, false));
  v = op(v, __builtin_amdgcn_update_dpp(v, v, kDppMirror16, 0xf, 0xf, false));
  const auto a = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
  v = op((int)a[0], (int)a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
  return op((int)b[0], (int)b[1]);
}
__device__ __forceinline__ int wave_min_int(int v) {
  return uniform(wave_reduce_int(v, [](int a, int b) { return min(a, b); }));
}
__device__ __forceinline__ int wave_max_int(int v) {
  return uniform(wave_reduce_int(v, [](int a, int b) { return max(a, b); }));
}
// Without ranges row_block says the same sooner (200 single tokens over up to 1500 keys, capped, 88.8 / 84.9 us; one over 1000 10.8 / 10.2); blocks of 32 rows have
// no registers for a second way (8 x 5 drafted tokens over up to 6000, with a bias, 36.2 / 37.1).
template <int BM> constexpr bool kLookAlways = BM == 32;
// row_block by what each of its tokens sees; by a whole wave, whose lanes look at a token each.  (One name for both, by the parameters' type.)
template <int BM>
__device__ __forceinline__ RowBlock block_of(const AttnParams& p, int b, int c0, int n, int L, int r0) {
  return row_block<BM>(p, b, c0, n, L, r0);
}
template <int BM>
__device__ __forceinline__ RowBlock block_of(const AttnModParams& p, int b, int c0, int n, int L, int r0) {
  if (!kLookAlways<BM> && !p.from && !p.to) return row_block<BM>(p, b, c0, n, L, r0);
  RowBlock k;
  const int G = p.group, lane = threadIdx.x & 63;
  k.b = b;
  k.tok0 = c0;
  k.n = n;
  k.L = L;
  k.r0 = r0;
  k.rows = min(n * G - r0, BM);
  const int last = k.rows > 0 ? (r0 + k.rows - 1) / G : -1;
  Seen s;
  for (int i = r0 / G + lane; i <= last; i += 64) s.add(row_range(p, c0 + i, L - n + i, L));
  k.end = wave_max_int(s.end);
  k.begin = k.end > 0 ? wave_min_int(s.begin) : 0;
  k.all_from = wave_max_int(s.all_from);
  k.all_to = min(wave_min_int(s.all_to), k.end);
  return k;
}

// whether a sequence is this kernel's (and one that can be)
__device__ __forceinline__ bool takes(const AttnParams& p, int c0, int n) {
  return n > 0 && c0 >= 0 && n <= p.c.tokens - c0 && n * p.group >= p.rows_from && n * p.group < p.rows_to;
}
// sum over the lanes up to each one
__device__ __forceinline__ int sum_upto(int v, int lane) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);     // 1, 2, 4 and 8 lanes before, within 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  const int a = __builtin_amdgcn_readlane(v, 15), b = __builtin_amdgcn_readlane(v, 31), c = __builtin_amdgcn_readlane(v, 47);
  return v + (lane >= 48 ? a + b + c : lane >= 32 ? a + b : lane >= 16 ? a : 0);
}

// A sequence: its first row of q, its new tokens, its keys, how many pieces of work it gives a key head, and how many those before it give.
struct Sequence { int b, c0, n, L, pieces, before; };

// The pieces of all sequences in a line.  Every wave for itself: a lane counts those of some sequences, and knows what lies before them.
// `count(c0, n, L)`: pieces of a sequence that is this kernel's.
template <class Count>
struct Line {
  const AttnParams& p;
  const Count& count;
  int l, b0, own, upto, total;
  Sequence s;                                                 // the lane's: the last that it looked at
  __device__ __forceinline__ void look(int b) {
    s.b = b;
    s.c0 = p.c.cu[b];
    s.n = p.c.cu[b + 1] - s.c0;
    s.L = p.c.len[b];
    s.pieces = takes(p, s.c0, s.n) ? count(s.c0, s.n, s.L) : 0;
  }
  __device__ __forceinline__ Line(const AttnParams& q, const Count& c, int lane) : p(q), count(c), l(lane), own(0), s{} {
    const int per = (p.c.seqs + 63) / 64;
    b0 = l * per;
    for (int i = min(per, p.c.seqs - b0) - 1; i >= 0; --i) {  // (the first one last)
      look(b0 + i);
      own += s.pieces;
    }
    upto = sum_upto(own, l);
    total = __builtin_amdgcn_readlane(upto, 63);
  }
  // the sequence that piece `at` (0 <= at < total) is of
  __device__ __forceinline__ Sequence find(int at) {
    const int lane = __builtin_ctzll(__ballot(own > 0 && at >= upto - own && at < upto));
    int before = upto - own;
    if (l == lane && own > s.pieces) {                        // several sequences: which of them
      look(b0);
      while (at >= before + s.pieces) {
        before += s.pieces;
        look(s.b + 1);
      }
    }
    Sequence x;
    x.b = __builtin_amdgcn_readlane(s.b, lane);
    x.c0 = __builtin_amdgcn_readlane(s.c0, lane);
    x.n = __builtin_amdgcn_readlane(s.n, lane);
    x.L = __builtin_amdgcn_readlane(s.L, lane);
    x.pieces = __builtin_amdgcn_readlane(s.pieces, lane);
    x.before = __builtin_amdgcn_readlane(before, lane);
    return x;
  }
};

// device memory behind an address that is put together from numbers (a plain pointer would be taken for one that may also point into LDS)
typedef __attribute__((address_space(1))) const char GlobalByte;
typedef __attribute__((address_space(1))) const u4 GlobalPiece;

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

constexpr float kLog2e = 1.44269504088896341f;

// Weights are 16-bit numbers where they meet V.  bf16 has exponents for all of them; fp16 ends at 2^16 and loses bits below 2^-14, so there the reference lies
// 9 lower in the exponent: weights are at most 2^15, and of full precision down to 2^-23 of the reference's own.  (Else 60000 keys
// 20.5 below in the exponent, 2^-20.5 being 11.3 of the type's smallest steps, would each count as 11.)
template <int DT> constexpr float kHeadroom = DT == SERQ_F16 ? 9.0f : 0.0f;
template <int DT> __device__ __forceinline__ float reference(float score, float c) { return fmaxf(score * c - kHeadroom<DT>, -FLT_MAX); }
// what makes a score one in the exponent of 2 (not 0, which would make NaN of a masked score)
__device__ __forceinline__ float score_factor(float scale, float k_scale) { return fmaxf(scale * k_scale * kLog2e, FLT_MIN); }
// by how much a score may exceed the reference before that is raised: 2^6 in weight
__device__ __forceinline__ float score_slack(float c) { return fminf(6.0f / c, 1e30f); }

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

// whether any of 8 values is not finite: its exponent's bits are all ones, so that one more of the lowest runs into the sign's place
template <int DT>
__device__ __forceinline__ bool any_odd(const u4& x) {
  constexpr uint32_t STEP = DT == SERQ_BF16 ? 0x00800080u : 0x04000400u;
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m |= (x[i] & 0x7fff7fffu) + STEP;
  return (m & 0x80008000u) != 0;
}

// Values of keys that some rows of a block see and others do not.  A weight of zero does not make NaN or infinity zero, so in the tiles that hold such keys
// what is not finite is taken out before the products, and added at the end for the rows that do see it.
template <int DT>
__device__ __forceinline__ u4 take_out(u4 x, bool& odd) {
  constexpr uint32_t M = DT == SERQ_BF16 ? 0x7f80u : 0x7c00u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool a = (x[i] & M) == M, b = (x[i] & (M << 16)) == (M << 16);
    odd |= a || b;
    x[i] = (a ? 0u : x[i] & 0xffffu) | (b ? 0u : x[i] & 0xffff0000u);
  }
  return x;
}
// What was taken out of channel d of key j of sequence b, 0 if nothing was.
template <int DT, bool F8>
__device__ __forceinline__ float taken_out(const AttnParams& p, int b, int h, int j, int d) {
  const int page = min(max(p.c.table[b * p.c.table_ld + (j >> p.c.page_shift)], 0), p.c.pages - 1);
  const char* row = p.c.v + h * p.c.v_head + page * p.c.v_page + (j & ((1 << p.c.page_shift) - 1)) * p.c.v_token;
  float v;
  if constexpr (F8) v = __builtin_amdgcn_cvt_f32_fp8((int)(uint8_t)row[d], 0);
  else v = Elem<DT>::ld(row, d);
  return __builtin_isfinite(v) ? 0.0f : v;
}

template <int DT>
__device__ __forceinline__ uint32_t pack16(float a, float b) { return DT == SERQ_BF16 ? f32x2_to_bf16x2(a, b) : f32x2_to_f16x2(a, b); }

// what is written for a row whose weighted sum is o and whose weights sum to l
__device__ __forceinline__ float row_factor(float l, float v_scale) { return l == 0.0f ? 0.0f : v_scale / l; }
// logarithm of the softmax' sum: m is the running reference in the exponent of 2
__device__ __forceinline__ float row_lse(float m, float l) {
  return l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.693147180559945309f;
}

// ---- scores before the softmax --------------------------------------------------------------------------------------------------
// Biased: a slope times the distance is a number of score units that is there before the first product: the sums of the matrix instruction begin with it.
// `slope` in units of a score (score_slope), `d` the row's position less the key's.
__device__ __forceinline__ float score_slope(float slope, float c) { return fminf(fmaxf(slope * kLog2e / c, -FLT_MAX), FLT_MAX); }
__device__ __forceinline__ float distance_bias(float slope, float d) { return -slope * fabsf(d); }

// The reference of such scores lies higher by 2^-22 of its size where that is large: a product s c that is as large as a bias can be is rounded in m and not in s c - m, and what is
// left may not make a weight infinite in keys so far off that they weigh nothing in the end.
template <int MOD, int DT>
__device__ __forceinline__ float reference_of(float score, float c) {
  const float m = reference<DT>(score, c);
  if constexpr (MOD == kBiased) return fabsf(m) > 4096.0f ? fminf(__builtin_fmaf(fabsf(m), 0x1p-22f, m), FLT_MAX) : m;
  else return m;
}

// Capped: cap tanh(x) = cap - 2 cap / (1 + e^(2 x)), x = score / cap.  What stands in a score's place from here on is -1 / (1 + e^(2 x)), which grows with the
// score, with 2 cap log2 e in the place of the scale's factor; the cap itself is the same for all keys of a row, so the softmax does not need it and the
// logarithm of its sum gets it at the end.  Good to some 2^-23 of 2 cap log2 e in the exponent: 2^-14 of a weight for a cap of 128.
// `rate`: 2 log2 e / cap of what a raw score stands for.
template <int MOD>
__device__ __forceinline__ float cap_rate(const ParamsOf<MOD>& p, float k_scale) {
  if constexpr (MOD == kCapped) return fminf(fmaxf(2.0f * kLog2e * p.scale * k_scale / p.cap, FLT_MIN), FLT_MAX);
  else return 0.0f;
}
__device__ __forceinline__ float capped(float s, float rate) { return -__builtin_amdgcn_rcpf(1.0f + exp2_fast(s * rate)); }
__device__ __forceinline__ float cap_factor(float cap) { return fmaxf(2.0f * cap * kLog2e, FLT_MIN); }
template <int MOD>
__device__ __forceinline__ float factor_of(const ParamsOf<MOD>& p, float k_scale) {
  if constexpr (MOD == kCapped) return cap_factor(p.cap);
  else return score_factor(p.scale, k_scale);
}
__device__ __forceinline__ float lse_of(const AttnParams&, float m, float l) { return row_lse(m, l); }
__device__ __forceinline__ float lse_of(const AttnModParams& p, float m, float l) { return l == 0.0f ? -INFINITY : row_lse(m, l) + p.cap; }   // (cap 0: none)

constexpr int kMaxSlices = 256;          // of the kernel for few rows
constexpr int kMaxTileSlices = 32;       // of the kernel for many
constexpr int kTileRows = 128;

// ---- where the slices of a row block meet -------------------------------------------------------------------------------------
// A slice leaves its weighted sums and the statistics (m, l) of its rows in a slot of the workspace: rows x D floats in an order of the kernel's own,
// then [rows][2].  The slots are written and read past the caches that workgroups of different dies do not share (accesses at the
// device's scope).
__device__ __forceinline__ void put2(float* p, float a, float b) {
  const uint64_t v = (uint64_t)__float_as_uint(a) | (uint64_t)__float_as_uint(b) << 32;
  __hip_atomic_store((uint64_t*)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ v2f get2(const float* p) {
  const uint64_t v = __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return (v2f){__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))};
}
// A workgroup's stores are done before it takes its ticket, and who draws the last one finds all of them; the count is left at zero.
__device__ __forceinline__ bool last_to_arrive(uint32_t* ticket, int ns, int tid, uint32_t* shared) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) {
    const uint32_t n = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (n == (uint32_t)(ns - 1)) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *shared = n;
  }
  __syncthreads();
  return *shared == (uint32_t)(ns - 1);
}
size_t paged_attn_few_slot_floats(int nb, int D);
int paged_attn_few_resident(int nb, bool f8, int D);          // workgroups that a compute unit runs together
int launch_paged_attn_few(const AttnParams& p, int dtype, bool f8, int D, int nb, int workgroups, hipStream_t st);
// heads of 64 channels one a time, or two where the line has `long_line` pieces: workgroups of either, and slice_keys of two
struct PairPlan { int one, two, long_line, two_keys; };
int launch_paged_attn_pairs(const AttnParams& p, int dtype, const PairPlan& n, hipStream_t st);
size_t paged_attn_tile_slot_floats(int D);
int launch_paged_attn_tile(const AttnParams& p, int dtype, bool f8, int D, int blocks, hipStream_t st);
int launch_paged_attn_mixed(const AttnParams& many, const AttnParams& few, int dtype, bool f8, int D, int blocks, int shares, hipStream_t st);
// the same three with what stands between scores and softmax; one or two of them: a call's whole launch
struct ModLaunch {
  const AttnModParams* many; const AttnModParams* few;        // null: none
  int dtype; bool f8; int D, nb, blocks, shares;              // blocks: of the kernel for many rows, shares: workgroups of the one for few
  PairPlan pairs;                                             // few rows alone: two key heads of 64 channels a time (`two` is 0: no)
};
int launch_paged_attn_ranges(const ModLaunch& a, hipStream_t st);
int launch_paged_attn_capped(const ModLaunch& a, hipStream_t st);
int launch_paged_attn_biased(const ModLaunch& a, hipStream_t st);

}  // namespace serq
