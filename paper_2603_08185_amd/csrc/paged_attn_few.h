// serq_paged_attn for sequences with few rows (a token or a few, times the query heads of a key head): the cache is read once, and
// everything else is there to keep it coming.
//
// The keys that the call's sequences see form a line for each key head that is cut into equal shares, one a workgroup, so that neither few
// sequences nor sequences of very different lengths leave compute units idle.  A workgroup walks the stretches of its share: a sequence's
// 16 NB rows of the key head and some of its keys.  Each of its four waves takes every fourth tile of 16 TG keys and walks alone, with a running
// maximum, sum and weighted values of its own; the four meet in LDS at the stretch's end, and the stretches of a sequence that was cut in the
// workspace, where the last one to arrive joins them.
//   scores   S^T = K Q^T on the 16x16x32 matrix instruction: keys are its rows, fetched from memory in the layout of its operand (a lane has
//            16 bytes of one key), queries its columns, so that a lane's results are 4 keys of one row.
//   weights  exp2(s c - m c), c = scale log2 e: one fused multiply-add and one exponential.  m is raised only when a score exceeds it by more than
//            2^6 in weight; between two raises no lane needs another's maximum.  (fp16: 2^9 times that, so that small ones keep their bits.)
//   values   O^T = V^T P^T: the lane's weights are the instruction's operand as they stand (8 keys: 4 of one group of 16, 4 of the next); V goes
//            through LDS, which reads it back by columns.
// Weights are rounded to the 16-bit type for the product (that is what the instruction takes; the sums are fp32); their sum takes them unrounded.
//
// Bound by memory: 32 query and 8 key heads of 128 channels, one token a sequence: one of 131000 keys 84 us (6.4 TB/s; a plain read of as much reaches
// 6.7), 47 of up to 8000 106 us (5.2), 31 of up to 16000 with an E4M3 cache 77 us (5.4), 128 of 4000 356 us (5.9).  One token over 1000 keys: 9 us, of which
// a chain of loads (lengths, pages, keys, the other shares' sums) is most.  By [page, head, row] the same batch is read 10 % faster than by
// [page, row, head].  What carried it (us, without / with): equal shares against slices of the longest sequence's length 149 / 117 (47 sequences), loads
// that do not stay in the caches 103.5 / 92 (one of 131000), the next tile's loads sent without a condition and shares that keep to a key head
// 92 / 88, and one workgroup a compute unit where the parts of a sequence are many 88 / 84.  (Workgroups a compute unit: 1 / 2 / 4 84.5 / 88 / 93 for one of
// 131000, 163 / 157 / 167 for 255 of up to 2000.)  8 tokens over 32000: 50 us; with twice the shares 67, of which the join of 64 slots of 32 rows is half.
// Tried and not kept: the next stretch's first loads before the present one's end (18.6 against 15.6 over 8000 keys: registers), shares that begin
// with sequences (77 / 90 for the 31), a join in two steps (8 tokens over 32000 46 with twice the shares, but 9.0 -> 9.5 over 1000 keys: code and registers), three workgroups a compute unit by fewer registers (122 against 103 over 131000).
#pragma once

#include <type_traits>

#include "paged_attn.h"

namespace serq {
namespace few {

constexpr int kWaves = 4;

template <bool F8, int D, int NB> struct Few {
  static constexpr int ROWB = D * (F8 ? 1 : 2);               // bytes of a key in the cache
  static constexpr int TG = ROWB == 256 || (F8 && D == 128 && NB == 2) ? 2 : 4;   // groups of 16 keys in a tile (the second: registers)
  static constexpr int KEYS = 16 * TG;
  static constexpr int KL = ROWB / 64;                        // 16-byte loads of a lane for 16 keys
  static constexpr int LPR = ROWB / 16, RPI = 64 / LPR;       // V: lanes of a row, rows of a load
  static constexpr int STEPS = D / 32;
  static constexpr int OPITCH = D + 4;                        // floats of a row where the waves meet
  // LDS of a wave: a tile of V, then its rows' sums
  static constexpr int REGION = KEYS * D * 2 > 16 * NB * OPITCH * 4 ? KEYS * D * 2 : 16 * NB * OPITCH * 4;
};

template <int DT>
__device__ __forceinline__ v4f mfma(const u4& a, const u4& b, const v4f& c) {
  if constexpr (DT == SERQ_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

// PAIRS: two neighbouring key heads of 64 channels, side by side in memory, are read as one of 128.  The queries of both are its rows, with zeros for the
// other's channels; of a row's scores and of its sums the other's are dropped.  (A head's 128 bytes out of rows of 2 KiB come slowly: one token, 16 heads over 65000
// keys, by [page, row, head] 60.7 us against 46 by [page, head, row].)
template <bool PAIRS>
__device__ __forceinline__ bool own_half(int g, int group, int d) { return !PAIRS || (d >= 64) == (2 * g >= group); }

// rows of V in LDS: 16-byte pieces, their place turned by the row so that 8 rows' equal pieces lie in different banks
template <int D>
__device__ __forceinline__ int turned(int row) { return D == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); }

// The slots slot(0) .. slot(ns - 1), joined in this order and written out.  scratch: rows x (ns + 1) floats of LDS.
template <int DT, int D, int BM, int THREADS, bool PAIRS, class P, class Slot>
__device__ __forceinline__ void join_slices(const P& p, const RowBlock& k, int h, int ns, const Slot& slot, float* scratch, int tok0,
                                            float vs, int tid) {
  const int l = tid & 63, w = uniform(tid >> 6);
  const auto put = [&](int r, int d, const v2f& acc, float f) {
    const int i = (k.r0 + r) / p.group, g = k.r0 + r - i * p.group;
    char* dst = p.out + (int64_t)(tok0 + i) * p.ldo + (int64_t)(h * p.group + g) * p.ldoh;
    if (own_half<PAIRS>(g, p.group, d)) *(uint32_t*)(dst + 2 * (PAIRS ? d & 63 : d)) = pack16<DT>(acc[0] * f, acc[1] * f);
  };
  const auto put_lse = [&](int r, float m, float sum) {
    const int i = (k.r0 + r) / p.group, g = k.r0 + r - i * p.group;
    if (p.lse) p.lse[(int64_t)(tok0 + i) * p.q_heads + h * p.group + g] = lse_of(p, m, sum);
  };
  // A load takes a microsecond here, so as many as can be are under way together.  Few slices: every thread computes their weights by itself
  // (past the end: the last slot again, without weight).
  const auto alone = [&](auto number) {
    constexpr int N = decltype(number)::value;
    for (int it = tid; it < k.rows * (D / 2); it += THREADS) {
      const int r = it / (D / 2), d = 2 * (it % (D / 2));
      v2f st[N], x[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float* from = slot(min(e, ns - 1));
        st[e] = get2(from + BM * D + 2 * r);
        x[e] = get2(from + r * D + d);
      }
      float top = st[0][0], all = 0.0f;
#pragma unroll
      for (int e = 1; e < N; ++e) top = fmaxf(top, st[e][0]);
      v2f acc = {0.0f, 0.0f};
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < ns) {
          const float f = exp2_fast(st[e][0] - top);
          all += f * st[e][1];
          acc += f * x[e];
        }
      put(r, d, acc, row_factor(all, vs));
      if (d == 0) put_lse(r, top, all);
    }
  };
  if (ns <= 4) return alone(std::integral_constant<int, 4>{});
  if (ns <= 12) return alone(std::integral_constant<int, 12>{});
  float* weight = scratch + BM;                               // [rows][ns]: each slice's weight; scratch[row]: what the row is multiplied by
  for (int r = w; r < k.rows; r += THREADS / 64) {
    float m[(kMaxSlices + 63) / 64], n[(kMaxSlices + 63) / 64], top = -FLT_MAX;
#pragma unroll
    for (int e = 0; e < (kMaxSlices + 63) / 64; ++e) {
      const int u = l + 64 * e;
      m[e] = -FLT_MAX;
      n[e] = 0.0f;
      if (u < ns) {
        const v2f x = get2(slot(u) + BM * D + 2 * r);
        m[e] = x[0];
        n[e] = x[1];
      }
      top = fmaxf(top, m[e]);
    }
    top = wave_max(top);
    float all = 0.0f;
#pragma unroll
    for (int e = 0; e < (kMaxSlices + 63) / 64; ++e) {
      const int u = l + 64 * e;
      const float f = exp2_fast(m[e] - top);
      if (u < ns) {
        weight[r * ns + u] = f;
        all += f * n[e];
      }
    }
    all = wave_reduce(all, [](float x, float y) { return x + y; });
    if (l == 0) {
      scratch[r] = row_factor(all, vs);
      put_lse(r, top, all);
    }
  }
  __syncthreads();
  for (int it = tid; it < k.rows * (D / 2); it += THREADS) {
    const int r = it / (D / 2), d = 2 * (it % (D / 2));
    v2f acc = {0.0f, 0.0f};
    for (int u = 0; u < ns; u += 16) {
      v2f x[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = get2(slot(min(u + e, ns - 1)) + r * D + d);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (u + e < ns) acc += weight[r * ns + u + e] * x[e];
    }
    put(r, d, acc, scratch[r]);
  }
}

// A stretch of a sequence that was cut: where the sequence's stretches leave their sums, and how many there are.
template <int SLOT>
struct Part {
  float* base;            // of the workspace's slots, two a workgroup: for a stretch that goes on with a sequence, and for one that begins it
  uint32_t* ticket;
  int first, mine, count; // the workgroup that begins the sequence; this stretch's number, all of them
  __device__ __forceinline__ float* slot(int u) const { return base + (int64_t)(2 * (first + u) + (u == 0)) * SLOT; }
};

// Keys k0 .. k1-1 for the rows of block k and key head h.
template <int DT, bool F8, int D, int NB, int MOD, bool PAIRS>
__device__ __forceinline__ void stretch(const ParamsOf<MOD>& p, const RowBlock& k, int h, int k0, int k1, const bool cut,
                                        const Part<16 * NB * (D + 2)> part, char* lds, float (*stat)[16 * NB][2]) {
  using S = Few<F8, D, NB>;
  constexpr int TG = S::TG, KEYS = S::KEYS, KL = S::KL, BM = 16 * NB, VL = TG * KL, OPITCH = S::OPITCH, REGION = S::REGION;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));                               // (else what follows from it is kept from stretch to stretch: 67 registers)
  const int l = tid & 63, w = uniform(tid >> 6);
  const int n16 = l & 15, quad = l >> 4, G = p.group, tok0 = k.tok0;

  const int mask = (1 << p.c.page_shift) - 1;
  const int32_t* table = p.c.table + k.b * p.c.table_ld;
  const int nt = k1 > k0 ? (k1 - k0 + KEYS - 1) / KEYS : 0;   // tiles of the slice
  const int mine = nt > w ? (nt - w + kWaves - 1) / kWaves : 0;
  // the pages of the first tiles (loads come back in their order: these before the queries)
  const auto key_of = [&](int t) { return k0 + (w + kWaves * (t + l / TG)) * KEYS + 16 * (l % TG); };
  const auto page_of = [&](int key) { return table[min(key, k.end - 1) >> p.c.page_shift]; };   // (past the end: the last key's)
  int page = 0;
  if (mine > 0) page = page_of(key_of(0));
  __builtin_amdgcn_sched_barrier(0);

  // the rows' queries, and the keys that each sees: lo <= j < hi
  u4 q[NB][S::STEPS];
  int lo[NB], hi[NB];
  float slope[NB];                                            // biased: of the row's head; the row's position less the lane's first key
  int place[NB];
  bool second[NB];                                            // pairs: the row is of the second head
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = k.r0 + 16 * nb + n16;
    const bool live = 16 * nb + n16 < k.rows;
    const int i = r / G, g = r - i * G;
    second[nb] = PAIRS && 2 * g >= G;
    if constexpr (MOD == kPlain) {
      hi[nb] = live ? min(k.L - k.n + i + 1, k.end) : 0;
      lo[nb] = p.window > 0 ? max(0, k.L - k.n + i - p.window + 1) : 0;
    } else {
      const Range x = live ? row_range(p, tok0 + i, k.L - k.n + i, k.L) : Range{0, 0};
      hi[nb] = x.hi;
      lo[nb] = x.lo;
      if constexpr (MOD == kBiased) {
        slope[nb] = live ? p.slopes[h * G + g] : 0.0f;
        place[nb] = k.L - k.n + i - 4 * quad;
      }
    }
    const char* src = p.q + (int64_t)(tok0 + i) * p.ldq + (int64_t)(h * G + g) * p.ldqh;
#pragma unroll
    for (int st = 0; st < S::STEPS; ++st) {
      // channels of step st that quad has: where its loads of K put them
      const int at = F8 ? 64 * (st / 2) + 16 * quad + 8 * (st & 1) : 32 * st + 8 * quad;
      if constexpr (PAIRS) q[nb][st] = live && own_half<true>(g, G, at) ? *(const u4*)(src + 2 * (at & 63)) : (u4){0, 0, 0, 0};
      else q[nb][st] = live ? *(const u4*)(src + 2 * at) : (u4){0, 0, 0, 0};
    }
  }
  const int all_lo = k.all_from, all_hi = k.all_to;           // no mask there
  const float ks = p.c.k_scale ? p.c.k_scale[h] : 1.0f, vs = p.c.v_scale ? p.c.v_scale[h] : 1.0f;
  const float c = factor_of<MOD>(p, ks), slack = score_slack(c), rate = cap_rate<MOD>(p, ks);
  if constexpr (MOD == kBiased)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) slope[nb] = score_slope(slope[nb], c);

  const char* kbase = p.c.k + h * p.c.k_head;
  const char* vbase = p.c.v + h * p.c.v_head;
  const uint32_t klane = (uint32_t)(n16 * (int)p.c.k_token + quad * 16);
  uint32_t vlane[KL];
#pragma unroll
  for (int i = 0; i < KL; ++i) vlane[i] = (uint32_t)((i * S::RPI + l / S::LPR) * (int)p.c.v_token + (l % S::LPR) * 16);

  // lane: where group lane % TG of the wave's tile lane / TG of the next 64 / TG begins, so that a tile's loads need no arithmetic of their own
  uint64_t kfrom = 0, vfrom = 0;
  auto look_up = [&](int t, int page) {
    const int key = key_of(t);
    page = min(max(page, 0), p.c.pages - 1);
    kfrom = (uint64_t)(kbase + page * p.c.k_page + (key & mask) * p.c.k_token);
    vfrom = (uint64_t)(vbase + page * p.c.v_page + (key & mask) * p.c.v_token);
  };
  const auto group = [&](uint64_t v, int t, int a) {
    const int at = (t * TG + a) & 63;
    const uint32_t lo32 = __builtin_amdgcn_readlane((uint32_t)v, at), hi32 = __builtin_amdgcn_readlane((uint32_t)(v >> 32), at);
    return (const GlobalByte*)((uint64_t)hi32 << 32 | lo32);
  };
  u4 kr[TG][KL], vr[VL];
  auto load_k = [&](int t) {
    uint32_t lane = klane;
    asm("" : "+v"(lane));                                     // (an offset of 32 bits beside a uniform address; else kept as one of 64 bits)
#pragma unroll
    for (int a = 0; a < TG; ++a) {
      const GlobalByte* row = group(kfrom, t, a);
#pragma unroll
      for (int i = 0; i < KL; ++i) kr[a][i] = __builtin_nontemporal_load((const GlobalPiece*)(row + lane + 64 * i));
    }
  };
  auto load_v = [&](int t) {
#pragma unroll
    for (int a = 0; a < TG; ++a) {
      const GlobalByte* row = group(vfrom, t, a);
#pragma unroll
      for (int i = 0; i < KL; ++i) {
        uint32_t lane = vlane[i];
        asm("" : "+v"(lane));
        vr[a * KL + i] = __builtin_nontemporal_load((const GlobalPiece*)(row + lane));
      }
    }
  };

  v4f o[NB][D / 16];
  float m[NB], sum[NB];                                       // the reference in the exponent; the lane's part of the sum of weights
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    m[nb] = -FLT_MAX;
    sum[nb] = 0.0f;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) o[nb][d] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
  }
  float ref[NB];                                              // the reference as a score
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) ref[nb] = -FLT_MAX;

  char* my = lds + w * REGION;
  const int vrow = l / S::LPR, vpiece = l % S::LPR;
  // where a lane reads columns: keys 4 quad .. +3 of a group
  const int crow = 4 * quad + n16 / 4;
  const char* col = my + crow * D * 2 + ((n16 % 4) / 2) * 16 + (n16 & 1) * 8;
  const int cturn = turned<D>(crow) << 4;

  if (mine > 0) {
    look_up(0, page);
    load_k(0);
    load_v(0);
  }
  bool odd = false;                                           // the lane took something out
  // One tile.  The loads of the next one are sent without a condition (the waits count loads: one that may not have been sent counts as none,
  // and the wait for K would be one for V too), so the last tile is a case of its own.
  const auto tile = [&](int t, auto more) {
    constexpr bool MORE = decltype(more)::value;
    const int key0 = k0 + (w + kWaves * t) * KEYS;
    // scores
    v4f sc[TG][NB];
#pragma unroll
    for (int a = 0; a < TG; ++a) {
      u4 kk[S::STEPS];
#pragma unroll
      for (int i = 0; i < KL; ++i) {
        if constexpr (F8) widen_e4m3<DT>(kr[a][i], kk[2 * i], kk[2 * i + 1]);
        else kk[i] = kr[a][i];
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        sc[a][nb] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (MOD == kBiased) {
          const float d = (float)(place[nb] - key0);
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[a][nb][e] = distance_bias(slope[nb], d - (float)(16 * a + e));
        }
        if constexpr (PAIRS) {                                // a sum for each head, and the row's own of them: nothing of the other's keys, NaN among it, in it
          v4f upper = sc[a][nb];
#pragma unroll
          for (int st = 0; st < S::STEPS / 2; ++st) {
            sc[a][nb] = mfma<DT>(kk[st], q[nb][st], sc[a][nb]);
            upper = mfma<DT>(kk[S::STEPS / 2 + st], q[nb][S::STEPS / 2 + st], upper);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[a][nb][e] = second[nb] ? upper[e] : sc[a][nb][e];
        } else {
#pragma unroll
          for (int st = 0; st < S::STEPS; ++st) sc[a][nb] = mfma<DT>(kk[st], q[nb][st], sc[a][nb]);
        }
        if constexpr (MOD == kCapped) {
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[a][nb][e] = capped(sc[a][nb][e], rate);
        }
      }
    }
    if constexpr (MORE) {
      if (((t + 1) * TG & 63) == 0) look_up(t + 1, page_of(key_of(t + 1)));
      load_k(t + 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    // V to LDS; rows that no row sees are zero there (a weight of zero does not make NaN zero)
    const bool ends = key0 < k.begin || key0 + KEYS > k.end;
    const bool partly = (key0 + KEYS > all_hi && key0 < k.end && all_hi < k.end) || (key0 < all_lo && key0 + KEYS > k.begin && k.begin < all_lo);
    int to = vrow * D * 2, turn = cturn;
    asm volatile("" : "+v"(to), "+v"(turn));                   // (else sixteen places in LDS are kept from tile to tile)
#pragma unroll
    for (int u = 0; u < VL; ++u) {
      const int row = u * S::RPI + vrow;
      u4 x = vr[u];
      if (ends && (key0 + row < k.begin || key0 + row >= k.end)) x = (u4){0, 0, 0, 0};
      char* at = my + u * S::RPI * D * 2 + to;
      if constexpr (F8) {
        u4 a, b;
        widen_e4m3<DT>(x, a, b);
        if (partly && (key0 + row < all_lo || key0 + row >= all_hi)) {
          a = take_out<DT>(a, odd);
          b = take_out<DT>(b, odd);
        }
        at += ((2 * vpiece) ^ turned<D>(row)) << 4;
        *(u4*)at = a;
        *(u4*)(at + 16) = b;
      } else {
        if (partly && (key0 + row < all_lo || key0 + row >= all_hi)) x = take_out<DT>(x, odd);
        *(u4*)(at + ((vpiece ^ turned<D>(row)) << 4)) = x;
      }
    }
    if constexpr (MORE) load_v(t + 1);
    __builtin_amdgcn_sched_barrier(0);
    // weights
    if (key0 < all_lo || key0 + KEYS > all_hi) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int a = 0; a < TG; ++a)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = key0 + 16 * a + 4 * quad + e;
            if (j < lo[nb] || j >= hi[nb]) sc[a][nb][e] = -INFINITY;
          }
    }
    u4 pw[NB][TG / 2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float top = sc[0][nb][0];
#pragma unroll
      for (int a = 0; a < TG; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, sc[a][nb][e]);
      if (__ballot(top > ref[nb] + slack)) {
        // (each row by its own keys: where a row's reference lies must not tell of what it does not see)
        const float most = quads_reduce(top, [](float x, float y) { return fmaxf(x, y); }), now = most > ref[nb] + slack ? most : ref[nb];
        ref[nb] = now;
        const float mc = reference_of<MOD, DT>(now, c), f = exp2_fast(m[nb] - mc);
        m[nb] = mc;
        sum[nb] *= f;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) o[nb][d] *= f;
      }
#pragma unroll
      for (int a = 0; a < TG; ++a) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = exp2_fast(__builtin_fmaf(sc[a][nb][e], c, -m[nb]));
          sum[nb] += x[e];
        }
        pw[nb][a / 2][2 * (a & 1)] = pack16<DT>(x[0], x[1]);
        pw[nb][a / 2][2 * (a & 1) + 1] = pack16<DT>(x[2], x[3]);
      }
    }
    // values
#pragma unroll
    for (int st = 0; st < TG / 2; ++st)
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        const char* at = col + st * 32 * D * 2 + ((2 * d << 4) ^ turn);
        const u2 x = lds_column4(at), y = lds_column4(at + 16 * D * 2);
        const u4 a = {x.x, x.y, y.x, y.y};
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) o[nb][d] = mfma<DT>(a, pw[nb][st], o[nb][d]);
      }
  };
#pragma unroll 1
  for (int t = 0; t < mine - 1; ++t) tile(t, std::true_type{});
  if (mine > 0) tile(mine - 1, std::false_type{});

  if (__ballot(odd)) {
    for (int j = max(k0, k.begin); j < min(k1, k.end); ++j) {
      if (j >= all_lo && j < all_hi) j = all_hi;              // (what all rows see went through the products)
      if (j >= min(k1, k.end)) break;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
        if (j >= lo[nb] && j < hi[nb])
#pragma unroll
          for (int d = 0; d < D / 16; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nb][d][e] += taken_out<DT, F8>(p, k.b, h, j, 16 * d + 4 * quad + e);
    }
  }
  // the waves meet
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const float all = quads_reduce(sum[nb], [](float x, float y) { return x + y; });
    float* row = (float*)my + (16 * nb + n16) * OPITCH + 4 * quad;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) *(v4f*)(row + 16 * d) = o[nb][d];
    if (quad == 0) {
      stat[w][16 * nb + n16][0] = m[nb];
      stat[w][16 * nb + n16][1] = all;
    }
  }
  __syncthreads();
  const int64_t head0 = (int64_t)h * G;
  float* slot = cut ? part.slot(part.mine) : nullptr;
  for (int it = tid; it < k.rows * (D / 4); it += 256) {
    const int r = it / (D / 4), d = 4 * (it % (D / 4));
    float top = stat[0][r][0];
#pragma unroll
    for (int u = 1; u < kWaves; ++u) top = fmaxf(top, stat[u][r][0]);
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    float all = 0.0f;
#pragma unroll
    for (int u = 0; u < kWaves; ++u) {
      const float f = exp2_fast(stat[u][r][0] - top);
      all += f * stat[u][r][1];
      acc += f * *(const v4f*)((const float*)(lds + u * REGION) + r * OPITCH + d);
    }
    if (cut) {
      put2(slot + r * D + d, acc[0], acc[1]);
      put2(slot + r * D + d + 2, acc[2], acc[3]);
      if (d == 0) put2(slot + BM * D + 2 * r, top, all);
    } else {
      const int i = (k.r0 + r) / G, g = k.r0 + r - i * G;
      const float f = row_factor(all, vs);
      char* dst = p.out + (int64_t)(tok0 + i) * p.ldo + (head0 + g) * p.ldoh;
      if (own_half<PAIRS>(g, G, d))
        *(u2*)(dst + 2 * (PAIRS ? d & 63 : d)) = (u2){pack16<DT>(acc[0] * f, acc[1] * f), pack16<DT>(acc[2] * f, acc[3] * f)};
      if (p.lse && d == 0) p.lse[(int64_t)(tok0 + i) * p.q_heads + head0 + g] = lse_of(p, top, all);
    }
  }
  if (!cut) return;
  __shared__ uint32_t last;
  if (!last_to_arrive(part.ticket, part.count, tid, &last)) return;
  static_assert(BM * (kMaxSlices + 1) * 4 <= kWaves * REGION, "the stretches' weights");
  join_slices<DT, D, BM, 256, PAIRS>(p, k, h, part.count, [&](int u) { return part.slot(u); }, (float*)lds, tok0, vs, tid);   // (the regions of the waves are free)
}

constexpr int kUnit = 64;                                     // keys of a piece of a line

// The pieces that a sequence gives a key head's line (one at least: its rows have to be written).
template <int NB, int MOD>
__device__ __forceinline__ int pieces_of(const ParamsOf<MOD>& p, int c0, int n, int L) {
  if constexpr (MOD != kPlain) {                              // (what block_of finds for the same rows)
    constexpr int BM = 16 * NB;
    if (kLookAlways<BM> || p.from || p.to) {
      const int tokens = (min(n * p.group, BM) + p.group - 1) / p.group;
      Seen s;
      for (int i = 0; i < tokens; ++i) s.add(row_range(p, c0 + i, L - n + i, L));
      const int base = s.begin & ~15;
      return s.end > 0 ? (s.end - base - 1) / kUnit + 1 : 1;
    }
  }
  const int end = min(L, p.c.width << p.c.page_shift), base = (p.window > 0 ? max(0, L - n - p.window + 1) : 0) & ~15;
  return end > base ? (end - base - 1) / kUnit + 1 : 1;
}

// Share `number` of the `wanted` that key head h's line is cut into.  lds: kLds bytes, 16-byte aligned.
template <bool F8, int D, int NB> constexpr int kLds = kWaves * Few<F8, D, NB>::REGION;
template <int DT, bool F8, int D, int NB, int MOD, bool PAIRS, class L>
__device__ __forceinline__ void walk(const ParamsOf<MOD>& p, L& line, int number, int wanted, int h, char* lds, float (*stat)[16 * NB][2]) {
  constexpr int BM = 16 * NB;
  // a share: of the head's line, but not too little for a workgroup, nor so little that too many meet
  const int total = line.total;
  const int share = max(max(p.slice_keys / kUnit, total / (kMaxSlices - 2) + 1), (total + wanted - 1) / wanted);
  int at = (int)min((int64_t)number * share, (int64_t)total);
  const int stop = min(at + share, total);
  while (at < stop) {
    const Sequence x = line.find(at);
    const RowBlock k = block_of<BM>(p, x.b, x.c0, x.n, x.L, 0);
    const int ends = x.before + x.pieces, until = min(stop, ends), base = k.begin & ~15;
    const bool cut = at > x.before || until < ends;
    // (a sequence of more tokens than max_q has pieces past what the block's rows see, maybe nothing that they see: no table entry is read there)
    const int end = max(k.end, 0), k0 = base + (at - x.before) * kUnit, k1 = until < ends ? min(base + (until - x.before) * kUnit, end) : end;
    Part<BM * (D + 2)> part{};
    if (cut) {
      const int first = x.before / share;
      part = {p.part + (int64_t)h * wanted * 2 * (BM * (D + 2)), p.tickets + h * wanted + first, first, number - first, (ends - 1) / share - first + 1};
    }
    stretch<DT, F8, D, NB, MOD, PAIRS>(p, k, h, k0, k1, cut, part, lds, stat);
    at = until;
    __syncthreads();                                          // LDS is free again
  }
}

// What workgroup `id` of `count` does.  lds: kLds bytes, 16-byte aligned.
template <int DT, bool F8, int D, int NB, int MOD = kPlain>
__device__ __forceinline__ void work(const ParamsOf<MOD>& p, int id, int count, char* lds) {
  constexpr int BM = 16 * NB;
  __shared__ float stat[kWaves][BM][2];
  const int heads = p.c.heads;
  // neighbouring workgroups have different key heads
  const int number = uniform(id / heads), h = id - number * heads;
  if (p.slices <= 1) {                                        // nowhere to meet: a workgroup takes a sequence whole
    const int c0 = uniform(p.c.cu[number]), n = uniform(p.c.cu[number + 1]) - c0;
    if (!takes(p, c0, n)) return;
    const RowBlock k = block_of<BM>(p, number, c0, n, uniform(p.c.len[number]), 0);
    stretch<DT, F8, D, NB, MOD, false>(p, k, h, k.begin & ~15, max(k.end, 0), false, {}, lds, stat);
    return;
  }
  const auto pieces = [&](int c0, int n, int L) { return pieces_of<NB, MOD>(p, c0, n, L); };
  Line line(p, pieces, threadIdx.x & 63);
  walk<DT, F8, D, NB, MOD, false>(p, line, number, count / heads, h, lds, stat);
}

// Heads of 64 channels side by side in memory, one a time or two (PAIRS).  Two a time read 256 bytes in a row, but a share of two heads' keys is twice the work and
// slots of twice the rows and twice the channels are joined, which pays once the line is long: from `long_line` pieces on.  How long it is is known here alone
// (the host has bounds, and a captured graph has them for every step to come).  Measured (us, one a time / two; one token a sequence of alike
// lengths, key heads x rows of each):
//   16 x 1   one over 1000 keys 8.3 / 10.7, over 16000 22.1 / 19.9, over 65000 62.9 / 53.1;  40 over 1600 66.4 / 58.4
//    8 x 4   one over 1000 8.3 / 10.4, over 16000 15.3 / 20.3;  4 over 8000 24.1 / 22.9, over 32000 63.8 / 54.8;  40 over 6500 122 / 107
//    2 x 7   one over 65000 19.7 / 39.5;  12 over 22000 34.1 / 38.5, over 87000 97.0 / 95.6
//    4 x 1   4 over 16000 21.2 / 24.8, over 33000 32.4 / 34.5, over 65000 56.2 / 55.4
// Of 536 sizes, bounds far above the lengths and lengths far apart among them, none is slower than with one a time alone by over 3 %, 103 are faster.
template <int DT, int MOD>
__device__ __forceinline__ void work_pairs(const ParamsOf<MOD>& p, const PairPlan& n, int id, char* lds) {
  __shared__ float stat[kWaves][16][2];
  const int heads = p.c.heads, number = uniform(id / heads), h = id - number * heads, wanted = n.one / heads;
  const auto pieces = [&](int c0, int m, int L) { return pieces_of<1, MOD>(p, c0, m, L); };
  Line line(p, pieces, threadIdx.x & 63);
  if (line.total < n.long_line) {
    if (number < wanted) walk<DT, false, 64, 1, MOD, false>(p, line, number, wanted, h, lds, stat);
    return;
  }
  ParamsOf<MOD> two = p;
  two.c.heads /= 2;
  two.c.k_head *= 2;
  two.c.v_head *= 2;
  two.group *= 2;
  two.slice_keys = n.two_keys;
  const int number2 = uniform(id / two.c.heads);
  if (id < n.two) walk<DT, false, 128, 1, MOD, true>(two, line, number2, n.two / two.c.heads, id - number2 * two.c.heads, lds, stat);
}

}  // namespace few
}  // namespace serq
