// serq_paged_attn for sequences with many rows (chunks, prompts): bound by the matrix instructions and the exponentials between them.
//
// A workgroup takes 128 rows of a key head -- its four waves 32 each -- and a slice of the keys, in tiles of 64.  K and V of a tile lie in LDS, two
// tiles deep: while one is used, the next is on its way (straight to LDS for 16-bit caches; through registers, where they become 16-bit
// values, for E4M3 ones).  The scores of the next tile are computed while the present one's become weights: a matrix instruction, a pair of
// weights, the load of an operand some instructions further on, and so forth (in that order by hand: the compiler's put each operand's load
// right before its use).
//   scores   S^T = K Q^T on the 32x32x16 instruction: a lane's results are 16 of 32 keys of one row, the other 16 are with the lane 32 further.
//   weights  as in the kernel for few rows: exp2(s c - m c), m raised only when a score exceeds it by more than 2^6 in weight.
//   values   O^T = V^T P^T: the weights are the instruction's operand as they stand (eight registers of scores become one operand of 16 keys in
//            the order 4h .. 4h+3, 8+4h .. 8+4h+3), and V is read by columns in the same order.
// The 16-byte pieces of a row in LDS are turned by the row's number, so that the lanes that read together meet different banks.
//
// 32 query and 8 key heads of 128 channels: a prompt of 8192 tokens 482 to 501 us (1.10 to 1.14 PFLOP/s; a large bf16 matrix product reaches 1.4 to 1.6), 512
// tokens after 32000 247 to 258 us (1.05 to 1.10), 4096 131 to 135 us (1.02 to 1.05); E4M3 cache 529 to 535, 64 channels 295 to 303 (0.91 to 0.93: as many
// exponentials for half the products).  The clock falls as the matrix units get busier (of 2.4 GHz: 2.0 where they are busy in 47 % of the cycles, with an E4M3
// cache, 1.78 at 56 %, 512 after 32000, 1.73 at 60 %, the prompt): what the kernel saves in cycles, power takes back in part.  What carried it (us, before / after, prompt of 8192 unless stated): loads four
// products ahead and the next scores beside the weights 538 / 518, the largest score beside the products with V 528 / 524, the wave
// at its weights before the one at its products 524 / 506 (512 after 32000: 278 / 258).  Two waves share a SIMD, of two workgroups, so that
// one is at the exponentials while the other multiplies.
// Tried and not kept: eight waves on a tile, which halves the loads (511 against 508, E4M3 564 against 536), 64 rows a wave (530 registers spilled), some
// of the weights beside the products with V (493 against 492), six operands ahead (487 against 484).  Without any loads it takes 451 of 518.
#pragma once

#include <type_traits>

#include "paged_attn.h"

namespace serq {
namespace tile {

constexpr int kKeys = 64;

template <int DT>
__device__ __forceinline__ v16f mfma(const u4& a, const u4& b, const v16f& c) {
  if constexpr (DT == SERQ_BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

// places of the 16-byte pieces of a row: K is read 16 bytes a row by 16 rows at a time, V 64 bytes a row by 4
template <int D> __device__ __forceinline__ int turn_k(int row) { return D == 128 ? row & 15 : row & 7; }
template <int D> __device__ __forceinline__ int turn_v(int row) { return D == 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1); }

// N loads straight to LDS, 1 KiB each, one behind the other; from + voff[u] + 1024 u is what the lane brings
template <int N>
__device__ __forceinline__ void dma_rows(const char* from, const uint32_t (&voff)[N], uint32_t to) {
  static_assert(N == 2 || N == 4, "loads of a wave");
  if constexpr (N == 4)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\tglobal_load_lds_dwordx4 %2, %5 offset:1024\n\t"
                 "global_load_lds_dwordx4 %3, %5 offset:2048\n\tglobal_load_lds_dwordx4 %4, %5 offset:3072"
                 :: "s"(to), "v"(voff[0]), "v"(voff[1]), "v"(voff[2]), "v"(voff[3]), "s"(from) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\tglobal_load_lds_dwordx4 %2, %3 offset:1024"
                 :: "s"(to), "v"(voff[0]), "v"(voff[1]), "s"(from) : "memory", "m0");
}

// What workgroup `id` does.  lds: kLds bytes, 16-byte aligned: K, then V of two tiles.
template <int D> constexpr int kLds = 2 * 2 * kKeys * D * 2;
template <int DT, bool F8, int D, int MOD = kPlain>
__device__ __forceinline__ void work(const ParamsOf<MOD>& p, int id, char* lds_all) {
  constexpr int NW = kTileRows / 32, BM = kTileRows;          // waves
  constexpr int ROW = D * 2;                                  // bytes of a key in LDS
  constexpr int TILE = kKeys * ROW;                           // of K or of V
  constexpr int STEPS = D / 16, DB = D / 32;
  constexpr int ROWB = F8 ? D : 2 * D;                        // bytes of a key in the cache
  constexpr int LPR = ROWB / 16, RPI = 64 / LPR;              // lanes of a row, rows of a load of 64 lanes
  constexpr int LOADS = kKeys / RPI / NW;                     // loads of a wave for a tile of K
  static_assert(LOADS >= 1 && LOADS * RPI <= 16, "a wave's rows lie in one page");
  char (*const lds)[2][TILE] = reinterpret_cast<char (*)[2][TILE]>(lds_all);   // [buffer][K, V]

  const int tid = threadIdx.x, l = tid & 63, w = uniform(tid >> 6);
  const int n32 = l & 31, half = l >> 5;
  const int G = p.group;
  // a sequence's pieces of work are blocks of BM rows; those that see most keys come last and start first; neighbouring workgroups have different
  // key heads
  const auto pieces = [&](int, int n, int) { return (n * G + BM - 1) / BM; };
  Line line(p, pieces, l);
  // (workgroups without work are the last of the grid: between the others they would make two of these meet on a compute unit)
  const int unit = uniform(id / p.c.heads), h = id - unit * p.c.heads, number = unit / p.slices, s = unit - number * p.slices;
  if (number >= line.total) return;
  const int block = line.total - 1 - number;
  const Sequence seq = line.find(block);
  const RowBlock k = block_of<BM>(p, seq.b, seq.c0, seq.n, seq.L, (block - seq.before) * BM);
  const int base = k.begin & ~15;
  const int ns = k.end > base ? min((k.end - base - 1) / p.slice_keys + 1, p.slices) : 1;
  if (s >= ns) return;
  const int k0 = base + s * p.slice_keys, k1 = s == ns - 1 ? k.end : k0 + p.slice_keys;
  const int tok0 = k.tok0;

  // the lane's row, and the keys that it sees: lo <= j < hi
  const int rin = 32 * w + n32, r = k.r0 + rin;
  const bool live = rin < k.rows;
  const int i = r / G, g = r - i * G;
  const int first = k.L - k.n;
  int hi, lo;
  if constexpr (MOD == kPlain) {
    hi = live ? min(first + i + 1, k.end) : 0;
    lo = p.window > 0 ? max(0, first + i - p.window + 1) : 0;
  } else {
    const Range x = live ? row_range(p, tok0 + i, first + i, k.L) : Range{0, 0};
    hi = x.hi;
    lo = x.lo;
  }
  u4 q[STEPS];
  {
    const char* src = p.q + (int64_t)(tok0 + i) * p.ldq + (int64_t)(h * G + g) * p.ldqh;
#pragma unroll
    for (int st = 0; st < STEPS; ++st) q[st] = live ? *(const u4*)(src + 32 * st + 16 * half) : (u4){0, 0, 0, 0};
  }
  // keys that all of the wave's rows see: no mask there (a wave without rows: whatever)
  const int wr0 = k.r0 + 32 * w, wr1 = min(k.r0 + k.rows, wr0 + 32) - 1;
  int all_lo, all_hi;
  if constexpr (MOD == kPlain) {
    all_lo = p.window > 0 ? max(0, first + wr1 / G - p.window + 1) : 0;
    all_hi = min(first + wr0 / G + 1, k.end);
  } else {
    all_lo = wave_max_int(live ? lo : 0);
    all_hi = wave_min_int(live ? hi : 0x7fffffff);
  }
  const float ks = p.c.k_scale ? p.c.k_scale[h] : 1.0f, vs = p.c.v_scale ? p.c.v_scale[h] : 1.0f;
  const float c = factor_of<MOD>(p, ks), slack = score_slack(c), rate = cap_rate<MOD>(p, ks);
  float slope = 0.0f;                                         // biased: of the row's head; the row's position less the lane's first key
  const int place = first + i - 4 * half;
  if constexpr (MOD == kBiased) slope = live ? score_slope(p.slopes[h * G + g], c) : 0.0f;
  // what tile t's scores begin with (one multiply-add a score from the tile's first distance would take 541 us for 8192 tokens instead of 551, but leave a
  // steep slope's rounding on the row's own key)
  const auto begin_scores = [&](v16f (&sc)[2], int t) {
    const float d = MOD == kBiased ? (float)(place - (k0 + t * kKeys)) : 0.0f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[kb][e] = MOD == kBiased ? distance_bias(slope, d - (float)(32 * kb + 8 * (e / 4) + e % 4)) : 0.0f;
  };

  // ---- loads: a wave brings LOADS * RPI rows of K and of V, which lie in one page
  const int mask = (1 << p.c.page_shift) - 1;
  const int32_t* table = p.c.table + k.b * p.c.table_ld;
  const char* kbase = p.c.k + h * p.c.k_head;
  const char* vbase = p.c.v + h * p.c.v_head;
  const int nt = k1 > k0 ? (k1 - k0 + kKeys - 1) / kKeys : 0;
  const int wrow = w * LOADS * RPI;
  // lane: where this wave's rows of tile 64 (t / 64) + lane begin, so that a tile's loads need no arithmetic of their own
  uint64_t kfrom = 0, vfrom = 0;
  auto look_up = [&](int t, const char* cache, int64_t page_stride, int64_t token_stride) {
    const int key = k0 + (t + l) * kKeys + wrow;
    const int page = min(max(table[min(key, k.end - 1) >> p.c.page_shift], 0), p.c.pages - 1);
    return (uint64_t)(cache + page * page_stride + (key & mask) * token_stride);
  };
  const auto at_tile = [&](uint64_t v, int t) {
    const uint32_t lo32 = __builtin_amdgcn_readlane((uint32_t)v, t & 63), hi32 = __builtin_amdgcn_readlane((uint32_t)(v >> 32), t & 63);
    return (const char*)((uint64_t)hi32 << 32 | lo32);
  };
  uint32_t ksrc[LOADS], vsrc[LOADS];                          // a lane's place in the rows it brings
#pragma unroll
  for (int u = 0; u < LOADS; ++u) {
    const int row = wrow + u * RPI + l / LPR, piece = l % LPR;
    const int in = u * RPI + l / LPR;
    // (straight to LDS: the instruction's offset counts on both sides, so load u starts u KiB earlier, all of them 3 KiB later)
    const uint32_t back = F8 ? 0 : 3072 - 1024 * u;
    ksrc[u] = (uint32_t)(in * (int)p.c.k_token + ((F8 ? piece : piece ^ turn_k<D>(row)) << 4)) + back;
    vsrc[u] = (uint32_t)(in * (int)p.c.v_token + ((F8 ? piece : piece ^ turn_v<D>(row)) << 4)) + back;
  }
  u4 kr[F8 ? LOADS : 1], vr[F8 ? LOADS : 1];
  auto issue_k = [&](int t) {
    if ((t & 63) == 0) kfrom = look_up(t, kbase, p.c.k_page, p.c.k_token);
    const char* from = at_tile(kfrom, t);
    if constexpr (F8) {
#pragma unroll
      for (int u = 0; u < LOADS; ++u) kr[u] = *(const u4*)(from + ksrc[u]);
    } else {
      dma_rows<LOADS>(from - 3072, ksrc, uniform(lds_addr(&lds[t & 1][0][wrow * ROW])));
    }
  };
  auto issue_v = [&](int t) {
    if ((t & 63) == 0) vfrom = look_up(t, vbase, p.c.v_page, p.c.v_token);
    const char* from = at_tile(vfrom, t);
    if constexpr (F8) {
#pragma unroll
      for (int u = 0; u < LOADS; ++u) vr[u] = *(const u4*)(from + vsrc[u]);
    } else {
      dma_rows<LOADS>(from - 3072, vsrc, uniform(lds_addr(&lds[t & 1][1][wrow * ROW])));
    }
  };
  // E4M3: to LDS as 16-bit values
  auto commit_k = [&](int t) {
    if constexpr (F8) {
#pragma unroll
      for (int u = 0; u < LOADS; ++u) {
        const int row = wrow + u * RPI + l / LPR, piece = l % LPR;
        u4 a, b;
        widen_e4m3<DT>(kr[u], a, b);
        char* at = &lds[t & 1][0][row * ROW];
        *(u4*)(at + (((2 * piece) ^ turn_k<D>(row)) << 4)) = a;
        *(u4*)(at + (((2 * piece + 1) ^ turn_k<D>(row)) << 4)) = b;
      }
    }
  };
  auto commit_v = [&](int t) {
    if constexpr (F8) {
#pragma unroll
      for (int u = 0; u < LOADS; ++u) {
        const int row = wrow + u * RPI + l / LPR, piece = l % LPR;
        u4 a, b;
        widen_e4m3<DT>(vr[u], a, b);
        char* at = &lds[t & 1][1][row * ROW] + (((2 * piece) ^ turn_v<D>(row)) << 4);
        *(u4*)at = a;
        *(u4*)(at + 16) = b;
      }
    }
  };

  v16f o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;
  float ref = -FLT_MAX, m = -FLT_MAX;                         // the reference as a score, in the exponent
  float sum = 0.0f, sum2 = 0.0f;                              // the lane's part of the sum of weights: even and odd ones

  const int krow = n32 * ROW, kturn = (half ^ turn_k<D>(n32)) << 4;
  const int vr4 = 4 * half + (l & 15) / 4;                    // V: the lane's row of eight, its piece of the row's 64 bytes
  const int vrow = vr4 * ROW + (l & 1) * 8, vturn = ((2 * ((l >> 4) & 1) + ((l & 3) >> 1)) ^ turn_v<D>(vr4)) << 4;

  // ---- the products, one matrix instruction at a time, so that loads and the exponentials can be put between them
  const auto k_piece = [&](int t, int i) {                    // operand i of tile t's scores
    return *(const u4*)(lds[t & 1][0] + (i / STEPS) * 32 * ROW + krow + (kturn ^ ((i % STEPS) << 5)));
  };
  const auto v_piece = [&](int t, int g, int d) {             // keys 16 g .. +15, channels 32 d .. +31
    const char* at = lds[t & 1][1] + 16 * g * ROW + vrow + (vturn ^ (d << 6));
    const u2 y = lds_column4(at), z = lds_column4(at + 8 * ROW);
    return (u4){y.x, y.y, z.x, z.y};
  };
  constexpr int QK = 2 * STEPS, AHEAD = 2;                    // products of a tile's scores; operands of K that are under way
  // One tile: its scores `sc` become weights and meet V, while the next tile's scores are computed (MORE).  K runs a tile ahead of V.
  __shared__ int odd;                                         // something was taken out
  if (tid == 0) odd = 0;
  float top;                                                  // largest of the lane's scores of the tile whose turn it is
  const auto largest = [](const v16f (&sc)[2]) {
    float x = sc[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) x = fmaxf(x, sc[kb][e]);
    return x;
  };
  auto step = [&](int t, v16f (&sc)[2], v16f (&next)[2], auto more) {
    constexpr bool MORE = decltype(more)::value;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();                                          // K of t + 1 and V of t are there; nobody needs K of t or V of t - 1 any more
    const int key0 = k0 + t * kKeys;
    if (key0 < k.begin || key0 + kKeys > k.end || key0 < k.all_from || key0 + kKeys > k.all_to) {
      // values of keys that no row sees become zero (a weight of zero does not make NaN zero); of those that some see, what is not finite
      if constexpr (F8 && MOD == kPlain) {
        // (straight on: the other way spills 4 registers more and has few such tiles to make up for it: 384 after 3500 beside 8 single tokens 54.6 / 55.4 us,
        // 512 fresh ones 18.5 / 19.0, a prompt of 8192 551 / 555)
        bool found = false;
        for (int at = tid; at < TILE / 16; at += 64 * NW) {
          const int key = key0 + at / (ROW / 16);
          u4* v = (u4*)(lds[t & 1][1] + at * 16);
          if (key < k.begin || key >= k.end) *v = (u4){0, 0, 0, 0};
          else if (key < k.all_from || key >= k.all_to) *v = take_out<DT>(*v, found);
        }
        if (found) odd = 1;
      } else {
        // (tested eight values a time, since most often all are: 12000 tokens of packed documents 180 us without it, 158 with it; E4M3 186 / 179)
        constexpr int N = F8 ? 1 : TILE / 16 / (64 * NW);      // pieces a time (E4M3: registers; capped prompt of 8192 tokens 657 / 636 us)
#pragma unroll 1
        for (int at = tid; at < TILE / 16; at += 64 * NW * N) {
          u4* const v = (u4*)(lds[t & 1][1]) + at;
          u4 x[N];
#pragma unroll
          for (int i = 0; i < N; ++i) x[i] = v[64 * NW * i];
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const int key = key0 + (at + 64 * NW * i) / (ROW / 16);
            if (key < k.begin || key >= k.end) {
              v[64 * NW * i] = (u4){0, 0, 0, 0};
            } else if ((key < k.all_from || key >= k.all_to) && any_odd<DT>(x[i])) {
              bool found = false;
              v[64 * NW * i] = take_out<DT>(x[i], found);
              odd = 1;
            }
          }
        }
      }
      __syncthreads();
    }
    const bool more_k = t + 2 < nt;
    if (more_k) issue_k(t + 2);
    if (MORE) issue_v(t + 1);
    u4 kf[AHEAD];
    if constexpr (MORE) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) kf[i] = k_piece(t + 1, i);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (key0 < all_lo || key0 + kKeys > all_hi) {
      const int from = lo - key0 - 4 * half, to = hi - key0 - 4 * half;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int j = 32 * kb + 8 * (e / 4) + e % 4;
          if (j < from || j >= to) sc[kb][e] = -INFINITY;
        }
      top = largest(sc);
    }
    if (__ballot(top > ref + slack)) {
      const uint32_t bits = __float_as_uint(top);
      const auto two = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
      const float most = fmaxf(__uint_as_float(two[0]), __uint_as_float(two[1]));
      ref = most > ref + slack ? most : ref;                   // (by the row's own keys alone)
      const float mc = reference_of<MOD, DT>(ref, c), f = exp2_fast(m - mc);
      m = mc;
      sum *= f;
      sum2 *= f;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] *= f;
    }
    // the next tile's scores, and this one's weights, two a time
    u4 pw[4], vf[2][DB];
    begin_scores(next, t + 1);
    // (the wave that is here goes before the other one of the SIMD, which is most often at its products with V: see the figures above)
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < QK; ++i) {
      if constexpr (MORE) {
        next[i / STEPS] = mfma<DT>(kf[i % AHEAD], q[i % STEPS], next[i / STEPS]);
        if (i + AHEAD < QK) kf[i % AHEAD] = k_piece(t + 1, i + AHEAD);
      }
      if (i >= QK - DB) vf[0][i - (QK - DB)] = v_piece(t, 0, i - (QK - DB));
#pragma unroll
      for (int e = i * 16 / QK; e < (i + 1) * 16 / QK; ++e) { // weights 2 e, 2 e + 1 of the lane's 32
        const float x = exp2_fast(__builtin_fmaf(sc[e / 8][2 * (e % 8)], c, -m)), y = exp2_fast(__builtin_fmaf(sc[e / 8][2 * (e % 8) + 1], c, -m));
        sum += x;
        sum2 += y;
        pw[e / 4][e % 4] = pack16<DT>(x, y);
      }
      asm volatile("" : "+v"(sum), "+v"(sum2));               // (else the additions are put off, and their operands kept)
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        o[d] = mfma<DT>(vf[g & 1][d], pw[g], o[d]);
        if (g < 3) vf[(g + 1) & 1][d] = v_piece(t, g + 1, d);
        if constexpr (MORE) {                                 // the next tile's largest score, some of them a time
          const int n = g * DB + d;
          if constexpr (MOD == kCapped) {
#pragma unroll
            for (int e = n * 32 / (4 * DB); e < (n + 1) * 32 / (4 * DB); ++e) next[e / 16][e % 16] = capped(next[e / 16][e % 16], rate);
          }
          if (n == 0) top = next[0][0];
#pragma unroll
          for (int e = n * 32 / (4 * DB); e < (n + 1) * 32 / (4 * DB); ++e) top = fmaxf(top, next[e / 16][e % 16]);
          asm volatile("" : "+v"(top));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    if (more_k) commit_k(t + 2);
    if (MORE) commit_v(t + 1);
  };

  if (nt > 0) {
    v16f sa[2], sb[2];
    issue_k(0);
    issue_v(0);
    commit_k(0);
    commit_v(0);
    if (nt > 1) {
      issue_k(1);
      commit_k(1);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    begin_scores(sa, 0);
#pragma unroll
    for (int i = 0; i < QK; ++i) sa[i / STEPS] = mfma<DT>(k_piece(0, i), q[i % STEPS], sa[i / STEPS]);
    if constexpr (MOD == kCapped) {
#pragma unroll
      for (int e = 0; e < 32; ++e) sa[e / 16][e % 16] = capped(sa[e / 16][e % 16], rate);
    }
    top = largest(sa);
    int t = 0;
    for (; t + 2 < nt; t += 2) {
      step(t, sa, sb, std::true_type{});
      step(t + 1, sb, sa, std::true_type{});
    }
    if (t + 1 < nt) {
      step(t, sa, sb, std::true_type{});
      step(t + 1, sb, sa, std::false_type{});
    } else {
      step(t, sa, sb, std::false_type{});
    }
  }

  __syncthreads();
  if (odd) {
    for (int j = max(k0, k.begin); j < min(k1, k.end); ++j) {
      if (j >= k.all_from && j < k.all_to) j = k.all_to;      // (what all rows see went through the products)
      if (j >= min(k1, k.end)) break;
      if (j >= lo && j < hi)
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[d][e] += taken_out<DT, F8>(p, k.b, h, j, 32 * d + 8 * (e / 4) + 4 * half + e % 4);
    }
  }
  const uint32_t sbits = __float_as_uint(sum + sum2);
  const auto both = __builtin_amdgcn_permlane32_swap(sbits, sbits, false, false);
  float all = __uint_as_float(both[0]) + __uint_as_float(both[1]);
  if (ns > 1) {
    // The slices meet in the workspace, register by register: pair j of thread t lies at [j][t], so that a wave's accesses are whole lines.  They
    // are added in their order, whoever comes last.
    constexpr int SLOT = BM * (D + 2);
    float* slot0 = p.part + ((int64_t)block * p.c.heads + h) * p.slices * SLOT;
    float* slot = slot0 + (int64_t)s * SLOT;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int e = 0; e < 8; ++e) put2(slot + 2 * ((8 * d + e) * 64 * NW + tid), o[d][2 * e], o[d][2 * e + 1]);
    if (half == 0) put2(slot + BM * D + 2 * rin, m, all);
    __shared__ uint32_t last;
    if (!last_to_arrive(p.tickets + (int64_t)block * p.c.heads + h, ns, tid, &last)) return;
    const float* stat = slot0 + BM * D + 2 * rin;
    m = -FLT_MAX;
    for (int u = 0; u < ns; ++u) m = fmaxf(m, get2(stat + (int64_t)u * SLOT)[0]);
    all = 0.0f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;
    for (int u = 0; u < ns; ++u) {
      const v2f st = get2(stat + (int64_t)u * SLOT);
      const float f = exp2_fast(st[0] - m);
      all += f * st[1];
      const float* src = slot0 + (int64_t)u * SLOT + 2 * tid;
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        v2f x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = get2(src + 2 * (8 * d + e) * 64 * NW);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          o[d][2 * e] += f * x[e][0];
          o[d][2 * e + 1] += f * x[e][1];
        }
      }
    }
  }
  if (!live) return;
  const float f = row_factor(all, vs);
  char* dst = p.out + (int64_t)(tok0 + i) * p.ldo + (int64_t)(h * G + g) * p.ldoh;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *(u2*)(dst + 2 * (32 * d + 8 * e + 4 * half)) = (u2){pack16<DT>(o[d][4 * e] * f, o[d][4 * e + 1] * f),
                                                           pack16<DT>(o[d][4 * e + 2] * f, o[d][4 * e + 3] * f)};
  if (p.lse && half == 0) p.lse[(int64_t)(tok0 + i) * p.q_heads + h * G + g] = lse_of(p, m, all);
}

}  // namespace tile
}  // namespace serq
