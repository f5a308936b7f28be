// serq_paged_attn for sequences with many rows (chunks, prompts): bound by the matrix instructions and the exponentials between them.
//
// A workgroup takes 128 rows of a key head -- its waves 32 each -- and a slice of the keys, in tiles of 64.  K and V of a tile lie in LDS, two
// tiles deep: while one is used, the next is on its way (straight to LDS for 16-bit caches; through registers, where they become 16-bit
// values, for E4M3 ones).
//   scores   S^T = K Q^T on the 32x32x16 instruction: a lane's results are 16 of 32 keys of one row, the other 16 are with the lane 32 further.
//   weights  as in the kernel for few rows: exp2(s c - m c), m raised only when a score exceeds it by more than 2^6 in weight.
//   values   O^T = V^T P^T: the weights are the instruction's operand as they stand (eight registers of scores become one operand of 16 keys in
//            the order 4h .. 4h+3, 8+4h .. 8+4h+3), and V is read by columns in the same order.
// The 16-byte pieces of a row in LDS are turned by the row's number, so that the lanes that read together meet different banks.
#include "paged_attn.h"

namespace serq {
namespace {

constexpr int kKeys = 64;

template <int DT>
__device__ __forceinline__ v16f mfma(const u4& a, const u4& b, const v16f& c) {
  if constexpr (DT == SERQ_BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

// places of the 16-byte pieces of a row: K is read 16 bytes a row by 32 rows at a time, V 64 bytes a row by 8
template <int D> __device__ __forceinline__ int turn_k(int row) { return D == 128 ? row & 15 : row & 7; }
template <int D> __device__ __forceinline__ int turn_v(int row) { return D == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); }

template <int DT, bool F8, int D, int NW>
__global__ __launch_bounds__(64 * NW, 2) void paged_attn_tile_kernel(AttnParams p) {
  constexpr int BM = 32 * NW;
  constexpr int ROW = D * 2;                                  // bytes of a key in LDS
  constexpr int TILE = kKeys * ROW;                           // of K or of V
  constexpr int STEPS = D / 16, DB = D / 32;
  constexpr int ROWB = F8 ? D : 2 * D;                        // bytes of a key in the cache
  constexpr int LPR = ROWB / 16, RPI = 64 / LPR;              // lanes of a row, rows of a load of 64 lanes
  constexpr int LOADS = kKeys / RPI / NW;                     // loads of a wave for a tile of K
  static_assert(LOADS >= 1 && LOADS * RPI <= 16, "a wave's rows lie in one page");
  __shared__ __align__(16) char lds[2][2][TILE];              // [buffer][K, V]

  const int tid = threadIdx.x, l = tid & 63, w = uniform(tid >> 6);
  const int n32 = l & 31, half = l >> 5;
  const int G = p.group;
  // the rows that see most keys come last in a sequence and start first; neighbouring workgroups have different key heads
  const int units = gridDim.x / p.c.heads;
  const int h = blockIdx.x % p.c.heads, block = units - 1 - blockIdx.x / p.c.heads, s = blockIdx.z;
  const RowBlock k = row_block<BM, false>(p, block, l);
  if (k.rows <= 0) return;
  const int base = k.begin & ~15;
  const int ns = k.end > base ? min((k.end - base - 1) / p.slice_keys + 1, p.slices) : 1;
  if (s >= ns) return;
  const int k0 = base + s * p.slice_keys, k1 = s == ns - 1 ? k.end : k0 + p.slice_keys;
  const int tok0 = uniform(p.c.cu[k.b]);

  // the lane's row, and the keys that it sees: lo <= j < hi
  const int rin = 32 * w + n32, r = k.r0 + rin;
  const bool live = rin < k.rows;
  const int i = r / G, g = r - i * G;
  const int first = k.L - k.n;
  const int hi = live ? min(first + i + 1, k.end) : 0, lo = p.window > 0 ? max(0, first + i - p.window + 1) : 0;
  u4 q[STEPS];
  {
    const char* src = p.q + (int64_t)(tok0 + i) * p.ldq + (int64_t)(h * G + g) * p.ldqh;
#pragma unroll
    for (int st = 0; st < STEPS; ++st) q[st] = live ? *(const u4*)(src + 32 * st + 16 * half) : (u4){0, 0, 0, 0};
  }
  // of the wave's rows: keys that any sees, keys that all see (a wave without rows: none)
  const int wr0 = k.r0 + 32 * w, wr1 = min(k.r0 + k.rows, wr0 + 32) - 1;
  const int any_lo = p.window > 0 ? max(0, first + wr0 / G - p.window + 1) : 0, any_hi = wr1 < wr0 ? 0 : min(first + wr1 / G + 1, k.end);
  const int all_lo = p.window > 0 ? max(0, first + wr1 / G - p.window + 1) : 0, all_hi = min(first + wr0 / G + 1, k.end);
  const float ks = p.c.k_scale ? p.c.k_scale[h] : 1.0f, vs = p.c.v_scale ? p.c.v_scale[h] : 1.0f;
  const float c = p.scale * ks * kLog2e, slack = score_slack(c);

  // ---- loads: a wave brings LOADS * RPI rows of K and of V, which lie in one page
  const int mask = (1 << p.c.page_shift) - 1;
  const int32_t* table = p.c.table + k.b * p.c.table_ld;
  const char* kbase = p.c.k + h * p.c.k_head;
  const char* vbase = p.c.v + h * p.c.v_head;
  const int nt = k1 > k0 ? (k1 - k0 + kKeys - 1) / kKeys : 0;
  const int wrow = w * LOADS * RPI;
  int pages = 0;                                              // lane: the page of this wave's rows in tile 64 (t / 64) + lane
  auto look_up = [&](int t) {
    const int key = min(k0 + (t + l) * kKeys + wrow, k.end - 1);
    pages = min(max(table[key >> p.c.page_shift], 0), p.c.pages - 1);
  };
  uint32_t ksrc[LOADS], vsrc[LOADS];                          // a lane's place in the rows it brings
#pragma unroll
  for (int u = 0; u < LOADS; ++u) {
    const int row = wrow + u * RPI + l / LPR, piece = l % LPR;
    const int in = u * RPI + l / LPR;
    ksrc[u] = (uint32_t)(in * (int)p.c.k_token + ((F8 ? piece : piece ^ turn_k<D>(row)) << 4));
    vsrc[u] = (uint32_t)(in * (int)p.c.v_token + ((F8 ? piece : piece ^ turn_v<D>(row)) << 4));
  }
  u4 kr[F8 ? LOADS : 1], vr[F8 ? LOADS : 1];
  auto issue = [&](int t) {
    if ((t & 63) == 0) look_up(t);
    const int row0 = (k0 + t * kKeys + wrow) & mask, pg = __builtin_amdgcn_readlane(pages, t & 63);
    const char* ka = kbase + pg * p.c.k_page + row0 * p.c.k_token;
    const char* va = vbase + pg * p.c.v_page + row0 * p.c.v_token;
    if constexpr (F8) {
#pragma unroll
      for (int u = 0; u < LOADS; ++u) kr[u] = *(const u4*)(ka + ksrc[u]);
#pragma unroll
      for (int u = 0; u < LOADS; ++u) vr[u] = *(const u4*)(va + vsrc[u]);
    } else {
      const uint32_t kd = lds_addr(&lds[t & 1][0][wrow * ROW]), vd = lds_addr(&lds[t & 1][1][wrow * ROW]);
#pragma unroll
      for (int u = 0; u < LOADS; ++u) dma16(ka, ksrc[u], uniform(kd + u * 1024));
#pragma unroll
      for (int u = 0; u < LOADS; ++u) dma16(va, vsrc[u], uniform(vd + u * 1024));
    }
  };
  auto commit = [&](int t) {                                  // E4M3: to LDS as 16-bit values
    if constexpr (F8) {
#pragma unroll
      for (int u = 0; u < LOADS; ++u) {
        const int row = wrow + u * RPI + l / LPR, piece = l % LPR;
        u4 a, b;
        widen_e4m3<DT>(kr[u], a, b);
        char* at = &lds[t & 1][0][row * ROW];
        *(u4*)(at + (((2 * piece) ^ turn_k<D>(row)) << 4)) = a;
        *(u4*)(at + (((2 * piece + 1) ^ turn_k<D>(row)) << 4)) = b;
        widen_e4m3<DT>(vr[u], a, b);
        at = &lds[t & 1][1][row * ROW];
        *(u4*)(at + (((2 * piece) ^ turn_v<D>(row)) << 4)) = a;
        *(u4*)(at + (((2 * piece + 1) ^ turn_v<D>(row)) << 4)) = b;
      }
    }
  };

  v16f o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;
  float ref = -FLT_MAX, m = -FLT_MAX, sum = 0.0f;             // the reference as a score, times c; the lane's part of the sum of weights

  const int krow = n32 * ROW, kturn = (half ^ turn_k<D>(n32)) << 4;
  const int vr4 = 4 * half + (l & 15) / 4;                    // V: the lane's row of eight, its piece of the row's 64 bytes
  const int vrow = vr4 * ROW + (l & 1) * 8, vturn = ((2 * ((l >> 4) & 1) + ((l & 3) >> 1)) ^ turn_v<D>(vr4)) << 4;
  const int vturn8 = ((2 * ((l >> 4) & 1) + ((l & 3) >> 1)) ^ turn_v<D>(vr4 + 8)) << 4;

  if (nt > 0) {
    issue(0);
    commit(0);
  }
#pragma unroll 1
  for (int t = 0; t < nt; ++t) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const int key0 = k0 + t * kKeys;
    const char* kb0 = lds[t & 1][0];
    char* vb0 = lds[t & 1][1];
    if (key0 < k.begin || key0 + kKeys > k.end) {
      // values of keys that no row sees become zero (a weight of zero does not make NaN zero)
      for (int at = tid; at < TILE / 16; at += 64 * NW) {
        const int key = key0 + at / (ROW / 16);
        if (key < k.begin || key >= k.end) *(u4*)(vb0 + at * 16) = (u4){0, 0, 0, 0};
      }
      __syncthreads();
    }
    if (t + 1 < nt) issue(t + 1);
    if (key0 < any_hi && key0 + kKeys > any_lo) {
      v16f sc[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[kb][e] = 0.0f;
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
          const u4 a = *(const u4*)(kb0 + kb * 32 * ROW + krow + (kturn ^ (st << 5)));
          sc[kb] = mfma<DT>(a, q[st], sc[kb]);
        }
      }
      if (key0 < all_lo || key0 + kKeys > all_hi) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int j = key0 + 32 * kb + 8 * (e / 4) + 4 * half + e % 4;
            if (j < lo || j >= hi) sc[kb][e] = -INFINITY;
          }
      }
      float top = sc[0][0];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, sc[kb][e]);
      if (__ballot(top > ref + slack)) {
        const uint32_t bits = __float_as_uint(top);
        const auto two = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
        ref = fmaxf(ref, fmaxf(__uint_as_float(two[0]), __uint_as_float(two[1])));
        const float mc = fmaxf(ref * c, -FLT_MAX), f = exp2_fast(m - mc);
        m = mc;
        sum *= f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[d][e] *= f;
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] = exp2_fast(__builtin_fmaf(sc[kb][8 * st + e], c, -m));
            sum += x[e];
          }
          const u4 pw = {pack16<DT>(x[0], x[1]), pack16<DT>(x[2], x[3]), pack16<DT>(x[4], x[5]), pack16<DT>(x[6], x[7])};
          const char* v0 = vb0 + (32 * kb + 16 * st) * ROW + vrow;
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            const u2 y = lds_column4(v0 + (vturn ^ (d << 6))), z = lds_column4(v0 + 8 * ROW + (vturn8 ^ (d << 6)));
            o[d] = mfma<DT>((u4){y.x, y.y, z.x, z.y}, pw, o[d]);
          }
        }
    }
    if (t + 1 < nt) commit(t + 1);
  }

  const uint32_t sbits = __float_as_uint(sum);
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
  if (p.lse && half == 0) p.lse[(int64_t)(tok0 + i) * p.q_heads + h * G + g] = row_lse(m, all);
}

template <int DT, bool F8, int D>
int launch(const AttnParams& p, int blocks, hipStream_t st) {
  hipLaunchKernelGGL((paged_attn_tile_kernel<DT, F8, D, 4>), dim3((unsigned)(blocks * p.c.heads), 1, (unsigned)p.slices), dim3(256), 0, st, p);
  return hipGetLastError() == hipSuccess ? SERQ_OK : SERQ_EHIP;
}

}  // namespace

size_t paged_attn_tile_slot_floats(int D) { return (size_t)kTileRows * (D + 2); }

int launch_paged_attn_tile(const AttnParams& p, int dtype, bool f8, int D, int blocks, hipStream_t st) {
  const bool bf = dtype == SERQ_BF16;
  if (D == 128) {
    if (bf) return f8 ? launch<SERQ_BF16, true, 128>(p, blocks, st) : launch<SERQ_BF16, false, 128>(p, blocks, st);
    return f8 ? launch<SERQ_F16, true, 128>(p, blocks, st) : launch<SERQ_F16, false, 128>(p, blocks, st);
  }
  if (bf) return f8 ? launch<SERQ_BF16, true, 64>(p, blocks, st) : launch<SERQ_BF16, false, 64>(p, blocks, st);
  return f8 ? launch<SERQ_F16, true, 64>(p, blocks, st) : launch<SERQ_F16, false, 64>(p, blocks, st);
}

}  // namespace serq
