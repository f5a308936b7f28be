// Rotate queries and keys by their positions and put keys and values into the paged cache (serq_kv_append).
//
// Every new token is read and written once: (Hq + 2 Hkv) D elements in, as many out, and a row of the rotation's table; a few operations
// an element.  So it is bound by bytes, and for few tokens by the latency of one chain of loads: the sequence's end -> its length and
// number of new tokens -> the page -> the store.  A thread owns two pieces of 8 channels that the rotation mixes (the same piece of both
// halves, or 16 neighbours), so that nothing is exchanged between threads and every access is 16 bytes wide.
#include "kv_cache.h"

namespace serq {
namespace {

struct AppendParams {
  const char* q; const char* k; const char* v; char* qo;      // strides in bytes
  int64_t ldq, ldqh, ldk, ldkh, ldv, ldvh, ldqo, ldqoh;
  const float* cos; const float* sin; const int32_t* positions;
  int rows, rot, q_heads, items;                              // items: pairs of pieces of a token
  KvView c;
};

template <int DT>
__device__ __forceinline__ u4 to16(const float v[8]) {
  u4 o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = DT == SERQ_BF16 ? f32x2_to_bf16x2(v[2 * i], v[2 * i + 1]) : f32x2_to_f16x2(v[2 * i], v[2 * i + 1]);
  return o;
}
__device__ __forceinline__ u2 to_e4m3(const float v[8], float scale) {
  u2 o;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t w = pack_e4m3<false>(v[4 * i] / scale, v[4 * i + 1] / scale, 0u);
    o[i] = pack_e4m3<true>(v[4 * i + 2] / scale, v[4 * i + 3] / scale, w);
  }
  return o;
}

// (x, y) -> (x c - y s, y c + x s), every operation rounded by itself
__device__ __forceinline__ void turn(float& x, float& y, float c, float s) {
#pragma clang fp contract(off)
  const float xc = x * c, ys = y * s, yc = y * c, xs = x * s;
  x = xc - ys;
  y = yc + xs;
}

// One token a workgroup, one pair of pieces a thread (more where a token has more pairs than threads).  What does not hang on the token's place is
// asked for before that is known: the token's values with the ends and lengths of the sequences, then the page with the rotation.
template <int DT, bool F8, int D, bool INTER>
__global__ __launch_bounds__(512) void kv_append_kernel(AppendParams p) {
  constexpr int PP = D / 16;                                  // pairs of a head
  const int t = blockIdx.x, lane = threadIdx.x & 63;

  struct Item {
    int h, d0, d1;                                            // head of its kind, first channels of the two pieces
    bool is_q, is_k, rotated;
    Raw8<DT> x, y;
  };
  const auto fetch = [&](int it) {
    Item m;
    const int head = it / PP, j = it % PP;
    m.is_q = head < p.q_heads;
    m.is_k = !m.is_q && head < p.q_heads + p.c.heads;
    m.h = m.is_q ? head : m.is_k ? head - p.q_heads : head - p.q_heads - p.c.heads;
    m.rotated = (m.is_q || m.is_k) && j < p.rot / 16;
    const bool split = m.rotated && !INTER;                   // the two pieces lie rot / 2 channels apart
    m.d0 = split ? 8 * j : 16 * j;
    m.d1 = split ? m.d0 + p.rot / 2 : m.d0 + 8;
    const char* src = m.is_q ? p.q + t * p.ldq + m.h * p.ldqh : m.is_k ? p.k + t * p.ldk + m.h * p.ldkh : p.v + t * p.ldv + m.h * p.ldvh;
    m.x.a = *(const u4*)(src + 2 * m.d0);
    m.y.a = *(const u4*)(src + 2 * m.d1);
    return m;
  };
  // (the sequences first: loads come back in their order)
  const auto ask = [&](int b, int& end, int& len) {
    const int i = min(b + lane, p.c.seqs - 1);
    end = p.c.cu[i + 1];
    len = p.c.len[i];
  };
  int b = 0, pos, end, len;
  const int first = p.c.cu[0];                                // rows before it are of no sequence
  ask(0, end, len);
  int it = threadIdx.x;
  Item m{};
  if (it < p.items) m = fetch(it);
  __builtin_amdgcn_sched_barrier(0);

  // the token's sequence: the first that ends behind it
  if (t < first) return;
  for (;;) {
    const int c = __builtin_popcountll(__ballot(b + lane < p.c.seqs && end <= t));
    b += c;
    if (b >= p.c.seqs) return;                                // a row of no sequence
    if (c < 64) {
      pos = __builtin_amdgcn_readlane(len, c) - __builtin_amdgcn_readlane(end, c) + t;
      break;
    }
    ask(b, end, len);
  }
  const int turned = min(max(p.positions ? p.positions[t] : pos, 0), p.rows - 1);
  const int slot = pos >> p.c.page_shift;                     // (negative for a negative position)
  int page = -1;
  if (slot >= 0 && slot < p.c.width) page = p.c.table[b * p.c.table_ld + slot];
  if (page >= p.c.pages) page = -1;
  const int row = pos & ((1 << p.c.page_shift) - 1);

  for (; it < p.items;) {
    float a[8], e[8];
    values8<DT>(m.x, a);
    values8<DT>(m.y, e);
    if (m.rotated) {
      const int64_t at = (int64_t)turned * (p.rot / 2) + (INTER ? m.d0 / 2 : m.d0);
      float c[8], s[8];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const v4f cc = *(const v4f*)(p.cos + at + 4 * i), ss = *(const v4f*)(p.sin + at + 4 * i);
#pragma unroll
        for (int n = 0; n < 4; ++n) { c[4 * i + n] = cc[n]; s[4 * i + n] = ss[n]; }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (INTER) {                                // pairs (0,1) .. (6,7) of the first piece, then of the second
          if (i < 4) turn(a[2 * i], a[2 * i + 1], c[i], s[i]);
          else turn(e[2 * i - 8], e[2 * i - 7], c[i], s[i]);
        } else {
          turn(a[i], e[i], c[i], s[i]);
        }
      }
    }
    if (m.is_q) {
      char* dst = p.qo + t * p.ldqo + m.h * p.ldqoh;
      *(u4*)(dst + 2 * m.d0) = to16<DT>(a);
      *(u4*)(dst + 2 * m.d1) = to16<DT>(e);
    } else if (page >= 0) {
      char* dst = m.is_k ? p.c.k + page * p.c.k_page + row * p.c.k_token + m.h * p.c.k_head
                         : p.c.v + page * p.c.v_page + row * p.c.v_token + m.h * p.c.v_head;
      if constexpr (F8) {
        const float* sc = m.is_k ? p.c.k_scale : p.c.v_scale;
        const float scale = sc ? sc[m.h] : 1.0f;
        *(u2*)(dst + m.d0) = to_e4m3(a, scale);
        *(u2*)(dst + m.d1) = to_e4m3(e, scale);
      } else {
        *(u4*)(dst + 2 * m.d0) = to16<DT>(a);
        *(u4*)(dst + 2 * m.d1) = to16<DT>(e);
      }
    }
    it += blockDim.x;
    if (it < p.items) m = fetch(it);
  }
}

template <int DT, bool F8, int D>
void launch(const AppendParams& p, bool inter, hipStream_t st) {
  const int threads = p.items >= 512 ? 512 : (p.items + 63) & ~63;
  if (inter) hipLaunchKernelGGL((kv_append_kernel<DT, F8, D, true>), dim3(p.c.tokens), dim3(threads), 0, st, p);
  else hipLaunchKernelGGL((kv_append_kernel<DT, F8, D, false>), dim3(p.c.tokens), dim3(threads), 0, st, p);
}

}  // namespace
}  // namespace serq

using namespace serq;

extern "C" int serq_kv_append(const void* q, int64_t ldq, int64_t ldqh, int q_heads,
                              const void* k, int64_t ldk, int64_t ldkh, const void* v, int64_t ldv, int64_t ldvh, int dtype,
                              const float* cos_table, const float* sin_table, int64_t table_rows, int rot_dim, int interleaved,
                              const int32_t* positions, const serq_kv_cache* cache, const serq_kv_batch* batch,
                              void* q_out, int64_t ldqo, int64_t ldqoh, void* stream) {
  AppendParams p{};
  int rc = kv_check(cache, batch, dtype, p.c);
  if (rc != SERQ_OK) return rc;
  const int D = cache->dim;
  if (q_heads < 0 || q_heads > 65536) return SERQ_ESHAPE;
  if (rot_dim < 0 || rot_dim > D || (rot_dim % 16) != 0 || table_rows < 0 || table_rows > 0x7fffffff) return SERQ_ESHAPE;
  if (rot_dim > 0 && table_rows == 0) return SERQ_ESHAPE;
  if (batch->tokens == 0 || batch->seqs == 0) return SERQ_OK;
  if (q_heads > 0) {
    if ((rc = kv_check_rows(q, ldq, ldqh, q_heads, D)) != SERQ_OK) return rc;
    if ((rc = kv_check_rows(q_out, ldqo, ldqoh, q_heads, D)) != SERQ_OK) return rc;
    if (q == q_out && (ldq != ldqo || ldqh != ldqoh)) return SERQ_ESHAPE;
  }
  if ((rc = kv_check_rows(k, ldk, ldkh, cache->heads, D)) != SERQ_OK) return rc;
  if ((rc = kv_check_rows(v, ldv, ldvh, cache->heads, D)) != SERQ_OK) return rc;
  if (rot_dim > 0) {
    if (!cos_table || !sin_table) return SERQ_ENULL;
    if (!kv_aligned(cos_table, 16) || !kv_aligned(sin_table, 16)) return SERQ_EALIGN;
  }
  if (!kv_aligned(positions, 4)) return SERQ_EALIGN;
  p.q = (const char*)q; p.k = (const char*)k; p.v = (const char*)v; p.qo = (char*)q_out;
  p.ldq = 2 * ldq; p.ldqh = 2 * ldqh; p.ldk = 2 * ldk; p.ldkh = 2 * ldkh; p.ldv = 2 * ldv; p.ldvh = 2 * ldvh;
  p.ldqo = 2 * ldqo; p.ldqoh = 2 * ldqoh;
  p.cos = cos_table; p.sin = sin_table; p.positions = positions;
  p.rows = (int)table_rows; p.rot = rot_dim; p.q_heads = q_heads;
  p.items = (q_heads + 2 * cache->heads) * (D / 16);
  const bool f8 = cache->dtype == SERQ_F8, bf = dtype == SERQ_BF16, inter = interleaved != 0;
  hipStream_t st = (hipStream_t)stream;
  if (D == 128) {
    if (bf) f8 ? launch<SERQ_BF16, true, 128>(p, inter, st) : launch<SERQ_BF16, false, 128>(p, inter, st);
    else f8 ? launch<SERQ_F16, true, 128>(p, inter, st) : launch<SERQ_F16, false, 128>(p, inter, st);
  } else {
    if (bf) f8 ? launch<SERQ_BF16, true, 64>(p, inter, st) : launch<SERQ_BF16, false, 64>(p, inter, st);
    else f8 ? launch<SERQ_F16, true, 64>(p, inter, st) : launch<SERQ_F16, false, 64>(p, inter, st);
  }
  return hipGetLastError() == hipSuccess ? SERQ_OK : SERQ_EHIP;
}
