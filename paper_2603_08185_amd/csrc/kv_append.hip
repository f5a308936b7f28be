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

// One token a workgroup, one pair of pieces a thread (more where a token has more pairs than threads).
template <int DT, bool F8, int D, bool INTER>
__global__ __launch_bounds__(512) void kv_append_kernel(AppendParams p) {
  constexpr int PP = D / 16;                                  // pairs of a head
  const int t = blockIdx.x;
  const int lane = threadIdx.x & 63;
  const int b = sequences_before(t, p.c.seqs, lane, [&](int i) { return p.c.cu[i + 1]; });
  if (b >= p.c.seqs) return;                                  // a row of no sequence
  const int pos = p.c.len[b] - p.c.cu[b + 1] + t;
  const int turned = min(max(p.positions ? p.positions[t] : pos, 0), p.rows - 1);
  const int slot = pos >> p.c.page_shift;                     // (negative for a negative position)
  int page = -1;
  if (slot >= 0 && slot < p.c.width) page = p.c.table[b * p.c.table_ld + slot];
  if (page >= p.c.pages) page = -1;
  const int row = pos & ((1 << p.c.page_shift) - 1);

  for (int it = threadIdx.x; it < p.items; it += blockDim.x) {
    const int head = it / PP, j = it % PP;
    const bool is_q = head < p.q_heads, is_k = !is_q && head < p.q_heads + p.c.heads;
    const int h = is_q ? head : is_k ? head - p.q_heads : head - p.q_heads - p.c.heads;
    const bool rotated = (is_q || is_k) && j < p.rot / 16;
    const bool split = rotated && !INTER;                     // the two pieces lie rot / 2 channels apart
    const int d0 = split ? 8 * j : 16 * j, d1 = split ? d0 + p.rot / 2 : d0 + 8;
    const char* src = is_q ? p.q + t * p.ldq + h * p.ldqh : is_k ? p.k + t * p.ldk + h * p.ldkh : p.v + t * p.ldv + h * p.ldvh;
    Raw8<DT> x, y;
    x.a = *(const u4*)(src + 2 * d0);
    y.a = *(const u4*)(src + 2 * d1);
    float a[8], e[8];
    values8<DT>(x, a);
    values8<DT>(y, e);
    if (rotated) {
      const int64_t at = (int64_t)turned * (p.rot / 2) + 8 * j;
      float c[8], s[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) { c[i] = p.cos[at + i]; s[i] = p.sin[at + i]; }
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
    if (is_q) {
      char* dst = p.qo + t * p.ldqo + h * p.ldqoh;
      *(u4*)(dst + 2 * d0) = to16<DT>(a);
      *(u4*)(dst + 2 * d1) = to16<DT>(e);
    } else if (page >= 0) {
      char* dst = is_k ? p.c.k + page * p.c.k_page + row * p.c.k_token + h * p.c.k_head
                       : p.c.v + page * p.c.v_page + row * p.c.v_token + h * p.c.v_head;
      if constexpr (F8) {
        const float* sc = is_k ? p.c.k_scale : p.c.v_scale;
        const float scale = sc ? sc[h] : 1.0f;
        *(u2*)(dst + d0) = to_e4m3(a, scale);
        *(u2*)(dst + d1) = to_e4m3(e, scale);
      } else {
        *(u4*)(dst + 2 * d0) = to16<DT>(a);
        *(u4*)(dst + 2 * d1) = to16<DT>(e);
      }
    }
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
