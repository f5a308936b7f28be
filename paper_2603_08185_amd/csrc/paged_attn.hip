// Attention of new tokens over the paged cache (serq_paged_attn): one pass over the keys with the running maximum and sum of the softmax.
//
// First form: a wave per new token and query head.  64 keys at a time, a lane computes one key's score; then a lane owns D / 64 channels and
// adds the 64 weighted values.
#include "kv_cache.h"

namespace serq {
namespace {

struct AttnParams {
  const char* q; char* out; float* lse;                       // strides in bytes
  int64_t ldq, ldqh, ldo, ldoh;
  int q_heads, group, window;
  float scale;
  KvView c;
};

template <int DT, bool F8>
__device__ __forceinline__ float ld_elem(const char* p, int d) {
  if constexpr (F8) return __builtin_amdgcn_cvt_f32_fp8((int)(uint8_t)p[d], 0);
  else return Elem<DT>::ld(p, d);
}

template <int DT, bool F8, int D>
__global__ __launch_bounds__(64) void paged_attn_simple_kernel(AttnParams p) {
  const int t = blockIdx.x, head = blockIdx.y, h = head / p.group, lane = threadIdx.x;
  const int b = sequences_before(t, p.c.seqs, lane, [&](int i) { return p.c.cu[i + 1]; });
  if (b >= p.c.seqs) return;
  const int pos = p.c.len[b] - p.c.cu[b + 1] + t;
  const int64_t most = (int64_t)p.c.width << p.c.page_shift;
  const int end = (int)min((int64_t)pos + 1, most);
  const int begin = p.window > 0 ? max(0, pos - p.window + 1) : 0;
  const char* q = p.q + t * p.ldq + head * p.ldqh;
  const float ks = p.c.k_scale ? p.c.k_scale[h] : 1.0f, vs = p.c.v_scale ? p.c.v_scale[h] : 1.0f;
  float m = -INFINITY, l = 0.0f, o[D / 64] = {};
  for (int j0 = begin; j0 < end; j0 += 64) {
    const int j = j0 + lane;
    int page = 0;
    float s = -INFINITY;
    if (j < end) {
      page = min(max(p.c.table[b * p.c.table_ld + (j >> p.c.page_shift)], 0), p.c.pages - 1);
      const char* k = p.c.k + page * p.c.k_page + (j & ((1 << p.c.page_shift) - 1)) * p.c.k_token + h * p.c.k_head;
      s = 0.0f;
      for (int d = 0; d < D; ++d) s += Elem<DT>::ld(q, d) * ld_elem<DT, F8>(k, d);
      s *= p.scale * ks;
    }
    const float mn = fmaxf(m, wave_max(s));
    const float f = expf(m - mn), w = j < end ? expf(s - mn) : 0.0f;
    m = mn;
    l = l * f + wave_reduce(w, [](float a, float c) { return a + c; });
    for (int i = 0; i < D / 64; ++i) o[i] *= f;
    const int n = min(64, end - j0);
    for (int i = 0; i < n; ++i) {
      const int pg = __shfl(page, i), jj = j0 + i;
      const float pw = __shfl(w, i);
      const char* v = p.c.v + pg * p.c.v_page + (jj & ((1 << p.c.page_shift) - 1)) * p.c.v_token + h * p.c.v_head;
      for (int e = 0; e < D / 64; ++e) o[e] += pw * ld_elem<DT, F8>(v, lane + 64 * e);
    }
  }
  uint16_t* out = (uint16_t*)(p.out + t * p.ldo + head * p.ldoh);
  for (int e = 0; e < D / 64; ++e) {
    const float r = l > 0.0f || l != l ? o[e] * vs / l : 0.0f;
    out[lane + 64 * e] = DT == SERQ_BF16 ? f32_to_bf16_rne(r) : f32_to_f16_rne(r);
  }
  if (p.lse && lane == 0) p.lse[(int64_t)t * p.q_heads + head] = l > 0.0f || l != l ? m + logf(l) : -INFINITY;
}

template <int DT, bool F8, int D>
int launch(const AttnParams& p, hipStream_t st) {
  hipLaunchKernelGGL((paged_attn_simple_kernel<DT, F8, D>), dim3(p.c.tokens, p.q_heads), dim3(64), 0, st, p);
  return hipGetLastError() == hipSuccess ? SERQ_OK : SERQ_EHIP;
}

}  // namespace
}  // namespace serq

using namespace serq;

extern "C" {

size_t serq_paged_attn_workspace_bytes(int64_t tokens, int seqs, int max_q, int64_t max_kv, int q_heads, int kv_heads, int dim) {
  if (tokens < 0 || tokens > (1 << 24) || seqs < 0 || seqs > 65536 || max_q < 0 || max_kv < 0 || kv_heads < 1 || kv_heads > 1024 ||
      q_heads < 1 || q_heads > 65536 || q_heads % kv_heads || (dim != 64 && dim != 128))
    return 0;
  return 16;
}

int serq_paged_attn(const void* q, int64_t ldq, int64_t ldqh, int q_heads, int dtype, const serq_kv_cache* cache,
                    const serq_kv_batch* batch, int max_q, int64_t max_kv, float scale, int window,
                    void* out, int64_t ldo, int64_t ldoh, float* lse,
                    void* workspace, size_t workspace_bytes, void* stream) {
  AttnParams p{};
  int rc = kv_check(cache, batch, dtype, p.c);
  if (rc != SERQ_OK) return rc;
  const int D = cache->dim;
  if (q_heads < 1 || q_heads > 65535 || q_heads % cache->heads || window < 0 || max_q < 0 || max_kv < 0) return SERQ_ESHAPE;
  if (batch->tokens * (q_heads / cache->heads) > 0x7fffffff) return SERQ_ESHAPE;
  if (!(scale > 0.0f) || !(scale <= 3.4028234e38f)) return SERQ_ESHAPE;
  if (batch->tokens == 0 || batch->seqs == 0) return SERQ_OK;
  if ((rc = kv_check_rows(q, ldq, ldqh, q_heads, D)) != SERQ_OK) return rc;
  if ((rc = kv_check_rows(out, ldo, ldoh, q_heads, D)) != SERQ_OK) return rc;
  if (!kv_aligned(lse, 4) || !kv_aligned(workspace, 16)) return SERQ_EALIGN;
  (void)workspace_bytes;
  p.q = (const char*)q; p.out = (char*)out; p.lse = lse;
  p.ldq = 2 * ldq; p.ldqh = 2 * ldqh; p.ldo = 2 * ldo; p.ldoh = 2 * ldoh;
  p.q_heads = q_heads; p.group = q_heads / cache->heads; p.window = window; p.scale = scale;
  const bool f8 = cache->dtype == SERQ_F8, bf = dtype == SERQ_BF16;
  hipStream_t st = (hipStream_t)stream;
  if (D == 128) {
    if (bf) return f8 ? launch<SERQ_BF16, true, 128>(p, st) : launch<SERQ_BF16, false, 128>(p, st);
    return f8 ? launch<SERQ_F16, true, 128>(p, st) : launch<SERQ_F16, false, 128>(p, st);
  }
  if (bf) return f8 ? launch<SERQ_BF16, true, 64>(p, st) : launch<SERQ_BF16, false, 64>(p, st);
  return f8 ? launch<SERQ_F16, true, 64>(p, st) : launch<SERQ_F16, false, 64>(p, st);
}

}  // extern "C"
