// serq_paged_attn: argument checks, the choice of kernel and of the slices of a long cache (include/serq_kv.h; the kernels say what they do).
#include "paged_attn.h"

namespace serq {
namespace {

constexpr int kTickets = 4096;                                // words at the start of a workspace, whatever the call

struct Plan {
  int nb, blocks, slices, slice_keys, direct;
  size_t bytes;
};

// keys: most that a row block can see
Plan plan_few(int64_t tokens, int seqs, int max_q, int64_t max_kv, int window, int heads, int group, int D) {
  Plan k{};
  const int64_t rows = (int64_t)max_q * group;
  k.nb = rows <= 16 ? 1 : 2;
  const int BM = 16 * k.nb;
  k.direct = rows <= BM;
  k.blocks = k.direct ? seqs : (int)(tokens * group / BM) + seqs;
  const int64_t units = (int64_t)k.blocks * heads;
  int64_t keys = max_kv;
  if (window > 0 && keys > (int64_t)window + max_q) keys = (int64_t)window + max_q;
  k.slices = 1;
  k.slice_keys = 0x7fffff00;
  k.bytes = 16;
  const int64_t want = 4 * (int64_t)device_cu_count();
  if (units > 0 && units < want && units <= kTickets && keys > 256) {
    int64_t n = (want + units - 1) / units;
    if (n > kMaxSlices) n = kMaxSlices;
    k.bytes = kTickets * 4 + (size_t)units * n * paged_attn_few_slot_floats(k.nb, D) * 4;   // (the same with and without a window)
    int64_t each = ((keys + n - 1) / n + 255) & ~(int64_t)255;
    n = (keys + each - 1) / each;
    if (n > 1) {
      k.slices = (int)n;
      k.slice_keys = (int)each;
    }
  }
  return k;
}

}  // namespace
}  // namespace serq

using namespace serq;

extern "C" {

size_t serq_paged_attn_workspace_bytes(int64_t tokens, int seqs, int max_q, int64_t max_kv, int q_heads, int kv_heads, int dim) {
  if (tokens < 0 || tokens > (1 << 24) || seqs < 0 || seqs > 65536 || max_q < 0 || max_kv < 0 || kv_heads < 1 || kv_heads > 1024 ||
      q_heads < 1 || q_heads > 65535 || q_heads % kv_heads || (dim != 64 && dim != 128) || tokens * (q_heads / kv_heads) > 0x7fffffff)
    return 0;
  return plan_few(tokens, seqs, max_q, max_kv, 0, kv_heads, q_heads / kv_heads, dim).bytes;
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
  if (!(scale > 0.0f) || !(scale <= FLT_MAX)) return SERQ_ESHAPE;
  if (batch->tokens == 0 || batch->seqs == 0) return SERQ_OK;
  if ((rc = kv_check_rows(q, ldq, ldqh, q_heads, D)) != SERQ_OK) return rc;
  if ((rc = kv_check_rows(out, ldo, ldoh, q_heads, D)) != SERQ_OK) return rc;
  if (!kv_aligned(lse, 4) || !kv_aligned(workspace, 16)) return SERQ_EALIGN;
  p.q = (const char*)q; p.out = (char*)out; p.lse = lse;
  p.ldq = 2 * ldq; p.ldqh = 2 * ldqh; p.ldo = 2 * ldo; p.ldoh = 2 * ldoh;
  p.q_heads = q_heads; p.group = q_heads / cache->heads; p.window = window; p.scale = scale;
  if (max_q > batch->tokens) max_q = (int)batch->tokens;
  const Plan k = plan_few(batch->tokens, batch->seqs, max_q, max_kv, window, cache->heads, p.group, D);
  p.direct = k.direct;
  p.rows_from = 0; p.rows_to = 0x7fffffff;
  const bool sliced = k.slices > 1 && workspace && workspace_bytes >= k.bytes;
  p.slices = sliced ? k.slices : 1;
  p.slice_keys = sliced ? k.slice_keys : 0x7fffff00;
  p.tickets = (uint32_t*)workspace;
  p.part = (float*)workspace + kTickets;
  return launch_paged_attn_few(p, dtype, cache->dtype == SERQ_F8, D, k.nb, k.blocks, (hipStream_t)stream);
}

}  // extern "C"
