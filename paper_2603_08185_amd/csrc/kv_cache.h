// What the kernels over the paged cache share: the cache and the batch as they are handed to a kernel, the checks of both, and where a
// token, a position and a page are found (include/serq_kv.h has the definitions).
#pragma once

#include "../../include/serq_kv.h"
#include "serq_device.h"

namespace serq {

struct KvView {
  char* k; char* v;
  const float* k_scale; const float* v_scale;
  int64_t k_page, k_token, k_head, v_page, v_token, v_head;   // bytes
  int pages, page_shift, heads;
  const int32_t* cu; const int32_t* len; const int32_t* table;
  int64_t table_ld;
  int width, seqs, tokens;
};

constexpr int64_t kKvTokens = 1 << 22;   // of a call (a workgroup of up to 512 threads each: a grid's threads are counted in 32 bits)

// of a table: positions are 32-bit numbers, and the kernels look up to 64 tiles past a sequence's end before they cut a position to it, and
// a window short of it and kKvTokens before its start
constexpr int64_t kKvPositions = (1ll << 31) - (1 << 23);

inline bool kv_aligned(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// q, k, v, out: a token's and a head's stride in elements
inline int kv_check_rows(const void* p, int64_t ld, int64_t ldh, int heads, int dim) {
  if (!p) return SERQ_ENULL;
  if (ld < 0 || ldh < 0 || (heads > 1 && ldh < dim)) return SERQ_ESHAPE;
  if (ld > ((int64_t)1 << 31) || ldh > ((int64_t)1 << 31)) return SERQ_ESHAPE;
  if ((ld % 8) != 0 || (ldh % 8) != 0 || !kv_aligned(p, 16)) return SERQ_EALIGN;
  return SERQ_OK;
}

inline int kv_check(const serq_kv_cache* c, const serq_kv_batch* b, int dtype, KvView& view) {
  if (!c || !b) return SERQ_ENULL;
  if (dtype != SERQ_F16 && dtype != SERQ_BF16) return SERQ_EDTYPE;
  if (c->dtype != dtype && c->dtype != SERQ_F8) return SERQ_EDTYPE;
  if (c->dim != 64 && c->dim != 128) return SERQ_ESHAPE;
  if (c->heads < 1 || c->heads > 1024 || c->pages < 0 || c->pages > 0x7fffffff) return SERQ_ESHAPE;
  if (c->page_size < 16 || c->page_size > 65536 || (c->page_size & (c->page_size - 1))) return SERQ_ESHAPE;
  if (b->seqs < 0 || b->seqs > 65536 || b->tokens < 0 || b->tokens > kKvTokens || b->table_width < 0) return SERQ_ESHAPE;
  if ((int64_t)b->table_width * c->page_size > kKvPositions || b->table_ld < b->table_width) return SERQ_ESHAPE;
  const int64_t unit = c->dtype == SERQ_F8 ? 16 : 8, es = c->dtype == SERQ_F8 ? 1 : 2;
  const int64_t st[6] = {c->k_page, c->k_token, c->k_head, c->v_page, c->v_token, c->v_head};
  for (int64_t s : st) {
    if (s < 0 || s > ((int64_t)1 << 40)) return SERQ_ESHAPE;
    if (s % unit) return SERQ_EALIGN;
  }
  if (c->k_token > (1 << 26) || c->v_token > (1 << 26)) return SERQ_ESHAPE;    // (16 rows lie within 2^31 bytes)
  if (b->tokens > 0 && b->seqs > 0) {
    if (!b->cu_q || !b->kv_len) return SERQ_ENULL;
    if (b->table_width > 0 && !b->table) return SERQ_ENULL;
    if (c->pages > 0 && (!c->k || !c->v)) return SERQ_ENULL;
  }
  if (!kv_aligned(c->k, 16) || !kv_aligned(c->v, 16) || !kv_aligned(b->cu_q, 4) || !kv_aligned(b->kv_len, 4) || !kv_aligned(b->table, 4))
    return SERQ_EALIGN;
  if (c->dtype == SERQ_F8 && (!kv_aligned(c->k_scale, 4) || !kv_aligned(c->v_scale, 4))) return SERQ_EALIGN;
  view.k = (char*)c->k; view.v = (char*)c->v;
  view.k_scale = c->dtype == SERQ_F8 ? c->k_scale : nullptr;
  view.v_scale = c->dtype == SERQ_F8 ? c->v_scale : nullptr;
  view.k_page = c->k_page * es; view.k_token = c->k_token * es; view.k_head = c->k_head * es;
  view.v_page = c->v_page * es; view.v_token = c->v_token * es; view.v_head = c->v_head * es;
  view.pages = (int)c->pages; view.heads = c->heads;
  view.page_shift = __builtin_ctz((unsigned)c->page_size);
  view.cu = b->cu_q; view.len = b->kv_len; view.table = b->table; view.table_ld = b->table_ld;
  // (without pages there is nothing to address: no position has one)
  view.width = c->pages > 0 ? b->table_width : 0;
  view.seqs = b->seqs; view.tokens = (int)b->tokens;
  return SERQ_OK;
}

// two fp32 values as E4M3 bytes in the low (HI = false) or high half of `old`: clipped to +-448, ties to even, NaN stays NaN
__device__ __forceinline__ float clip_e4m3(float x) { return x != x ? x : fminf(fmaxf(x, -448.0f), 448.0f); }
template <bool HI>
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, uint32_t old) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clip_e4m3(a), clip_e4m3(b), (int)old, HI);
}

}  // namespace serq
