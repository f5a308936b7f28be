/*
 * serq_kv.h -- what lies between the q/k/v projection and the o projection of a decoder block, exported by
 * libserq.so: the rotation of queries and keys by their positions, a paged cache of keys and values, and the
 * attention of new tokens over it.  (The paper times whole models, Sec. 4.3 and Table 3, and takes these steps
 * as given; their arithmetic below is the usual one.)
 *
 * Conventions are those of serq.h: device pointers, work enqueued on `stream`, nothing allocated, no waiting,
 * SERQ_OK or a negative SERQ_E* code, nothing throws.  The structures themselves are read on the host during the
 * call.  Data pointers are 16-byte aligned, int32 and float arrays 4-byte aligned.
 *
 * One call serves a ragged batch: seqs sequences, of which sequence b has n_b = cu_q[b+1] - cu_q[b] >= 0 new tokens
 * (rows cu_q[b] .. cu_q[b+1]-1 of q, k, v and out) and kv_len[b] = L_b keys in the cache once the new ones are in.  New
 * token i of sequence b is at position p = L_b - n_b + i.  Position p of sequence b lives in page table[b, p / page_size],
 * row p % page_size.  cu_q, kv_len and table lie in device memory, so that a captured graph can be replayed for the
 * next step; they are not checked on the host.  A sequence without new tokens is an empty slot.  cu_q must not decrease.
 * Rows of q, k and v before cu_q[0] and from cu_q[seqs] on belong to no sequence: nothing is written for them.  So a later part of
 * cu_q, kv_len and table serves some of a batch's sequences over the buffers of all.
 */
#ifndef SERQ_KV_H_
#define SERQ_KV_H_

#include "serq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* dtype of a cache: OCP E4M3 (finite: largest value 448), value = code * scale of the key head */
#define SERQ_F8   4

typedef struct serq_kv_cache {
  void*        k;                 /* element (page, row, head, d) at page*k_page + row*k_token + head*k_head + d */
  void*        v;
  const float* k_scale;           /* SERQ_F8: [heads] fp32 each, positive, NULL = ones; else ignored */
  const float* v_scale;
  int64_t      k_page, k_token, k_head;   /* strides in elements, multiples of 16 bytes; k_token, v_token up to 2^26 */
  int64_t      v_page, v_token, v_head;
  int64_t      pages;             /* page numbers in table are 0 .. pages-1 */
  int32_t      page_size;         /* a power of two, 16 .. 65536 */
  int32_t      heads;             /* key heads, 1 .. 1024 */
  int32_t      dim;               /* channels of a head: 64 or 128 */
  int32_t      dtype;             /* the dtype of q (SERQ_F16 or SERQ_BF16), or SERQ_F8 */
} serq_kv_cache;

typedef struct serq_kv_batch {
  const int32_t* cu_q;            /* [seqs+1] */
  const int32_t* kv_len;          /* [seqs] */
  const int32_t* table;           /* [seqs, table_width], row stride table_ld */
  int64_t        table_ld;
  int64_t        tokens;          /* rows of q, k, v and out: 0 .. 2^22 */
  int32_t        table_width;     /* table_width * page_size up to 2^31 - 2^23 */
  int32_t        seqs;            /* 0 .. 65536 */
} serq_kv_batch;

/*
 * Rotate and append: for every new token
 *   q_out[t,h,:] = rot(q[t,h,:]),  K[slot,h,:] = rot(k[t,h,:]),  V[slot,h,:] = v[t,h,:]
 * where rot turns `rot_dim` channels of a head, frequency f < rot_dim/2, by the angle whose cosine and sine are
 * cos_table[p', f] and sin_table[p', f]:  (x, y) -> (x c - y s, y c + x s), the pair being channels (f, f + rot_dim/2), or
 * (2f, 2f+1) if `interleaved`; the other channels pass unchanged.  p' is the token's position, or positions[t] where
 * `positions` is given; it is clamped to the table's rows.  Every product and sum is one fp32 operation, rounded once to
 * the type it is stored in.  A SERQ_F8 cache stores rne(clip(x / scale, -448, 448)) (NaN stays NaN).
 *   q [tokens, q_heads, dim], k, v [tokens, cache->heads, dim] in dtype (SERQ_F16 / SERQ_BF16), strides in elements
 *     (multiples of 8) of a token (ldq) and of a head (ldqh): parts of one fused buffer, for instance.
 *   q_out like q; it may be q itself (same strides).  q_heads = 0: keys and values only (q, q_out ignored).
 *   rot_dim a multiple of 16 up to dim; 0: no rotation (tables ignored).  Tables [table_rows, rot_dim/2] fp32, contiguous.
 * A token whose position is negative, or whose page number is missing from the table (position >= table_width *
 * page_size) or outside 0 .. pages-1, stores no key and no value: page -1 marks such a hole.  Two tokens of one call must not share
 * a slot, and the cache must not overlap k, v, q or q_out.
 */
int serq_kv_append(const void* q, int64_t ldq, int64_t ldqh, int q_heads,
                   const void* k, int64_t ldk, int64_t ldkh, const void* v, int64_t ldv, int64_t ldvh, int dtype,
                   const float* cos_table, const float* sin_table, int64_t table_rows, int rot_dim, int interleaved,
                   const int32_t* positions, const serq_kv_cache* cache, const serq_kv_batch* batch,
                   void* q_out, int64_t ldqo, int64_t ldqoh, void* stream);

/*
 * The same for models that normalise the queries and keys of every head: before the rotation
 *   x[d] = fl(fl(x[d] * r) * weight[d]),   r = 1 / sqrt(mean_d x[d]^2 + eps) over the head's dim channels,
 * r formed in 64 bits, rounded to fp32, at most the largest finite number (0 where the root is 0 or infinite: a head with an
 * infinite channel becomes NaN there and 0 elsewhere before the rotation, one with NaN becomes NaN).  q_weight for queries, k_weight for keys: [dim] fp32,
 * 16-byte aligned, the same for all heads; NULL: those are not normalised (both NULL: serq_kv_append).  Values are never normalised.  eps finite, not
 * negative.  Everything else as serq_kv_append.
 */
int serq_kv_append_norm(const void* q, int64_t ldq, int64_t ldqh, int q_heads,
                        const void* k, int64_t ldk, int64_t ldkh, const void* v, int64_t ldv, int64_t ldvh, int dtype,
                        const float* q_weight, const float* k_weight, float eps,
                        const float* cos_table, const float* sin_table, int64_t table_rows, int rot_dim, int interleaved,
                        const int32_t* positions, const serq_kv_cache* cache, const serq_kv_batch* batch,
                        void* q_out, int64_t ldqo, int64_t ldqoh, void* stream);

/*
 * Attention over the cache: query head h reads key head h / (q_heads / cache->heads),
 *   s_j = scale * q[t,h,:] . K_j,   out[t,h,:] = sum_j softmax(s)_j V_j,   lse[t,h] = log sum_j exp(s_j),
 * over the positions j with 0 <= j <= p and, where window > 0, j > p - window.  A row that sees no key (p < 0) gives out = 0,
 * lse = -inf.  What a row does not see does not reach its result, whatever it holds, NaN and infinities among it; pages that hold no
 * position that a token of the call sees are not read, and their table entries may be anything.  A key whose score is -inf
 * weighs nothing, and a row that sees only such keys is as one that sees none.  (Else NaN or infinite values that a row does see make its result NaN or
 * infinite, which of the two is not defined.)  Page numbers outside 0 .. pages-1 are clamped, lengths past
 * table_width * page_size cut (nothing is read out of bounds; the result is then meaningless).
 *   q, out [tokens, q_heads, dim] in dtype (SERQ_F16 / SERQ_BF16), strides as above; q_heads a multiple of cache->heads.  tokens * q_heads is
 *          at most 2^30, seqs * cache->heads 2^22.
 *   scale  positive and finite.
 *   max_q, max_kv  upper bounds of n_b and L_b, by which the kernel and the number of slices are chosen (host values).  Results differ with them as
 *          sums of another order and weights rounded against another running maximum do, within the errors below.  More tokens or keys than that give SERQ_OK and wrong results, but
 *          nothing is read or written out of bounds.
 *   lse    [tokens, q_heads] fp32, or NULL.
 * Scores, statistics and sums are fp32.  The softmax' weights are rounded to `dtype` for their product with V, as the matrix instruction takes them; their
 * sum takes them unrounded.  So a result is within about 2^-8 (bf16) or 2^-11 (fp16) of sum_j softmax_j |V_j|, and rounded once.
 *   workspace  serq_paged_attn_workspace_bytes(...) bytes prepared by serq_workspace_init: where the slices of long caches meet.  What it
 *          returns serves every call of up to as many tokens and sequences, max_q and max_kv, with the same heads: sized once for the largest step.
 *          NULL / 0, or too little, makes the call do without slices, or with fewer.  Left ready for the next call; two calls that share one
 *          must not overlap in time.  It is this function's own: what it keeps zero and what it leaves behind lie elsewhere than the layers' (serq_linear and
 *          the like), so a buffer that goes from one to the other has to pass through serq_workspace_init in between.
 */
int serq_paged_attn(const void* q, int64_t ldq, int64_t ldqh, int q_heads, int dtype, const serq_kv_cache* cache,
                    const serq_kv_batch* batch, int max_q, int64_t max_kv, float scale, int window,
                    void* out, int64_t ldo, int64_t ldoh, float* lse,
                    void* workspace, size_t workspace_bytes, void* stream);
size_t serq_paged_attn_workspace_bytes(int64_t tokens, int seqs, int max_q, int64_t max_kv, int q_heads, int kv_heads, int dim);

/*
 * The same with what some models put between the scores and the softmax.  A row of token t at position p has the scores
 *   s_j = scale * q.K_j                             (plain)
 *   s_j = cap * tanh(scale * q.K_j / cap)           (cap > 0)
 *   s_j = scale * q.K_j - slopes[h] * |p - j|       (slopes)
 * over the keys j with see_from[t] <= j < see_to[t] that lie in the sequence (0 <= j < L_b) and, where window > 0, j > p - window.  Without see_from
 * rows see from 0, without see_to up to their own position (p + 1): several documents one after the other in a sequence have the start of each row's
 * own in see_from; a prefix that all its rows see, both ways, has its length in see_to of those rows; a row of padding has 0 there.  A row that
 * sees no key gives out = 0, lse = -inf; lse is of the scores as above.
 *   mod NULL, or all of it zero: serq_paged_attn.  cap and slopes together: SERQ_EUNSUPPORTED.
 * What a row does not see does not reach its result, as above.  Pages between the first and the last key that a sequence's rows see may be read whatever lies between
 * (their page numbers are clamped); pages outside are not.  With a cap a product of -inf has the score -cap and weighs as such.  A capped score is good to
 * cap * 2^-20 beside what scale * q.K_j is; a biased one is an fp32 sum that the bias is part of, so it is good to about
 * 2^-24 (dim + 8) slopes[h] |p - j| (of no account where a row sees keys near its own; a row whose nearest key has a bias beyond 2^24 may count as one that sees none).
 * Chunks over a long cache are cut into slices by max_kv, not by what their rows see: where that is little of it, few of the slices have work.
 * Everything else (workspace, bounds, types) as serq_paged_attn.
 */
#define SERQ_ATTN_MAX_CAP 1024.0f
typedef struct serq_attn_mod {
  const float*   slopes;          /* [q_heads] fp32, finite, or NULL */
  const int32_t* see_from;        /* [tokens], or NULL */
  const int32_t* see_to;          /* [tokens], or NULL */
  float          cap;             /* up to SERQ_ATTN_MAX_CAP; 0: none */
} serq_attn_mod;

int serq_paged_attn_mod(const void* q, int64_t ldq, int64_t ldqh, int q_heads, int dtype, const serq_kv_cache* cache,
                        const serq_kv_batch* batch, int max_q, int64_t max_kv, float scale, int window, const serq_attn_mod* mod,
                        void* out, int64_t ldo, int64_t ldoh, float* lse,
                        void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SERQ_KV_H_ */
