// serq_paged_attn: argument checks, the choice of kernel and of the slices of a long cache (include/serq_kv.h; the kernels say what they do).
#include <math.h>

#include "paged_attn.h"

namespace serq {
namespace {

// A workspace: the tickets of the kernel for few rows, those of the kernel for many, whatever the call; then the slots of the first, those of the second.
constexpr int kTickets = 4096;
constexpr size_t kTicketBytes = 2 * kTickets * 4;

// Keys of a share of the kernel for few rows, at least: a share of its own costs its start and the meeting, a longer one more rounds of loads.
// Measured with 128 / 256 / 512 / 1024 (us, one token, 8 key heads): 1000 keys 8.4 / 8.8 / 10.9 / 13.7, 8000 keys 16.1 / 13.4 / 16.1 / 23.2.
// Whoever joins a sequence reads a slot of all its rows for each of its shares, so the time that grows with the keys of a share stands against one that grows
// with rows and shares: the least of both lies where the square of a share's keys is as rows times keys.  Measured (us, 256 / such shares / their keys
// squared twice that): 8 tokens of 4 rows over 32000 keys, 8 key heads, 66.9 / 50.1 / 53.7; one token over 60000, one key head of 32 rows 124.7 / 53.4 / 54.9,
// of 8 rows 40.5 / 27.6 / 28.0; over 30000, two key heads of 16 rows, 41.6 / 29.8 / 30.6.
constexpr int kFewKeys = 256;
int64_t few_keys(int64_t rows, int64_t keys) {
  const int64_t n = (int64_t)sqrt((double)rows * (double)keys);
  return n > kFewKeys ? (n + 63) / 64 * 64 : kFewKeys;
}

// (rows fit 31 bits, the threads of a grid 32)
bool counts_ok(int64_t tokens, int64_t seqs, int q_heads, int heads) {
  return tokens * q_heads <= (1 << 30) && seqs * heads <= (1 << 22);
}

// One kernel's share of a call.
struct Plan {
  int blocks, slices, slice_keys;
  size_t bytes;           // of slots
};

constexpr size_t kManyRoom = 46u << 20;                        // most that its slices take

// The kernel for many rows: blocks of rows times key heads are the workgroups; where they would leave compute units idle, the keys (at most `keys` that
// a row block sees) are cut into slices.  Taken is the number of slices with the shortest time.  A tile of 64 keys takes a workgroup 1.08 us on a
// compute unit of its own, 1.85 beside another; to begin takes 5 us, to begin and to meet 8 and one a slice.  `blocks` counts a block more for each
// sequence than may be needed (every sequence's last one is half empty on average); `full` is about what there is.
// Measured (32 query and 8 key heads; us with 1 / 2 / 3 / 4 / 5 / 8 slices): 384 tokens after 3500 66.6 / 43.1 / 44.8 / 45.5 / 45.2 / 48.4, 100 after 30000
// 469 / 245 / 171 / 134 / 114 / 87, 512 fresh ones 14.9 / 16.9 / 17.3 / 21.5; 512 after 32000 with 2 / 4 292 / 272, 256 after 8000 with 3 / 4 56.5 / 50.6.
constexpr int64_t kGrain = 128;                                // keys of a slice are a multiple of it
Plan plan_many(int blocks, int64_t full, int heads, int64_t keys, int64_t cus, size_t slot_floats, size_t room) {
  Plan k{blocks, 1, 0x7fffff00, 0};
  const int64_t units = (int64_t)blocks * heads, slot = (int64_t)slot_floats * 4, bytes_most = (int64_t)(room < kManyRoom ? room : kManyRoom);
  if (units <= 0 || units > kTickets || keys <= kGrain) return k;
  double least = 0;
  for (int64_t n = 1; n <= kMaxTileSlices && (n == 1 || units * n * slot <= bytes_most); ++n) {
    const int64_t each = ((keys + n - 1) / n + kGrain - 1) / kGrain * kGrain;
    if ((keys + each - 1) / each != n) continue;
    const double a_unit = (double)(full * heads * n) / (double)cus;
    const double slow = a_unit <= 1.0 ? 1.08 : a_unit <= 2.0 ? 1.85 : 0.93 * a_unit + 0.4;
    const double time = slow * (double)((each + 63) / 64 + (n > 1 ? 8 + n : 5));
    if (n == 1 || time < 0.95 * least) {
      least = time;
      k.slices = (int)n;
      k.slice_keys = (int)each;
    }
  }
  if (k.slices > 1) k.bytes = (size_t)(units * k.slices * slot);
  else k.slice_keys = 0x7fffff00;
  return k;
}

// Workgroups of the kernel for few rows for a key head, where `together` run together.
int64_t few_shares(int64_t together, int seqs, int heads, int64_t keys) {
  const int64_t most = seqs * ((keys + kFewKeys - 1) / kFewKeys + 1);
  int64_t each = (together + heads - 1) / heads;
  if (each > most) each = most;
  return each > kTickets / heads ? kTickets / heads : each;
}
size_t few_slots_bytes(int64_t each, int heads, int nb, int D) { return (size_t)(each * heads) * 2 * paged_attn_few_slot_floats(nb, D) * 4; }
int many_blocks(int64_t tokens, int seqs, int group) { return (int)(tokens * group / kTileRows) + seqs; }

struct Plans {
  bool few, many;         // which kernels have work
  int few_rows, nb;       // sequences with up to few_rows rows are the first one's where both have; its blocks have 16 nb
  Plan f, m;
};

// room: bytes of the workspace
Plans plans(int64_t tokens, int seqs, int max_q, int64_t max_kv, int window, int heads, int group, int D, bool f8, size_t room) {
  Plans k{};
  if (max_q > tokens) max_q = (int)tokens;
  if (max_kv > 0x7fffffff) max_kv = 0x7fffffff;
  const int64_t rows = (int64_t)max_q * group;
  // The kernel for few rows holds 16 or 32 of them.  Measured on sequences of 17 to 32 (us, few rows / many; 4 rows a token): 1 of 8 tokens after 4000
  // 25.1 / 27.9, 1 of 6 after 30000 56.3 / 68.1, 1 of 5 after 300 13.1 / 10.2, 4 of 5 after 3000 29.3 / 26.1: it holds its own where keys are many, and
  // one launch then serves drafts beside single tokens.
  k.many = rows > 32;
  k.few = !k.many || (seqs > 1 && tokens < (int64_t)max_q * seqs);   // (a sequence alone, or all alike: none is short)
  // beside a chunk, what is short is a token or a few
  k.few_rows = k.many && group <= 16 ? 16 : 32;
  k.nb = rows <= 16 || k.few_rows == 16 ? 1 : 2;
  int64_t keys = max_kv;
  if (window > 0 && keys > (int64_t)window + max_q) keys = (int64_t)window + max_q;
  const int64_t cus = device_cu_count();
  room = room > kTicketBytes ? room - kTicketBytes : 0;
  if (k.few) {
    // As many workgroups as run together, each with an equal share of a head's keys; or a workgroup for every sequence and head, where sequences are
    // many and short: a share then is several stretches, each of which has to get going, and the longest sequence is soon done with.  Measured (us, shares
    // / whole sequences, 8 key heads, 512 run together, lengths up to 16 times apart): 70 up to 8000 140 / 232, 200 up to 4000 223 / 264, 250 up to
    // 2000 141 / 151, 300 up to 1000 104 / 101, 600 up to 600 140 / 113, 1200 up to 600 309 / 238; 128 of 4000 356 / 359.
    const int64_t together = cus * paged_attn_few_resident(k.nb, f8, D), whole = (int64_t)seqs * heads;
    const int64_t slots = (int64_t)few_slots_bytes(1, heads, k.nb, D);                    // bytes of a workgroup for each head
    // Where a sequence's parts and rows are many, a workgroup for every compute unit: half as many slots meet, and a unit streams as fast alone.  Measured (us,
    // as many as run together / one a unit, 8 key heads): 1 token over 131000 88.3 / 84.3, over 32000 32.8 / 29.9, 8 over 130000 134.9 / 115.9, 4 of 8
    // tokens over 8000 53.5 / 44.4; one token each of 255 sequences of up to 2000 157 / 163.
    const int64_t rows_few = rows <= k.few_rows ? rows : group;
    int64_t each = (together + heads - 1) / heads;
    each = few_shares(seqs > 0 && each / seqs * rows_few >= 256 ? cus : together, seqs, heads, keys);
    if (each > (int64_t)room / slots) each = (int64_t)room / slots;
    k.f = Plan{(int)whole, 1, 0, 0};
    if (whole * 256 < keys * together && each > 0) k.f = Plan{(int)each * heads, 2, (int)few_keys(rows_few, keys), (size_t)(each * slots)};
    room -= k.f.bytes;
  }
  if (k.many) {
    const int blocks = many_blocks(tokens, seqs, group);
    // (sequences of about the longest one's length, and half of the last block of each)
    const int64_t alike = 2 * tokens / max_q < seqs ? 2 * tokens / max_q : seqs;
    k.m = plan_many(blocks, (tokens * group + kTileRows - 1) / kTileRows + (alike - 1) / 2, heads, keys, cus, paged_attn_tile_slot_floats(D), room);
  }
  return k;
}

// The most that a call of up to these sizes, with either cache and any window, takes of a workspace: a caller who sizes one for its largest step decodes with
// the same one, so what matters is not this step's own plan (a long prompt alone needs no slices).
size_t most_bytes(int64_t tokens, int seqs, int max_q, int64_t max_kv, int heads, int group, int D) {
  const int64_t rows = (max_q < tokens ? max_q : tokens) * group, cus = device_cu_count();
  if (max_kv > kKvPositions) max_kv = kKvPositions;
  const int nb = rows > 16 ? 2 : 1;
  const int resident = nb > 1 ? paged_attn_few_resident(nb, false, D) : paged_attn_few_resident(nb, true, D);   // (the larger one: E4M3)
  size_t bytes = kTicketBytes + few_slots_bytes(few_shares(cus * resident, seqs, heads, max_kv), heads, nb, D);
  if (rows > 32 && max_kv > kGrain) {
    int64_t units = (int64_t)many_blocks(tokens, seqs, group) * heads, slices = (max_kv + kGrain - 1) / kGrain;
    if (units > kTickets) units = kTickets;
    if (slices > kMaxTileSlices) slices = kMaxTileSlices;
    const size_t slots = (size_t)(units * slices) * paged_attn_tile_slot_floats(D) * 4;
    bytes += slots < kManyRoom ? slots : kManyRoom;
  }
  return bytes;
}

}  // namespace
}  // namespace serq

using namespace serq;

extern "C" {

size_t serq_paged_attn_workspace_bytes(int64_t tokens, int seqs, int max_q, int64_t max_kv, int q_heads, int kv_heads, int dim) {
  if (tokens < 0 || tokens > kKvTokens || seqs < 0 || seqs > 65536 || max_q < 0 || max_kv < 0 || kv_heads < 1 || kv_heads > 1024 ||
      q_heads < 1 || q_heads > 65535 || q_heads % kv_heads || (dim != 64 && dim != 128) || !counts_ok(tokens, seqs, q_heads, kv_heads))
    return 0;
  return most_bytes(tokens, seqs, max_q, max_kv, kv_heads, q_heads / kv_heads, dim);
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
  if (!counts_ok(batch->tokens, batch->seqs, q_heads, cache->heads)) return SERQ_ESHAPE;
  if (!(scale > 0.0f) || !(scale <= FLT_MAX)) return SERQ_ESHAPE;
  if (batch->tokens == 0 || batch->seqs == 0) return SERQ_OK;
  if ((rc = kv_check_rows(q, ldq, ldqh, q_heads, D)) != SERQ_OK) return rc;
  if ((rc = kv_check_rows(out, ldo, ldoh, q_heads, D)) != SERQ_OK) return rc;
  if (!kv_aligned(lse, 4) || !kv_aligned(workspace, 16)) return SERQ_EALIGN;
  p.q = (const char*)q; p.out = (char*)out; p.lse = lse;
  p.ldq = 2 * ldq; p.ldqh = 2 * ldqh; p.ldo = 2 * ldo; p.ldoh = 2 * ldoh;
  p.q_heads = q_heads; p.group = q_heads / cache->heads; p.window = window; p.scale = scale;
  const bool f8 = cache->dtype == SERQ_F8;
  // (as wide as the table or wider: it hides nothing, and the position of a token before the start less such a window would not fit 32 bits)
  if (window >= (int64_t)batch->table_width * cache->page_size) p.window = window = 0;
  if (!workspace) workspace_bytes = 0;
  const Plans k = plans(batch->tokens, batch->seqs, max_q, max_kv, window, cache->heads, p.group, D, f8, workspace_bytes);
  AttnParams few = p, many = p;
  few.slices = k.f.slices; few.slice_keys = k.f.slice_keys;
  few.rows_from = 0; few.rows_to = k.many ? k.few_rows + 1 : 0x7fffffff;
  few.tickets = (uint32_t*)workspace;
  few.part = (float*)((char*)workspace + kTicketBytes);
  many.slices = k.m.slices; many.slice_keys = k.m.slice_keys;
  many.rows_from = k.few ? k.few_rows + 1 : 0; many.rows_to = 0x7fffffff;
  many.tickets = few.tickets + kTickets;
  many.part = (float*)((char*)workspace + kTicketBytes + k.f.bytes);
  hipStream_t st = (hipStream_t)stream;
  if (k.few && k.many && k.nb == 1) return launch_paged_attn_mixed(many, few, dtype, f8, D, k.m.blocks, k.f.blocks, st);
  if (k.many && (rc = launch_paged_attn_tile(many, dtype, f8, D, k.m.blocks, st)) != SERQ_OK) return rc;
  return k.few ? launch_paged_attn_few(few, dtype, f8, D, k.nb, k.f.blocks, st) : SERQ_OK;
}

}  // extern "C"
