"""The paged cache where a call is not the ordinary one: a later part of a batch over the whole batch's buffers, more tokens than were announced, windows, scales and
weights at the ends of their ranges, a workspace sized for another step, long caches, many query heads a key head."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as orc
from paper_2603_08185_amd import binding as serq
from tests._kv import DEV, Batch, check_attention
from tests.test_gpu_kv import _bits, _expected_append, _tables

pytestmark = pytest.mark.gpu

# the first sequence that is left has more keys than there are rows before it, so that a row taken for one of its own would find a place
PART = [(3, 5), (2, 33), (1, 40), (0, 9), (17, 60), (1, 100)]
CHUNKS = [(3, 5), (40, 90), (1, 70), (33, 150), (0, 0), (2, 300)]


def _later(B, n):
    """The sequences from n on; the rows of those before them belong to no sequence now."""
    B.cu, B.len, B.table, B.seqs = B.cu[n:], B.len[n:], B.table[n:], B.seqs[n:]
    B.d_cu, B.d_len, B.d_table = B.d_cu[n:], B.d_len[n:], B.d_table[n:]
    return B


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("first", [1, 2, 4, 6])
def test_append_a_later_part_of_a_batch(first, fp8):
    B = _later(Batch(PART, 8, 2, 128, 16, fp8=fp8, extra=2, seed=21), first)
    cos, sin = _tables(100, 128)
    want_q, want_K, want_V, seq = _expected_append(B, cos, sin, False)
    q_out = torch.full((B.T, 8, 128), 7.0, dtype=B.dt, device=DEV)
    serq.kv_append(B.q, B.k, B.v, *B.args(), cos, sin, k_scale=B.k_scale, v_scale=B.v_scale, q_out=q_out)
    mine = torch.from_numpy(seq >= 0)
    assert int(mine.sum()) == B.cu[-1] - B.cu[0] and (q_out[~mine.to(DEV)] == 7).all()
    assert torch.equal(_bits(q_out.cpu()[mine]), _bits(want_q[mine]))
    for got, want in ((B.K, want_K), (B.V, want_V)):              # (places that nothing was appended to hold NaN)
        got, nan = got.cpu().contiguous(), torch.isnan(want.float())
        assert torch.equal(nan, torch.isnan(got.float())) and torch.equal(_bits(got)[~nan], _bits(want)[~nan])


@pytest.mark.parametrize("seqs", [PART, CHUNKS])
@pytest.mark.parametrize("first", [1, 2, 3])
def test_attention_a_later_part_of_a_batch(seqs, first):
    B = Batch(seqs, 8, 2, 128, 16, extra=1, seed=22).fill()
    B.kv, B = B.kv[first:], _later(B, first)
    ws = serq.paged_attention_workspace(B.T, len(B.seqs), B.max_q, B.max_kv, 8, 2, 128, DEV)
    for use in (None, ws):
        out, lse = torch.full((B.T, 8, 128), 7.0, dtype=B.dt, device=DEV), torch.full((B.T, 8), 7.0, device=DEV)
        serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, out=out, lse=lse, ws=use)
        none = torch.ones(B.T, dtype=torch.bool, device=DEV)
        none[B.cu[0]:B.cu[-1]] = False
        assert (out[none] == 7).all() and (lse[none] == 7).all()
        out[none], lse[none] = 0, -float("inf")                   # (as the oracle has a row of no sequence)
        check_attention(B, out, lse, what=f"from sequence {first} on")


@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("n,L", [(1000, 500), (700, 5000), (300, 0), (90, 89)])
def test_more_tokens_than_max_q_stay_in_bounds(n, L, window):
    """Wrong results are all that such a call may give: a sequence whose first tokens lie before its start (a length that has been cut) has no key that its
    first block of rows sees, though its length counts many.  Nothing beside the batch's rows is written, and the workspace is ready for the next call."""
    good = Batch([(1, 700), (2, 900)], 8, 2, 128, 16, window=window, seed=23).fill()
    B = Batch([(1, 300), (n, max(L, n)), (2, 90)], 8, 2, 128, 16, window=window, seed=24, extra=3)
    B.d_len[1] = L
    table = torch.zeros((B.d_table.shape[0], B.width + 8), dtype=torch.int32, device=DEV)[:, :B.width]
    ws = serq.paged_attention_workspace(B.T, len(B.seqs), 2, max(L, 900), 8, 2, 128, DEV)
    for use in (None, ws):
        big = torch.full((B.T, 9, 136), 7.0, dtype=B.dt, device=DEV)
        lse = torch.full((B.T, 8), 7.0, device=DEV)
        serq.paged_attention(B.q, B.K, B.V, table, B.d_cu, B.d_len, 2, max(L, 900), window=window, out=big[:, :8, :128], lse=lse, ws=use)
        assert (big[:, 8:] == 7).all() and (big[:, :, 128:] == 7).all() and (big[-3:] == 7).all() and (lse[-3:] == 7).all()
    lse = torch.empty((good.T, 8), device=DEV)
    out = serq.paged_attention(good.q, *good.args(), good.max_q, good.max_kv, window=window, lse=lse, ws=ws)
    check_attention(good, out, lse, what="the call after it")


@pytest.mark.parametrize("seqs", [[(3, 2), (8, 3), (1, 50), (5, 5)], [(60, 20), (1, 50), (40, 40)]])
@pytest.mark.parametrize("window", [(1 << 31) - 1, (1 << 31) - 3, 1 << 30, 101])
def test_a_window_that_reaches_past_the_start_is_none(seqs, window):
    """Also where the first new tokens lie before the start of their sequence."""
    B = Batch(seqs, 8, 2, 128, 16, seed=25, extra=0).fill()
    ws = serq.paged_attention_workspace(B.T, len(B.seqs), B.max_q, B.max_kv, 8, 2, 128, DEV)
    for use in (None, ws):
        lse = torch.full((B.T, 8), 7.0, device=DEV)
        out = serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, window=window, lse=lse, ws=use)
        check_attention(B, out, lse, what=f"window {window}")


def _sink(n, L, Hq, Hkv, D, gap, page=64, seed=0):
    """A key that dominates, and L - 1 others that each weigh 2^-gap of it and together a good part of the sum: q is one channel of ones, the first key is 0
    there and the others -gap ln 2 / scale.  Values: 0 for the first key, 1 + |noise| / 4 for the others, so that what their weights lose shows."""
    B = Batch([(n, L)], Hq, Hkv, D, page, torch.float16, seed=seed).fill()
    B.qkv[:, :Hq * D] = 0
    B.q[..., 0] = 1
    k = torch.zeros(L, Hkv, D)
    k[1:, :, 0] = -gap * float(np.log(2.0)) * D ** 0.5
    v = 1 + torch.randn(L, Hkv, D, generator=torch.Generator().manual_seed(seed)).abs() / 4
    v[0] = 0
    at = np.arange(L)
    where, row = torch.from_numpy(B.table[0, at // page]).to(DEV), torch.from_numpy(at % page).to(DEV)
    for cache, x in ((B.K, k), (B.V, v)):
        cache[where, row] = x.half().to(DEV)
    B.kv = [[x.half().double().numpy() for x in (k, v)]]
    return B


# gap: weights of 2^-gap of the largest; 2^-20.5 is 11.3 steps of an fp16 number below 2^-14, 2^-24.4 three quarters of one
@pytest.mark.parametrize("gap", [17.97, 20.5, 24.4])
@pytest.mark.parametrize("n,Hq,Hkv,sliced", [(1, 4, 1, True), (1, 4, 1, False), (40, 2, 1, False), (40, 2, 1, True)])
def test_small_weights_beside_a_large_one_in_fp16(n, Hq, Hkv, sliced, gap):
    """Weights meet V as 16-bit numbers: bits of them may go, not parts of the result.  Errors, derived: the result's rounding, 2^-11 |out|; a weight's, 2^-11 of it or,
    below 2^-23 of the largest, half a step there, 2^-34 of the largest; the score, one product that is exact but for 2^-23 of its 17 to 25 in the exponent, twice: 2^-17
    of a weight; exponential, running factors and sums (32 + L / 16) 2^-22."""
    L, D = 60000, 128
    B = _sink(n, L, Hq, Hkv, D, gap)
    ws = serq.paged_attention_workspace(B.T, 1, n, L, Hq, Hkv, D, DEV) if sliced else None
    lse = torch.empty((n, Hq), device=DEV)
    out = serq.paged_attention(B.q, *B.args(), n, L, lse=lse, ws=ws).double().cpu().numpy()
    want, wlse, mag, _ = B.attention64()
    rel = 2.0 ** -11 + 2.0 ** (gap - 34) + 2.0 ** -17 + (32 + L / 16) * 2.0 ** -22
    assert (np.abs(out - want) <= 2.0 ** -11 * np.abs(want) + rel * mag).all(), np.abs(out / want - 1).max()
    assert (np.abs(lse.double().cpu().numpy() - wlse) <= 2.0 ** -17 + (32 + L / 16) * 2.0 ** -22 + 2.0 ** -20).all()


@pytest.mark.parametrize("seqs", [[(3, 5), (1, 40), (8, 130)], [(40, 90), (1, 70)]])
@pytest.mark.parametrize("scale", [1.5e-45, 1e-40, 1e-37])
def test_attention_the_smallest_scales(seqs, scale):
    """Products of the scale with the cache's own that 32 bits do not hold: every key a row sees weighs the same."""
    B = Batch(seqs, 8, 2, 128, 16, fp8=True, seed=26).fill()
    lse = torch.empty((B.T, 8), device=DEV)
    out = serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, scale=scale, k_scale=B.k_scale, v_scale=B.v_scale, lse=lse)
    check_attention(B, out, lse, scale, what=f"scale {scale}")


@pytest.mark.parametrize("seqs", [[(1, 9000)], [(5, 6000)], [(1, 4000), (1, 700), (1, 90)], [(100, 4000), (1, 700)], [(40, 3000)]])
def test_the_workspace_of_the_largest_step_serves_the_others(seqs):
    """Sized for a prompt of 8192 tokens, a long cache and a few users: smaller steps run as with all the room there could be."""
    B = Batch(seqs, 8, 2, 128, 16, seed=27).fill()
    ws = serq.paged_attention_workspace(8192, 4, 8192, 131072, 8, 2, 128, DEV)
    room = torch.zeros(256 << 20, dtype=torch.uint8, device=DEV)
    lse = torch.empty((B.T, 8), device=DEV)
    want = serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, ws=room)
    out = serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, lse=lse, ws=ws)
    check_attention(B, out, lse, what="workspace of the largest step")
    assert torch.equal(out, want)


def test_a_buffer_goes_between_attention_and_a_layer_through_init():
    """The workspaces of serq_paged_attn and of the layers are different things; initialised in between, one buffer is either."""
    N, K, r = 512, 4096, 32                                        # few channels, one token: the layer's slices meet in its workspace
    g = torch.Generator(device=DEV).manual_seed(0)
    pk = serq.pack_weights(torch.randn((N, K), generator=g, device=DEV).bfloat16() * K ** -0.5, None, r,
                           torch.arange(K, dtype=torch.int32, device=DEV), torch.bfloat16)
    xq, sc = serq.quantize_act(torch.randn((1, K), generator=g, device=DEV).bfloat16(), pk.s_inv, 8)
    B = Batch([(1, 9000)], 8, 2, 128, 16, seed=28).fill()
    own = serq.workspace(1, N, K, r, 8, DEV), serq.paged_attention_workspace(1, 1, 1, 9000, 8, 2, 128, DEV)
    one = torch.empty(max(w.numel() for w in own), dtype=torch.uint8, device=DEV)

    def layer(ws):
        return serq.linear(xq, sc, 8, pk.Wq, pk.wscale, 1, N, K, Rp=pk.Rp, r=r, ws=ws).clone()

    def attention(ws):
        return serq.paged_attention(B.q, *B.args(), 1, 9000, ws=ws)

    want = layer(own[0]), attention(own[1])
    for _ in range(3):
        for call, y in zip((layer, attention), want):
            serq._check("serq_workspace_init", serq.lib().serq_workspace_init(one.data_ptr(), one.numel(), serq._stream()))
            assert torch.equal(call(one), y) and torch.equal(call(one), y)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("seqs", [[(1, 9), (1, 3000), (2, 40)], [(40, 90), (1, 33), (130, 300)]])
def test_scores_of_minus_infinity_weigh_nothing(seqs, dt):
    """Keys of -inf in a channel where every query is 1: as if they were not there; a row that sees no other key is as one that sees none."""
    B = Batch(seqs, 8, 2, 128, 16, dt, seed=29).fill()
    B.q[..., 0] = 1
    hidden = []
    for b, (n, L) in enumerate(B.seqs):
        j = np.unique(np.concatenate([np.arange(0, L, 3), np.arange(L - n, L - n + n // 2), np.arange(L if b == 0 else 0)]))   # (of the first one: all)
        page, row = torch.from_numpy(B.table[b, j // 16]).to(DEV), torch.from_numpy(j % 16).to(DEV)
        B.K[page, row, :, 0] = -float("inf")
        hidden.append(j)
    q = B.q.double().cpu().numpy()
    ws = serq.paged_attention_workspace(B.T, len(B.seqs), B.max_q, B.max_kv, 8, 2, 128, DEV)
    for use in (None, ws):
        lse = torch.empty((B.T, 8), device=DEV)
        out = serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, lse=lse, ws=use).double().cpu().numpy()
        got = lse.double().cpu().numpy()
        for b, (n, L) in enumerate(B.seqs):
            for i in range(n):
                t, keys = B.cu[b] + i, np.setdiff1d(np.arange(L - n + i + 1), hidden[b])
                if len(keys) == 0:
                    assert not out[t].any() and np.isneginf(got[t]).all()
                    continue
                want, wl, mag, big = orc.attention(q[t:t + 1], B.kv[b][0][keys], B.kv[b][1][keys], 128 ** -0.5, len(keys) - 1)
                u = 2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -11
                esc = 136 * 2.0 ** -24 * big
                tol = u * np.abs(want) + (2 * u + 2 * esc[..., None] + (32 + L / 16) * 2.0 ** -22) * mag * 1.01 + 2.0 ** -24
                assert (np.abs(out[t] - want[0]) <= tol[0]).all()
                assert (np.abs(got[t] - wl[0]) <= esc[0] + (32 + L / 16) * 2.0 ** -22 + 2.0 ** -22 * np.abs(wl[0]) + 2.0 ** -21).all()


LONG = [  # new tokens, keys, query heads, key heads, with a workspace
    (40, 9000, 2, 1, False),                                       # the kernel for many rows, one slice: 141 tiles, whose places are looked up 64 a time
    (40, 9000, 2, 1, True),
    (3, 20000, 4, 1, False),                                       # the one for few, a sequence a workgroup
    (1, 131000, 8, 1, True),                                       # more parts than a wave has lanes
    (1, 131000, 1, 1, True),                                       # ... and as many as may meet
    (8, 60000, 4, 1, True),                                        # 32 rows
]


@pytest.mark.parametrize("n,L,Hq,Hkv,sliced", LONG)
@pytest.mark.parametrize("dt,fp8,D", [(torch.float16, False, 128), (torch.bfloat16, True, 128), (torch.bfloat16, False, 64), (torch.float16, True, 64)])
def test_attention_long_caches(n, L, Hq, Hkv, sliced, dt, fp8, D):
    B = Batch([(n, L)], Hq, Hkv, D, 64, dt, fp8, "hnd", seed=30).fill()
    ws = serq.paged_attention_workspace(n, 1, n, L, Hq, Hkv, D, DEV) if sliced else None
    for _ in range(2 if sliced else 1):
        lse = torch.empty((n, Hq), device=DEV)
        out = serq.paged_attention(B.q, *B.args(), n, L, k_scale=B.k_scale, v_scale=B.v_scale, lse=lse, ws=ws)
        check_attention(B, out, lse, what=f"{n} tokens over {L} keys")


@pytest.mark.parametrize("seqs", [[(1, 5000)], [(1, 700), (1, 33), (0, 0), (1, 1)], [(2, 40), (1, 300), (70, 200), (1, 9)], [(5, 900), (1, 1200)]])
@pytest.mark.parametrize("Hq,Hkv", [(64, 1), (33, 1), (80, 2), (130, 1)])
@pytest.mark.parametrize("window,fp8", [(0, False), (50, True)])
def test_attention_many_query_heads_a_key_head(seqs, Hq, Hkv, window, fp8):
    B = Batch(seqs, Hq, Hkv, 128, 16, window=window, fp8=fp8, seed=31, extra=1).fill()
    ws = serq.paged_attention_workspace(B.T, len(B.seqs), B.max_q, B.max_kv, Hq, Hkv, 128, DEV)
    for use in (None, ws, ws):
        lse = torch.empty((B.T, Hq), device=DEV)
        out = serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, window=window, k_scale=B.k_scale, v_scale=B.v_scale, lse=lse, ws=use)
        check_attention(B, out, lse, what=f"{Hq} query heads, {Hkv} key heads")


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_append_every_16_bit_value_passes_unchanged(dt):
    """Subnormal numbers, signed zeros and infinities among them; NaN stays NaN."""
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dt).view(1024, 1, 64).to(DEV)
    B = Batch([(1024, 1024)], 1, 1, 64, 16, dt)
    q = serq.kv_append(x, x, x, *B.args())
    page, row = (torch.from_numpy(a).to(DEV) for a in orc.slots(*orc.positions(B.cu, B.len, 1024), B.table, 16, B.pages))
    nan = torch.isnan(x)
    for got in (q, B.K[page, row], B.V[page, row]):
        assert torch.equal(torch.isnan(got), nan) and torch.equal(_bits(got)[~nan], _bits(x)[~nan])
