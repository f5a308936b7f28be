"""The paged cache on the GPU: rotation and append against the same fp32 operations one by one (bit for bit) and against 64 bits; attention
against 64 bits, with NaN in everything that a call must not look at."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as orc
from paper_2603_08185_amd import binding as serq
from tests._kv import DEV, Batch, check_attention
from tests._util import replay_check

pytestmark = pytest.mark.gpu

RAGGED = [(3, 5), (0, 0), (1, 1), (17, 40), (0, 9), (2, 33), (1, 16), (5, 5), (1, 100)]


def _tables(rows, rot, seed=0):
    g = torch.Generator().manual_seed(seed)
    a = torch.rand(rows, rot // 2, generator=g, dtype=torch.float64) * 6.28
    return a.cos().float().to(DEV), a.sin().float().to(DEV)


def _expected_append(B, cos, sin, inter, at=None):
    """fp32, operation by operation; q_out and the caches as 16-bit / E4M3 tensors on the host."""
    c, s = (x.cpu().numpy() if x is not None else np.zeros((1, 0), np.float32) for x in (cos, sin))
    rot = 2 * c.shape[1]
    seq, pos = orc.positions(B.cu, B.len, B.T)
    turned = np.clip(pos if at is None else at, 0, c.shape[0] - 1)
    page, row = orc.slots(seq, pos, B.table, B.page, B.pages)
    q, k = (orc.rotate(x.float().cpu().numpy(), c[turned], s[turned], rot, inter, np.float32) for x in (B.q, B.k))
    v = B.v.float().cpu().numpy()
    K, V = B.K.cpu().contiguous(), B.V.cpu().contiguous()
    for t in range(B.T):
        if page[t] < 0:
            continue
        for cache, x, sc in ((K, k, B.k_scale), (V, v, B.v_scale)):
            y = torch.from_numpy(x[t])
            if B.fp8:
                y = (y / sc.cpu()[:, None]).clamp(-448, 448).to(cache.dtype)
                cache.view(torch.uint8)[page[t], row[t]] = y.view(torch.uint8)
            else:
                cache[page[t], row[t]] = y.to(cache.dtype)
    return torch.from_numpy(q).to(B.dt), K, V, seq


def _bits(x):
    return x.contiguous().view(torch.uint8 if x.element_size() == 1 else torch.int16)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D,rot,page,order", [(8, 2, 128, 128, 16, "nhd"), (3, 1, 128, 64, 32, "hnd"), (4, 4, 64, 16, 16, "hnd"),
                                                     (14, 2, 64, 64, 64, "nhd"), (64, 8, 128, 128, 32, "hnd"), (2, 2, 64, 0, 128, "nhd")])
def test_append(dt, fp8, inter, Hq, Hkv, D, rot, page, order):
    B = Batch(RAGGED, Hq, Hkv, D, page, dt, fp8, order, extra=2, seed=Hq + D)
    for b in range(len(B.seqs)):                                  # every page of a sequence that appends is its own
        assert all(0 <= B.table[b, i] < B.pages for i in range(-(-B.seqs[b][1] // page))) or B.seqs[b][0] == 0
    cos, sin = _tables(100, rot) if rot else (None, None)
    want_q, want_K, want_V, seq = _expected_append(B, cos, sin, inter)
    big = torch.full((B.T, Hq + 1, D + 8), 7.0, dtype=dt, device=DEV)
    q_out = big[:, :Hq, :D]                                        # strides of its own
    serq.kv_append(B.q, B.k, B.v, *B.args(), cos, sin, interleaved=inter, k_scale=B.k_scale, v_scale=B.v_scale, q_out=q_out)
    mine = torch.from_numpy(seq >= 0)
    assert torch.equal(_bits(q_out.cpu()[mine]), _bits(want_q[mine]))
    assert (big[:, Hq:] == 7).all() and (big[:, :, D:] == 7).all() and (q_out[~mine.to(DEV)] == 7).all()
    for got, want in ((B.K, want_K), (B.V, want_V)):
        got = got.cpu().contiguous()
        nan = torch.isnan(want.float())
        assert torch.equal(nan, torch.isnan(got.float()))
        assert torch.equal(_bits(got)[~nan], _bits(want)[~nan])


def test_append_against_64_bits():
    B = Batch([(40, 90), (1, 64)], 8, 2, 128, 16, seed=3)
    cos, sin = _tables(100, 128)
    q_out = serq.kv_append(B.q, B.k, B.v, *B.args(), cos, sin)
    seq, pos = orc.positions(B.cu, B.len, B.T)
    c, s = cos.double().cpu().numpy()[pos], sin.double().cpu().numpy()[pos]
    x = B.q.double().cpu().numpy()
    want = orc.rotate(x, c, s, 128, False)
    ax, ac, as_ = np.abs(x), np.abs(c), np.abs(s)
    size = np.concatenate([orc.rotate(ax, ac, -as_, 128, False)[..., :64], orc.rotate(ax, ac, as_, 128, False)[..., 64:]], -1)   # |x c| + |y s|
    err = np.abs(q_out.double().cpu().numpy() - want)
    assert (err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -22 * size + 2.0 ** -133).all()


def test_append_positions_in_place_and_keys_only():
    B = Batch(RAGGED, 8, 2, 128, 16, seed=5)
    cos, sin = _tables(50, 128)
    at = np.random.RandomState(1).randint(-3, 60, B.T).astype(np.int32)   # some past the table, some negative: its ends
    want_q, want_K, want_V, _ = _expected_append(B, cos, sin, False, at)
    q = B.q.clone()
    got = serq.kv_append(q, B.k, B.v, *B.args(), cos, sin, positions=torch.from_numpy(at).to(DEV), q_out=q)
    assert got is q and torch.equal(_bits(q.cpu()), _bits(want_q))
    for a, b in ((B.K, want_K), (B.V, want_V)):
        nan = torch.isnan(b)
        assert torch.equal(nan, torch.isnan(a.cpu())) and torch.equal(_bits(a.cpu())[~nan], _bits(b)[~nan])
    C = Batch(RAGGED, 8, 2, 128, 16, seed=5)
    assert serq.kv_append(None, C.k, C.v, *C.args(), cos, sin, positions=torch.from_numpy(at).to(DEV)) is None
    assert torch.equal(_bits(C.K).view(torch.uint8), _bits(B.K).view(torch.uint8)) and torch.equal(_bits(C.V), _bits(B.V))


def test_append_holes_and_ends():
    """A token without a place -- a hole or a wild number in the table, a position past the table or before the start -- leaves the cache alone."""
    B = Batch([(4, 40), (3, 2), (20, 64), (2, 32)], 4, 2, 64, 16, seed=9, width=3)       # the third reaches one page too far
    B.table[0, 2], B.table[2, 2], B.table[3, 1] = -1, 1 << 30, B.pages
    B.d_table.copy_(torch.from_numpy(B.table.astype(np.int32)))
    cos, sin = _tables(100, 64)
    want_q, want_K, want_V, _ = _expected_append(B, cos, sin, False)
    q_out = serq.kv_append(B.q, B.k, B.v, *B.args(), cos, sin)
    assert torch.equal(_bits(q_out.cpu()), _bits(want_q))
    for a, b in ((B.K, want_K), (B.V, want_V)):
        nan = torch.isnan(b)
        assert (~nan).any() and torch.equal(nan, torch.isnan(a.cpu())) and torch.equal(_bits(a.cpu())[~nan], _bits(b)[~nan])


def test_append_e4m3_every_code_tie_and_special():
    """Values on, beside and between all E4M3 numbers, past the largest, infinite and NaN."""
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    codes = codes[torch.isfinite(codes)].unique()
    mid = (codes[1:] + codes[:-1]) / 2
    x = torch.cat([codes, mid, mid * (1 + 2.0 ** -8), mid * (1 - 2.0 ** -8), torch.tensor([449.0, 464.0, 480.0, 1e4, -1e4, float("inf"), -float("inf"), float("nan")])])
    x = x.to(torch.bfloat16)
    n = -(-x.numel() // 64)
    x = torch.cat([x, torch.zeros(n * 64 - x.numel(), dtype=x.dtype)]).view(n, 1, 64).to(DEV)
    B = Batch([(n, n)], 1, 1, 64, 16, fp8=True)
    serq.kv_append(None, x, x, *B.args())
    want = torch.where(torch.isnan(x.float()), x.float(), x.float().clamp(-448, 448)).cpu().to(torch.float8_e4m3fn)
    page, row = orc.slots(*orc.positions(B.cu, B.len, n), B.table, 16, B.pages)
    for cache in (B.K, B.V):
        got = cache.cpu().view(torch.uint8)[torch.from_numpy(page), torch.from_numpy(row)].view(torch.float8_e4m3fn).float()
        w = want.float()
        assert torch.equal(torch.isnan(got), torch.isnan(w)) and torch.equal(got[~torch.isnan(w)], w[~torch.isnan(w)])


SETS = {
    "ones": [(1, 1), (1, 2), (1, 15), (1, 16), (1, 17), (1, 31), (1, 33), (1, 64), (1, 257), (1, 1000)],
    "slots": [(1, 70), (0, 0), (1, 0), (1, 300), (0, 50), (1, 1)],                  # empty slots, a new token without any key
    "few": [(2, 2), (5, 77), (3, 2), (8, 400), (1, 130), (4, 4)],                   # (3, 2): its first row sees nothing
    "chunk": [(33, 33), (70, 200), (1, 90), (129, 129), (0, 0), (16, 1000)],
    "long": [(1, 5000), (3, 2500)],
    "prompt": [(300, 300), (260, 700)],
}


@pytest.mark.parametrize("name", list(SETS))
@pytest.mark.parametrize("Hq,Hkv,D,page,order", [(8, 2, 128, 16, "nhd"), (4, 4, 64, 32, "hnd"), (7, 1, 128, 64, "hnd"), (16, 2, 64, 16, "nhd"),
                                                 (48, 2, 128, 128, "nhd")])
@pytest.mark.parametrize("dt,fp8", [(torch.bfloat16, False), (torch.float16, False), (torch.bfloat16, True), (torch.float16, True)])
def test_attention(name, Hq, Hkv, D, page, order, dt, fp8):
    if name in ("long", "prompt") and Hq > 8:
        Hq, Hkv = Hq // Hkv, 1
    B = Batch(SETS[name], Hq, Hkv, D, page, dt, fp8, order, seed=len(name) + Hq, extra=1).fill()
    ws = serq.paged_attention_workspace(B.T, len(B.seqs), B.max_q, B.max_kv, Hq, Hkv, D, DEV)
    for use in (None, ws, ws):                                     # without slices, and twice with them: the workspace stays ready
        big = torch.full((B.T, Hq + 1, D + 8), 7.0, dtype=dt, device=DEV)
        out, lse = big[:, :Hq, :D], torch.full((B.T, Hq), 7.0, device=DEV)
        serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, k_scale=B.k_scale, v_scale=B.v_scale, out=out, lse=lse, ws=use)
        check_attention(B, out, lse, what=f"{name}, {'with' if use is not None else 'without'} workspace")
        assert (big[:, Hq:] == 7).all() and (big[:, :, D:] == 7).all() and (out[-1] == 7).all() and (lse[-1] == 7).all()


@pytest.mark.parametrize("name", ["ones", "few", "chunk", "long"])
@pytest.mark.parametrize("window", [1, 16, 100])
@pytest.mark.parametrize("fp8", [False, True])
def test_attention_window(name, window, fp8):
    """Pages that no row's window reaches have wild numbers, and keys before the first window hold NaN."""
    B = Batch(SETS[name], 4, 2, 128, 16, torch.bfloat16, fp8, "hnd", window=window, seed=window).fill()
    ws = serq.paged_attention_workspace(B.T, len(B.seqs), B.max_q, B.max_kv, 4, 2, 128, DEV)
    lse = torch.empty((B.T, 4), device=DEV)
    for use in (None, ws):
        out = serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, window=window, k_scale=B.k_scale, v_scale=B.v_scale, lse=lse, ws=use)
        check_attention(B, out, lse, what=f"{name}, window {window}")


@pytest.mark.parametrize("name", ["ones", "few", "chunk"])
@pytest.mark.parametrize("scale,gain", [(1e-3, 1.0), (1.0, 4.0), (0.3, 30.0)])
def test_attention_scales(name, scale, gain):
    """Flat and peaked softmax: scores of a few thousandths, of a hundred, of thousands."""
    B = Batch(SETS[name], 8, 2, 64, 16, seed=11, gain=gain).fill(gain=gain)
    lse = torch.empty((B.T, 8), device=DEV)
    out = serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, scale=scale, lse=lse)
    check_attention(B, out, lse, scale, what=f"{name}, scale {scale}, gain {gain}")


@pytest.mark.parametrize("name", ["few", "chunk", "prompt", "ones"])
@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("dt,fp8", [(torch.bfloat16, False), (torch.float16, False), (torch.bfloat16, True)])
def test_attention_nan_and_infinity_where_a_row_does_not_look(name, window, dt, fp8):
    """Single keys and values of the new tokens, and of keys just inside the first window, that are NaN or infinite: rows that do not see them
    keep their results, rows that see a value like that lose them."""
    r = np.random.RandomState(3)
    B = Batch(SETS[name], 4, 2, 128, 16, dt, fp8, "nhd", window=window, seed=13).fill()
    want = B._attention64(128 ** -0.5)[0]
    hit = np.zeros(B.T, bool)
    for b, (n, L) in enumerate(B.seqs):
        if n < 2:
            continue
        lo = B.first[b]
        spots = {L - 1, max(L - n + n // 2, lo), *( [lo] if window and lo > 0 else [])}
        for i, j in enumerate(sorted(spots)):
            page, row = int(B.table[b, j // 16]), j % 16
            d = int(r.randint(0, 128))
            v = float("nan") if fp8 or i % 2 == 0 else (float("inf") if i % 4 == 1 else -float("inf"))
            if fp8:
                B.V.view(torch.uint8)[page, row, :, d] = 0x7f
            else:
                B.V[page, row, :, d] = v
            if i % 2 == 1 and not fp8:
                B.K[page, row, :, (d + 1) % 128] = float("nan")
            t = np.arange(n)
            sees = (L - n + t >= j) & (True if not window else L - n + t - window < j)
            hit[B.cu[b]:B.cu[b + 1]] |= sees
    ws = serq.paged_attention_workspace(B.T, len(B.seqs), B.max_q, B.max_kv, 4, 2, 128, DEV)
    u = 2.0 ** -8 if dt == torch.bfloat16 else 2.0 ** -11
    for use in (None, ws):
        out = serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, window=window, k_scale=B.k_scale, v_scale=B.v_scale, ws=use).double().cpu().numpy()
        fine = np.isfinite(out).all((1, 2))
        assert np.array_equal(fine, ~hit), f"rows {np.argwhere(fine == hit).ravel()[:10]}"
        assert np.abs(out[~hit] - want[~hit]).max(initial=0) <= 8 * u       # (values of a few: the exact bounds are the other tests')


def test_attention_far_pages():
    """A cache of more than 2^32 bytes: keys whose offsets pass 32 bits."""
    D, page, Hkv = 128, 256, 8
    pages = (5 << 30) // (page * Hkv * D * 2)
    B = Batch([(1, 700), (40, 600)], 8, Hkv, D, page, seed=2).fill()
    K, V = (torch.empty((pages, page, Hkv, D), dtype=B.dt, device=DEV) for _ in range(2))
    used = np.unique(B.table[(B.table >= 0) & (B.table < B.pages)])
    far = {int(u): pages - 1 - 3 * i for i, u in enumerate(used)}
    for u, f in far.items():
        K[f].copy_(B.K[u])
        V[f].copy_(B.V[u])
    table = torch.from_numpy(np.vectorize(lambda x: far.get(int(x), -1))(B.table).astype(np.int32)).to(DEV)
    lse = torch.empty((B.T, 8), device=DEV)
    out = serq.paged_attention(B.q, K, V, table, B.d_cu, B.d_len, B.max_q, B.max_kv, lse=lse)
    check_attention(B, out, lse, what="far pages")
    cos, sin = _tables(700, D)
    got = serq.kv_append(B.q, B.k, B.v, K, V, table, B.d_cu, B.d_len, cos, sin)
    near = serq.kv_append(B.q, B.k, B.v, *B.args(), cos, sin)
    assert torch.equal(got, near)
    for u, f in far.items():
        a, b = _bits(K[f]), _bits(B.K[u])
        assert torch.equal(a[~torch.isnan(B.K[u])], b[~torch.isnan(B.K[u])])


def test_attention_bounds_larger_than_the_batch():
    """max_q and max_kv are bounds only; results may differ in the last bits of fp32 sums."""
    B = Batch(SETS["few"], 8, 2, 128, 16, seed=4).fill()
    for mq, mk in ((B.max_q, B.max_kv), (64, 4000), (300, 100000)):
        ws = serq.paged_attention_workspace(B.T, len(B.seqs), mq, mk, 8, 2, 128, DEV)
        lse = torch.empty((B.T, 8), device=DEV)
        out = serq.paged_attention(B.q, *B.args(), mq, mk, lse=lse, ws=ws)
        check_attention(B, out, lse, what=f"bounds {mq}, {mk}")


def test_attention_many_sequences():
    """More sequences than one wave looks through at a time."""
    r = np.random.RandomState(0)
    seqs = [(int(r.randint(0, 3)), 0) for _ in range(150)]
    seqs = [(n, n + int(r.randint(0, 60))) for n, _ in seqs]
    B = Batch(seqs, 4, 2, 64, 16, seed=8).fill()
    lse = torch.empty((B.T, 4), device=DEV)
    out = serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, lse=lse)
    check_attention(B, out, lse, what="many sequences")
    cos, sin = _tables(70, 64)
    C = Batch(seqs, 4, 2, 64, 16, seed=8)
    want_q, want_K, _, _ = _expected_append(C, cos, sin, True)
    assert torch.equal(_bits(serq.kv_append(C.q, C.k, C.v, *C.args(), cos, sin, interleaved=True).cpu()), _bits(want_q))
    nan = torch.isnan(want_K)
    assert torch.equal(_bits(C.K.cpu())[~nan], _bits(want_K)[~nan])


@pytest.mark.parametrize("name", ["ones", "few", "chunk", "long"])
def test_replays(name):
    """Append and attention recorded into a graph; lengths and pages change between replays."""
    B = Batch(SETS[name], 8, 2, 128, 16, seed=6).fill()
    for t in (B.K, B.V):
        t.nan_to_num_(nan=0.0)
    table = torch.where((B.d_table < 0) | (B.d_table >= B.pages), 0, B.d_table)
    cos, sin = _tables(B.max_kv, 128)
    ws = serq.paged_attention_workspace(B.T, len(B.seqs), B.max_q, B.max_kv, 8, 2, 128, DEV)
    q, out, lse = torch.empty_like(B.q), torch.empty_like(B.q), torch.empty((B.T, 8), device=DEV)
    kv_len = B.d_len.clone()

    def step():
        serq.kv_append(B.q, B.k, B.v, B.K, B.V, table, B.d_cu, kv_len, cos, sin, q_out=q)
        serq.paged_attention(q, B.K, B.V, table, B.d_cu, kv_len, B.max_q, B.max_kv, out=out, lse=lse, ws=ws)

    def mutate(it):
        B.qkv.mul_(-0.7)
        kv_len.copy_((B.d_len - it).clamp(min=0))

    replay_check(step, [q, out, lse], mutate)


def test_other_stream():
    B = Batch(SETS["long"], 8, 2, 128, 16, seed=6).fill()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    ws = serq.paged_attention_workspace(B.T, len(B.seqs), B.max_q, B.max_kv, 8, 2, 128, DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        lse = torch.empty((B.T, 8), device=DEV)
        out = serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, lse=lse, ws=ws)
    st.synchronize()
    check_attention(B, out, lse, what="another stream")


def test_attention_many_sequences_chunks_among_them():
    """More sequences than lanes, with a workspace: both kernels in one launch, single tokens and chunks in any order, empty slots between them."""
    r = np.random.RandomState(1)
    seqs = [(int(r.choice([0, 1, 1, 1, 2, 9, 40])), int(r.randint(0, 300))) for _ in range(140)]
    seqs = [(n, n + c) for n, c in seqs]
    for window, Hq, Hkv in ((0, 8, 2), (50, 4, 4)):
        B = Batch(seqs, Hq, Hkv, 64, 16, window=window, seed=14, order="hnd").fill()
        ws = serq.paged_attention_workspace(B.T, len(seqs), B.max_q, B.max_kv, Hq, Hkv, 64, DEV)
        lse = torch.empty((B.T, Hq), device=DEV)
        for use in (None, ws, ws):
            out = serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, window=window, lse=lse, ws=use)
            check_attention(B, out, lse, what=f"many with chunks, window {window}")


@pytest.mark.parametrize("name", ["ones", "few", "chunk", "long"])
def test_attention_any_workspace(name):
    """A workspace of any size serves, and the same one serves calls of any kind, one after the other."""
    B = Batch(SETS[name], 8, 2, 128, 16, seed=15).fill()
    C = Batch(SETS["chunk"], 4, 4, 64, 16, torch.float16, seed=16).fill()
    full = serq.paged_attention_workspace(B.T, len(B.seqs), B.max_q, B.max_kv, 8, 2, 128, DEV).numel()
    for n in (16, 32 << 10, (32 << 10) + 40000, (32 << 10) + 400000, full // 2, full, 2 * full + 1000000):
        ws = torch.zeros(n, dtype=torch.uint8, device=DEV)
        for X in (B, C, B):
            lse = torch.empty((X.T, X.Hq), device=DEV)
            out = serq.paged_attention(X.q, *X.args(), X.max_q, X.max_kv, lse=lse, ws=ws)
            check_attention(X, out, lse, what=f"workspace of {n}")


def test_attention_is_the_same_from_run_to_run():
    """Slices are added in their order, whoever comes last."""
    for seqs in ([(1, 9000)], [(100, 4000), (1, 700)], [(5, 3000), (2, 900)]):
        B = Batch(seqs, 8, 2, 128, 16, seed=17).fill()
        ws = serq.paged_attention_workspace(B.T, len(seqs), B.max_q, B.max_kv, 8, 2, 128, DEV)
        want = serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, ws=ws)
        for _ in range(20):
            assert torch.equal(serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, ws=ws), want)


def test_lengths_past_the_table_are_cut():
    B = Batch([(2, 64), (40, 64), (1, 30)], 4, 2, 64, 16, seed=18).fill()
    B.seqs = [(2, 90), (40, 70), (1, 30)]                          # the table ends at 64
    B.len = np.array([90, 70, 30], np.int32)
    B.d_len.copy_(torch.from_numpy(B.len))
    lse = torch.empty((B.T, 4), device=DEV)
    out = serq.paged_attention(B.q, *B.args(), 40, 90, lse=lse)
    check_attention(B, out, lse, what="cut")


def test_nothing_to_do():
    B = Batch([(0, 5), (0, 0)], 4, 2, 64, 16, seed=19)
    assert serq.paged_attention(B.q, *B.args(), 0, 5).shape == (0, 4, 64)
    assert serq.kv_append(B.q, B.k, B.v, *B.args()).shape == (0, 4, 64)
    C = Batch([(3, 5)], 4, 2, 64, 16, seed=19)
    none = torch.zeros((0, 1), dtype=torch.int32, device=DEV)
    out = torch.full_like(C.q, 7.0)
    serq.paged_attention(C.q, C.K, C.V, none, C.d_cu[:1], C.d_len[:0], 3, 5, out=out)
    assert (out == 7).all()
    # a cache without pages: no key can be seen
    empty = torch.empty((0, 16, 2, 64), dtype=C.dt, device=DEV)
    lse = torch.empty((3, 4), device=DEV)
    assert not serq.paged_attention(C.q, empty, empty, C.d_table, C.d_cu, C.d_len, 3, 5, lse=lse).any() and torch.isneginf(lse).all()


class _General:
    def __getattr__(self, name):
        return lambda *a: None


def test_both_ways_from_python(monkeypatch):
    """The extension module and ctypes: the same results, the same errors."""
    B = Batch(RAGGED, 8, 2, 128, 16, fp8=True, seed=20).fill()
    cos, sin = _tables(100, 128)
    fast, got = serq._fast, []
    for mod in (fast, _General()):
        monkeypatch.setattr(serq, "_fast", mod)
        K, V = B.K.clone(), B.V.clone()
        q = serq.kv_append(B.q, B.k, B.v, K, V, *B.args()[2:], cos, sin, k_scale=B.k_scale, v_scale=B.v_scale)
        ws = serq.paged_attention_workspace(B.T, len(B.seqs), B.max_q, B.max_kv, 8, 2, 128, DEV)
        lse = torch.empty((B.T, 8), device=DEV)
        out = serq.paged_attention(q, K, V, *B.args()[2:], B.max_q, B.max_kv, lse=lse, ws=ws, k_scale=B.k_scale, v_scale=B.v_scale)
        got.append([q, K.view(torch.uint8), V.view(torch.uint8), out, lse])
        for call, code in ((lambda: serq.paged_attention(B.q, *B.args(), 1, 1, scale=0.0), -3), (lambda: serq.paged_attention(B.q, *B.args(), 1, 1, window=-1), -3),
                           (lambda: serq.paged_attention(B.q[:, :7], *B.args(), 1, 1), -3), (lambda: serq.kv_append(B.q, B.k, B.v, *B.args(), cos[:0], sin[:0]), -3),
                           (lambda: serq.kv_append(B.q, B.k, B.v, *B.args(), cos[:, :4].contiguous(), sin[:, :4].contiguous()), -3)):
            with pytest.raises(serq.SerqError) as e:
                call()
            assert e.value.code == code
        t32 = B.d_table.long()
        for call in (lambda: serq.paged_attention(B.q, B.K, B.V, t32, B.d_cu, B.d_len, 1, 1), lambda: serq.paged_attention(B.q, B.K, B.V[:1], *B.args()[2:], 1, 1),
                     lambda: serq.paged_attention(B.q, *B.args()[:3], B.d_cu[:-1], B.d_len, 1, 1), lambda: serq.paged_attention(B.q.half(), B.K.float().bfloat16(), B.V.float().bfloat16(), *B.args()[2:], 1, 1),
                     lambda: serq.paged_attention(B.q[..., :64], *B.args(), 1, 1), lambda: serq.paged_attention(B.q, *B.args(), 1, 1, out=B.q[:1]),
                     lambda: serq.paged_attention(B.q, *B.args(), 1, 1, lse=torch.empty((B.T, 7), device=DEV)), lambda: serq.paged_attention(B.q, *B.args(), 1, 1, ws=torch.empty(64, device=DEV)),
                     lambda: serq.paged_attention(B.q, *B.args(), 1, 1, k_scale=B.k_scale[:1]), lambda: serq.kv_append(B.q, B.k, B.v[:1], *B.args()),
                     lambda: serq.kv_append(B.q, B.q, B.q, *B.args()), lambda: serq.kv_append(B.q, B.k, B.v, *B.args(), cos),
                     lambda: serq.kv_append(B.q, B.k, B.v, *B.args(), cos.double(), sin.double()), lambda: serq.kv_append(B.q, B.k, B.v, *B.args(), cos, sin, positions=B.d_cu[:3])):
            with pytest.raises(ValueError):
                call()
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("fp8", [False, True])
def test_a_block_of_a_decoder(fp8):
    """The example: prompts in one ragged call, then tokens through a replayed graph; against the same steps with plain attention on the cache."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_block.py")
    spec = importlib.util.spec_from_file_location("attention_block", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    block = ex.AttentionBlock(hidden=512, q_heads=8, kv_heads=2, dim=64, rank=32, pages=64, page=16, fp8=fp8)
    prompts = [70, 3, 130]
    seen = {}
    real = serq.paged_attention

    def spy(q, K, V, table, cu, kv_len, *a, **kw):
        out = real(q, K, V, table, cu, kv_len, *a, **kw)
        seen["last"] = (q, table, cu, kv_len, out)
        if "first" not in seen:
            seen["first"] = [t.clone() for t in seen["last"]]
        return out

    serq.paged_attention = spy
    try:
        first, y, kv_len, table, _ = ex.run(block, prompts, 5)
    finally:
        serq.paged_attention = real
    assert kv_len.tolist() == [p + 1 + 5 for p in prompts] and torch.isfinite(first).all() and torch.isfinite(y).all()
    for key, n in (("first", prompts), ("last", [1, 1, 1])):
        q, tb, cu, ln, out = seen[key]
        at = 0
        for b in range(3):
            L = int(ln[b])
            p = torch.arange(L, device=DEV)
            page, row = tb[b].long()[p // 16], p % 16
            k, v = ((x.float() * (s[:, None] if s is not None else 1.0))[page, row].double().cpu().numpy() for x, s in ((block.K, block.k_scale), (block.V, block.v_scale)))
            want, _, mag, big = orc.attention(q[at:at + n[b]].double().cpu().numpy(), k, v, 64 ** -0.5, L - n[b])
            tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -7 + 2 * 72 * 2.0 ** -24 * big[..., None] + 2.0 ** -15) * mag
            assert (np.abs(out[at:at + n[b]].double().cpu().numpy() - want) <= tol).all(), (key, b)
            at += n[b]
