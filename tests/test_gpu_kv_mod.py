"""Attention over the paged cache with capped scores, biases by distance and rows that see ranges of their own, against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2603_08185_amd import binding as serq
from tests._kv import DEV
from tests._kv_mod import ModBatch, check_mod, docs, prefix, wild
from tests._util import replay_check

pytestmark = pytest.mark.gpu

SETS = {"ones": [(1, 1), (1, 40), (0, 0), (1, 333), (1, 17), (1, 64), (1, 2000)],
        "few": [(3, 5), (2, 40), (0, 9), (5, 333), (1, 17), (4, 64), (8, 8)],
        "chunk": [(100, 100), (1, 130), (0, 0), (33, 290), (3, 65), (70, 71), (1, 1)],
        "long": [(1, 9000), (2, 5000), (150, 3000)]}
MODS = {"cap": dict(cap=30.0), "small cap": dict(cap=0.5), "bias": dict(bias=1.0), "docs": dict(ranges=docs), "prefix": dict(ranges=prefix),
        "wild": dict(ranges=wild), "cap docs": dict(cap=5.0, ranges=docs), "bias prefix": dict(bias=0.25, ranges=prefix), "cap wild": dict(cap=50.0, ranges=wild),
        "bias wild": dict(bias=0.5, ranges=wild), "cap window": dict(cap=20.0, window=50), "bias window": dict(bias=0.1, window=33),
        "docs window": dict(ranges=docs, window=20), "wild window": dict(ranges=wild, window=64), "growing": dict(bias=-0.01)}


def _run(B, ws=True, **kw):
    lse = torch.full((B.T, B.Hq), 7.0, device=DEV)
    out = torch.full((B.T, B.Hq, B.D), 7.0, dtype=B.dt, device=DEV)
    if ws is True:
        ws = serq.paged_attention_workspace(B.T, len(B.seqs), B.max_q, B.max_kv, B.Hq, B.Hkv, B.D, DEV)
    serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, out=out, lse=lse, ws=ws if ws is not None else None, **B.call(**kw))
    return out, lse


@pytest.mark.parametrize("mod", MODS)
@pytest.mark.parametrize("name", SETS)
def test_modifications(name, mod):
    for i, (Hq, Hkv, D, dt, fp8, order) in enumerate(((8, 2, 128, torch.bfloat16, False, "nhd"), (4, 4, 64, torch.float16, False, "hnd"),
                                                      (8, 1, 64, torch.bfloat16, True, "hnd"), (6, 2, 128, torch.float16, True, "nhd"))):
        B = ModBatch(SETS[name], Hq, Hkv, D, 16 << (i % 3), dt, fp8, order, extra=2, seed=i, gain=2.0, **MODS[mod])
        for ws in (True, None):
            out, lse = _run(B, ws)
            check_mod(B, out, lse, what=f"{Hq} {Hkv} {D} {dt} fp8 {fp8} ws {ws}")
            assert (out[B.cu[-1]:] == 7).all() and (lse[B.cu[-1]:] == 7).all()


@pytest.mark.parametrize("mod", ["cap", "bias", "wild"])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (7, 1), (16, 1), (33, 1), (24, 8), (64, 8), (5, 5)])
def test_heads(mod, Hq, Hkv):
    for seqs in ([(1, 70), (4, 9)], [(40, 200), (1, 5)]):
        B = ModBatch(seqs, Hq, Hkv, 128, 32, seed=Hq, **MODS[mod])
        check_mod(B, *_run(B), what=f"{Hq} {Hkv} {seqs}")


@pytest.mark.parametrize("mod", ["cap", "bias", "docs", "prefix", "wild"])
@pytest.mark.parametrize("L", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 511, 513])
def test_lengths(mod, L):
    for n in sorted({1, min(2, L), min(L, 9), L}):
        B = ModBatch([(n, L)], 4, 2, 64, 16, seed=L, **MODS[mod])
        check_mod(B, *_run(B), what=f"{n} of {L}")


def test_rows_of_nothing():
    """All rows empty, in every kernel: zeros and -inf."""
    nothing = lambda r, n, L: (np.full(n, 5), np.full(n, 5))
    for name in SETS:
        for more in ({}, dict(cap=3.0), dict(bias=1.0)):
            B = ModBatch(SETS[name], 8, 2, 128, 16, seed=2, ranges=nothing, **more)
            out, lse = _run(B)
            assert not out[:B.cu[-1]].any() and torch.isneginf(lse[:B.cu[-1]]).all()


def test_only_one_of_the_ends():
    B = ModBatch(SETS["chunk"], 8, 2, 64, 16, seed=4, ranges=lambda r, n, L: (np.maximum(np.arange(L - n, L) - 9, 0), np.arange(L - n, L) + 1))
    check_mod(B, *_run(B, see_to=None), what="from alone")
    B = ModBatch(SETS["chunk"], 8, 2, 64, 16, seed=4, ranges=lambda r, n, L: (np.zeros(n, int), np.minimum(np.arange(L - n, L) + 1, 30)))
    check_mod(B, *_run(B, see_from=None), what="to alone")


def test_ranges_of_everything_are_the_plain_attention():
    """Ranges that say what the causal mask says, a bias of slopes zero, and no modification at all: the same bits as the plain call."""
    for name in SETS:
        for window in (0, 40):
            B = ModBatch(SETS[name], 8, 2, 128, 16, seed=5, window=window, ranges=lambda r, n, L: (np.zeros(n, int), np.arange(L - n, L) + 1))
            want = _run(B, see_from=None, see_to=None)
            zero = torch.zeros(8, device=DEV)
            for got in (_run(B), _run(B, see_to=None), _run(B, see_from=None, see_to=None, slopes=zero), _run(B, slopes=zero)):
                for a, b in zip(got, want):
                    assert torch.equal(a.nan_to_num(), b.nan_to_num())


def test_scores_past_the_cap_and_specials():
    """Scores a thousand times the cap, infinite ones: capped to +-cap; NaN makes its own rows NaN and no others."""
    B = ModBatch([(1, 100), (40, 130)], 4, 2, 64, 16, seed=6, cap=2.0, gain=60.0)
    check_mod(B, *_run(B), what="far past")
    B = ModBatch([(40, 130)], 4, 2, 64, 16, seed=7, cap=2.0)
    page, row = int(B.table[0, 3]), 5                              # position 53: seen by all rows, all of whose products with it are infinite
    B.K[page, row] = float("inf")
    B.kv[0][0][53] = np.nan
    out, lse = _run(B)
    q = B.q.double().cpu().numpy()
    mixed = torch.from_numpy(((q > 0).any(-1) & (q < 0).any(-1)))
    assert torch.isnan(out.cpu()[mixed]).all()                     # inf - inf
    B.K[page, row] = 0
    B.K[page, row, :, 0] = float("inf")                            # alone: its score is +-inf, capped
    B.kv[0][0][53] = 0
    B.kv[0][0][53, :, 0] = 1e30
    sure = torch.from_numpy(np.abs(q[..., 0]) > 0)
    out, lse = _run(B)
    want, wlse, mag, eo, el = B.mod64()
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -7 + 2.0 ** -14) * mag + 2.0 ** -14 * mag
    off = np.abs(out.double().cpu().numpy() - want) <= tol
    assert off[sure.numpy()].all()


def test_what_a_row_does_not_see_cannot_reach_it():
    """NaN and infinities in keys and values that some rows of a block see and others do not."""
    for fp8 in (False, True):
        for more in (dict(cap=4.0), dict(bias=0.1), {}):
            B = ModBatch([(100, 100)], 4, 1, 64, 16, fp8=fp8, seed=8, ranges=lambda r, n, L: (np.where(np.arange(n) < 50, 0, 50), np.where(np.arange(n) < 50, 50, 100)), **more)
            clean, _ = _run(B)
            page, row = int(B.table[0, 1]), 4                      # position 20: the first half's
            if fp8:
                B.V.view(torch.uint8)[page, row] = 0x7f
            else:
                B.V[page, row] = float("nan")
            out, lse = _run(B)
            assert torch.isnan(out[:50].float()).all() and torch.equal(out[50:], clean[50:])
            if fp8:
                B.K.view(torch.uint8)[page, row] = 0x7f
            else:
                B.K[page, row] = float("nan")
            out, lse = _run(B)
            assert torch.isnan(out[:50].float()).all() and torch.equal(out[50:], clean[50:])


@pytest.mark.parametrize("cap", [2.0 ** -20, 0.01, 1.0, 50.0, 300.0, 1024.0])
def test_caps(cap):
    for dt in (torch.bfloat16, torch.float16):
        B = ModBatch([(1, 300), (2, 80), (60, 200)], 4, 2, 64, 16, dt, seed=9, cap=cap, gain=3.0)
        check_mod(B, *_run(B), what=f"cap {cap}")
        check_mod(B, *_run(B, scale=3.0), scale=3.0, what=f"cap {cap}, scale 3")


@pytest.mark.parametrize("bias", [1e-4, 0.03, 2.0, 50.0, 1e30])
def test_slopes(bias):
    for dt in (torch.bfloat16, torch.float16):
        B = ModBatch([(1, 3000), (2, 80), (60, 200)], 4, 2, 64, 16, dt, seed=10, bias=bias)
        check_mod(B, *_run(B), what=f"slope {bias}")


@pytest.mark.parametrize("mod", ["cap", "bias", "docs", "bias wild"])
@pytest.mark.parametrize("name", ["ones", "few", "chunk", "long"])
def test_replays(name, mod):
    """Recorded into a graph; lengths and ranges change between replays."""
    B = ModBatch(SETS[name], 8, 2, 128, 16, seed=11, **MODS[mod])
    for t in (B.K, B.V):
        t.nan_to_num_(nan=0.0)
    B.d_table = torch.where((B.d_table < 0) | (B.d_table >= B.pages), 0, B.d_table)
    ws = serq.paged_attention_workspace(B.T, len(B.seqs), B.max_q, B.max_kv, 8, 2, 128, DEV)
    out, lse = torch.empty_like(B.q), torch.empty((B.T, 8), device=DEV)
    q = B.q.clone()
    kw = B.call(out=out, lse=lse, ws=ws)

    def step():
        serq.paged_attention(q, B.K, B.V, B.d_table, B.d_cu, B.d_len, B.max_q, B.max_kv, **kw)

    def mutate(it):
        q.mul_(-0.7)
        B.d_len.sub_(1).clamp_(min=0)
        if B.see_from is not None:
            B.see_from.add_(it)
            B.see_to.sub_(1)

    replay_check(step, [out, lse], mutate)


def test_append_then_attend():
    """A block's middle as a server runs it: heads normalised, rotated and appended, then attention with each modification over what was written."""
    for mod in ("cap", "bias", "docs", "prefix"):
        B = ModBatch(SETS["chunk"], 8, 2, 64, 16, seed=12, **MODS[mod])
        table = torch.zeros_like(B.d_table)
        at = 0
        for b, (n, L) in enumerate(B.seqs):
            m = -(-L // 16)
            table[b, :m] = torch.arange(at, at + m, device=DEV)
            at += m
        K, V = (torch.zeros((at, 16, 2, 64), dtype=B.dt, device=DEV) for _ in range(2))
        g = torch.Generator(device=DEV).manual_seed(3)
        every = torch.cat([torch.zeros(1, dtype=torch.int32), torch.tensor([L for _, L in B.seqs], dtype=torch.int32).cumsum(0, dtype=torch.int32)]).to(DEV)
        kv = [torch.randn((int(every[-1]), 2, 64), generator=g, device=DEV).to(B.dt) for _ in range(2)]
        w = torch.rand(64, generator=g, device=DEV) + 0.5
        pos = torch.arange(2100, device=DEV)[:, None] * 10000.0 ** (-torch.arange(32, device=DEV) / 32)
        cos, sin = pos.cos().contiguous(), pos.sin().contiguous()
        serq.kv_append(None, *kv, K, V, table, every, B.d_len, cos, sin, k_norm=w)                 # what was there: all keys
        q = serq.kv_append(B.q, kv[0][:B.T], kv[1][:B.T], torch.zeros_like(K), torch.zeros_like(V), table, B.d_cu, B.d_len, cos, sin, q_norm=w, k_norm=w)
        for b, (n, L) in enumerate(B.seqs):
            p = torch.arange(L, device=DEV)
            B.kv[b] = [c[table[b].long()[p // 16], p % 16].double().cpu().numpy() for c in (K, V)]
        B.q, B.K, B.V, B.d_table = q, K, V, table
        check_mod(B, *_run(B), what=mod)


def test_same_from_run_to_run():
    for seqs in ([(1, 9000)], [(100, 4000), (1, 700)], [(5, 3000), (2, 900)]):
        for mod in ("cap", "bias", "docs"):
            B = ModBatch(seqs, 8, 2, 128, 16, seed=13, **MODS[mod])
            ws = serq.paged_attention_workspace(B.T, len(seqs), B.max_q, B.max_kv, 8, 2, 128, DEV)
            want, _ = _run(B, ws)
            for _ in range(10):
                assert torch.equal(_run(B, ws)[0], want)


class _General:
    def __getattr__(self, name):
        return lambda *a: None


def test_both_ways_from_python(monkeypatch):
    B = ModBatch(SETS["chunk"], 8, 2, 128, 16, fp8=True, seed=14, ranges=docs)
    slopes = torch.rand(8, device=DEV)
    fast, got = serq._fast, []
    for mod in (fast, _General()):
        monkeypatch.setattr(serq, "_fast", mod)
        got.append([*_run(B), *_run(B, cap=3.0), *_run(B, slopes=slopes)])
        for kw, code in ((dict(cap=-1.0), -3), (dict(cap=float("nan")), -3), (dict(cap=1025.0), -3), (dict(cap=2.0, slopes=slopes), -7)):
            with pytest.raises(serq.SerqError) as e:
                _run(B, **kw)
            assert e.value.code == code
        for kw in (dict(slopes=slopes[:7]), dict(slopes=slopes.double()), dict(see_from=B.see_from[:-1]), dict(see_to=B.see_to.long()),
                   dict(see_to=B.see_to.cpu()), dict(slopes=slopes.repeat(2)[::2])):
            with pytest.raises(ValueError):
                _run(B, **kw)
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("mod", ["none", "cap", "bias", "wild", "bias prefix"])
@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (6, 6), (16, 4), (32, 8), (8, 1), (12, 4)])
def test_narrow_heads_side_by_side(mod, Hq, Hkv):
    """Heads of 64 channels next to one another in memory are read two a time: none sees the other's keys or values, NaN and infinities among them."""
    for dt in (torch.bfloat16, torch.float16):
        for seqs in ([(1, 700), (1, 40), (0, 3), (1, 1)], [(2, 90), (1, 300)], [(1, 5000)]):
            kw = dict(MODS[mod]) if mod != "none" else {}
            B = ModBatch(seqs, Hq, Hkv, 64, 16, dt, seed=Hq, order="nhd", extra=1, **kw)
            assert B.K.stride(2) == 64
            for ws in (None, True):                                # (with the workspace last: what follows is compared with it bit by bit)
                clean, lse = _run(B, ws)
                check_mod(B, clean, lse, what=f"{seqs}")
                assert (clean[B.cu[-1]:] == 7).all()
            if Hkv < 2:
                continue
            K, V, G = B.K.clone(), B.V.clone(), Hq // Hkv
            for bad in (float("nan"), float("inf")):
                B.K[:, :, 1::2], B.V[:, :, 0::2] = bad, bad       # odd heads' keys, even heads' values: every head has something of its own spoilt
                out, l2 = _run(B)
                for h in range(0, Hkv, 2):                         # an even head's softmax does not change
                    a, b = l2[:, h * G:(h + 1) * G], lse[:, h * G:(h + 1) * G]
                    assert torch.equal(a, b)
                B.K.copy_(K)
                B.V.copy_(V)
                B.V[:, :, 1::2] = bad
                out, _ = _run(B)
                for h in range(0, Hkv, 2):
                    assert torch.equal(out[:, h * G:(h + 1) * G], clean[:, h * G:(h + 1) * G])
                B.V.copy_(V)


def test_narrow_heads_other_strides():
    """Keys side by side and values not, a gap between heads, an odd number of heads: heads one a time, the same results within the bounds."""
    for Hkv, where in ((4, "gap"), (4, "values"), (3, "odd")):
        B = ModBatch([(1, 300), (1, 77)], 2 * Hkv, Hkv, 64, 16, seed=3, cap=9.0)
        if where != "odd":
            for name in (("K", "V") if where == "gap" else ("V",)):
                x = getattr(B, name)
                wide = torch.full((*x.shape[:2], Hkv, 72), float("nan"), dtype=x.dtype, device=DEV)
                wide[..., :64] = x
                setattr(B, name, wide[..., :64])
        check_mod(B, *_run(B), what=where)


def test_pages_far_apart():
    """Pages 4 GiB apart: offsets past 32 bits, heads one and two at a time, few rows and many."""
    for Hq, Hkv, seqs in ((4, 2, [(1, 40), (2, 20)]), (8, 1, [(40, 48)])):
        B = ModBatch(seqs, Hq, Hkv, 64, 16, seed=5, cap=6.0, ranges=prefix)
        clean, lse = _run(B)
        far = []
        for x in (B.K, B.V):
            apart = 1 << 31                                        # elements
            wide = torch.empty(apart * (B.pages - 1) + 16 * Hkv * 64, dtype=x.dtype, device=DEV).as_strided(x.shape, (apart, Hkv * 64, 64, 1))
            wide.copy_(x)
            far.append(wide)
        B.K, B.V = far
        out, l2 = _run(B)
        assert torch.equal(out, clean) and torch.equal(l2, lse)
        check_mod(B, out, l2)


def test_another_stream():
    for mod in ("cap", "bias", "docs"):
        B = ModBatch(SETS["long"], 8, 2, 128, 16, seed=6, **MODS[mod])
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            out, lse = _run(B)
        st.synchronize()
        check_mod(B, out, lse, what=mod)


def test_one_workspace_for_all_kinds():
    """Plain and modified calls of several shapes, one after the other on the same workspace, sized for the largest."""
    Bs = [ModBatch(SETS[n], 4, 2, 64, 16, seed=i, **MODS[m]) for i, (n, m) in enumerate((("long", "cap"), ("ones", "bias"), ("chunk", "docs"), ("few", "wild"), ("ones", "cap")))]
    most = [max(f(B) for B in Bs) for f in (lambda B: B.T, lambda B: len(B.seqs), lambda B: B.max_q, lambda B: B.max_kv)]
    ws = serq.paged_attention_workspace(*most, 4, 2, 64, DEV)
    for B in Bs + Bs[::-1]:
        plain = serq.paged_attention(B.q, *B.args(), B.max_q, B.max_kv, ws=ws)
        assert plain.shape == B.q.shape
        check_mod(B, *_run(B, ws))


@pytest.mark.parametrize("mod", ["none", "cap", "bias", "docs"])
@pytest.mark.parametrize("Hq,Hkv,D,dt", [(4, 2, 128, torch.bfloat16), (4, 4, 64, torch.float16), (2, 1, 64, torch.bfloat16)])
def test_keys_of_other_rows_change_no_bit(mod, Hq, Hkv, D, dt):
    """Large scores with keys that only the later rows of a block see: the earlier rows' weights are rounded as before, too."""
    for n, L in ((4, 1200), (16, 300), (100, 700)):
        kw = dict(MODS[mod]) if mod != "none" else {}
        if mod == "docs":
            kw = dict(ranges=lambda r, n, L: (np.zeros(n, int), np.where(np.arange(n) < n // 2, L - n, L)))
        B = ModBatch([(n, L), (1, 50)], Hq, Hkv, D, 16, dt, seed=n, **kw)
        want, lse = _run(B)
        late, half = L - n + n // 2, n // 2                           # the first key that rows half, half + 1, ... see and those before do not
        for factor in (30.0, -30.0, 0.0):
            for j in range(late, L):
                page = int(B.table[0, j // 16])
                B.K[page, j % 16] *= factor
            out, l2 = _run(B)
            assert torch.equal(out[:half], want[:half]) and torch.equal(l2[:half], lse[:half]), (n, factor)
            assert torch.equal(out[n:], want[n:]) and torch.equal(l2[n:], lse[n:])


def test_caps_too_small_for_fp32(monkeypatch):
    """A cap that is 0 in fp32 is refused, not taken for none; 0 of either sign or type is none."""
    B = ModBatch(SETS["few"], 4, 2, 64, 16, seed=3)
    fast = serq._fast
    for mod in (fast, _General()):
        monkeypatch.setattr(serq, "_fast", mod)
        for cap in (1e-50, -1e-50, 5e-324, 2.0 ** -151):
            for more in ({}, dict(slopes=torch.ones(4, device=DEV)), dict(see_from=torch.zeros(B.T, dtype=torch.int32, device=DEV))):
                with pytest.raises(ValueError):
                    _run(B, cap=cap, **more)
        want = _run(B, cap=0.0)
        for cap in (0, -0.0):
            for a, b in zip(_run(B, cap=cap), want):
                assert torch.equal(a, b)
        _run(B, cap=2.0 ** -149)


def test_plain_calls_between_modified_ones():
    """Plain calls on a workspace that modified ones leave behind, and the other way round: each as on a workspace of its own, bit by bit."""
    Bs = [ModBatch(SETS[n], 4, 2, 64, 16, seed=i, **MODS[m]) for i, (n, m) in enumerate((("long", "cap"), ("ones", "bias"), ("chunk", "docs"), ("few", "wild"), ("ones", "cap")))]
    most = [max(f(B) for B in Bs) for f in (lambda B: B.T, lambda B: len(B.seqs), lambda B: B.max_q, lambda B: B.max_kv)]
    room = lambda: serq.paged_attention_workspace(*most, 4, 2, 64, DEV)

    def plain(B, ws):
        lse = torch.empty((B.T, 4), device=DEV)
        table = torch.where((B.d_table < 0) | (B.d_table >= B.pages), 0, B.d_table)    # (a plain row sees pages that the modified ones do not)
        return serq.paged_attention(B.q, B.K, B.V, table, B.d_cu, B.d_len, B.max_q, B.max_kv, lse=lse, ws=ws), lse

    for B in Bs:
        for t in (B.K, B.V):
            t.nan_to_num_(nan=0.25)
    alone = [(plain(B, room()), _run(B, room())) for B in Bs]
    assert all(torch.isfinite(x.float()).all() for (a, _) in alone for x in a)
    ws = room()
    for i in (0, 1, 2, 3, 4, 4, 3, 2, 1, 0):
        for got, want in zip((plain(Bs[i], ws), _run(Bs[i], ws)), alone[i]):
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), i
