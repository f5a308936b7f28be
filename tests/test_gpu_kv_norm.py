"""The append of a model that normalises the heads of q and k: against the same fp32 operations one by one (the root in 64 bits), bit for bit."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as orc
from paper_2603_08185_amd import binding as serq
from tests._kv import DEV, Batch
from tests._util import replay_check

pytestmark = pytest.mark.gpu

RAGGED = [(3, 5), (0, 0), (1, 1), (17, 40), (0, 9), (2, 33), (1, 16), (5, 5), (1, 100)]


def _weights(D, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.rand(D, generator=g) * 1.5 + 0.25).to(DEV) for _ in range(2)]


def _tables(rows, rot, seed=0):
    g = torch.Generator().manual_seed(seed)
    a = torch.rand(rows, rot // 2, generator=g, dtype=torch.float64) * 6.28
    return a.cos().float().to(DEV), a.sin().float().to(DEV)


def _expected(B, cos, sin, inter, qw, kw, eps, at=None):
    c, s = (x.cpu().numpy() if x is not None else np.zeros((1, 0), np.float32) for x in (cos, sin))
    rot = 2 * c.shape[1]
    seq, pos = orc.positions(B.cu, B.len, B.T)
    turned = np.clip(pos if at is None else at, 0, c.shape[0] - 1)
    page, row = orc.slots(seq, pos, B.table, B.page, B.pages)
    done = []
    for x, w in ((B.q, qw), (B.k, kw)):
        x = x.float().cpu().numpy()
        x = x if w is None else orc.normed(x, w.cpu().numpy(), eps)
        done.append(orc.rotate(x, c[turned], s[turned], rot, inter, np.float32))
    q, k = done
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
    return torch.from_numpy(q).to(B.dt), K, V, torch.from_numpy(seq >= 0)


def _bits(x):
    return x.contiguous().view(torch.uint8 if x.element_size() == 1 else torch.int16)


def _same(B, q_out, want, what=""):
    want_q, want_K, want_V, mine = want
    assert torch.equal(_bits(q_out.cpu()[mine]), _bits(want_q[mine])), f"{what}: q"
    for name, got, ref in (("K", B.K, want_K), ("V", B.V, want_V)):
        got = got.cpu().contiguous()
        nan = torch.isnan(ref.float())
        assert torch.equal(nan, torch.isnan(got.float())), f"{what}: {name}"
        assert torch.equal(_bits(got)[~nan], _bits(ref)[~nan]), f"{what}: {name}"


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D,rot,page,order", [(8, 2, 128, 128, 16, "nhd"), (3, 1, 128, 64, 32, "hnd"), (4, 4, 64, 16, 16, "hnd"),
                                                     (14, 2, 64, 64, 64, "nhd"), (64, 8, 128, 128, 32, "hnd"), (2, 2, 64, 0, 128, "nhd"), (1, 1, 64, 64, 16, "nhd")])
def test_append(dt, fp8, inter, Hq, Hkv, D, rot, page, order):
    B = Batch(RAGGED, Hq, Hkv, D, page, dt, fp8, order, extra=2, seed=Hq + D, gain=3.0)
    cos, sin = _tables(100, rot) if rot else (None, None)
    qw, kw = _weights(D, Hq)
    want = _expected(B, cos, sin, inter, qw, kw, 1e-6)
    big = torch.full((B.T, Hq + 1, D + 8), 7.0, dtype=dt, device=DEV)
    q_out = big[:, :Hq, :D]
    serq.kv_append(B.q, B.k, B.v, *B.args(), cos, sin, interleaved=inter, k_scale=B.k_scale, v_scale=B.v_scale, q_out=q_out, q_norm=qw, k_norm=kw)
    _same(B, q_out, want)
    assert (big[:, Hq:] == 7).all() and (big[:, :, D:] == 7).all() and (q_out[~want[3].to(DEV)] == 7).all()


@pytest.mark.parametrize("which", ["q", "k", "neither"])
def test_one_of_both(which):
    B = Batch(RAGGED, 8, 2, 128, 16, seed=5, gain=0.3)
    cos, sin = _tables(50, 128)
    qw, kw = _weights(128)
    qw, kw = qw if which == "q" else None, kw if which == "k" else None
    at = np.random.RandomState(1).randint(-3, 60, B.T).astype(np.int32)
    want = _expected(B, cos, sin, False, qw, kw, 1e-5, at)
    q = B.q.clone()
    got = serq.kv_append(q, B.k, B.v, *B.args(), cos, sin, positions=torch.from_numpy(at).to(DEV), q_out=q, q_norm=qw, k_norm=kw, eps=1e-5)
    assert got is q
    _same(B, q, want, which)


def test_keys_only():
    B = Batch(RAGGED, 8, 2, 64, 16, seed=6)
    cos, sin = _tables(100, 64)
    qw, kw = _weights(64)
    want = _expected(B, cos, sin, True, qw, kw, 1e-6)
    assert serq.kv_append(None, B.k, B.v, *B.args(), cos, sin, interleaved=True, q_norm=qw, k_norm=kw) is None
    _same(B, want[0], want)


@pytest.mark.parametrize("eps", [0.0, 1e-6, 1.0])
def test_heads_of_zeros_and_extremes(eps):
    """Zero heads (0 without an eps too), one channel alone, the smallest and the largest numbers of the type."""
    for dt in (torch.bfloat16, torch.float16):
        B = Batch([(6, 9)], 4, 2, 128, 16, dt, seed=7)
        top = torch.finfo(dt).max
        for x in (B.q, B.k):
            x[0] = 0
            x[1] = 0
            x[1, :, 77] = -3.0
            x[2] = torch.finfo(dt).smallest_normal
            x[3] = 2.0 ** -24 if dt == torch.float16 else 1e-38
            x[4] = top
            x[5, :, ::2] = -top
        qw, kw = _weights(128, 3)
        want = _expected(B, None, None, False, qw, kw, eps)
        q_out = serq.kv_append(B.q, B.k, B.v, *B.args(), q_norm=qw, k_norm=kw, eps=eps)
        assert torch.isfinite(q_out.float()).all() and not q_out[0].any()
        _same(B, q_out, want, f"{dt} {eps}")


def test_against_64_bits_and_through_the_graph():
    B = Batch([(40, 90), (1, 64)], 8, 2, 128, 16, seed=3)
    cos, sin = _tables(100, 128)
    qw, kw = _weights(128)
    q_out = serq.kv_append(B.q, B.k, B.v, *B.args(), cos, sin, q_norm=qw, k_norm=kw)
    seq, pos = orc.positions(B.cu, B.len, B.T)
    c, s = cos.double().cpu().numpy()[pos], sin.double().cpu().numpy()[pos]
    x = B.q.double().cpu().numpy()
    x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + 1e-6) * qw.double().cpu().numpy()
    want = orc.rotate(x, c, s, 128, False)
    ax, ac, as_ = np.abs(x), np.abs(c), np.abs(s)
    size = np.concatenate([orc.rotate(ax, ac, -as_, 128, False)[..., :64], orc.rotate(ax, ac, as_, 128, False)[..., 64:]], -1)   # |x c| + |y s|
    err = np.abs(q_out.double().cpu().numpy() - want)
    # one rounding to bf16 (2^-8); the root, two products and the rotation's three operations in fp32 (six times 2^-24, of which 2^-21 is more)
    assert (err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -21 * size + 2.0 ** -133).all()
    for t in (B.K, B.V):
        t.nan_to_num_(nan=0.0)
    out = torch.empty_like(q_out)
    replay_check(lambda: serq.kv_append(B.q, B.k, B.v, *B.args(), cos, sin, q_out=out, q_norm=qw, k_norm=kw), [out, B.K, B.V],
                 lambda i: B.qkv.mul_(-0.7))


class _General:
    def __getattr__(self, name):
        return lambda *a: None


def test_both_ways_from_python(monkeypatch):
    """The extension module and ctypes: the same results, the same errors."""
    B = Batch(RAGGED, 8, 2, 128, 16, fp8=True, seed=20)
    cos, sin = _tables(100, 128)
    qw, kw = _weights(128)
    fast, got = serq._fast, []
    for mod in (fast, _General()):
        monkeypatch.setattr(serq, "_fast", mod)
        K, V = B.K.clone(), B.V.clone()
        q = serq.kv_append(B.q, B.k, B.v, K, V, *B.args()[2:], cos, sin, k_scale=B.k_scale, v_scale=B.v_scale, q_norm=qw, k_norm=kw)
        got.append([q, K.view(torch.uint8), V.view(torch.uint8)])
        for bad in (dict(eps=-1.0), dict(eps=float("nan"))):
            with pytest.raises(serq.SerqError) as e:
                serq.kv_append(B.q, B.k, B.v, *B.args(), cos, sin, q_norm=qw, k_norm=kw, **bad)
            assert e.value.code == -3
        wide = torch.ones(130, device=DEV)
        for bad in (dict(q_norm=qw[:64]), dict(k_norm=kw.double()), dict(q_norm=qw.cpu()), dict(k_norm=kw[None]), dict(q_norm=wide[::2][:64])):
            with pytest.raises(ValueError):
                serq.kv_append(B.q, B.k, B.v, *B.args(), cos, sin, **bad)
        with pytest.raises(serq.SerqError) as e:
            serq.kv_append(B.q, B.k, B.v, *B.args(), cos, sin, q_norm=wide[1:129])         # 4 bytes past a 16-byte boundary
        assert e.value.code == -4
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,rot", [(128, 128), (64, 32), (128, 0)])
def test_heads_that_are_not_finite(fp8, inter, D, rot):
    """An infinite channel: NaN there, zeros in the head's other channels, before the rotation; NaN: the whole head.  Other heads as ever."""
    for dt in (torch.bfloat16, torch.float16):
        B = Batch([(6, 9), (1, 3)], 4, 2, D, 16, dt, fp8, seed=9)
        for x in (B.q, B.k):
            x[0, 0, 5] = float("inf")
            x[1, 1, D - 3] = -float("inf")
            x[2, 0, 3] = float("nan")
            x[3] = float("nan")
            x[4, 1, 1], x[4, 1, 2] = float("inf"), float("nan")
        cos, sin = _tables(20, rot) if rot else (None, None)
        qw, kw = _weights(D, 3)
        with np.errstate(invalid="ignore"):
            want = _expected(B, cos, sin, inter, qw, kw, 1e-6)
        assert want[0][0, 0].isnan().sum() == (2 if rot else 1) and (want[0][0, 0].nan_to_num() == 0).all() and want[0][2, 0].isnan().all()
        q_out = serq.kv_append(B.q, B.k, B.v, *B.args(), cos, sin, interleaved=inter, k_scale=B.k_scale, v_scale=B.v_scale, q_norm=qw, k_norm=kw).cpu()
        nan = want[0].isnan()
        assert torch.equal(q_out.isnan(), nan) and torch.equal(_bits(q_out)[~nan], _bits(want[0])[~nan])
        _same(B, torch.where(nan.to(DEV), want[0].to(DEV), q_out.to(DEV)), want, f"{dt}")
