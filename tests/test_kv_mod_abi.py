"""What the attention with capped scores, biases and ranges refuses, before any launch; its oracle by hand; on the CPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import kv_oracle as orc
from paper_2603_08185_amd import binding as serq
from tests.test_kv_abi import ODD, OFF4, P, _batch, _cache


def _call(q=P, Hq=8, dt=2, scale=0.1, window=0, o=P, lse=None, ws=None, wsb=0, c=None, b=None, mod=True, **m):
    cc, bb = _cache(**(c or {})), _batch(**(b or {}))
    mm = serq._AttnMod(**m)
    return serq.lib().serq_paged_attn_mod(q, 1024, 128, Hq, dt, C.addressof(cc), C.addressof(bb), 1, 40, scale, window, C.addressof(mm) if mod else None, o,
                                          1024, 128, lse, ws, wsb, None)


def test_refuses():
    for bad in (dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(cap=1024.5), dict(Hq=7), dict(scale=0.0), dict(window=-1)):
        assert _call(**bad) == -3, bad
    assert _call(cap=1.0, slopes=P) == -7
    for bad in (dict(slopes=ODD), dict(see_from=ODD), dict(see_to=ODD), dict(q=OFF4), dict(ws=OFF4)):
        assert _call(**bad) == -4, bad
    for bad in (dict(q=None), dict(o=None)):
        assert _call(cap=1.0, **bad) == -1, bad
    assert _call(dt=0) == -2 and _call(c=dict(dim=96)) == -3
    assert _call(b=dict(tokens=0), cap=1.0) == 0 and _call(b=dict(seqs=0), mod=False) == 0


def test_binding_refuses_host_tensors():
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    K = torch.zeros((2, 16, 4, 64), dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="device memory"):
        serq.paged_attention(q, K, K, i[:, None], i, i[:1], 1, 16, cap=3.0)
    serq.lib()
    assert serq._fast.paged_attention_mod(q, K, K, i[:, None], i, i[:1], 1, 16, 0.1, 0, None, None, q, None, None, 3.0, None, None, None) is None
    with pytest.raises(TypeError):
        serq._fast.paged_attention_mod(q)


def test_oracle_by_hand():
    """One row, two keys with the products 0 and ln 3: weights 1/4, 3/4; a cap of 1 makes the second tanh(ln 3) = 4/5; a slope of ln 3 a key undoes it."""
    q = np.ones((1, 1, 1))
    K, V = np.array([0.0, np.log(3)]).reshape(2, 1, 1), np.array([0.0, 4.0]).reshape(2, 1, 1)
    got = lambda first=1, lo=0, hi=2, **kw: orc.attention_mod(q, K, V, 1.0, first, [lo], [hi], **kw)
    assert np.isclose(got()[0], 3) and np.isclose(got()[1], np.log(4))
    e = np.exp(0.8)
    assert np.isclose(got(cap=1.0)[0], 4 * e / (1 + e)) and np.isclose(got(cap=1.0)[1], np.log(1 + e))
    assert np.isclose(got(first=0, slopes=[np.log(3)])[0], 2) and np.isclose(got(first=0, slopes=[np.log(3)])[1], np.log(2))
    assert np.isclose(got(first=1, slopes=[np.log(3)])[0], 4 * 9 / 10)
    out, lse, mag, _, _ = got(lo=1, hi=1)
    assert out[0] == 0 and lse[0] == -np.inf
    assert got(lo=1)[0] == 4
    a, b = orc.attention(np.random.RandomState(0).randn(3, 4, 8), np.random.RandomState(1).randn(9, 2, 8), np.random.RandomState(2).randn(9, 2, 8), 0.3, 6, 4), \
        orc.attention_mod(np.random.RandomState(0).randn(3, 4, 8), np.random.RandomState(1).randn(9, 2, 8), np.random.RandomState(2).randn(9, 2, 8), 0.3, 6,
                          [3, 4, 5], [7, 8, 9])
    assert np.allclose(a[0], b[0]) and np.allclose(a[1], b[1])
