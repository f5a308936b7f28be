"""What the normalising append refuses, before any launch; on the CPU."""
import ctypes as C

import pytest
import torch

from paper_2603_08185_amd import binding as serq
from tests.test_kv_abi import ODD, OFF4, P, _batch, _cache


def _call(q=P, ldq=1024, ldqh=128, Hq=8, k=P, ldk=256, ldkh=128, v=P, ldv=256, ldvh=128, dt=2, qw=P, kw=P, eps=1e-6, cos=P, sin=P, rows=10, rot=128,
          inter=0, pos=None, qo=P + 1024, ldqo=1024, ldqoh=128, c=None, b=None):
    cc, bb = _cache(**(c or {})), _batch(**(b or {}))
    return serq.lib().serq_kv_append_norm(q, ldq, ldqh, Hq, k, ldk, ldkh, v, ldv, ldvh, dt, qw, kw, eps, cos, sin, rows, rot, inter, pos,
                                          C.addressof(cc), C.addressof(bb), qo, ldqo, ldqoh, None)


def test_refuses():
    for bad in (dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")), dict(rot=8), dict(Hq=-1), dict(ldqh=64), dict(qo=P, ldqo=2048)):
        assert _call(**bad) == -3, bad
    for bad in (dict(qw=OFF4), dict(kw=ODD), dict(cos=OFF4), dict(q=ODD)):
        assert _call(**bad) == -4, bad
    for bad in (dict(k=None), dict(cos=None)):
        assert _call(**bad) == -1, bad
    assert _call(dt=0) == -2 and _call(c=dict(dim=96)) == -3
    assert _call(b=dict(tokens=0)) == 0 and _call(b=dict(seqs=0)) == 0


def test_binding_refuses_host_tensors():
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    K = torch.zeros((2, 16, 4, 64), dtype=torch.bfloat16)
    i, w = torch.zeros(2, dtype=torch.int32), torch.ones(64)
    with pytest.raises(ValueError, match="device memory"):
        serq.kv_append(q, q, q, K, K, i[:, None], i, i[:1], q_norm=w, k_norm=w)
    serq.lib()
    assert serq._fast.kv_append_norm(q, q, q, K, K, i[:, None], i, i[:1], None, None, 0, None, None, None, q, w, w, 1e-6) is None
    with pytest.raises(TypeError):
        serq._fast.kv_append_norm(q)
