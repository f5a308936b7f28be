"""What the paged cache's entry points refuse, before any launch; on the CPU."""
import ctypes as C

import pytest
import torch

from paper_2603_08185_amd import binding as serq

_buf = (C.c_char * 4096)()
_a = (C.addressof(_buf) + 15) & ~15
P, ODD, OFF4 = _a, _a + 2, _a + 4


def _cache(**kw):
    d = dict(k=P, v=P, k_scale=None, v_scale=None, k_page=16 * 256, k_token=256, k_head=128, v_page=16 * 256, v_token=256, v_head=128, pages=4,
             page_size=16, heads=2, dim=128, dtype=2)
    d.update(kw)
    return serq._KvCache(**d)


def _batch(**kw):
    d = dict(cu_q=P, kv_len=P, table=P, table_ld=3, tokens=5, table_width=3, seqs=2)
    d.update(kw)
    return serq._KvBatch(**d)


def _append(q=P, ldq=1024, ldqh=128, Hq=8, k=P, ldk=256, ldkh=128, v=P, ldv=256, ldvh=128, dt=2, cos=P, sin=P, rows=10, rot=128, inter=0, pos=None,
            qo=P + 1024, ldqo=1024, ldqoh=128, cache=True, batch=True, c=None, b=None):
    cc, bb = _cache(**(c or {})), _batch(**(b or {}))
    return serq.lib().serq_kv_append(q, ldq, ldqh, Hq, k, ldk, ldkh, v, ldv, ldvh, dt, cos, sin, rows, rot, inter, pos,
                                     C.addressof(cc) if cache else None, C.addressof(bb) if batch else None, qo, ldqo, ldqoh, None)


def _attn(q=P, ldq=1024, ldqh=128, Hq=8, dt=2, max_q=1, max_kv=40, scale=0.1, window=0, o=P, ldo=1024, ldoh=128, lse=None, ws=None, wsb=0,
          cache=True, batch=True, c=None, b=None):
    cc, bb = _cache(**(c or {})), _batch(**(b or {}))
    return serq.lib().serq_paged_attn(q, ldq, ldqh, Hq, dt, C.addressof(cc) if cache else None, C.addressof(bb) if batch else None, max_q, max_kv,
                                      scale, window, o, ldo, ldoh, lse, ws, wsb, None)


@pytest.mark.parametrize("call", [_append, _attn])
def test_cache_and_batch_are_checked(call):
    assert call(cache=False) == -1 and call(batch=False) == -1
    assert call(dt=0) == -2 and call(dt=3) == -2 and call(c=dict(dtype=1)) == -2 and call(c=dict(dtype=0)) == -2
    for bad in (dict(dim=96), dict(dim=256), dict(heads=0), dict(heads=1025), dict(pages=-1), dict(page_size=8), dict(page_size=24),
                dict(page_size=131072), dict(k_page=-8), dict(v_head=-128), dict(k_token=(1 << 26) + 16)):
        assert call(c=bad) == -3, bad
    for bad in (dict(seqs=-1), dict(seqs=65537), dict(tokens=-1), dict(tokens=(1 << 22) + 1), dict(table_width=-1), dict(table_ld=2),
                dict(table_width=1 << 30, table_ld=1 << 30)):
        assert call(b=bad) == -3, bad
    for bad in (dict(k_token=260), dict(v_page=4), dict(k=ODD), dict(v=OFF4), dict(dtype=4, k_token=264), dict(dtype=4, v_scale=ODD)):
        assert call(c=bad) == -4, bad
    for bad in (dict(cu_q=ODD), dict(kv_len=ODD), dict(table=ODD)):
        assert call(b=bad) == -4, bad
    for bad in (dict(cu_q=None), dict(kv_len=None), dict(table=None)):
        assert call(b=bad) == -1, bad
    assert call(c=dict(k=None)) == -1 and call(c=dict(v=None)) == -1
    assert call(b=dict(tokens=0)) == 0 and call(b=dict(seqs=0)) == 0        # nothing to do
    assert call(b=dict(tokens=0, cu_q=None, kv_len=None, table=None), c=dict(k=None, v=None)) == 0


def test_append_refuses():
    for bad in (dict(rot=8), dict(rot=-16), dict(rot=144), dict(rows=0), dict(rows=-1), dict(Hq=-1), dict(Hq=65537), dict(ldqh=64), dict(ldkh=120),
                dict(ldv=-256), dict(ldqoh=8), dict(qo=P, ldqo=2048)):
        assert _append(**bad) == -3, bad
    for bad in (dict(q=None), dict(qo=None), dict(k=None), dict(v=None), dict(cos=None), dict(sin=None)):
        assert _append(**bad) == -1, bad
    for bad in (dict(ldq=1028), dict(ldk=260), dict(ldvh=132), dict(q=OFF4), dict(k=ODD), dict(v=ODD), dict(qo=ODD), dict(cos=OFF4), dict(pos=ODD)):
        assert _append(**bad) == -4, bad


def test_attention_refuses():
    for bad in (dict(Hq=0), dict(Hq=7), dict(Hq=65536), dict(window=-1), dict(max_q=-1), dict(max_kv=-1), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(ldqh=64), dict(ldo=-8), dict(ldoh=120),
                dict(Hq=2048, b=dict(tokens=1 << 22)), dict(Hq=1024, b=dict(seqs=65536), c=dict(heads=128))):
        assert _attn(**bad) == -3, bad
    for bad in (dict(q=None), dict(o=None)):
        assert _attn(**bad) == -1, bad
    for bad in (dict(ldq=1028), dict(ldoh=132), dict(q=OFF4), dict(o=ODD), dict(lse=ODD), dict(ws=OFF4)):
        assert _attn(**bad) == -4, bad
    size = serq.lib().serq_paged_attn_workspace_bytes
    assert size(1, 1, 1, 1000, 32, 8, 128) > 0 and size(0, 0, 0, 0, 8, 8, 64) > 0
    for bad in ((-1, 1, 1, 1, 8, 8, 64), (1, -1, 1, 1, 8, 8, 64), (1, 1, -1, 1, 8, 8, 64), (1, 1, 1, -1, 8, 8, 64), (1, 1, 1, 1, 9, 8, 64),
                (1, 1, 1, 1, 8, 0, 64), (1, 1, 1, 1, 8, 8, 80), (1, 1, 1, 1, 0, 8, 64)):
        assert size(*bad) == 0, bad


def test_binding_refuses_host_tensors():
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    K = torch.zeros((2, 16, 4, 64), dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="device memory"):
        serq.kv_append(q, q, q, K, K, i[:, None], i, i[:1])
    with pytest.raises(ValueError, match="device memory"):
        serq.paged_attention(q, K, K, i[:, None], i, i[:1], 1, 16)
    serq.lib()
    assert serq._fast.kv_append(q, q, q, K, K, i[:, None], i, i[:1], None, None, 0, None, None, None, q) is None
    assert serq._fast.paged_attention(q, K, K, i[:, None], i, i[:1], 1, 16, 0.1, 0, None, None, q, None, None) is None
    for f in (serq._fast.kv_append, serq._fast.paged_attention, serq._fast.bind_kv):
        with pytest.raises(TypeError):
            f(q)
    with pytest.raises(ValueError):
        serq._fast.bind_kv(0, 0)
