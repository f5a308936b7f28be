"""What the fused norm's entry points refuse, before any launch; on the CPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import serq_oracle as orc
from paper_2603_08185_amd import binding as serq

_buf = (C.c_char * 4096)()
P = (C.addressof(_buf) + 15) & ~15
ODD, OFF4, OFF8 = P + 2, P + 4, P + 8


def _sym(x=P, res=P + 1024, dt=2, gain=P, eps=1e-6, M=1, K=64, ldx=64, ldr=64, h=P + 2048, ldh=64, abits=8, xq=P, sc=P, zero=P):
    return serq.lib().serq_rmsnorm_quantize_act(x, res, dt, gain, eps, M, K, ldx, ldr, h, ldh, abits, xq, sc, None)


def _asym(x=P, res=P + 1024, dt=2, gain=P, eps=1e-6, M=1, K=64, ldx=64, ldr=64, h=P + 2048, ldh=64, abits=8, xq=P, sc=P, zero=P):
    return serq.lib().serq_rmsnorm_quantize_act_asym(x, res, dt, gain, eps, M, K, ldx, ldr, h, ldh, abits, xq, sc, zero, None)


def _mx(x=P, res=P + 1024, dt=2, gain=P, eps=1e-6, M=1, K=64, ldx=64, ldr=64, h=P + 2048, ldh=64, abits=4, xq=P, sc=P, zero=P):
    return serq.lib().serq_mx_rmsnorm_quantize_act(x, res, dt, gain, eps, M, K, ldx, ldr, h, ldh, xq, sc, None)


@pytest.mark.parametrize("call", [_sym, _asym, _mx])
def test_refuses(call):
    for bad in (dict(dt=3), dict(dt=4), dict(dt=-1)):
        assert call(**bad) == -2, bad
    for bad in (dict(K=0), dict(K=96, ldx=96, ldr=96, ldh=96), dict(K=131136, ldx=131136, ldr=131136, ldh=131136), dict(M=-1), dict(M=(1 << 30) + 1),
                dict(ldx=56), dict(ldr=56), dict(ldh=56), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(res=None), dict(x=P + 2048, ldx=72), dict(res=P + 2048, ldr=72)):
        assert call(**bad) == -3, bad
    for bad in (dict(ldx=68), dict(ldr=68), dict(ldh=68), dict(x=ODD), dict(res=OFF8), dict(gain=OFF4), dict(h=OFF8), dict(xq=OFF8), dict(sc=ODD)):
        assert call(**bad) == -4, bad
    for bad in (dict(x=None), dict(h=None), dict(xq=None), dict(sc=None)):
        assert call(**bad) == -1, bad
    assert call(M=0, x=None, res=None, h=None, xq=None, sc=None, zero=None) == 0
    assert call(M=0, ldr=56) == -3


def test_refuses_by_form():
    assert _sym(abits=5) == -2 and _asym(abits=3) == -2
    assert _asym(zero=None) == -1 and _asym(zero=ODD) == -4
    assert _mx(sc=OFF4) == -4                                       # the layer reads block scales in pieces of 16 bytes


def test_binding_refuses():
    x, g = torch.zeros((2, 64), dtype=torch.bfloat16), torch.ones(64)
    for call in (lambda **k: serq.rmsnorm_quantize_act(x, g, 1e-6, 8, **k), lambda **k: serq.rmsnorm_quantize_act_asym(x, g, 1e-6, 8, **k),
                 lambda **k: serq.mx_rmsnorm_quantize_act(x, g, 1e-6, **k)):
        with pytest.raises(ValueError, match="device memory"):
            call()
        with pytest.raises(ValueError, match="device memory"):
            call(residual=x, h=x)
    serq.lib()
    u8, f, i = torch.zeros(256, dtype=torch.uint8), torch.zeros(16), torch.zeros(16, dtype=torch.int32)
    assert serq._fast.rmsnorm_quantize_act(x, g, 1e-6, 8, None, None, u8, f) is None
    assert serq._fast.rmsnorm_quantize_act_asym(x, g, 1e-6, 8, None, None, u8, f, i) is None
    assert serq._fast.mx_rmsnorm_quantize_act(x, g, 1e-6, None, None, u8, u8) is None
    for f in (serq._fast.rmsnorm_quantize_act, serq._fast.rmsnorm_quantize_act_asym, serq._fast.mx_rmsnorm_quantize_act, serq._fast.bind_norm):
        with pytest.raises(TypeError):
            f(x)
    with pytest.raises(ValueError):
        serq._fast.bind_norm(0, 0, 0, 0, 0)


def test_oracle_by_hand():
    """h = (3, 4, 0 ...) of 64 channels: mean square 25 / 64, root 5 / 8; gain 2 doubles u, not the root."""
    h = np.zeros((3, 64), np.float32)
    h[0, :2] = 3, 4
    h[2] = 1
    gain = np.full(64, 2, np.float32)
    u, rstd = orc.rmsnorm_rows(h, gain, 0.0)
    assert u[0, 0] == 6 and u[0, 1] == 8 and rstd[0] == np.float32(1.6) and rstd[1] == 0 and rstd[2] == 1
    codes, scale = orc.rmsnorm_quantize_act(h, gain, 0.0, 8)
    assert list(codes[0, :2]) == [95, 127] and scale[0] == np.float32(8) * (np.float32(1) / np.float32(127)) * np.float32(1.6)
    assert scale[1] == 1 and not codes[1].any()
    codes, E = orc.mx_rmsnorm_quantize_act(h, gain, 0.0)              # 9.6, 12.8: 2^3 over the largest code's 2^2 -> 2^1: 4.8, 6.4 -> 4, 6
    assert E[0, 0] == 128 and list(codes[0, :2]) == [6, 7]
    codes, scale, zero = orc.rmsnorm_quantize_act_asym(h, gain, 0.0, 4)
    assert list(codes[0, :2]) == [11 - 8, 15 - 8] and zero[0] == -8
