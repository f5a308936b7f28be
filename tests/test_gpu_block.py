"""The steps of a block's attention half together, as the example runs them: sum and norm with the codes, the projection, head norms, rotation and append,
capped attention, the o projection; every step against the same arithmetic in 64 bits on what the one before it gave."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import kv_oracle as kvo
from oracle import serq_oracle as orc
from paper_2603_08185_amd import binding as serq
from tests._util import f32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_block.py")
    spec = importlib.util.spec_from_file_location("attention_block", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    return ex


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("cap", [0.0, 4.0])
def test_a_block_with_norms(fp8, cap, monkeypatch):
    ex = _example()
    block = ex.AttentionBlock(hidden=512, q_heads=8, kv_heads=2, dim=64, rank=32, pages=64, page=16, fp8=fp8, norms=True, cap=cap)
    seen = []
    for name in ("rmsnorm_quantize_act", "kv_append", "paged_attention"):
        def spy(*a, _real=getattr(serq, name), _name=name, **kw):
            before = [t.clone() if isinstance(t, torch.Tensor) else t for t in a], {k: t.clone() if isinstance(t, torch.Tensor) else t for k, t in kw.items()}
            out = _real(*a, **kw)
            if len(seen) < 6:                                     # the prompts' step and the first token's
                seen.append((_name, before, a, kw, [t.clone() if isinstance(t, torch.Tensor) else t for t in (out if isinstance(out, tuple) else (out,))]))
            return out
        monkeypatch.setattr(serq, name, spy)
    prompts = [70, 3, 130]
    first, y, kv_len, table, _ = ex.run(block, prompts, 5)
    assert kv_len.tolist() == [p + 1 + 5 for p in prompts] and torch.isfinite(first).all() and torch.isfinite(y).all()
    assert [s[0] for s in seen] == ["rmsnorm_quantize_act", "kv_append", "paged_attention"] * 2
    for name, (a, kw), _, now, out in seen:
        if name == "rmsnorm_quantize_act":
            h = (a[0].float() + kw["residual"].float()).to(a[0].dtype)
            codes, scale = orc.rmsnorm_quantize_act(f32(h), f32(a[1]), a[2], 8)
            M, K = a[0].shape
            assert torch.equal(out[2], h) and np.array_equal(out[0].view(torch.int8)[:M * K].view(M, K).cpu().numpy(), codes)
            assert np.array_equal(out[1][:M].cpu().numpy(), scale)
        elif name == "kv_append":
            q, k, v, K, V, tb, cu, ln, cos, sin = a
            seq, pos = kvo.positions(cu.cpu().numpy(), ln.cpu().numpy(), q.shape[0])
            want = kvo.rotate(kvo.normed(f32(q), f32(kw["q_norm"]), 1e-6), f32(cos)[pos], f32(sin)[pos], 64, False, np.float32)
            assert torch.equal(out[0].cpu(), torch.from_numpy(want).to(q.dtype))
        else:
            q, K, V, tb, cu, ln = a[:6]
            for b in range(3):
                L, rows = int(ln[b]), slice(int(cu[b]), int(cu[b + 1]))
                n, p = rows.stop - rows.start, torch.arange(L, device=DEV)
                page, row = tb[b].long()[p // 16], p % 16
                kk, vv = ((x.float() * (s[:, None] if s is not None else 1.0))[page, row].double().cpu().numpy() for x, s in ((K, kw["k_scale"]), (V, kw["v_scale"])))
                at = np.arange(L - n, L)
                want, _, mag, eo, _ = kvo.attention_mod(q[rows].double().cpu().numpy(), kk, vv, 64 ** -0.5, L - n, np.zeros(n), at + 1, cap)
                tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -7 + 2.0 ** -15) * mag + 2 * eo
                assert (np.abs(out[0][rows].double().cpu().numpy() - want) <= tol).all(), b


def test_what_the_block_gives_goes_back_into_the_stream():
    """The example's graph against the same steps one by one: each step's output is the next one's x, which is added to the stream."""
    ex = _example()
    blocks = [ex.AttentionBlock(hidden=512, q_heads=8, kv_heads=2, dim=64, rank=32, pages=64, page=16, norms=True, cap=6.0) for _ in range(2)]
    prompts, steps = [70, 3, 130], 4
    first, y, kv_len, table, _ = ex.run(blocks[0], prompts, steps)
    block, g = blocks[1], torch.Generator(device=DEV).manual_seed(1)
    torch.randperm(block.K.shape[0], generator=g, device=DEV)
    new = lambda n: torch.randn((n, block.hidden), generator=g, device=DEV).to(block.dtype)
    cu = torch.tensor([0, 70, 73, 203], dtype=torch.int32, device=DEV)
    lens = torch.tensor(prompts, dtype=torch.int32, device=DEV)
    x, most = new(203), max(prompts) + steps + 1
    out = block.step(x, table, cu, lens, block.buffers(203, 3, 130, 130), torch.zeros_like(x))
    assert torch.equal(out, first)
    x, one, b = new(3), torch.arange(4, dtype=torch.int32, device=DEV), block.buffers(3, 3, 1, most)
    stream = torch.zeros_like(x)
    for _ in range(steps + 1):
        lens += 1
        before = stream.clone()
        out = block.step(x, table, one, lens, b, stream).clone()
        assert torch.equal(stream, (x.float() + before.float()).to(x.dtype))
        x = out
    assert torch.equal(lens, kv_len) and torch.equal(out, y)
    for a, c in ((blocks[0].K, block.K), (blocks[0].V, block.V)):
        assert torch.equal(a, c)


@pytest.mark.parametrize("fp8", [False, True])
def test_what_the_append_writes(fp8, monkeypatch):
    """Keys and values of a block's steps as they lie in the cache: normalised and rotated keys, values as they are, each in its own slot, bit for bit, and
    every other slot as it was."""
    ex = _example()
    block = ex.AttentionBlock(hidden=512, q_heads=8, kv_heads=2, dim=64, rank=32, pages=64, page=16, fp8=fp8, norms=True)
    for cache in (block.K, block.V):
        cache.view(torch.uint8).random_(0, 120, generator=torch.Generator(device=DEV).manual_seed(2))
    seen, real = [], serq.kv_append

    def spy(q, k, v, K, V, *a, **kw):
        if len(seen) == 2:                                        # the prompts' step, the first token's; then the graph's
            return real(q, k, v, K, V, *a, **kw)
        before = [t.clone() for t in (q, k, v, K, V, a[1], a[2])]
        out = real(q, k, v, K, V, *a, **kw)
        seen.append((before, a, kw, K.clone(), V.clone()))
        return out

    monkeypatch.setattr(serq, "kv_append", spy)
    ex.run(block, [70, 3, 130], 2)
    bits = lambda t: t.contiguous().view(torch.uint8).cpu()
    for (q, k, v, K, V, cu, ln), (table, _, _, cos, sin), kw, K1, V1 in seen:
        seq, pos = kvo.positions(cu.cpu().numpy(), ln.cpu().numpy(), k.shape[0])
        page, row = (torch.from_numpy(np.asarray(x)).to(DEV) for x in kvo.slots(seq, pos, table.cpu().numpy(), 16, 64))
        assert (page >= 0).all() and len(set(zip(page.tolist(), row.tolist()))) == k.shape[0]
        keys = kvo.rotate(kvo.normed(f32(k), f32(kw["k_norm"]), 1e-6), f32(cos)[pos], f32(sin)[pos], 64, False, np.float32)
        for cache, after, x, s in ((K, K1, keys, kw["k_scale"]), (V, V1, f32(v), kw["v_scale"])):
            want = cache.clone()
            x = torch.from_numpy(x).to(DEV)
            x = (x / s[:, None]).clamp(-448, 448) if fp8 else x
            want.view(torch.uint8)[page, row] = x.to(cache.dtype).view(torch.uint8)
            assert torch.equal(bits(after), bits(want))
