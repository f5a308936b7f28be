"""The attention half of a decoder block, served with 4-bit weights: prompts, then token after token.

    python examples/attention_block.py [--fp8] [--tokens 32]

Every step runs what a server runs for a layer: quantise the residual stream, the fused q/k/v projection, rotate and append to the paged
cache, attention over it, quantise, the o projection.  Sequences of different lengths share the cache's pages; the prompts go through in
one ragged call, the tokens after them one a sequence, recorded into a graph once and replayed (lengths live in device memory).
Weights are random: the numbers show the path, not a language.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2603_08185_amd import binding as serq  # noqa: E402


class AttentionBlock:
    """One layer's projections and cache."""

    def __init__(self, hidden=4096, q_heads=32, kv_heads=8, dim=128, rank=64, pages=256, page=64, fp8=False, dtype=torch.bfloat16, dev="cuda", seed=0):
        g = torch.Generator(device=dev).manual_seed(seed)
        self.hidden, self.q_heads, self.kv_heads, self.dim, self.rank, self.dtype, self.dev = hidden, q_heads, kv_heads, dim, rank, dtype, dev
        w = lambda n, k: (torch.randn((n, k), generator=g, device=dev) * k ** -0.5).to(dtype)
        self.width = (q_heads + 2 * kv_heads) * dim
        # (the identity as channel order: the projections' inputs here come in their own order)
        order = lambda k: torch.arange(k, dtype=torch.int32, device=dev)
        self.qkv = serq.pack_weights(w(self.width, hidden), None, rank, order(hidden), dtype)
        self.o = serq.pack_weights(w(hidden, q_heads * dim), None, rank, order(q_heads * dim), dtype)
        kind = torch.float8_e4m3fn if fp8 else dtype
        pool = lambda: torch.zeros((pages, kv_heads, page, dim), device=dev).to(kind).transpose(1, 2)      # [pages, page, heads, dim]
        self.K, self.V, self.page = pool(), pool(), page
        self.k_scale = torch.full((kv_heads,), 0.05, device=dev) if fp8 else None
        self.v_scale = torch.full((kv_heads,), 0.05, device=dev) if fp8 else None
        angle = torch.arange(pages * page, device=dev, dtype=torch.float64)[:, None] * 500000.0 ** (-torch.arange(dim // 2, device=dev) / (dim / 2))
        self.cos, self.sin = angle.cos().float(), angle.sin().float()

    def buffers(self, tokens, seqs, max_q, max_kv):
        """What a server allocates once for steps of up to these sizes."""
        e = lambda *s, dt=self.dtype: torch.empty(s, dtype=dt, device=self.dev)
        ws = lambda n, k: serq.workspace(tokens, n, k, self.rank, 8, self.dev)
        return {"xq": e(tokens * max(self.hidden, self.q_heads * self.dim), dt=torch.uint8), "sc": e(tokens, dt=torch.float32),
                "qkv": e(tokens, self.width), "att": e(tokens, self.q_heads, self.dim), "y": e(tokens, self.hidden),
                "ws_qkv": ws(self.width, self.hidden), "ws_o": ws(self.hidden, self.q_heads * self.dim), "max": (max_q, max_kv),
                "ws": serq.paged_attention_workspace(tokens, seqs, max_q, max_kv, self.q_heads, self.kv_heads, self.dim, self.dev)}

    def step(self, x, table, cu_q, kv_len, b):
        """x [tokens, hidden]: the new tokens of all sequences; returns the attention half's contribution to the residual stream."""
        T, H, Hk, D = x.shape[0], self.q_heads, self.kv_heads, self.dim
        serq.quantize_act(x, self.qkv.s_inv, 8, b["xq"], b["sc"])
        serq.linear(b["xq"], b["sc"], 8, self.qkv.Wq, self.qkv.wscale, T, self.width, self.hidden, Rp=self.qkv.Rp, r=self.rank, Y=b["qkv"], ws=b["ws_qkv"])
        q, k, v = (t.view(T, -1, D) for t in b["qkv"].split([H * D, Hk * D, Hk * D], 1))
        serq.kv_append(q, k, v, self.K, self.V, table, cu_q, kv_len, self.cos, self.sin, k_scale=self.k_scale, v_scale=self.v_scale, q_out=q)
        serq.paged_attention(q, self.K, self.V, table, cu_q, kv_len, *b["max"], k_scale=self.k_scale, v_scale=self.v_scale, out=b["att"], ws=b["ws"])
        serq.quantize_act(b["att"].view(T, H * D), self.o.s_inv, 8, b["xq"], b["sc"])
        return serq.linear(b["xq"], b["sc"], 8, self.o.Wq, self.o.wscale, T, self.hidden, H * D, Rp=self.o.Rp, r=self.rank, Y=b["y"], ws=b["ws_o"])


def run(block, prompts, steps, seed=1):
    """Prompts of the given lengths, then `steps` tokens each; returns the outputs of the prompts and of the last step, and seconds a step."""
    dev, B = block.dev, len(prompts)
    g = torch.Generator(device=dev).manual_seed(seed)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    most = max(prompts) + steps + 1
    width = -(-most // block.page)
    table = torch.randperm(block.K.shape[0], generator=g, device=dev)[:B * width].view(B, width).to(torch.int32).contiguous()
    new = lambda n: torch.randn((n, block.hidden), generator=g, device=dev).to(block.dtype)

    T = sum(prompts)
    cu = i32([sum(prompts[:b]) for b in range(B + 1)])
    first = block.step(new(T), table, cu, i32(prompts), block.buffers(T, B, max(prompts), max(prompts))).clone()

    x, one, kv_len, b = new(B), i32(list(range(B + 1))), i32(prompts), block.buffers(B, B, 1, most)
    kv_len += 1
    block.step(x, table, one, kv_len, b)                          # warm, and the token that the graph's first replay follows
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        kv_len += 1
        y = block.step(x, table, one, kv_len, b)
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(steps):
        graph.replay()
    torch.cuda.synchronize()
    return first, y, kv_len, table, (time.perf_counter() - began) / max(steps, 1)


def main():
    a = argparse.ArgumentParser()
    a.add_argument("--fp8", action="store_true", help="an E4M3 cache")
    a.add_argument("--tokens", type=int, default=32)
    a = a.parse_args()
    block = AttentionBlock(fp8=a.fp8)
    prompts = [700, 33, 1500, 256]
    _, y, kv_len, _, s = run(block, prompts, a.tokens)
    assert torch.isfinite(y).all()
    print(f"prompts of {prompts} tokens, then {a.tokens} tokens each ({'E4M3' if a.fp8 else '16-bit'} cache): {s * 1e6:.1f} us a step of "
          f"{len(prompts)} tokens, lengths now {kv_len.tolist()}")


if __name__ == "__main__":
    main()
