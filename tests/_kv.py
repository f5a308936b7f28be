"""Batches for the tests of the paged cache: whatever a call must not look at holds NaN, and page numbers that it must not read are wild."""
from __future__ import annotations

import numpy as np
import torch

from oracle import kv_oracle as orc

DEV = "cuda:0"
WILD = (-7, 1 << 30, -(1 << 31))


def f8_values(x: torch.Tensor) -> np.ndarray:
    return x.float().double().cpu().numpy()


class Batch:
    """seqs: (new tokens, keys with them) of every sequence."""

    def __init__(self, seqs, Hq, Hkv, D, page=16, dt=torch.bfloat16, fp8=False, order="nhd", window=0, extra=0, seed=0, width=None, gain=1.0):
        g = torch.Generator().manual_seed(seed)
        r = np.random.RandomState(seed)
        self.seqs, self.Hq, self.Hkv, self.D, self.page, self.dt, self.fp8, self.window = seqs, Hq, Hkv, D, page, dt, fp8, window
        self.cu = np.concatenate([[0], np.cumsum([n for n, _ in seqs])]).astype(np.int32)
        self.len = np.array([L for _, L in seqs], np.int32)
        self.T = int(self.cu[-1]) + extra                        # `extra` rows of no sequence
        self.max_q, self.max_kv = max([n for n, _ in seqs] + [0]), max([L for _, L in seqs] + [0])
        need = [-(-L // page) for _, L in seqs]
        self.width = max(need + [1]) if width is None else width
        self.pages = sum(need) + 2
        perm = r.permutation(self.pages)
        self.table = r.choice(WILD, size=(len(seqs), self.width)).astype(np.int64)
        at = 0
        self.first = []                                          # first key that any new token of a sequence sees
        for b, (n, L) in enumerate(seqs):
            lo = max(0, L - n - window + 1) if window else 0
            if n == 0:
                lo = L
            self.first.append(min(lo, L))
            for i in range(min(need[b], self.width)):
                if i >= lo // page or n == 0:
                    self.table[b, i] = perm[at + i]
                if n == 0 or i < lo // page:
                    self.table[b, i] = WILD[i % 3]
            at += need[b]
        ct = torch.float8_e4m3fn if fp8 else dt
        shape = (self.pages, page, Hkv, D) if order == "nhd" else (self.pages, Hkv, page, D)

        def pool():
            x = torch.full(shape, float("nan")).to(ct).to(DEV)
            return x if order == "nhd" else x.transpose(1, 2)

        self.K, self.V = pool(), pool()
        self.k_scale = (torch.rand(Hkv, generator=g) * 0.02 + 0.04).to(DEV) if fp8 else None
        self.v_scale = (torch.rand(Hkv, generator=g) * 0.02 + 0.02).to(DEV) if fp8 else None
        qkv = torch.randn(self.T, (Hq + 2 * Hkv) * D + 24, generator=g) * gain
        self.qkv = qkv.to(dt).to(DEV)
        self.q = self.qkv[:, :Hq * D].view(self.T, Hq, D)
        self.k = self.qkv[:, Hq * D:(Hq + Hkv) * D].view(self.T, Hkv, D)
        self.v = self.qkv[:, (Hq + Hkv) * D:(Hq + 2 * Hkv) * D].view(self.T, Hkv, D)
        self.d_table = torch.from_numpy(self.table.astype(np.int32)).to(DEV)
        self.d_cu, self.d_len = torch.from_numpy(self.cu).to(DEV), torch.from_numpy(self.len).to(DEV)
        self._g = g

    def fill(self, gain=1.0):
        """Keys and values at every position that a new token may see; the rest keeps its NaN."""
        self.kv = []
        for b, (n, L) in enumerate(self.seqs):
            lo = self.first[b]
            k = torch.randn(L - lo, self.Hkv, self.D, generator=self._g) * gain
            v = torch.randn(L - lo, self.Hkv, self.D, generator=self._g)
            p = np.arange(lo, L)
            vals = []
            for cache, x, s in ((self.K, k, self.k_scale), (self.V, v, self.v_scale)):
                x = x.to(DEV)
                x = (x / s[:, None]).clamp(-448, 448).to(cache.dtype) if self.fp8 else x.to(cache.dtype)
                page = torch.from_numpy(self.table[b, p // self.page]).to(DEV)
                row = torch.from_numpy(p % self.page).to(DEV)
                if len(p) and self.fp8:
                    cache.view(torch.uint8)[page, row] = x.view(torch.uint8)
                elif len(p):
                    cache[page, row] = x
                x = x.float().double().cpu().numpy()
                x = x * s.double().cpu().numpy()[:, None] if self.fp8 else x
                vals.append(np.concatenate([np.full((lo, self.Hkv, self.D), np.nan), x]))
            self.kv.append(vals)
        return self

    def args(self):
        return self.K, self.V, self.d_table, self.d_cu, self.d_len

    def attention64(self, scale=None):
        scale = self.D ** -0.5 if scale is None else scale
        if getattr(self, "_known", (None,))[0] != scale:
            self._known = (scale, self._attention64(scale))
        return self._known[1]

    def _attention64(self, scale):
        out = np.zeros((self.T, self.Hq, self.D))
        mag, lse, big = out.copy(), np.full((self.T, self.Hq), -np.inf), np.zeros((self.T, self.Hq))
        q = self.q.double().cpu().numpy()
        for b, (n, L) in enumerate(self.seqs):
            s = slice(self.cu[b], self.cu[b + 1])
            out[s], lse[s], mag[s], big[s] = orc.attention(q[s], self.kv[b][0], self.kv[b][1], scale, L - n, self.window)
        return out, lse, mag, big


def check_attention(B, out, lse, scale=None, what=""):
    """Bounds: u half a unit in the last place of the 16-bit type, as a part of the value.  The result is rounded once (u |out|); the softmax'
    weights may be rounded to the 16-bit type before they meet V (u each, and u more for a sum formed from rounded ones: 2 u sum p |v|); a
    score is an fp32 sum of D products (at worst (D + 8) 2^-24 of sum |q k|, twice for the difference to the maximum), and the
    exponential, the running factors and the sum over n keys are good to (32 + n / 16) 2^-22 together.  fp16 weights below 2^-14 are off by up to 2^-25 of the
    largest one, each of them: 2^-25 n max |v|."""
    want, wlse, mag, big = B.attention64(scale)
    u, tiny = (2.0 ** -8, 2.0 ** -133) if B.dt == torch.bfloat16 else (2.0 ** -11, 2.0 ** -24)
    n = max(B.max_kv, 1)
    esc = (B.D + 8) * 2.0 ** -24 * big
    rel = 2 * esc + (32 + n / 16) * 2.0 ** -22
    sub = 2.0 ** -25 * n * 6.0 if B.dt == torch.float16 else 0.0
    tol = u * np.abs(want) + (2 * u + rel[..., None]) * mag * 1.01 + tiny + np.where(mag.max(-1, keepdims=True) > 0, sub, 0.0)
    got = out.double().cpu().numpy()
    rows = B.cu[-1]
    bad = ~(np.abs(got[:rows] - want[:rows]) <= tol[:rows])
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[:rows][bad][0]} for {want[:rows][bad][0]}"
    if lse is not None:
        gl = lse.double().cpu().numpy()[:rows]
        none = np.isneginf(wlse[:rows])
        assert np.array_equal(none, np.isneginf(gl)), f"{what}: rows without keys"
        d = np.abs(gl[~none] - wlse[:rows][~none])
        lim = (esc[:rows] + (32 + n / 16) * 2.0 ** -22 + 2.0 ** -22 * np.abs(np.where(np.isneginf(wlse[:rows]), 0, wlse[:rows])) + 2.0 ** -21)[~none]
        assert (d <= lim).all(), f"{what}: lse off by {d.max()} (bound {lim[d.argmax()]})"
