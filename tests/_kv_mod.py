"""Batches for the tests of the attention with capped scores, biases and ranges: every key that no row sees holds NaN, and page numbers outside what a
sequence's rows see are wild."""
from __future__ import annotations

import numpy as np
import torch

from oracle import kv_oracle as orc
from tests._kv import DEV, WILD, Batch


def docs(rng, n, L):
    """Documents of 1 to 60 keys in a row; some rows of padding."""
    p = np.arange(L - n, L)
    starts = [0]
    while starts[-1] < L:
        starts.append(starts[-1] + int(rng.randint(1, 60)))
    frm = np.array(starts)[np.searchsorted(starts, p, side="right") - 1]
    to = np.where(rng.rand(n) < 0.1, 0, p + 1)
    return frm, to


def prefix(rng, n, L):
    p = np.arange(L - n, L)
    return np.zeros(n, int), np.maximum(p + 1, int(rng.randint(0, L + 1)))


def wild(rng, n, L):
    """Any range: empty ones, reversed ones, past the end, before the start, one key, keys behind the row's own."""
    frm = rng.randint(-5, L + 5, n)
    to = np.where(rng.rand(n) < 0.3, frm + 1, rng.randint(-5, L + 40, n))
    frm = np.where(rng.rand(n) < 0.3, -(1 << 31), frm)
    to = np.where(rng.rand(n) < 0.2, (1 << 31) - 1, to)
    return frm, to


class ModBatch(Batch):
    def __init__(self, seqs, Hq, Hkv, D, page=16, dt=torch.bfloat16, fp8=False, order="nhd", window=0, cap=0.0, bias=None, ranges=None, extra=0, seed=0,
                 gain=1.0):
        super().__init__(seqs, Hq, Hkv, D, page, dt, fp8, order, 0, extra, seed, gain=gain)
        super().fill(gain)
        self.cap, self.win = cap, window
        r = np.random.RandomState(seed + 1)
        self.slopes = None if bias is None else (np.array([bias * 2.0 ** (-8.0 * (h % 16) / 16) for h in range(Hq)], np.float32))
        frm, to = np.zeros(self.T, np.int64), np.zeros(self.T, np.int64)
        self.lo, self.hi = [], []
        for b, (n, L) in enumerate(seqs):
            s, p = slice(self.cu[b], self.cu[b + 1]), np.arange(L - n, L)
            frm[s], to[s] = ranges(r, n, L) if ranges else (0, p + 1)
            lo, hi = np.maximum(frm[s], 0), np.minimum(to[s], min(L, self.width * page))
            if window:
                lo = np.maximum(lo, p - window + 1)
            some = hi > lo
            self.lo.append(np.where(some, lo, 0))
            self.hi.append(np.where(some, hi, 0))
            seen = np.zeros(L + 1, bool)
            for a, z in zip(self.lo[-1], self.hi[-1]):
                seen[a:z] = True
            hidden = np.nonzero(~seen[:L])[0]
            if n and len(hidden):                                       # what no row sees is NaN, in the caches and in what the oracle reads
                at, row = torch.from_numpy(self.table[b, hidden // page]).to(DEV), torch.from_numpy(hidden % page).to(DEV)
                for cache in (self.K, self.V):
                    if fp8:
                        cache.view(torch.uint8)[at, row] = 0x7f
                    else:
                        cache[at, row] = float("nan")
                for x in self.kv[b]:
                    x[hidden] = np.nan
            which = np.nonzero(seen)[0]
            keep = (which[0] // page, which[-1] // page) if len(which) else (1, 0)
            for i in range(self.width):
                if not keep[0] <= i <= keep[1]:
                    self.table[b, i] = WILD[i % 3]
        self.d_table = torch.from_numpy(self.table.astype(np.int32)).to(DEV)
        i32 = lambda x: torch.from_numpy(np.clip(x, -(1 << 31), (1 << 31) - 1).astype(np.int32)).to(DEV)
        self.see_from = self.see_to = None
        if ranges:
            self.see_from, self.see_to = i32(frm), i32(to)

    def call(self, **kw):
        return dict(window=self.win, k_scale=self.k_scale, v_scale=self.v_scale, cap=self.cap, see_from=self.see_from, see_to=self.see_to,
                    slopes=None if self.slopes is None else torch.from_numpy(self.slopes).to(DEV)) | kw

    def mod64(self, scale=None):
        scale = self.D ** -0.5 if scale is None else scale
        if getattr(self, "_mod", (None,))[0] != scale:
            got = [np.zeros((self.T, self.Hq, self.D)), np.full((self.T, self.Hq), -np.inf), np.zeros((self.T, self.Hq, self.D)),
                   np.zeros((self.T, self.Hq, self.D)), np.zeros((self.T, self.Hq))]
            q = self.q.double().cpu().numpy()
            for b, (n, L) in enumerate(self.seqs):
                s = slice(self.cu[b], self.cu[b + 1])
                for g, x in zip(got, orc.attention_mod(q[s], *self.kv[b], scale, L - n, self.lo[b], self.hi[b], self.cap, self.slopes)):
                    g[s] = x
            self._mod = (scale, got)
        return self._mod[1]


def check_mod(B, out, lse, scale=None, what=""):
    """Bounds as check_attention's (u half a unit in the last place of the 16-bit type as a part of the value: the result u, the weights 2 u; the
    exponential, the running factors and the sum over n keys (32 + n / 16) 2^-22; fp16 weights below 2^-14 up to 2^-25 n max |v|), with the errors of the
    scores key by key: twice the oracle's, for the difference to the reference."""
    want, wlse, mag, eo, el = B.mod64(scale)
    u, tiny = (2.0 ** -8, 2.0 ** -133) if B.dt == torch.bfloat16 else (2.0 ** -11, 2.0 ** -24)
    n = max(B.max_kv, 1)
    run = (32 + n / 16) * 2.0 ** -22
    sub = 2.0 ** -25 * n * 6.0 if B.dt == torch.float16 else 0.0
    tol = u * np.abs(want) + ((2 * u + run) * mag + 2 * eo) * 1.01 + tiny + np.where(mag.max(-1, keepdims=True) > 0, sub, 0.0)
    got, rows = out.double().cpu().numpy(), B.cu[-1]
    bad = ~(np.abs(got[:rows] - want[:rows]) <= tol[:rows])
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[:rows][bad][0]} for {want[:rows][bad][0]}"
    if lse is not None:
        gl, none = lse.double().cpu().numpy()[:rows], np.isneginf(wlse[:rows])
        assert np.array_equal(none, np.isneginf(gl)), f"{what}: rows without keys"
        some = ~none
        d = np.abs(gl[some] - wlse[:rows][some])
        lim = 2 * el[:rows][some] + run + 2.0 ** -22 * (np.abs(wlse[:rows][some]) + 4 * B.cap) + 2.0 ** -21
        assert (d <= lim).all(), f"{what}: lse off by {d.max()} (bound {lim[d.argmax()]})"
