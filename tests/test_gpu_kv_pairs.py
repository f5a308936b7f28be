"""Heads of 64 channels side by side in memory, one a time or two where the sequences' keys are many: lines on both sides of that length, against 64 bits.
Sequences share their pages, so that long lines cost little."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as orc
from paper_2603_08185_amd import binding as serq
from tests._kv import DEV, WILD
from tests._kv_mod import check_mod
from tests._util import replay_check

pytestmark = pytest.mark.gpu
D, PAGE = 64, 16


def least(rows):
    """Keys times key heads from which on two heads go together; rows: of one head."""
    return max(6, 2 * rows) << 17


class Shared:
    """lens: keys of every sequence, all of them the first of the same pages; n new tokens each (0: an empty slot)."""

    def __init__(self, lens, Hq, Hkv, dt=torch.bfloat16, new=None, cap=0.0, bias=None, window=0, ranges=None, seed=0, gain=1.0):
        g, r = torch.Generator().manual_seed(seed), np.random.RandomState(seed)
        self.lens, self.Hq, self.Hkv, self.D, self.dt, self.cap, self.win = lens, Hq, Hkv, D, dt, cap, window
        new = new or [1] * len(lens)
        self.new, self.cu = new, np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.T, self.max_q, self.max_kv = int(self.cu[-1]), max(new), max(lens)
        pages = -(-self.max_kv // PAGE)
        perm = r.permutation(pages + 2)[:pages]
        need = [-(-L // PAGE) for L in lens]
        table = r.choice(WILD, size=(len(lens), pages)).astype(np.int64)
        for b, m in enumerate(need):
            table[b, :m] = perm[:m]
        self.table = torch.from_numpy(table.astype(np.int32)).to(DEV)
        self.K, self.V = (torch.full((pages + 2, PAGE, Hkv, D), float("nan"), dtype=dt, device=DEV) for _ in range(2))
        self.kv = []
        for cache, m in ((self.K, gain), (self.V, 1.0)):
            x = (torch.randn(pages * PAGE, Hkv, D, generator=g) * m).to(dt)
            cache[torch.from_numpy(perm).to(DEV)] = x.view(pages, PAGE, Hkv, D).to(DEV)
            self.kv.append(x.double().numpy())
        self.q = torch.randn(self.T, Hq, D, generator=g).to(dt).to(DEV)
        self.d_cu, self.d_len = torch.from_numpy(self.cu).to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.slopes = None if bias is None else np.array([bias * 2.0 ** (-8.0 * (h % 16) / 16) for h in range(Hq)], np.float32)
        self.lo, self.hi, frm, to = [], [], [], []
        for n, L in zip(new, lens):
            p = np.arange(L - n, L)
            a, z = ranges(r, n, L) if ranges else (np.zeros(n, int), p + 1)
            frm.append(a)
            to.append(z)
            lo, hi = np.maximum(a, 0), np.minimum(z, L)
            lo = np.maximum(lo, p - window + 1) if window else lo
            self.lo.append(np.where(hi > lo, lo, 0))
            self.hi.append(np.where(hi > lo, hi, 0))
        i32 = lambda x: torch.from_numpy(np.concatenate(x).astype(np.int32)).to(DEV)
        self.see_from, self.see_to = (i32(frm), i32(to)) if ranges else (None, None)

    def line(self):
        """Keys times key heads that the call's rows see, about."""
        return self.Hkv * sum(int(z.max() - a.min()) for a, z in zip(self.lo, self.hi) if len(z))

    def run(self, ws=True, max_kv=None):
        max_kv = max_kv or self.max_kv
        if ws is True:
            ws = serq.paged_attention_workspace(self.T, len(self.lens), self.max_q, max_kv, self.Hq, self.Hkv, D, DEV)
        lse = torch.full((self.T, self.Hq), 7.0, device=DEV)
        out = serq.paged_attention(self.q, self.K, self.V, self.table, self.d_cu, self.d_len, self.max_q, max_kv, window=self.win, lse=lse, ws=ws, cap=self.cap,
                                   slopes=None if self.slopes is None else torch.from_numpy(self.slopes).to(DEV), see_from=self.see_from, see_to=self.see_to)
        return out, lse

    def mod64(self, scale=None):
        if not hasattr(self, "_mod"):
            got = [np.zeros((self.T, self.Hq, D)), np.full((self.T, self.Hq), -np.inf), np.zeros((self.T, self.Hq, D)), np.zeros((self.T, self.Hq, D)),
                   np.zeros((self.T, self.Hq))]
            q = self.q.double().cpu().numpy()
            for b, (n, L) in enumerate(zip(self.new, self.lens)):
                s = slice(self.cu[b], self.cu[b + 1])
                for g, x in zip(got, orc.attention_mod(q[s], *self.kv, D ** -0.5, L - n, self.lo[b], self.hi[b], self.cap, self.slopes)):
                    g[s] = x
            self._mod = got
        return self._mod


def _lens(line, heads, window=0, most=6000):
    """Lengths of different sizes, whose seen keys times heads are `line` together."""
    left, out = line // heads, []
    while left > 0:
        out.append(min(left, most - 900 * (len(out) % 4) - len(out) % 7))
        left -= min(out[-1], window or out[-1])
    return out


MODS = {"none": {}, "cap": dict(cap=30.0), "bias": dict(bias=0.02), "bias window": dict(bias=0.1, window=5000), "cap window": dict(cap=9.0, window=4400),
        "ranges": dict(ranges=lambda r, n, L: (r.randint(0, 60, n), L - r.randint(0, 60, n))), "cap ranges": dict(cap=5.0, ranges=lambda r, n, L: (r.randint(-9, 60, n), L + r.randint(-60, 9, n))),
        "window": dict(window=5500)}


@pytest.mark.parametrize("mod", MODS)
@pytest.mark.parametrize("Hq,Hkv,n", [(2, 2, 1), (6, 6, 1), (32, 16, 1), (16, 4, 1), (14, 2, 1), (16, 16, 3), (8, 4, 4)])
def test_long_and_short_lines(mod, Hq, Hkv, n):
    for i, (part, dt) in enumerate(((1.3, torch.bfloat16), (1.3, torch.float16), (0.6, torch.float16))):
        lens = _lens(int(part * least(n * Hq // Hkv)), Hkv, MODS[mod].get("window", 0))
        new = [min(n, 1 + b % n) if n > 1 else 1 for b in range(len(lens))]
        new[3], new[4] = 0, n
        lens[5] = 3 + n
        B = Shared(lens, Hq, Hkv, dt, new, seed=Hq + i, **MODS[mod])
        assert (B.line() >= least(n * Hq // Hkv)) == (part > 1), "the other side"
        check_mod(B, *B.run(), what=f"{part} {dt}")
        if i == 0:
            check_mod(B, *B.run(ws=None), what="no workspace")
            for less in (70000, 1 << 20):                            # room for some of the slots
                ws = serq.paged_attention_workspace(B.T, len(lens), n, B.max_kv, Hq, Hkv, D, DEV)[:less]
                check_mod(B, *B.run(ws=ws), what=f"{less} bytes of workspace")


@pytest.mark.parametrize("mod", ["none", "cap", "bias", "ranges"])
@pytest.mark.parametrize("part", [1.2, 0.5])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (16, 4), (28, 4)])
def test_no_head_sees_its_neighbour(mod, part, Hq, Hkv):
    """What the keys and values of every other head hold, NaN and infinities, reaches no bit of the rest: even heads and odd ones, keys and values alike."""
    G = Hq // Hkv
    B = Shared(_lens(int(part * least(G)), Hkv), Hq, Hkv, seed=3, **MODS[mod])
    clean, lse = B.run()
    assert torch.isfinite(clean.float()).all()
    keep = B.K.clone(), B.V.clone()
    for spoilt in (0, 1):
        rest = [h for g in range(1 - spoilt, Hkv, 2) for h in range(g * G, (g + 1) * G)]
        hit = [h for g in range(spoilt, Hkv, 2) for h in range(g * G, (g + 1) * G)]
        for bad in (float("nan"), float("inf"), -float("inf")):
            for which in ("K", "V", "KV"):
                for name in which:
                    getattr(B, name)[:, :, spoilt::2] = bad
                out, l2 = B.run()
                assert torch.equal(out[:, rest], clean[:, rest]) and torch.equal(l2[:, rest], lse[:, rest]), (spoilt, bad, which)
                assert not torch.isfinite(out[:, hit].float()).any() or (mod == "cap" and which == "K") or (bad < 0 and which == "K"), (spoilt, bad, which)
                B.K.copy_(keep[0])
                B.V.copy_(keep[1])


def test_bounds_far_above_the_lengths():
    """max_kv of a captured graph that serves every step to come: short sequences, the same results within the bounds; more keys than the line's least, too."""
    for Hq, Hkv in ((16, 16), (16, 4)):
        for lens in ([1], [40], [300, 7, 64, 65], [5000], [900] * 30, _lens(int(1.1 * least(Hq // Hkv)), Hkv)):
            for mod in ("none", "cap", "bias"):
                B = Shared(lens, Hq, Hkv, seed=len(lens), **MODS[mod])
                check_mod(B, *B.run(max_kv=1 << 20), what=f"{len(lens)} {mod}")


@pytest.mark.parametrize("mod", ["none", "cap", "ranges"])
def test_replays_across_the_length(mod):
    """One graph whose sequences grow past the length and shrink again, on one workspace."""
    B = Shared(_lens(int(1.02 * least(1)), 8), 8, 8, seed=5, **MODS[mod])
    whole = B.d_len.clone()
    ws = serq.paged_attention_workspace(B.T, len(B.lens), 1, B.max_kv, 8, 8, D, DEV)
    out, lse = torch.empty_like(B.q), torch.empty((B.T, 8), device=DEV)
    for t in (B.K, B.V):
        t.nan_to_num_(nan=0.0)
    table = B.table.clamp(0, B.K.shape[0] - 1)

    def step():
        serq.paged_attention(B.q, B.K, B.V, table, B.d_cu, B.d_len, 1, B.max_kv, out=out, lse=lse, ws=ws, cap=B.cap, see_from=B.see_from, see_to=B.see_to)

    def mutate(it):
        B.d_len.copy_(whole if it % 2 else whole * 2 // 3)
        B.q.mul_(-0.9)

    replay_check(step, [out, lse], mutate)


def test_same_from_run_to_run():
    for part in (0.7, 1.3):
        B = Shared(_lens(int(part * least(4)), 4), 16, 4, seed=8)
        ws = serq.paged_attention_workspace(B.T, len(B.lens), 1, B.max_kv, 16, 4, D, DEV)
        want, lse = B.run(ws)
        for _ in range(10):
            out, l2 = B.run(ws)
            assert torch.equal(out, want) and torch.equal(l2, lse)
