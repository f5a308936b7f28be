"""The work by which three steps of a decoder block are judged that go past the plain layer and the plain attention.

  norm       what stands before a quantised projection: the residual sum, its root-mean-square norm, flattening and quantisation, in one pass
             (`rmsnorm_quantize_act` and its forms for asymmetric codes and for MXFP4).
  append     `kv_append` of a model that normalises the queries and keys of every head before it rotates them.
  attention  `paged_attention` with what some models put between the scores and the softmax: scores capped by a tanh, a bias that grows with the
             distance, rows that see a range of keys of their own (packed documents, prefixes that are seen both ways, padding).

A pass is one call that a model server makes for one layer and one batch of new tokens.  Weights, the cache, the page table, lengths, tables,
output buffers and the workspace are what such a program keeps.

A case of norm:
  M, K        tokens, channels
  inp, form   type of the stream; "a8", "a4" (symmetric codes), "asym8", "asym4", "mx"
  res         whether there is a residual to add (the first layer has none)
A case of append or attention:
  B, n, mix   sequences, new tokens of the first one, and how many the others have: "same" (n each), "ragged" (1 to n), "ones" (1 each, a
              chunk that rides along with decoding).  In a batch of 8 or more that is not "same" the last sequence is an empty slot.
  ctx, fill   keys that the cache holds before the call: ctx for the first sequence, for the others "same" or "ragged" (ctx / 16 to ctx)
  Hq, Hkv, D  query heads, key heads, channels of a head
  page        tokens of a page
  inp, cache  type of q, k, v and of the cache ("fp8": E4M3 with a scale per key head)
  order       the cache's memory: "nhd" [page, token, head, channel] or "hnd" [page, head, token, channel]
  rot, inter  append: channels of a head that are rotated, and whether pairs are neighbours (else: the halves)
  window      attention: keys that a query sees at most (0: all before it)
  cap, bias   attention: the cap of the scores (0: none), whether the distance counts
  mask        attention: "causal"; "docs" (several documents in a row, each blind to those before it, some rows of padding at the end); "prefix" (the
              first part of a sequence is seen by all of its rows)
  lse         attention: the logarithm of the softmax' sum is asked for too
"""
import math
import random

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
WORKSPACE = 64 << 20
EPS = 1e-6


def _norm(name, M, K, inp, form, res):
    return {"name": name, "op": "norm", "M": M, "K": K, "inp": inp, "form": form, "res": res}


def _append(name, B, n, mix, ctx, fill, Hq, Hkv, D, page, inp, cache, order, rot, inter):
    return {"name": name, "op": "append", "B": B, "n": n, "mix": mix, "ctx": ctx, "fill": fill, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page,
            "inp": inp, "cache": cache, "order": order, "rot": rot, "inter": inter}


def _attention(name, B, n, mix, ctx, fill, Hq, Hkv, D, page, inp, cache, order, window=0, cap=0.0, bias=False, mask="causal", lse=False):
    return {"name": name, "op": "attention", "B": B, "n": n, "mix": mix, "ctx": ctx, "fill": fill, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page,
            "inp": inp, "cache": cache, "order": order, "window": window, "cap": cap, "bias": bias, "mask": mask, "lse": lse}


def listed():
    return [
        # one token of one user before the fused q/k/v projection of the benchmark's block: latency
        _norm("norm_one", 1, 4096, "bf16", "a8", True),
        # a decode batch in the 4-bit block format, a wider model
        _norm("norm_decode_b48_mx", 48, 8192, "bf16", "mx", True),
        # a ragged chunk at a first layer (nothing to add), an odd width, 4-bit codes with a zero point
        _norm("norm_chunk_asym4", 777, 2624, "fp16", "asym4", False),
        # whole prompts of several users
        _norm("norm_prompts", 16384, 4096, "bf16", "a8", True),
        # one token of one user, 32 + 8 + 8 heads of 128: latency
        _append("append_one", 1, 1, "same", 1000, "same", 32, 8, 128, 64, "bf16", "bf16", "nhd", 128, False),
        # a decode batch with an 8-bit cache, a small fp16 model, part of a head rotated, neighbouring pairs
        _append("append_decode_b60_fp8", 60, 1, "ragged", 6000, "ragged", 16, 4, 64, 32, "fp16", "fp8", "hnd", 32, True),
        # whole prompts of several users
        _append("append_prompts", 6, 4096, "ragged", 0, "same", 32, 8, 128, 64, "bf16", "bf16", "hnd", 128, False),
        # a decode batch of users at different points, capped scores
        _attention("cap_decode_b40", 40, 1, "ragged", 8000, "ragged", 32, 8, 128, 64, "bf16", "bf16", "hnd", cap=50.0),
        # one token of one user, a very long document, a bias by distance, no shared heads
        _attention("bias_decode_long", 1, 1, "same", 65000, "same", 16, 16, 64, 64, "fp16", "fp16", "nhd", bias=True),
        # prompts put together from several documents, padded at the end
        _attention("docs_prompts", 2, 6000, "same", 0, "same", 32, 8, 128, 64, "bf16", "bf16", "hnd", mask="docs", lse=True),
        # a chunk of a sequence with a prefix that is seen both ways, beside seven users' decoding and an empty slot, 8-bit cache
        _attention("prefix_mixed_b9_fp8", 9, 700, "ones", 2500, "ragged", 32, 8, 128, 64, "bf16", "fp8", "hnd", mask="prefix"),
        # a whole prompt with capped scores, the largest case
        _attention("cap_prompt_8192", 1, 8192, "same", 0, "same", 32, 8, 128, 64, "bf16", "bf16", "hnd", cap=30.0),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _lengths(case):
    """(new tokens, keys in the cache with them) of each sequence: part of the case, so that its work is known without a seed."""
    B, n, ctx = case["B"], case["n"], case["ctx"]
    rng = random.Random(1000003 * B + 1009 * n + ctx)
    got = []
    for b in range(B):
        new = n if b == 0 or case["mix"] == "same" else 1 if case["mix"] == "ones" else rng.randint(1, n)
        old = ctx if b == 0 or case["fill"] == "same" or ctx == 0 else round(_log(rng, max(1, ctx / 16), ctx))
        got.append((new, old + new))
    if B >= 8 and case["mix"] != "same":
        got[-1] = (0, 0)
    return got


def _ranges(case):
    """What the mask says of every new token, by sequence: it sees from <= j < to, before the window is looked at."""
    rng = random.Random(7919 * case["B"] + 104729 * case["n"] + case["ctx"])
    got = []
    for n, L in _lengths(case):
        p = np.arange(L - n, L)
        frm, to = np.zeros(n, np.int64), p + 1
        if case["mask"] == "docs":
            starts = [0]
            while starts[-1] < L:
                starts.append(starts[-1] + round(_log(rng, 16, 2048)))
            frm = np.array(starts)[np.searchsorted(starts, p, side="right") - 1]
            to = np.where(np.arange(n) >= n - n // 32, 0, to)
        elif case["mask"] == "prefix":
            to = np.maximum(to, min(L, round(L * rng.uniform(0.1, 0.9))))
        got.append((p, frm, to))
    return got


def work(case):
    if case["op"] == "norm":
        M, K = case["M"], case["K"]
        code = {"a8": 1, "a4": 0.5, "asym8": 1, "asym4": 0.5, "mx": 0.5 + 1 / 32}[case["form"]]
        es = 4 if case["inp"] == "fp32" else 2
        return {"bytes": round(M * K * (es * (3 if case["res"] else 1) + code) + 4 * K + 8 * M), "flops": 6 * M * K}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    ec = 1 if case["cache"] == "fp8" else 2
    T = sum(n for n, _ in _lengths(case))
    if case["op"] == "append":
        return {"bytes": T * ((Hq + 2 * Hkv) * D * 2 + Hq * D * 2 + 2 * Hkv * D * ec + case["rot"] * 4) + 8 * D,
                "flops": T * (Hq + Hkv) * (case["rot"] * 3 + 4 * D)}
    read = seen = 0
    for p, frm, to in _ranges(case):
        if case["window"]:
            frm = np.maximum(frm, p - case["window"] + 1)
        some = to > frm
        seen += int((to - frm)[some].sum())
        if some.any():                                   # keys that any row sees
            lo, hi = frm[some], to[some]
            mark = np.zeros(int(hi.max()) + 1, np.int64)
            np.add.at(mark, lo, 1)
            np.add.at(mark, hi, -1)
            read += int((np.cumsum(mark) > 0).sum())
    more = 0 if case["mask"] == "causal" else 8
    return {"bytes": T * Hq * (2 * D * 2 + (4 if case["lse"] else 0)) + T * more + read * 2 * Hkv * D * ec, "flops": 4 * D * Hq * seen}


def _heads(rng):
    while True:
        Hkv = rng.choice([1, 2, 4, 8, 8, 8, 16, 32])
        Hq = Hkv * rng.choice([1, 2, 3, 4, 4, 4, 7, 8])
        if Hq <= 64:
            return Hq, Hkv


def draw(rng):
    op = rng.choice(["norm", "append", "attention", "attention"])
    most = {c["op"]: work(c) for c in listed() if c["name"] in ("norm_prompts", "append_prompts", "cap_prompt_8192")}[op]
    while True:
        if op == "norm":
            K = 64 * round(_log(rng, 4, 256))
            case = _norm("", max(1, round(_log(rng, 1, 16384))), K, rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                         rng.choice(["a8", "a8", "a4", "asym8", "asym4", "mx"]), rng.random() < 0.75)
            if work(case)["bytes"] <= most["bytes"]:
                del case["name"]
                return case
            continue
        kind = rng.choice(["one", "few", "chunk", "prompts", "mixed"])
        B = max(1, round(_log(rng, 1, 64 if kind in ("one", "few") else 8)))
        n = {"one": 1, "few": rng.randint(2, 8)}.get(kind) or round(_log(rng, 9, 8192))
        ctx = 0 if kind == "prompts" else round(_log(rng, 1, 65000))
        mix = "ones" if kind == "mixed" else rng.choice(["same", "ragged"])
        Hq, Hkv = _heads(rng)
        D, page, inp = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128, 256]), rng.choice(["bf16", "bf16", "fp16"])
        cache, order, fill = rng.choice([inp, inp, "fp8"]), rng.choice(["nhd", "hnd"]), rng.choice(["same", "ragged"])
        if op == "append":
            case = _append("", B, n, mix, min(ctx, 32000), fill, Hq, Hkv, D, page, inp, cache, order, rng.choice([D, D, D // 2]),
                           rng.random() < 0.4)
        else:
            window, mask = rng.choice([0, 0, 0, round(_log(rng, 16, 8192))]), rng.choice(["causal", "causal", "docs", "prefix"])
            what = rng.choice(["cap", "cap", "bias", "bias", ""]) if mask == "causal" else rng.choice(["cap", "bias", "", ""])
            if mask == "causal" and not what:
                continue                                 # (the plain attention)
            case = _attention("", B, n, mix, ctx, fill, Hq, Hkv, D, page, inp, cache, order, window,
                              rng.choice([15.0, 30.0, 50.0]) if what == "cap" else 0.0, what == "bias", mask, rng.random() < 0.3)
        longest = ctx + n
        cells = B * longest * (Hq * n if op == "attention" else 0)
        held = 4 * B * longest * Hkv * D                 # K and V of all sequences, at their longest, in 16 bits
        if cells > 8192 * 8192 * 32 or held > 2 << 30:
            continue
        w = work(case)
        if w["flops"] <= most["flops"] if op == "attention" else w["bytes"] <= most["bytes"]:
            del case["name"]
            return case


# ---- what a server holds ------------------------------------------------------------------------------------------------------------
def _random(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    def uniform(n, lo, hi):
        return torch.rand(n, generator=gen, device="cuda", dtype=torch.float32) * (hi - lo) + lo
    return gen, normal, uniform


def _code_bytes(case):
    return case["M"] * case["K"] * (8 if case["form"] in ("a8", "asym8") else 4) // 8


def _prepare_norm(case, seed):
    gen, normal, uniform = _random(seed)
    M, K, dt = case["M"], case["K"], DT[case["inp"]]
    loud = torch.ones(K, device="cuda")                  # a few channels of the stream are far larger than the others
    loud[torch.randint(0, K, (max(1, K // 100),), generator=gen, device="cuda")] = 30.0
    st = {"case": case, "x": (normal(M, K) * (1.0 if case["res"] else loud)).to(dt), "residual": (normal(M, K) * loud).to(dt) if case["res"] else None,
          "h": torch.empty((M, K), dtype=dt, device="cuda") if case["res"] else None,
          # the norm's weight over the flattening factor, which is larger where the channel is
          "gain": uniform(K, 0.5, 1.5) / (uniform(K, 0.5, 2.0) * loud.sqrt()),
          "codes": torch.empty(_code_bytes(case), dtype=torch.uint8, device="cuda")}
    if case["form"] == "mx":
        st["scale"] = torch.empty(-(-K // 256) * (M + M % 2) * 8, dtype=torch.uint8, device="cuda")
    else:
        st["scale"] = torch.empty(M, dtype=torch.float32, device="cuda")
    if case["form"] in ("asym8", "asym4"):
        st["zero"] = torch.empty(M, dtype=torch.int32, device="cuda")
    return st


def prepare(case, seed):
    if case["op"] == "norm":
        return _prepare_norm(case, seed)
    gen, normal, uniform = _random(seed)
    dev = "cuda"
    B, Hq, Hkv, D, P = (case[k] for k in ("B", "Hq", "Hkv", "D", "page"))
    dt = DT[case["inp"]]
    lens = _lengths(case)
    T = sum(n for n, _ in lens)
    longest = max(L for _, L in lens)

    # every sequence's pages, scattered over a pool that holds some pages of others too
    need = [-(-L // P) for _, L in lens]
    pages = sum(need) + 3
    where = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)
    width = max(need)
    first = torch.tensor([sum(need[:b]) for b in range(B)], device=dev)
    has = torch.tensor(need, device=dev)
    col = torch.arange(width, device=dev)
    table = torch.where(col < has[:, None], where[(first[:, None] + col).clamp(max=pages - 1)], torch.zeros((), dtype=torch.int32, device=dev)).contiguous()
    cu = torch.tensor([sum(n for n, _ in lens[:b]) for b in range(B + 1)], dtype=torch.int32, device=dev)
    kv_len = torch.tensor([L for _, L in lens], dtype=torch.int32, device=dev)

    # keys have a few channels that are larger than the others
    loud = torch.ones((Hkv, 1, D), device=dev)
    loud.scatter_(2, torch.randint(0, D, (Hkv, 1, 2), generator=gen, device=dev), 4.0)
    st = {"case": case, "table": table, "cu": cu, "kv_len": kv_len, "max_q": max(n for n, _ in lens), "max_kv": longest,
          "k_scale": None, "v_scale": None}
    if case["cache"] == "fp8":
        st["k_scale"], st["v_scale"] = uniform(Hkv, 0.04, 0.06), uniform(Hkv, 0.012, 0.02)

    def pool(mult, scale):
        x = normal(pages, Hkv, P, D)
        if mult is not None:
            x.mul_(mult)
        x = (x / scale[:, None, None]).clamp_(-448, 448).to(torch.float8_e4m3fn) if scale is not None else x.to(dt)
        return x.transpose(1, 2) if case["order"] == "hnd" else x.transpose(1, 2).contiguous()    # [pages, P, Hkv, D]

    st["K"], st["V"] = pool(loud, st["k_scale"]), pool(None, st["v_scale"])
    qkv = normal(T, (Hq + 2 * Hkv) * D)                  # the projection's output: q, k and v side by side
    qkv[:, Hq * D:(Hq + Hkv) * D] *= loud.reshape(-1)
    if case["op"] == "append":
        qkv *= torch.exp(normal(T, 1))                   # what the norms take out again
    qkv = qkv.to(dt)
    q = qkv[:, :Hq * D].view(T, Hq, D)
    if case["op"] == "append":
        st["q"], st["k"], st["v"] = q, qkv[:, Hq * D:(Hq + Hkv) * D].view(T, Hkv, D), qkv[:, (Hq + Hkv) * D:].view(T, Hkv, D)
        st["q_norm"], st["k_norm"] = uniform(D, 0.5, 1.5), uniform(D, 0.5, 1.5)
        half = case["rot"] // 2
        angle = torch.arange(longest, device=dev, dtype=torch.float64)[:, None] * (
            500000.0 ** (-torch.arange(half, device=dev, dtype=torch.float64) / half))
        st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
        st["q_out"] = torch.empty((T, Hq, D), dtype=dt, device=dev)
        return st
    st["q"] = q.contiguous()
    st["out"] = torch.empty((T, Hq, D), dtype=dt, device=dev)
    st["lse"] = torch.empty((T, Hq), dtype=torch.float32, device=dev) if case["lse"] else None
    st["ws"] = torch.zeros(WORKSPACE, dtype=torch.uint8, device=dev)
    st["slopes"] = 2.0 ** (-8.0 * (torch.arange(Hq, device=dev) + 1) / Hq) if case["bias"] else None
    st["see_from"] = st["see_to"] = None
    if case["mask"] != "causal":
        ranges = _ranges(case)
        st["see_to"] = torch.from_numpy(np.concatenate([to for _, _, to in ranges]).astype(np.int32)).to(dev)
        if case["mask"] == "docs":
            st["see_from"] = torch.from_numpy(np.concatenate([frm for _, frm, _ in ranges]).astype(np.int32)).to(dev)
    return st


# ---- the plain forms ---------------------------------------------------------------------------------------------------------------
def _nibbles(c):
    """4-bit codes [M, K] as the layers take them: of 8 channels, byte j has channel j below and channel 4 + j above."""
    c = c.to(torch.uint8).bitwise_and_(15).view(c.shape[0], -1, 2, 4)
    return (c[:, :, 0] | (c[:, :, 1] << 4)).reshape(-1)


def _packed(c, bits):
    return c.to(torch.int8).view(c.shape[0], -1) if bits == 8 else _nibbles(c.to(torch.int8))


def _e2m1(t):
    a = t.abs()
    i = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int())
    return torch.where((t < 0) & (i > 0), i + 8, i)


def _plain_norm(st):
    """The codes of the sum times the gain do not hang on the norm, which goes into the token's scale; MXFP4's scales are powers of two, so there it
    goes into the values.  (The codes come back as the layers take them.  Each is defined to the bit, so both sides have to have the same bytes.)"""
    case, x = st["case"], st["x"]
    M, K, form = case["M"], case["K"], case["form"]
    h = (x.float() + st["residual"].float()).to(x.dtype) if case["res"] else x
    rstd = (1.0 / (h.double().square().mean(1) + EPS).sqrt()).float()
    u = h.float() * st["gain"]
    one = torch.ones((), device="cuda")
    out = {"h": h} if case["res"] else {}
    if form == "mx":
        v = (u * rstd[:, None]).view(M, K // 32, 32)
        amax = v.abs().amax(-1)
        E = torch.where(amax > 0, (torch.frexp(amax).exponent - 3).clamp(min=-127) + 127, torch.full((), 127, dtype=torch.int32, device="cuda"))
        code = _e2m1(torch.ldexp(v, (127 - E)[:, :, None])).view(M, K)
        tiles = -(-K // 256)
        scale = torch.full((M + M % 2, tiles * 8), 127, dtype=torch.uint8, device="cuda")
        scale[:M, :K // 32] = E.to(torch.uint8)
        return out | {"codes": _nibbles(code), "scale": scale.view(-1, tiles, 8).transpose(0, 1).reshape(-1)}
    if form in ("a8", "a4"):
        bits = int(form[1])
        qmax = 2 ** (bits - 1) - 1
        amax = u.abs().amax(1)
        s = torch.where(amax > 0, amax / qmax, one)
        c = (u / s[:, None]).round().clamp(-qmax, qmax)
        return out | {"codes": _packed(c, bits), "scale": torch.where(amax > 0, s * rstd, one)}
    bits = int(form[4])
    lo, hi = u.amin(1).clamp(max=0), u.amax(1).clamp(min=0)
    s = torch.where(hi > lo, (hi - lo) / (2 ** bits - 1), one)
    z = (-lo / s).round()
    c = ((u / s[:, None]).round() + z[:, None]).clamp(0, 2 ** bits - 1) - 2 ** (bits - 1)
    return out | {"codes": _packed(c, bits), "scale": torch.where(hi > lo, s * rstd, one), "zero": z.int() - 2 ** (bits - 1)}


def _place(st, T):
    """Sequence of every new token, its number in it, its position."""
    t = torch.arange(T, device="cuda")
    b = torch.bucketize(t, st["cu"][1:].long(), right=True)
    i = t - st["cu"].long()[b]
    n = (st["cu"][1:] - st["cu"][:-1]).long()
    return b, i, (st["kv_len"].long() - n)[b] + i


def _rotated(x, c, s, rot, inter):
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * c - b * s, b * c + a * s
    r = torch.stack((u, v), -1).flatten(-2) if inter else torch.cat((u, v), -1)
    return torch.cat((r, x[..., rot:]), -1)


def _normed(x, w):
    x = x.float()
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w


def _store(cache, page, row, x, scale):
    if scale is None:
        cache[page, row] = x.to(cache.dtype)
    else:
        cache.view(torch.uint8)[page, row] = (x / scale[:, None]).clamp(-448, 448).to(cache.dtype).view(torch.uint8)


def _plain_append(st):
    case = st["case"]
    b, _, pos = _place(st, st["q"].shape[0])
    page, row = st["table"][b, pos // case["page"]].long(), pos % case["page"]
    c, s = st["cos"][pos][:, None, :], st["sin"][pos][:, None, :]
    _store(st["K"], page, row, _rotated(_normed(st["k"], st["k_norm"]), c, s, case["rot"], case["inter"]), st["k_scale"])
    _store(st["V"], page, row, st["v"].float(), st["v_scale"])
    q = _rotated(_normed(st["q"], st["q_norm"]), c, s, case["rot"], case["inter"]).to(st["q"].dtype)
    return {"q": q, "K": st["K"], "V": st["V"]}


def _gathered(cache, page, row, live, scale):
    x = cache[page, row] if scale is None else cache.view(torch.uint8)[page, row].view(cache.dtype)
    x = x.float() if scale is None else x.float() * scale[:, None]
    return torch.where(live, x, torch.zeros((), device="cuda"))


def _plain_attention(st):
    case, q = st["case"], st["q"]
    T, Hq, D = q.shape
    B, Hkv, P, W = case["B"], case["Hkv"], case["page"], case["window"]
    G, n, S = Hq // Hkv, st["max_q"], st["max_kv"]
    zero = torch.zeros((), device="cuda")
    b, i, _ = _place(st, T)
    j = torch.arange(S, device="cuda")
    length = st["kv_len"].long()[:, None]
    new = (st["cu"][1:] - st["cu"][:-1]).long()[:, None]
    page, row, live = st["table"][:, j // P].long(), j % P, (j < length)[:, :, None, None]
    K = _gathered(st["K"], page, row, live, st["k_scale"])                     # [B, S, Hkv, D]
    V = _gathered(st["V"], page, row, live, st["v_scale"])
    rows = (st["cu"][:-1].long()[:, None] + torch.arange(n, device="cuda")).clamp(max=T - 1)
    Q = q.float()[rows].view(B, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, D)
    A = torch.matmul(Q, K.permute(0, 2, 3, 1)).mul_(1.0 / math.sqrt(D)).view(B, Hkv, G, n, S)
    at = (length - new + torch.arange(n, device="cuda"))[:, :, None]            # [B, n, 1]: positions
    if case["cap"]:
        A.div_(case["cap"]).tanh_().mul_(case["cap"])
    if case["bias"]:
        A.sub_(st["slopes"].view(Hkv, G, 1, 1) * (at - j).abs().float()[:, None, None])
    sees = (j < (at + 1 if st["see_to"] is None else st["see_to"].long()[rows][:, :, None])) & (j < length[:, :, None])
    if st["see_from"] is not None:
        sees &= j >= st["see_from"].long()[rows][:, :, None]
    if W:
        sees &= j > at - W
    A.masked_fill_(~sees[:, None, None], -math.inf)
    m = A.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, zero, m)
    E = A.sub_(m).exp_()
    total = E.sum(-1, keepdim=True)
    O = torch.matmul(E.view(B, Hkv, G * n, S), V.permute(0, 2, 1, 3)).view(B, Hkv, G, n, D)
    O = torch.where(total > 0, O / total, zero)
    out = {"out": O.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D)[b, i].to(q.dtype)}
    if case["lse"]:
        out["lse"] = (m + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(B, n, Hq)[b, i]
    return out


def _own(st):
    from paper_2603_08185_amd import binding as serq
    case = st["case"]
    if case["op"] == "norm":
        form, out = case["form"], {"h": st["h"]} if case["res"] else {}
        if form == "mx":
            serq.mx_rmsnorm_quantize_act(st["x"], st["gain"], EPS, residual=st["residual"], h=st["h"], Xq=st["codes"], xsc=st["scale"])
        elif form in ("a8", "a4"):
            serq.rmsnorm_quantize_act(st["x"], st["gain"], EPS, int(form[1]), residual=st["residual"], h=st["h"], Xq=st["codes"], scale=st["scale"])
        else:
            serq.rmsnorm_quantize_act_asym(st["x"], st["gain"], EPS, int(form[4]), residual=st["residual"], h=st["h"], Xq=st["codes"],
                                           scale=st["scale"], zero=st["zero"])
            out["zero"] = st["zero"]
        codes = st["codes"].view(torch.int8).view(case["M"], case["K"]) if form in ("a8", "asym8") else st["codes"]
        return out | {"codes": codes, "scale": st["scale"]}
    if case["op"] == "append":
        serq.kv_append(st["q"], st["k"], st["v"], st["K"], st["V"], st["table"], st["cu"], st["kv_len"], st["cos"], st["sin"],
                       interleaved=case["inter"], k_scale=st["k_scale"], v_scale=st["v_scale"], q_out=st["q_out"], q_norm=st["q_norm"],
                       k_norm=st["k_norm"], eps=EPS)
        return {"q": st["q_out"], "K": st["K"], "V": st["V"]}
    serq.paged_attention(st["q"], st["K"], st["V"], st["table"], st["cu"], st["kv_len"], st["max_q"], st["max_kv"], window=case["window"],
                         k_scale=st["k_scale"], v_scale=st["v_scale"], out=st["out"], lse=st["lse"], ws=st["ws"], cap=case["cap"],
                         slopes=st["slopes"], see_from=st["see_from"], see_to=st["see_to"])
    return {"out": st["out"], "lse": st["lse"]} if case["lse"] else {"out": st["out"]}


def run(st):
    if own:
        return _own(st)
    return {"norm": _plain_norm, "append": _plain_append, "attention": _plain_attention}[st["case"]["op"]](st)


# ---- from the definition, in 64 bits, one sequence at a time ---------------------------------------------------------------------------
def _exact_norm(st):
    """The sum and the tokens' scales; codes are whole numbers, whose neighbours' border 64 bits would draw elsewhere than the definition's 32 do."""
    case = st["case"]
    x, gain = st["x"].double(), st["gain"].double()
    total = x + st["residual"].double() if case["res"] else x
    h = total.to(st["x"].dtype).double()                 # what the norm is of: the stream as it is stored
    got = {"h": total} if case["res"] else {}
    got |= {"codes": None, "scale": None}
    if case["form"] == "mx":
        return got
    y = h * gain / (torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / case["K"] + EPS) ** 0.5
    if case["form"] in ("a8", "a4"):
        top = y.abs().max(1).values / (127 if case["form"] == "a8" else 7)
    else:
        got["zero"] = None
        top = (y.max(1).values.clamp(min=0) - y.min(1).values.clamp(max=0)) / (255 if case["form"] == "asym8" else 15)
    got["scale"] = torch.where(top > 0, top, torch.ones_like(top))
    return got


def _slots(st, b, positions):
    p = torch.as_tensor(positions, device="cuda", dtype=torch.long)
    return st["table"][b].long()[p // st["case"]["page"]], p % st["case"]["page"]


def _exact_append(st, lens):
    case, R = st["case"], st["case"]["rot"]
    K, V = (x.to(torch.float32).double() for x in (st["K"], st["V"]))
    v = st["v"].double()
    q, k = (x.double() / (torch.linalg.vector_norm(x.double(), dim=-1, keepdim=True) ** 2 / case["D"] + EPS) ** 0.5 * w.double()
            for x, w in ((st["q"], st["q_norm"]), (st["k"], st["k_norm"])))
    cos, sin = st["cos"].double(), st["sin"].double()
    pairs = [(2 * f, 2 * f + 1) if case["inter"] else (f, f + R // 2) for f in range(R // 2)]
    first, second = [a for a, _ in pairs], [a for _, a in pairs]
    t = 0
    for b, (n, L) in enumerate(lens):
        if n == 0:
            continue
        c, s = cos[L - n:L].unsqueeze(1), sin[L - n:L].unsqueeze(1)
        for x in (q, k):
            part = x[t:t + n]
            x0, x1 = part[:, :, first].clone(), part[:, :, second].clone()
            part[:, :, first] = x0 * c - x1 * s
            part[:, :, second] = x1 * c + x0 * s
        page, row = _slots(st, b, range(L - n, L))
        for cache, new, scale in ((K, k, st["k_scale"]), (V, v, st["v_scale"])):
            new = new[t:t + n]
            cache[page, row] = new if scale is None else torch.clamp(new / scale.double().view(-1, 1), -448, 448)
        t += n
    return {"q": q, "K": K, "V": V}


def _exact_attention(st, lens):
    case = st["case"]
    T, Hq, D = st["q"].shape
    G = Hq // case["Hkv"]
    out = torch.zeros((T, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device="cuda")
    ranges = _ranges(case)
    t = 0
    for b, (n, L) in enumerate(lens):
        if n == 0:
            continue
        page, row = _slots(st, b, range(L))
        key = torch.arange(L, device="cuda")
        for h in range(case["Hkv"]):
            K, V = (x[:, :, h][page, row] if s is None else x.view(torch.uint8)[:, :, h][page, row].view(x.dtype) for x, s in (
                (st["K"], st["k_scale"]), (st["V"], st["v_scale"])))
            K, V = K.to(torch.float32).double(), V.to(torch.float32).double()
            if st["k_scale"] is not None:
                K, V = K * st["k_scale"][h].double(), V * st["v_scale"][h].double()
            heads = slice(h * G, (h + 1) * G)
            for i0 in range(0, n, 2048):
                i1 = min(n, i0 + 2048)
                p, frm, to = (torch.from_numpy(np.ascontiguousarray(x[i0:i1])).to("cuda")[:, None, None] for x in ranges[b])
                Q = st["q"][t + i0:t + i1, heads].double()                      # [i, G, D]
                A = (Q.reshape(-1, D) @ K.T.contiguous()).view(i1 - i0, G, L) / math.sqrt(D)
                if case["cap"]:
                    A = case["cap"] * torch.tanh(A / case["cap"])
                if case["bias"]:
                    A = A - st["slopes"][heads].double().view(1, G, 1) * (p - key).abs()
                hidden = (key < frm) | (key >= to)
                if case["window"]:
                    hidden = hidden | (key <= p - case["window"])
                A = A.masked_fill(hidden, -math.inf)
                total = torch.logsumexp(A, -1)
                lse[t + i0:t + i1, heads] = total
                A = torch.exp(A - torch.where(total == -math.inf, torch.zeros_like(total), total)[:, :, None])
                out[t + i0:t + i1, heads] = (A.reshape(-1, L) @ V).view(i1 - i0, G, D)
        t += n
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(st)
    lens = _lengths(case)
    return _exact_append(st, lens) if case["op"] == "append" else _exact_attention(st, lens)
