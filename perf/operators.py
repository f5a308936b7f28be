"""The work by which the cache operators are judged: what lies between the q/k/v projection and the o projection of a decoder block.

A pass is one call that a model server makes for one layer and one batch of new tokens: `kv_append` (rotate q and k by their positions, put k
and v into the paged cache) or `paged_attention` (the new tokens' queries over the cache).  The cache, the page table and the lengths of the
sequences, the rotation's table, the output buffers and the workspace are what such a program keeps.

A case:
  op          "append" or "attention"
  B, n, mix   sequences, new tokens of the first one, and how many the others have: "same" (n each), "ragged" (1 to n), "ones" (1 each, a
              chunk that rides along with decoding).  In a batch of 8 or more that is not "same" the last sequence is an empty slot.
  ctx, fill   keys that the cache holds before the call: ctx for the first sequence, for the others "same" or "ragged" (ctx / 16 to ctx)
  Hq, Hkv, D  query heads, key heads, channels of a head
  page        tokens of a page
  inp, cache  type of q, k, v and of the cache ("fp8": E4M3 with a scale per key head)
  order       the cache's memory: "nhd" [page, token, head, channel] or "hnd" [page, head, token, channel]
  rot, inter  append: channels of a head that are rotated, and whether pairs are neighbours (else: the halves)
  window      attention: keys that a query sees at most (0: all before it)
  lse         attention: the logarithm of the softmax' sum is asked for too
"""
import math
import random

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
WORKSPACE = 64 << 20


def _append(name, B, n, mix, ctx, fill, Hq, Hkv, D, page, inp, cache, order, rot, inter):
    return {"name": name, "op": "append", "B": B, "n": n, "mix": mix, "ctx": ctx, "fill": fill, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page,
            "inp": inp, "cache": cache, "order": order, "rot": rot, "inter": inter}


def _attention(name, B, n, mix, ctx, fill, Hq, Hkv, D, page, inp, cache, order, window=0, lse=False):
    return {"name": name, "op": "attention", "B": B, "n": n, "mix": mix, "ctx": ctx, "fill": fill, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page,
            "inp": inp, "cache": cache, "order": order, "window": window, "lse": lse}


def listed():
    return [
        # one token of one user, the fused q/k/v projection of the benchmark's block (6144 = 32 + 8 + 8 heads of 128): latency
        _append("append_one", 1, 1, "same", 1000, "same", 32, 8, 128, 64, "bf16", "bf16", "nhd", 128, False),
        # a decode batch with an 8-bit cache
        _append("append_decode_b48_fp8", 48, 1, "ragged", 8000, "ragged", 32, 8, 128, 32, "bf16", "fp8", "hnd", 128, False),
        # a ragged chunk of a small fp16 model without shared heads, part of a head rotated, neighbouring pairs, short pages
        _append("append_chunk_d64", 1, 777, "same", 500, "same", 32, 32, 64, 16, "fp16", "fp16", "nhd", 32, True),
        # whole prompts of several users
        _append("append_prompts", 6, 4096, "ragged", 0, "same", 32, 8, 128, 64, "bf16", "bf16", "hnd", 128, False),
        # one token of one user, a short conversation: latency
        _attention("decode_one", 1, 1, "same", 1000, "same", 32, 8, 128, 64, "bf16", "bf16", "nhd"),
        # one token of one user, a very long document: the cache's stream from one sequence
        _attention("decode_long", 1, 1, "same", 131000, "same", 32, 8, 128, 64, "bf16", "bf16", "hnd"),
        # a decode batch of users at different points
        _attention("decode_b48", 48, 1, "ragged", 8000, "ragged", 32, 8, 128, 16, "bf16", "bf16", "nhd"),
        # a decode batch with an 8-bit cache
        _attention("decode_b32_fp8", 32, 1, "ragged", 16000, "ragged", 32, 8, 128, 64, "bf16", "fp8", "hnd"),
        # five drafted tokens a sequence, a small fp16 model with a sliding window
        _attention("draft_b12_d64", 12, 5, "same", 4000, "ragged", 32, 4, 64, 32, "fp16", "fp16", "nhd", window=1024),
        # the next chunk of a long prompt
        _attention("chunk_512", 1, 512, "same", 32000, "same", 32, 8, 128, 64, "bf16", "bf16", "nhd"),
        # a chunk that rides along with seven users' decoding and an empty slot, 8-bit cache
        _attention("mixed_b9_fp8", 9, 384, "ones", 3500, "ragged", 32, 8, 128, 64, "bf16", "fp8", "hnd", lse=True),
        # a whole prompt, the largest case
        _attention("prompt_8192", 1, 8192, "same", 0, "same", 32, 8, 128, 64, "bf16", "bf16", "hnd"),
    ]


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


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _seen(n, length, window):
    """Keys that the n newest of `length` positions see, in all."""
    total = 0
    if n > 0:
        a, b = length - n + 1, length                    # visible keys of the first and the last token, without a window
        if not window:
            total = (a + b) * n // 2
        else:
            k = max(0, min(b, window) - a + 1)            # tokens whose window reaches back to the start
            total = (a + a + k - 1) * k // 2 + window * (n - k)
    return total


def work(case):
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    ec = 1 if case["cache"] == "fp8" else 2
    lens = _lengths(case)
    T = sum(n for n, _ in lens)
    if case["op"] == "append":
        return {"bytes": T * ((Hq + 2 * Hkv) * D * 2 + Hq * D * 2 + 2 * Hkv * D * ec + case["rot"] * 4),
                "flops": T * (Hq + Hkv) * case["rot"] * 3}
    W = case["window"]
    read = sum(min(L, W + n - 1) if W else L for n, L in lens if n)
    return {"bytes": T * Hq * (2 * D * 2 + (4 if case["lse"] else 0)) + read * 2 * Hkv * D * ec,
            "flops": 4 * D * Hq * sum(_seen(n, L, W) for n, L in lens)}


def _heads(rng):
    while True:
        Hkv = rng.choice([1, 2, 4, 8, 8, 8, 16, 32])
        Hq = Hkv * rng.choice([1, 2, 3, 4, 4, 4, 7, 8])
        if Hq <= 64:
            return Hq, Hkv


def draw(rng):
    op = rng.choice(["append", "attention", "attention"])
    most = {c["op"]: work(c) for c in listed() if c["name"] in ("append_prompts", "prompt_8192")}[op]
    stream = work(next(c for c in listed() if c["name"] == "decode_long"))["bytes"]
    while True:
        kind = rng.choice(["one", "few", "chunk", "prompts", "mixed"])
        B = max(1, round(_log(rng, 1, 64 if kind in ("one", "few") else 8)))
        n = {"one": 1, "few": rng.randint(2, 8)}.get(kind) or round(_log(rng, 9, 8192))
        ctx = 0 if kind == "prompts" else round(_log(rng, 1, 131000))
        mix = "ones" if kind == "mixed" else rng.choice(["same", "ragged"])
        Hq, Hkv = _heads(rng)
        D, page, inp = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128, 256]), rng.choice(["bf16", "bf16", "fp16"])
        cache, order, fill = rng.choice([inp, inp, "fp8"]), rng.choice(["nhd", "hnd"]), rng.choice(["same", "ragged"])
        if op == "append":
            case = _append("", B, n, mix, min(ctx, 32000), fill, Hq, Hkv, D, page, inp, cache, order, rng.choice([D, D, D // 2]),
                           rng.random() < 0.4)
        else:
            window = rng.choice([0, 0, 0, round(_log(rng, 16, 8192))])
            case = _attention("", B, n, mix, ctx, fill, Hq, Hkv, D, page, inp, cache, order, window, rng.random() < 0.3)
        w, longest = work(case), ctx + n
        cells = B * longest * (Hq * n if op == "attention" else 0)
        held = 4 * B * longest * Hkv * D                 # K and V of all sequences, at their longest, in 16 bits
        if cells <= 8192 * 8192 * 32 and held <= 2 << 30 and (
                w["bytes"] <= stream and w["flops"] <= most["flops"] if op == "attention" else w["bytes"] <= most["bytes"]):
            del case["name"]
            return case


def prepare(case, seed):
    """What a server holds for a layer and a batch: the cache, the sequences' pages and lengths, the new tokens' q, k and v, the buffers."""
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    B, Hq, Hkv, D, P = (case[k] for k in ("B", "Hq", "Hkv", "D", "page"))
    dt = DT[case["inp"]]
    lens = _lengths(case)
    T = sum(n for n, _ in lens)
    longest = max(L for _, L in lens)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32)

    def uniform(n, lo, hi):
        return torch.rand(n, generator=gen, device=dev, dtype=torch.float32) * (hi - lo) + lo

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
    qkv = qkv.to(dt)
    q = qkv[:, :Hq * D].view(T, Hq, D)
    if case["op"] == "append":
        st["q"], st["k"], st["v"] = q, qkv[:, Hq * D:(Hq + Hkv) * D].view(T, Hkv, D), qkv[:, (Hq + Hkv) * D:].view(T, Hkv, D)
        half = case["rot"] // 2
        angle = torch.arange(longest, device=dev, dtype=torch.float64)[:, None] * (
            500000.0 ** (-torch.arange(half, device=dev, dtype=torch.float64) / half))
        st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
        st["q_out"] = torch.empty((T, Hq, D), dtype=dt, device=dev)
    else:
        st["q"] = q.contiguous()
        st["out"] = torch.empty((T, Hq, D), dtype=dt, device=dev)
        st["lse"] = torch.empty((T, Hq), dtype=torch.float32, device=dev) if case["lse"] else None
        st["ws"] = torch.zeros(WORKSPACE, dtype=torch.uint8, device=dev)
    return st


# ---- the plain forms ---------------------------------------------------------------------------------------------------------------
def _place(st, T):
    """Sequence of every new token, its number in it, its position."""
    t = torch.arange(T, device="cuda")
    b = torch.bucketize(t, st["cu"][1:].long(), right=True)
    i = t - st["cu"].long()[b]
    n = (st["cu"][1:] - st["cu"][:-1]).long()
    return b, i, (st["kv_len"].long() - n)[b] + i


def _rotated(x, c, s, rot, inter):
    x = x.float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * c - b * s, b * c + a * s
    r = torch.stack((u, v), -1).flatten(-2) if inter else torch.cat((u, v), -1)
    return torch.cat((r, x[..., rot:]), -1)


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
    _store(st["K"], page, row, _rotated(st["k"], c, s, case["rot"], case["inter"]), st["k_scale"])
    _store(st["V"], page, row, st["v"].float(), st["v_scale"])
    q = _rotated(st["q"], c, s, case["rot"], case["inter"]).to(st["q"].dtype)
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
    sees = (j <= at) & (j < length[:, :, None])
    if W:
        sees &= j > at - W
    A.masked_fill_(~sees[:, None, None], -math.inf)
    m = A.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros((), device="cuda"), m)
    E = A.sub_(m).exp_()
    total = E.sum(-1, keepdim=True)
    O = torch.matmul(E.view(B, Hkv, G * n, S), V.permute(0, 2, 1, 3)).view(B, Hkv, G, n, D)
    O = torch.where(total > 0, O / total, torch.zeros((), device="cuda"))
    out = {"out": O.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D)[b, i].to(q.dtype)}
    if case["lse"]:
        out["lse"] = (m + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(B, n, Hq)[b, i]
    return out


def run(st):
    case = st["case"]
    if not own:
        return _plain_append(st) if case["op"] == "append" else _plain_attention(st)
    from paper_2603_08185_amd import binding as serq
    if case["op"] == "append":
        serq.kv_append(st["q"], st["k"], st["v"], st["K"], st["V"], st["table"], st["cu"], st["kv_len"], st["cos"], st["sin"],
                       interleaved=case["inter"], k_scale=st["k_scale"], v_scale=st["v_scale"], q_out=st["q_out"])
        return {"q": st["q_out"], "K": st["K"], "V": st["V"]}
    serq.paged_attention(st["q"], st["K"], st["V"], st["table"], st["cu"], st["kv_len"], st["max_q"], st["max_kv"], window=case["window"],
                         k_scale=st["k_scale"], v_scale=st["v_scale"], out=st["out"], lse=st["lse"], ws=st["ws"])
    return {"out": st["out"], "lse": st["lse"]} if case["lse"] else {"out": st["out"]}


# ---- from the definition, in 64 bits, one sequence at a time ---------------------------------------------------------------------------
def _slots(st, b, positions):
    p = torch.as_tensor(positions, device="cuda", dtype=torch.long)
    return st["table"][b].long()[p // st["case"]["page"]], p % st["case"]["page"]


def _exact_append(st, lens):
    case, R = st["case"], st["case"]["rot"]
    K, V = (x.to(torch.float32).double() for x in (st["K"], st["V"]))
    q = st["q"].double().clone()
    k, v = st["k"].double().clone(), st["v"].double()
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
    t = 0
    for b, (n, L) in enumerate(lens):
        if n == 0:
            continue
        page, row = _slots(st, b, range(L))
        for h in range(case["Hkv"]):
            K, V = (x[:, :, h][page, row] if s is None else x.view(torch.uint8)[:, :, h][page, row].view(x.dtype) for x, s in (
                (st["K"], st["k_scale"]), (st["V"], st["v_scale"])))
            K, V = K.to(torch.float32).double(), V.to(torch.float32).double()
            if st["k_scale"] is not None:
                K, V = K * st["k_scale"][h].double(), V * st["v_scale"][h].double()
            for i0 in range(0, n, 2048):
                i1 = min(n, i0 + 2048)
                heads = slice(h * G, (h + 1) * G)
                Q = st["q"][t + i0:t + i1, heads].double()                      # [i, G, D]
                A = (Q.reshape(-1, D) @ K.T.contiguous()).view(i1 - i0, G, L) / math.sqrt(D)
                p = torch.arange(L - n + i0, L - n + i1, device="cuda")[:, None, None]
                key = torch.arange(L, device="cuda")
                hidden = key > p
                if case["window"]:
                    hidden = hidden | (key <= p - case["window"])
                A = A.masked_fill(hidden, -math.inf)
                lse[t + i0:t + i1, heads] = torch.logsumexp(A, -1)
                A = torch.softmax(A, -1)
                out[t + i0:t + i1, heads] = (A.reshape(-1, L) @ V).view(i1 - i0, G, D)
        t += n
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def exact(case, seed):
    st = prepare(case, seed)
    lens = _lengths(case)
    return _exact_append(st, lens) if case["op"] == "append" else _exact_attention(st, lens)
