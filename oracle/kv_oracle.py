"""Plain NumPy oracle of the paged cache's operators, one sequence at a time: the rotation and append of keys and values, and the
attention over the cache, from their definitions in 64 bits (include/serq_kv.h states them)."""
from __future__ import annotations

import numpy as np


def rotate(x, cos, sin, rot, interleaved, dtype=np.float64):
    """x [T, H, D], cos / sin [T, rot/2]: every product and sum is one operation in `dtype`."""
    y = np.array(x, dtype=dtype)
    c, s = np.asarray(cos, dtype)[:, None, :], np.asarray(sin, dtype)[:, None, :]
    f = np.arange(rot // 2)
    i, j = (2 * f, 2 * f + 1) if interleaved else (f, f + rot // 2)
    a, b = y[..., i].copy(), y[..., j].copy()
    y[..., i] = a * c - b * s
    y[..., j] = b * c + a * s
    return y


def normed(x, weight, eps):
    """Every head of x [T, H, D] (fp32 values) by its root mean square: r = 1 / sqrt(mean x^2 + eps) formed in fp64 and rounded to fp32 (0 where the
    root is 0 or infinite), then two fp32 products."""
    x = np.asarray(x, np.float32)
    ms = (x.astype(np.float64) ** 2).sum(-1, keepdims=True) / x.shape[-1] + np.float64(np.float32(eps))
    with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
        r = np.minimum(np.where(ms == 0, 0.0, 1.0 / np.sqrt(ms)).astype(np.float32), np.finfo(np.float32).max)
    with np.errstate(invalid="ignore"):
        return (x * r).astype(np.float32) * np.asarray(weight, np.float32)


def positions(cu, kv_len, T):
    """(sequence, position) of the rows 0 .. T-1; sequence -1: a row of none."""
    seq, pos = np.full(T, -1), np.zeros(T, np.int64)
    for b, L in enumerate(kv_len):
        n = int(cu[b + 1] - cu[b])
        seq[cu[b]:cu[b + 1]] = b
        pos[cu[b]:cu[b + 1]] = np.arange(n) + int(L) - n
    return seq, pos


def slots(seq, pos, table, page_size, pages):
    """(page, row) of every position; page -1: it has none."""
    page = np.full(len(seq), -1)
    for t, (b, p) in enumerate(zip(seq, pos)):
        if b >= 0 and 0 <= p < table.shape[1] * page_size:
            g = int(table[b, p // page_size])
            page[t] = g if 0 <= g < pages else -1
    return page, np.asarray(pos) % page_size


def attention(q, K, V, scale, first, window=0):
    """One sequence: q [n, Hq, D] at positions first, first + 1, ...; K, V [L, H, D].  Returns out [n, Hq, D], lse [n, Hq] and, for
    error bounds, sum_j softmax_j |v_j| and the largest scale * sum_d |q_d k_d| a row meets."""
    n, Hq, D = q.shape
    L, H, _ = K.shape
    G = Hq // H
    out, mag = np.zeros((n, Hq, D)), np.zeros((n, Hq, D))
    lse, big = np.full((n, Hq), -np.inf), np.zeros((n, Hq))
    for i in range(n):
        p = first + i
        lo, hi = (max(0, p - window + 1) if window else 0), min(p + 1, L)
        if hi <= lo:
            continue
        x = q[i].reshape(H, G, D)
        k, v = K[lo:hi].transpose(1, 2, 0), V[lo:hi].transpose(1, 0, 2)        # [H, D, keys], [H, keys, D]
        s = scale * (x @ k)                                                  # [H, G, keys]
        m = s.max(-1, keepdims=True)
        e = np.exp(s - m)
        total = e.sum(-1, keepdims=True)
        lse[i] = (m + np.log(total)).reshape(Hq)
        out[i] = (e @ v / total).reshape(Hq, D)
        mag[i] = (e @ np.abs(v) / total).reshape(Hq, D)
        big[i] = scale * (np.abs(x) @ np.abs(k)).max(-1).reshape(Hq)
    return out, lse, mag, big


def attention_mod(q, K, V, scale, first, lo, hi, cap=0.0, slopes=None, rnd=2.0 ** -24):
    """One sequence: row i, at position first + i, sees the keys lo[i] <= j < hi[i]; scores cap tanh(s / cap), or s - slopes[h] |p - j|.  Returns
    out, lse, sum_j softmax_j |v_j| and two error bounds of what fp32 scores do: to out (sum_j p_j e_j |v_j| + sum_j p_j e_j sum_j p_j |v_j|)
    and to lse (sum_j p_j e_j), where e_j is the error of score j: (D + 8) rnd (scale sum_d |q_d k_d| + the bias), 3 rnd of the bias for its own products,
    and 12 rnd cap for a capped score (the reciprocal, the exponential, their arguments and the sum: 2.75 2^-22 cap)."""
    n, Hq, D = q.shape
    H = K.shape[1]
    G = Hq // H
    out, mag, eo = np.zeros((n, Hq, D)), np.zeros((n, Hq, D)), np.zeros((n, Hq, D))
    lse, el = np.full((n, Hq), -np.inf), np.zeros((n, Hq))
    sl = None if slopes is None else np.asarray(slopes, np.float64).reshape(H, G, 1)
    for i in range(n):
        a, b = int(lo[i]), int(hi[i])
        if b <= a:
            continue
        x = q[i].reshape(H, G, D)
        k, v = K[a:b].transpose(1, 2, 0), V[a:b].transpose(1, 0, 2)              # [H, D, keys], [H, keys, D]
        s = scale * (x @ k)                                                      # [H, G, keys]
        e = (D + 8) * rnd * scale * (np.abs(x) @ np.abs(k))
        if cap:
            s = cap * np.tanh(s / cap)
            e = e + 12 * rnd * cap
        if sl is not None:
            far = sl * np.abs(first + i - np.arange(a, b))
            s = s - far
            e = e + (D + 11) * rnd * np.abs(far)
        m = s.max(-1, keepdims=True)
        p = np.exp(s - m)
        total = p.sum(-1, keepdims=True)
        lse[i] = (m + np.log(total)).reshape(Hq)
        p = p / total
        off = (p * e).sum(-1, keepdims=True)
        out[i] = (p @ v).reshape(Hq, D)
        mag[i] = (p @ np.abs(v)).reshape(Hq, D)
        eo[i] = ((p * e) @ np.abs(v) + off * (p @ np.abs(v))).reshape(Hq, D)
        el[i] = off.reshape(Hq)
    return out, lse, mag, eo, el
