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
