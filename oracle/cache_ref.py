"""A paged cache of keys and values in 64 bits, written from the formulas: the rotation by position, what an append stores, and attention of new tokens over what their sequences hold.
NumPy only; values come in as float64 arrays."""
from __future__ import annotations

import numpy as np


def tokens(seq_rows, lengths):
    """(row, sequence, position) of every new token."""
    for s in range(len(lengths)):
        n = int(seq_rows[s + 1]) - int(seq_rows[s])
        for i in range(n):
            yield int(seq_rows[s]) + i, s, int(lengths[s]) - n + i


def place(table, page, pages, s, p):
    """(page, slot) of position p of sequence s; None: it has none, or its page is no page."""
    if not 0 <= p < table.shape[1] * page:
        return None
    at = int(table[s, p // page])
    return (at, p % page) if 0 <= at < pages else None


def rotate(x, cos, sin, style):
    """x (heads, D) turned by R / 2 angles."""
    y, h = x.copy(), len(cos)
    a, b = (np.arange(h), np.arange(h) + h) if style == "halves" else (2 * np.arange(h), 2 * np.arange(h) + 1)
    y[:, a] = x[:, a] * cos - x[:, b] * sin
    y[:, b] = x[:, b] * cos + x[:, a] * sin
    return y


def append(q, k, v, angles, seq_rows, lengths, table, page, pages, style):
    """({row: rotated q}, {(page, slot): rotated k}, {(page, slot): v}) of the new tokens that have a place."""
    R = angles.shape[1]
    out, ks, vs = {}, {}, {}
    for t, s, p in tokens(seq_rows, lengths):
        if not 0 <= p < table.shape[1] * page:
            continue
        cos, sin = angles[p, :R // 2], angles[p, R // 2:]
        out[t] = rotate(q[t], cos, sin, style)
        at = place(table, page, pages, s, p)
        if at is not None:
            ks[at], vs[at] = rotate(k[t], cos, sin, style), v[t]
    return out, ks, vs


def attention(q, k_cache, v_cache, seq_rows, lengths, table, scale, causal=True, window=0):
    """(out, spread, reach) for q (T, heads, D) over caches (pages, slots, kv heads, D): out as defined (zeros where nothing is seen; rows of no sequence: NaN), spread = sum_j w_j |v_j| of the same
    shape, reach (T, heads) = the largest sum_d |q_d k_jd| scale of a seen key: what the rounding of terms and of scores is measured by; and the number of seen keys (T)."""
    T, Hq, D = q.shape
    pages, page, Hkv, _ = k_cache.shape
    out, spread = np.full(q.shape, np.nan), np.zeros(q.shape)
    reach, seen = np.zeros((T, Hq)), np.zeros(T, dtype=np.int64)
    for t, s, p in tokens(seq_rows, lengths):
        keys = [j for j in range(max(0, min(int(lengths[s]), table.shape[1] * page))) if (not causal or j <= p) and (not window or j > p - window)]
        at = [place(table, page, pages, s, j) for j in keys]
        at = [x for x in at if x is not None]
        out[t] = 0
        seen[t] = len(at)
        if not at:
            continue
        pg, sl = (np.array(x) for x in zip(*at))
        for h in range(Hq):
            K, V = k_cache[pg, sl, h // (Hq // Hkv)], v_cache[pg, sl, h // (Hq // Hkv)]
            x = K @ q[t, h] * scale
            w = np.exp(x - x.max())
            w /= w.sum()
            out[t, h], spread[t, h] = w @ V, w @ np.abs(V)
            reach[t, h] = (np.abs(K) @ np.abs(q[t, h])).max() * scale
    return out, spread, reach, seen
