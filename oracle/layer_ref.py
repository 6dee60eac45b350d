"""What stands around the experts' products, in 64 bits, written from the formulas: root-mean-square norm, quantisation of 128 columns, routing,
rows in the experts' order, and the gradients of each.  NumPy only; values come in as float64 arrays."""
from __future__ import annotations

import numpy as np

E4M3_MAX = 448.0
F32_MAX = float(np.finfo(np.float32).max)


def rmsnorm(h, w, eps):
    """(y, rho) of rows h (T, H)."""
    rho = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    return h * rho * w, rho


def rmsnorm_backward(dy, h, w, eps, dsum=None):
    """(dx, dw)."""
    H = h.shape[1]
    rho = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    dx = np.zeros_like(h)
    for t in range(h.shape[0]):
        u = dy[t] * w
        dx[t] = rho[t] * u - rho[t] ** 3 * h[t] * (u @ h[t]) / H
    if dsum is not None:
        dx = dx + dsum
    return dx, (dy * h * rho).sum(0)


def scales(y, kind):
    """One scale per row and 128 columns, "f32" or "e8m0" (as values)."""
    T, H = y.shape
    out = np.ones((T, -(-H // 128)))
    for b in range(out.shape[1]):
        part = np.abs(y[:, 128 * b:128 * b + 128])
        most = np.where(np.isnan(part), 0.0, np.minimum(part, F32_MAX)).max(1)
        s = most / E4M3_MAX
        if kind == "e8m0":
            s = np.exp2(np.ceil(np.log2(np.where(s > 0, s, 1.0))))
        out[:, b] = np.where(most > 0, np.maximum(s, 2.0 ** -126), 1.0)
    return out


def spread(s, H):
    """Scales (T, blocks) as one per column."""
    return np.repeat(s, 128, axis=1)[:, :H]


def scores(logits, kind):
    x = np.where(np.isnan(logits), -np.inf, np.minimum(logits, F32_MAX))
    if kind == "sigmoid":
        with np.errstate(over="ignore"):
            return 1.0 / (1.0 + np.exp(-x))
    top = x.max(1, keepdims=True)
    e = np.exp(x - np.where(np.isneginf(top), 0.0, top))
    total = e.sum(1, keepdims=True)
    return e / np.where(total > 0, total, 1.0)


def choices(logits, kind, bias=None):
    """What experts are chosen by; -inf: masked."""
    x = np.where(np.isnan(logits), -np.inf, logits)
    c = scores(logits, kind) + (0.0 if bias is None else bias)
    return np.where(np.isneginf(x) | np.isnan(c), -np.inf, c)


def route(logits, k, kind="softmax", bias=None, groups=1, kept=1, top2=False, renorm=True, scale=1.0):
    """(ids, weights), row by row."""
    T, E = logits.shape
    s, c = scores(logits, kind), choices(logits, kind, bias)
    ids, w = np.full((T, k), -1, dtype=np.int64), np.zeros((T, k))
    per = E // groups
    for t in range(T):
        order_by = np.where(np.isnan(logits[t]), -np.inf, np.minimum(logits[t], F32_MAX)) if kind == "softmax" and bias is None else c[t]
        left = [e for e in range(E) if c[t, e] > -np.inf]
        if groups > 1:
            gs = []
            for g in range(groups):
                members = sorted((c[t, e] for e in left if e // per == g), reverse=True)
                gs.append(-np.inf if not members else sum(members[:2]) if top2 else members[0])
            stay = sorted(range(groups), key=lambda g: (-gs[g], g))[:kept]
            left = [e for e in left if e // per in stay]
        left.sort(key=lambda e: (-order_by[e], e))
        pick = left[:k]
        ids[t, :len(pick)] = pick
        w[t, :len(pick)] = s[t, pick]
    if renorm:
        total = w.sum(1, keepdims=True)
        w = np.divide(w, total, out=np.zeros_like(w), where=total > 0)
    return ids, w * scale


def experts_order(ids, E):
    """(group_rows, row_of)."""
    T, k = ids.shape
    row_of = np.full((T, k), -1, dtype=np.int64)
    group_rows = [0]
    n = 0
    for e in range(E):
        for t, j in np.argwhere(ids == e):
            row_of[t, j] = n
            n += 1
        group_rows.append(n)
    return np.array(group_rows), row_of


def route_weights(logits, ids, kind, renorm, scale):
    """The weights as a function of the logits, ids fixed (what route_backward differentiates)."""
    s = scores(logits, kind)
    w = np.where(ids >= 0, np.take_along_axis(s, np.maximum(ids, 0), 1), 0.0)
    if renorm:
        total = w.sum(1, keepdims=True)
        w = np.divide(w, total, out=np.zeros_like(w), where=total > 0)
    return scale * w


def route_backward(logits, ids, g, kind, renorm, scale):
    T, E = logits.shape
    s = scores(logits, kind)
    out = np.zeros((T, E))
    for t in range(T):
        there = [j for j in range(ids.shape[1]) if 0 <= ids[t, j] < E]
        e = ids[t, there]
        gw = g[t, there] * scale
        total = s[t, e].sum()
        if renorm:
            gs = (gw - (gw * s[t, e]).sum() / total) / total if total > 0 else np.zeros(len(there))
        else:
            gs = gw
        ds = np.zeros(E)
        ds[e] = gs
        out[t] = s[t] * (ds - (s[t] * ds).sum()) if kind == "softmax" else s[t] * (1 - s[t]) * ds
    return out


def dispatch(x, row_of, M, fill=0.0):
    rows = np.full((M, x.shape[1]), float(fill))
    for t, j in np.argwhere((row_of >= 0) & (row_of < M)):
        rows[row_of[t, j]] = x[t]
    return rows


def combine(rows, row_of, w, add=None):
    T, k = row_of.shape
    out = np.zeros((T, rows.shape[1])) if add is None else add.copy()
    for t in range(T):
        for j in range(k):
            if 0 <= row_of[t, j] < rows.shape[0]:
                out[t] += w[t, j] * rows[row_of[t, j]]
    return out


def combine_backward(dout, rows, row_of, w, fill=0.0):
    d, dw = np.full(rows.shape, float(fill)), np.zeros(w.shape)
    for t, j in np.argwhere((row_of >= 0) & (row_of < rows.shape[0])):
        r = row_of[t, j]
        d[r] = w[t, j] * dout[t]
        dw[t, j] = rows[r] @ dout[t]
    return d, dw
