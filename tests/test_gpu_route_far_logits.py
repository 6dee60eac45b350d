"""Routing where scores saturate or vanish: experts whose sigmoids round to one fp32 number, scores below the smallest fp32 number, chosen experts far below the row's largest logit.

Tolerances.  U = 2^-24.  A weight is a quotient of scores exp(x) / (1 + exp(y)): two exponentials (2 U each, and U of the arguments' difference, which is exact for logits of like size), a
reciprocal, a product, a sum over k and a division: below 96 U of the value.  What is below the smallest normal fp32 number may be flushed: 2^-126."""
import numpy as np
import pytest
import torch

from oracle import layer_ref as R
from paper_2601_19092_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
CODE = {"bf16": B.AXE_BF16, "f16": B.AXE_F16, "f32": B.AXE_F32}
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def f64(t):
    return t.detach().cpu().to(torch.float32).double().numpy()


def spread_rows(T, E, lo, hi, dtype, seed):
    """Every row the same E values from lo to hi in an order of its own (equal ones where the type has no more between them)."""
    g = torch.Generator().manual_seed(seed)
    order = torch.stack([torch.randperm(E, generator=g) for _ in range(T)])
    return (lo + (hi - lo) * order.double() / max(E - 1, 1)).to(TORCH[dtype])


def far_logits(T, E, where, dtype, seed):
    if where == "high":
        return spread_rows(T, E, 14.0, 30.0, dtype, seed)
    if where == "low":
        return spread_rows(T, E, -95.0, -85.0, dtype, seed)
    x = spread_rows(T, E, -95.0, -85.0, dtype, seed)                   # low ones, and a few high
    x[:, ::9] = spread_rows(T, len(range(0, E, 9)), 16.0, 24.0, dtype, seed + 1)
    return x


def routed(logits, k, dtype, bias=None, order=True, **kw):
    T, E = logits.shape
    d = B.RouteDesc(T, E, k, CODE[dtype], bias=None if bias is None else bias.cuda(), **kw)
    ids, w = torch.zeros((T, k), dtype=torch.int32, device="cuda"), torch.zeros((T, k), device="cuda")
    rows, row_of = torch.zeros(E + 1, dtype=torch.int32, device="cuda"), torch.zeros((T, k), dtype=torch.int32, device="cuda")
    ws = torch.zeros(max(1, B.axe_route_workspace(d)), dtype=torch.int32, device="cuda")
    B.axe_route(d, logits.cuda(), ids, w, rows, row_of, ws)
    return ids.cpu().numpy(), f64(w), rows.cpu().numpy(), row_of.cpu().numpy()


def within(got, want, tol, what):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}"


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("where", ["high", "low", "both"])
@pytest.mark.parametrize("T,E,k", [(1, 128, 8), (70, 16, 4), (40, 256, 8), (33, 1024, 10), (65, 60, 6), (3, 5, 2), (2300, 96, 5), (2100, 200, 4)])
def test_sigmoid_choices_are_in_the_order_of_the_logits(T, E, k, where, dtype):
    logits = far_logits(T, E, where, dtype, T + E)
    for renorm in (True, False):
        ids, w, rows, row_of = routed(logits, k, dtype, score=B.AXE_ROUTE_SIGMOID, renorm=renorm, scale=1.5)
        want = np.argsort(-f64(logits), axis=1, kind="stable")[:, :k]  # (the sigmoid is monotone: the definition's order without its rounding)
        assert np.array_equal(ids, want)
        s = R.scores(f64(logits), "sigmoid")
        ww = np.take_along_axis(s, want, 1)
        ww = 1.5 * (ww / ww.sum(1, keepdims=True) if renorm else ww)
        within(w, ww, 96 * U * ww + 2.0 ** -126, "weights")
        gr, ro = R.experts_order(want, E) if T < 100 else (None, None)
        assert gr is None or (np.array_equal(rows, gr) and np.array_equal(row_of, ro))


@pytest.mark.parametrize("T,E,k,groups,kept", [(20, 64, 4, 8, 2), (20, 60, 5, 4, 2), (5, 256, 8, 8, 4), (2100, 128, 6, 4, 1)])
@pytest.mark.parametrize("where", ["high", "low", "both"])
def test_sigmoid_groups_by_their_largest_choice(T, E, k, groups, kept, where):
    logits = far_logits(T, E, where, "f32", E)
    ids, w, _, _ = routed(logits, k, "f32", score=B.AXE_ROUTE_SIGMOID, groups=groups, groups_kept=kept)
    l = f64(logits)
    best = l.reshape(T, groups, -1).max(2)
    stay = np.argsort(-best, axis=1, kind="stable")[:, :kept]
    keep = np.zeros((T, groups), bool)
    np.put_along_axis(keep, stay, True, 1)
    left = np.where(np.repeat(keep, E // groups, 1), l, -np.inf)
    want = np.argsort(-left, axis=1, kind="stable")[:, :k]
    assert np.array_equal(ids, want)
    ww = np.take_along_axis(R.scores(l, "sigmoid"), want, 1)
    ww /= ww.sum(1, keepdims=True)
    within(w, ww, 96 * U * ww, "weights")


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,k", [(1, 128, 8), (70, 16, 4), (40, 256, 8), (9, 1000, 12), (2100, 96, 5)])
def test_weights_of_experts_that_the_bias_chose(T, E, k, score):
    """Chosen by their bias, with logits some ninety below the others: their scores vanish in fp32, their weights are ordinary numbers."""
    logits = spread_rows(T, E, -1.0, 1.0, "f32", E)
    at = torch.randperm(E, generator=torch.Generator().manual_seed(T))[:k]
    logits[:, at] = spread_rows(T, k, -94.0, -91.0, "f32", T)
    bias = torch.zeros(E)
    bias[at] = 4.0 + torch.arange(k).float()                           # (far enough apart that the scores do not decide)
    want = at.flip(0).numpy()[None].repeat(T, 0)
    ids, w, _, _ = routed(logits, k, "f32", bias=bias, score=int(score == "sigmoid"))
    assert np.array_equal(ids, want)
    ww = np.take_along_axis(R.scores(f64(logits), score), want, 1)
    ww /= ww.sum(1, keepdims=True)
    within(w, ww, 96 * U * ww, "weights")


def test_rows_of_the_lowest_value_get_no_sigmoid_weights():
    logits = torch.full((70, 24), torch.finfo(torch.float32).min)
    logits[::2, 5] = -699.0
    for bias in (None, torch.zeros(24)):
        ids, w, _, _ = routed(logits, 3, "f32", bias=bias, score=B.AXE_ROUTE_SIGMOID)
        assert (w[1::2] == 0).all() and (ids[1::2] == np.arange(3)).all()
        if bias is None:
            assert (ids[::2, 0] == 5).all() and (w[::2] == [1.0, 0.0, 0.0]).all()


# ---- gradients ------------------------------------------------------------------------------------------------------------------------------------
# Unnormalised sigmoid: s (1 - s) g, three roundings more than two exponentials and reciprocals: 32 U of the value.  Renormalised: w (g - mean) (1 - s), w as above, the mean's error that of its
# magnitudes: 96 U of w (1 - s) 2 max |g|.

def gradient(logits, ids, g, dtype, score, renorm, scale=1.5):
    T, E = logits.shape
    d = B.RouteDesc(T, E, ids.shape[1], CODE[dtype], score=score, renorm=renorm, scale=scale)
    out = torch.full((T, E), 7.0, dtype=TORCH[dtype], device="cuda")
    B.axe_route_backward(d, logits.cuda(), torch.from_numpy(ids).int().cuda(), g.cuda(), out)
    return f64(out)


def other_side(l):
    """1 - sigmoid(l) without cancellation."""
    return 1.0 / (1.0 + np.exp(l))


def exact_gradient(l, ids, g, score, renorm, scale=1.5):
    """By the chosen logits, others 0: of renormalised weights, and of sigmoids."""
    out = np.zeros_like(l)
    c = np.take_along_axis(l, ids, 1)
    if renorm:
        top = c.max(1, keepdims=True)
        w = np.exp(c - top) / (1 + np.exp(c) if score else 1.0)
        w = w / w.sum(1, keepdims=True)
        d = w * (scale * g - (w * scale * g).sum(1, keepdims=True)) * (other_side(c) if score else 1.0)
    else:
        d = scale * g * other_side(c) * other_side(-c)
    np.put_along_axis(out, ids, d, 1)
    return out


@pytest.mark.parametrize("where", [(8.0, 20.0), (16.0, 60.0), (-95.0, -75.0), (-30.0, 30.0)])
@pytest.mark.parametrize("T,E,k", [(1, 128, 8), (70, 16, 4), (40, 256, 8), (9, 1000, 12), (8200, 96, 5)])
def test_sigmoid_gradient_far_out(T, E, k, where):
    logits = spread_rows(T, E, *where, "f32", T)
    ids = np.argsort(-f64(logits), axis=1, kind="stable")[:, :k]
    g = torch.randn((T, k), generator=torch.Generator().manual_seed(1))
    got, want = gradient(logits, ids, g, "f32", 1, False), exact_gradient(f64(logits), ids, f64(g), 1, False)
    within(got, want, 32 * U * np.abs(want) + 2.0 ** -126, "dlogits")


@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("size", [1.0, 1e8])
@pytest.mark.parametrize("where", [(8.0, 20.0), (-88.0, -80.0), (-95.0, -85.0), (-3.0, 3.0)])
@pytest.mark.parametrize("T,E,k", [(1, 128, 8), (70, 16, 4), (40, 256, 8), (9, 1000, 12), (8200, 96, 5)])
def test_renormalised_gradient_of_vanishing_scores(T, E, k, where, size, score):
    """Gradients of ordinary size, and scaled ones, of weights whose scores' sum vanishes (softmax: next to other experts around 0)."""
    logits = spread_rows(T, E, *where, "f32", T)
    if score == 0:
        logits[:, k:] = spread_rows(T, E - k, -1.0, 1.0, "f32", T + 1)
    ids = np.arange(k)[None].repeat(T, 0)
    g = size * torch.randn((T, k), generator=torch.Generator().manual_seed(1))
    l, gv = f64(logits), f64(g)
    got, want = gradient(logits, ids, g, "f32", score, True), exact_gradient(l, ids, gv, score, True)
    c = l[:, :k]
    top = c.max(1, keepdims=True)
    w = np.exp(c - top) / (1 + np.exp(c) if score else 1.0)
    mag = np.zeros_like(l)
    mag[:, :k] = w / w.sum(1, keepdims=True) * (other_side(c) if score else 1.0) * 2 * 1.5 * np.abs(gv).max()
    within(got, want, 96 * U * mag + 2.0 ** -126, "dlogits")


def test_gradient_of_rows_that_leave_nothing_is_zero():
    logits = torch.randn((70, 40), generator=torch.Generator().manual_seed(2))
    logits[::3] = -float("inf")
    ids = np.where(np.isneginf(f64(logits))[:, :5], -1, np.arange(5))
    ids[3] = np.arange(5)                                              # (named, but masked)
    for score in (0, 1):
        for renorm in (True, False):
            got = gradient(logits, ids, torch.ones((70, 5)), "f32", score, renorm)
            assert (got[::3] == 0).all() and np.isfinite(got).all(), (score, renorm)
            if not renorm:
                assert (got[1, :5] != 0).all()
