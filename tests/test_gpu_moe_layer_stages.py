"""The mixture-of-experts layer stage by stage, each from the buffer that the stage before it left, with weight scales that differ from block to block: a scale taken from another expert,
another block or the other axis is off by its own ratio, which no rounding hides."""
import pytest
import torch

from paper_2601_19092_amd import moe_layer as L

pytestmark = pytest.mark.gpu

HIDDEN, INTER, EXPERTS, TOPK = 512, 384, 12, 3                         # (blocks: 4 along hidden, 6 and 3 along the intermediate rows: no two axes alike)


def f64(t):
    return t.detach().cpu().to(torch.float32).double()


def made(tokens, fp8):
    g = torch.Generator(device="cuda").manual_seed(tokens + fp8)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")     # noqa: E731
    wt = torch.float8_e4m3fn if fp8 else torch.bfloat16
    gate_up = (normal(EXPERTS, 2 * INTER, HIDDEN) * (1 if fp8 else HIDDEN ** -0.5)).to(wt)
    down = (normal(EXPERTS, HIDDEN, INTER) * (1 if fp8 else INTER ** -0.5)).to(wt)
    s1 = s2 = None
    if fp8:                                                            # a factor of up to four either way
        s1 = HIDDEN ** -0.5 * torch.exp2(4 * torch.rand((EXPERTS, 2 * INTER // 128, HIDDEN // 128), generator=g, device="cuda") - 2)
        s2 = INTER ** -0.5 * torch.exp2(4 * torch.rand((EXPERTS, HIDDEN // 128, INTER // 128), generator=g, device="cuda") - 2)
    layer = L.MoeLayer(tokens, 1 + 0.1 * normal(HIDDEN), (normal(EXPERTS, HIDDEN) * HIDDEN ** -0.5).bfloat16(), gate_up, down, TOPK, s1, s2)
    return layer, normal(tokens, HIDDEN).bfloat16(), normal(tokens, HIDDEN).bfloat16(), gate_up, down, s1, s2


def dequantised(w, s):
    return f64(w) if s is None else f64(w) * f64(s).repeat_interleave(128, 1).repeat_interleave(128, 2)


def columns(s, n):
    return f64(s).repeat_interleave(128, 1)[:, :n]


# A product's result is rounded to bf16: 2^-9 of each value at most, hence of the norm; fp32 sums of up to 512 products, whose magnitudes add up to some 20 times the result, at most 512 roundings of
# 2^-24 of that each: below 2^-10.  The gate multiplies silu(g) by u, both within that sum's error: twice.
PRODUCT, GATED = 2.0 ** -9 + 2.0 ** -10, 2.0 ** -9 + 2.0 ** -9


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("tokens", [1, 5, 70, 333])
def test_stages(tokens, fp8):
    layer, stream, x, gate_up, down, s1, s2 = made(tokens, fp8)
    out = torch.zeros_like(stream)
    layer.forward(stream, x, out=out)
    torch.cuda.synchronize()
    rows, ids, row_of = layer.group_rows.cpu().long(), layer.ids.cpu().long(), layer.row_of.cpu().long()
    assert rows[-1] == tokens * TOPK
    y = f64(layer.y)
    by_row = torch.empty(tokens * TOPK, dtype=torch.long)
    by_row[row_of.reshape(-1)] = torch.arange(tokens * TOPK) // TOPK
    a = f64(layer.a)
    if fp8:                                                            # e4m3: half a step, 2^-4 of a value, or of the smallest normal number's step times the scale
        sc = columns(layer.a_scales, HIDDEN)
        assert ((a * sc - y[by_row]).abs() <= 2.0 ** -4 * y[by_row].abs() + 2.0 ** -10 * sc).all()
        a = a * sc
    else:
        assert torch.equal(a, y[by_row])
    g, d = dequantised(gate_up, s1), dequantised(down, s2)
    h, c = f64(layer.h), f64(layer.c)
    h_in = h
    if fp8:
        sc = columns(layer.h_scales, INTER)
        h_in = f64(layer.h8) * sc
        assert ((h_in - h).abs() <= 2.0 ** -4 * h.abs() + 2.0 ** -10 * sc).all()
    for e in range(EXPERTS):
        p = slice(int(rows[e]), int(rows[e + 1]))
        if rows[e] == rows[e + 1]:
            continue
        assert all((ids[t] == e).any() for t in by_row[p])
        pre = a[p] @ g[e].t()
        want = pre[:, :INTER] / (1 + torch.exp(-pre[:, :INTER])) * pre[:, INTER:]
        assert (h[p] - want).norm() <= GATED * want.norm(), e
        want = h_in[p] @ d[e].t()
        for b in range(HIDDEN // 128):                                 # (block by block: a wrong scale of one is not lost among the others)
            cols = slice(128 * b, 128 * b + 128)
            assert (c[p, cols] - want[:, cols]).norm() <= PRODUCT * want[:, cols].norm(), (e, b)
    w = f64(layer.weights)
    want = f64(stream) + (w[:, :, None] * c[row_of]).sum(1)
    mag = f64(stream).abs() + (w[:, :, None] * c[row_of]).abs().sum(1)
    assert ((f64(out) - want).abs() <= 2.0 ** -8 * want.abs() + (TOPK + 2) * 2.0 ** -24 * mag).all()
