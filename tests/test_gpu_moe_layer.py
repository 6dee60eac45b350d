"""A mixture-of-experts layer through the library's entry points, from the residual stream to the residual stream, against the same in 64 bits; and the gradients of
everything around the experts' products, chained, against automatic differentiation in 64 bits."""
import pytest
import torch

from paper_2601_19092_amd import binding as B
from paper_2601_19092_amd import moe_layer as L

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().cpu().to(torch.float32).double()


def plain(layer, stream, x, gate_up, down, s1=None, s2=None):
    """(stream + x, that plus the experts' sum) in 64 bits; the kernels' own choice of experts, so that a near tie does not decide the test."""
    s = f64(stream) + f64(x)
    y = s / torch.sqrt((s * s).mean(1, keepdim=True) + 1e-6) * f64(layer.norm_weight)
    logits = y @ f64(layer.router).t()
    p = torch.softmax(logits, 1)
    ids = layer.ids.cpu().long()
    w = p.gather(1, ids)
    w = w / w.sum(1, keepdim=True)
    g, d = f64(gate_up), f64(down)
    if s1 is not None:
        g = g * f64(s1).repeat_interleave(128, 1).repeat_interleave(128, 2)
        d = d * f64(s2).repeat_interleave(128, 1).repeat_interleave(128, 2)
    inter = d.shape[2]
    out = s.clone()
    for t in range(s.shape[0]):
        for j in range(ids.shape[1]):
            e = ids[t, j]
            pre = g[e] @ y[t]
            h = pre[:inter] / (1 + torch.exp(-pre[:inter])) * pre[inter:]
            out[t] += w[t, j] * (d[e] @ h)
    return s, out, logits, w


# relative Frobenius errors of what the experts add: bf16 rounds y, the rows between the products and the result of the second, 2^-9 at most and 2^-9 / sqrt(3) on
# average each, through a gate that at most doubles it: below 5e-3; e4m3 rounds the two products' rows by 2^-4 / sqrt(3) on average at most: below 6e-2
@pytest.mark.parametrize("fp8,tol", [(False, 5e-3), (True, 6e-2)])
@pytest.mark.parametrize("tokens", [1, 3, 70, 200])
def test_layer_against_64_bits(tokens, fp8, tol):
    hidden, inter, experts, topk = 512, 256, 16, 4
    g = torch.Generator(device="cuda").manual_seed(tokens)
    layer, stream, x = L.synthetic(tokens, fp8, hidden, inter, experts, topk, seed=3)
    gate_up = torch.randn((experts, 2 * inter, hidden), generator=g, device="cuda") * (1 if fp8 else hidden ** -0.5)
    gate_up = gate_up.to(torch.float8_e4m3fn if fp8 else torch.bfloat16)
    layer.gate_up = L.interleaved(gate_up)
    s0, out = stream.clone(), torch.zeros_like(stream)
    layer.forward(stream, x, out=out)
    s1 = torch.full((experts, 2 * inter // 128, hidden // 128), hidden ** -0.5) if fp8 else None
    s2 = torch.full((experts, hidden // 128, inter // 128), inter ** -0.5) if fp8 else None
    s, want, logits, w = plain(layer, s0, x, gate_up, layer.down, s1, s2)
    assert (f64(stream) - s).norm() <= 2 ** -8 * s.norm()
    # the chosen experts are the largest logits, as far as bf16's y can tell: each is within its error of the k-th largest
    kth = logits.topk(topk, 1).values[:, -1:]
    assert (logits.gather(1, layer.ids.cpu().long()) >= kth - 2 ** -6 * logits.abs().amax(1, keepdim=True)).all()
    assert (f64(layer.weights) - w).abs().max() <= 2 ** -6
    added, exact = f64(out) - f64(stream), want - s
    # (the sum itself is rounded to bf16: half a unit of the stream's values, over the norm of what is added)
    rounding = 2 ** -9 * want.norm() / exact.norm()
    assert (added - exact).norm() / exact.norm() <= tol + rounding + 2 ** -7
    # in place, from a graph, on another stream: the same bits
    again = s0.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.forward(again.clone(), x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(again, x)
    for _ in range(3):
        again.copy_(s0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(again, out)


def test_chained_gradients_against_automatic_differentiation():
    """loss = <combine(w, dispatch(y)) , g> with y = norm(x) wn, w = renormalised softmax weights of the chosen experts of y Wr: the rows' own experts left out, everything
    that the library has a gradient of is in it."""
    T, H, E, k = 37, 136, 24, 3
    gen = torch.Generator().manual_seed(5)
    x, wn, wr, g = (torch.randn(s, generator=gen) for s in ((T, H), (H,), (E, H), (T, H)))
    wr = wr * H ** -0.5
    scale_of_row = 1 + torch.arange(T * k).float() / (T * k)           # (stands for the experts: a factor for every row)
    dev = lambda t: t.cuda()                                           # noqa: E731
    nd, rd, wd = B.RmsNormDesc(T, H, B.AXE_F32, B.AXE_F32), B.RouteDesc(T, E, k, scale=1.5), B.RowsDesc(T, k, T * k, H, B.AXE_F32, B.AXE_F32)
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device="cuda")   # noqa: E731
    y = z(T, H)
    B.axe_rmsnorm(nd, dev(x), dev(wn), y)
    logits = y @ dev(wr).t().contiguous()
    ids, w, rows, ro = z(T, k, dt=torch.int32), z(T, k), z(E + 1, dt=torch.int32), z(T, k, dt=torch.int32)
    ws = z(max(1, B.axe_route_workspace(rd)), dt=torch.int32)
    B.axe_route(rd, logits, ids, w, rows, ro, ws)
    a, out = z(T * k, H), z(T, H)
    B.axe_rows_dispatch(wd, y, ro, a)
    c = a * dev(scale_of_row)[:, None]
    B.axe_rows_combine(wd, c, ro, w, out)
    dc, dw, dy, dlogits, dx, dwn = z(T * k, H), z(T, k), z(T, H), z(T, E), z(T, H), z(H)
    B.axe_rows_combine_backward(wd, dev(g), c, ro, w, dc, dw)
    B.axe_rows_combine(wd, dc * dev(scale_of_row)[:, None], ro, None, dy)
    B.axe_route_backward(rd, logits, ids, dw, dlogits)
    nws = z(max(1, B.axe_rmsnorm_workspace(nd)), dt=torch.int32)
    B.axe_rmsnorm_backward(nd, dy + dlogits @ dev(wr), dev(x), dev(wn), dx, dweight=dwn, workspace=nws)

    X, WN, WR = (t.double().requires_grad_() for t in (x, wn, wr))
    Y = X / torch.sqrt((X * X).mean(1, keepdim=True) + 1e-6) * WN
    P = torch.softmax(Y @ WR.t(), 1).gather(1, ids.cpu().long())
    P = 1.5 * P / P.sum(1, keepdim=True)
    S = scale_of_row.double()[ro.cpu().long()]
    loss = ((P * S).sum(1, keepdim=True) * Y * g.double()).sum()
    loss.backward()
    # fp32 throughout: a few hundred roundings of sums of some hundred numbers of like size
    for got, want in ((dx, X.grad), (dwn, WN.grad)):
        assert (f64(got) - want).norm() <= 2e-5 * want.norm()
    want_out = ((P * S).sum(1, keepdim=True) * Y).detach()
    assert (f64(out) - want_out).norm() <= 2e-6 * want_out.norm() * 4
