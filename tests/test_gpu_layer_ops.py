"""What stands around the experts' products on the GPU -- norm, routing, rows in the experts' order, each with its gradient -- against the same in 64 bits.

Tolerances.  U = 2^-24 is fp32's rounding.  A result in 16 bits is off by its own rounding (half a unit in its last place: 2^-9 of the value for bf16, 2^-12 for fp16, no less
than half of the smallest fp16 step, 2^-25) and by what fp32 does on the way; that is bounded by the number of roundings times U times the magnitudes that enter, and 64 U covers
sums over up to 32768 columns (32 in a lane's chain, 16 in a tree) with the divisions and the square root behind them."""
import numpy as np
import pytest
import torch

from oracle import layer_ref as R
from paper_2601_19092_amd import binding as B
from paper_2601_19092_amd import workloads as W

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
CODE = {"bf16": B.AXE_BF16, "f16": B.AXE_F16, "f32": B.AXE_F32, "fp8": B.AXE_FP8_E4M3}
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "fp8": torch.float8_e4m3fn}
HALF_ULP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": U}            # of the value: half a step is at most that share of it
EPS = 1e-6


def f64(t):
    return t.detach().cpu().to(torch.float32).double().numpy()


def draw(seed, shape, dtype, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(TORCH[dtype])


class Mat:
    """A matrix in a buffer of its own, at a pitch and an offset, the rest of the buffer a pattern that must survive."""

    def __init__(self, values, pitch=None, offset=0):
        rows, cols = values.shape
        self.shape, self.pitch, self.offset = (rows, cols), pitch or cols, offset
        n = offset + max(rows, 1) * self.pitch + 24
        eb = values.element_size()
        self.buf = torch.full((n * eb,), 0x5A, dtype=torch.uint8).view(values.dtype)
        self.view(self.buf)[:] = values
        self.buf = self.buf.cuda()
        self.before = self.buf.clone()
        self.layout = B.Layout(W.spec([(max(rows, 1), self.pitch, "m"), (cols, 1, "m")], O={"m": offset}), ["m"])

    def view(self, buf):
        return torch.as_strided(buf, self.shape, (self.pitch, 1), self.offset)

    def get(self):
        return self.view(self.buf).cpu()

    def rest_untouched(self):
        a, b = self.buf.clone().view(torch.uint8), self.before.clone().view(torch.uint8)
        eb = self.buf.element_size()
        mark = torch.ones(self.buf.numel(), dtype=torch.bool, device="cuda")
        torch.as_strided(mark, self.shape, (self.pitch, 1), self.offset)[:] = False
        mark = mark.repeat_interleave(eb)
        return bool((a[mark] == b[mark]).all())


def within(got, want, tol, what=""):
    got, want, tol = np.asarray(got), np.asarray(want), np.broadcast_to(tol, np.asarray(want).shape)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}, allowed {tol[bad][0]}"


def rounding(want, dtype):
    return np.abs(want) * HALF_ULP[dtype] + (2.0 ** -25 if dtype == "f16" else 0.0)


def check_quantised(q, stored, kind, y, err):
    """e4m3 rows q and their scales against y in 64 bits, itself known to `err` (relative to the row's largest)."""
    T, H = y.shape
    s64 = R.scales(y, kind)
    s = stored.cpu().numpy().astype(np.float64) if kind == "f32" else np.exp2(stored.cpu().numpy().astype(np.float64) - 127.0)
    s = s.reshape(s64.shape)
    if kind == "f32":
        within(s, s64, s64 * (err + 4 * U), "scales")
    else:                                                              # a maximum on a power of two's edge may fall to either side
        edge = np.abs(R.scales(y * (1 + 2 * err), kind) - R.scales(y * (1 - 2 * err), kind)) > 0
        assert ((s == s64) | (edge & ((s == 2 * s64) | (2 * s == s64)))).all()
    v = y / R.spread(s, H)
    got = f64(q)
    # e4m3 has steps of 2^-3 of a binade, 2^-9 below 2^-6
    within(got, np.clip(v, -448, 448), np.maximum(np.abs(v) * 2.0 ** -4, 2.0 ** -10) + np.abs(v) * (err + 4 * U) + 448 * err, "e4m3")


# ---- norm ---------------------------------------------------------------------------------------------------------------------------------------

def norm_inputs(T, H, dtype, seed, residual, pitched):
    x = draw(seed, (T, H), dtype, 1.5)
    r = draw(seed + 1, (T, H), dtype, 0.7) if residual else None
    w = 1.0 + 0.2 * draw(seed + 2, (H,), "f32")
    pad = [(H + p, o) for p, o in ((8, 16), (24, 8), (3, 1), (40, 32))] if pitched else [(None, 0)] * 4
    return x, r, w, pad


NORM_SHAPES = [(1, 1), (1, 2048), (3, 7), (5, 128), (2, 129), (1, 8192), (64, 2048), (7, 1999), (130, 768), (2, 5120), (3, 8200), (1, 16384), (2, 32768), (4100, 64), (33, 255), (2, 12345)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,H", NORM_SHAPES)
@pytest.mark.parametrize("residual,pitched", [(False, False), (True, False), (True, True)])
def test_norm_against_64_bits(T, H, dtype, residual, pitched):
    x, r, w, pad = norm_inputs(T, H, dtype, 11 * T + H, residual, pitched)
    X, Rm = Mat(x, *pad[0]), Mat(r, *pad[1]) if residual else None
    S, Y = Mat(torch.zeros_like(x), *pad[2]), Mat(torch.zeros_like(x), *pad[3])
    d = B.RmsNormDesc(T, H, CODE[dtype], CODE[dtype], eps=EPS, x=X.layout, residual=Rm and Rm.layout, sum=S.layout, y=Y.layout, x_elems=X.buf.numel(),
                      residual_elems=Rm.buf.numel() if Rm else None, sum_elems=S.buf.numel(), y_elems=Y.buf.numel())
    B.axe_rmsnorm(d, X.buf, w.cuda(), Y.buf, residual=Rm and Rm.buf, sum_out=S.buf)
    h = f64(x) + (f64(r) if residual else 0.0)
    y, _ = R.rmsnorm(h, f64(w), EPS)
    within(f64(S.get()), h, rounding(h, dtype) + np.abs(h) * 2 * U, "sum")
    within(f64(Y.get()), y, rounding(y, dtype) + np.abs(y) * 64 * U, "y")
    assert X.rest_untouched() and S.rest_untouched() and Y.rest_untouched() and torch.equal(X.get().view(torch.uint8), x.view(torch.uint8))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("T,H", [(1, 2048), (1, 1), (3, 130), (64, 2048), (9, 8192), (5, 1999), (2, 32768), (257, 384), (3, 4104)])
def test_norm_quantised(T, H, dtype, kind):
    x, r, w, _ = norm_inputs(T, H, dtype, 7 * T + H, True, False)
    nb = -(-H // 128)
    if H > 200:
        x[0, :128] = 0                                                 # a run of 128 zeros: scale 1
        r[0, :128] = 0
    q = torch.zeros((T, H), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    sc = torch.zeros((T, nb), dtype=torch.float32 if kind == "f32" else torch.uint8, device="cuda")
    d = B.RmsNormDesc(T, H, CODE[dtype], B.AXE_FP8_E4M3, eps=EPS, scale_dtype=B.AXE_SCALE_E8M0 if kind == "e8m0" else B.AXE_SCALE_F32)
    s = torch.zeros_like(x).cuda()
    B.axe_rmsnorm(d, x.cuda(), w.cuda(), q, residual=r.cuda(), sum_out=s, scales=sc)
    h = f64(x) + f64(r)
    y, _ = R.rmsnorm(h, f64(w), EPS)
    check_quantised(q, sc, kind, y, 64 * U)
    within(f64(s), h, rounding(h, dtype) + np.abs(h) * 2 * U, "sum")


@pytest.mark.parametrize("xt,yt,wt", [("f32", "bf16", "f32"), ("f32", "f16", "bf16"), ("bf16", "bf16", "bf16"), ("f16", "f16", "f16"), ("bf16", "bf16", "f16"), ("bf16", "bf16", None), ("f32", "fp8", None)])
def test_norm_mixed_types_and_no_weights(xt, yt, wt):
    T, H = 37, 640
    x = draw(5, (T, H), xt)
    w = None if wt is None else (1 + 0.2 * draw(6, (H,), "f32")).to(TORCH[wt])
    d = B.RmsNormDesc(T, H, CODE[xt], CODE[yt], eps=1e-3, weight_dtype=CODE[wt or "f32"])
    y = torch.zeros((T, H), dtype=torch.uint8 if yt == "fp8" else TORCH[yt], device="cuda")
    sc = torch.zeros((T, 5), device="cuda") if yt == "fp8" else None
    B.axe_rmsnorm(d, x.cuda(), None if w is None else w.cuda(), y, scales=sc)
    want, _ = R.rmsnorm(f64(x), 1.0 if w is None else f64(w), 1e-3)
    if yt == "fp8":
        check_quantised(y.view(torch.float8_e4m3fn), sc, "f32", want, 64 * U)
    else:
        within(f64(y), want, rounding(want, yt) + np.abs(want) * 64 * U)


def test_norm_of_zero_rows_infinities_and_nan():
    H = 512
    x = draw(3, (5, H), "f32")
    x[0] = 0
    x[1, 200] = float("nan")
    x[2, 300] = float("inf")
    x[3] = 1e-30
    w = torch.ones(H)
    y = torch.full((5, H), 7.0, device="cuda")
    d = B.RmsNormDesc(5, H, B.AXE_F32, B.AXE_F32, eps=EPS)
    B.axe_rmsnorm(d, x.cuda(), w.cuda(), y)
    got = y.cpu()
    assert (got[0] == 0).all() and got[1].isnan().all()                # a NaN reaches its own row, no other
    assert got[2, 300].isnan() and (got[2, :300] == 0).all()           # inf * 0
    want, _ = R.rmsnorm(f64(x[3:]), f64(w), EPS)
    within(f64(got[3:]), want, np.abs(want) * 64 * U)
    # the quantiser: rows in order, no norm
    q, sc = torch.zeros((5, H), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), torch.zeros((5, 4), device="cuda")
    x[4, 130] = float("-inf")
    rd = B.RowsDesc(5, 1, 5, H, B.AXE_F32, B.AXE_FP8_E4M3)
    B.axe_rows_dispatch(rd, x.cuda(), None, q, scales=sc)
    v, s = f64(q), sc.cpu().double().numpy()
    assert (v[0] == 0).all() and (s[0] == 1).all()
    assert np.isnan(v[1, 200]) and np.isfinite(np.delete(v[1], 200)).all()
    assert v[2, 300] == 448 and (np.delete(v[2, 256:384], 44) == 0).all() and v[4, 130] == -448
    clean = np.where(np.isfinite(f64(x)), f64(x), 0.0)
    for b in (0, 3):
        within(s[:, b], R.scales(clean, "f32")[:, b], s[:, b] * 4 * U, "scales")
    within(s[1], R.scales(clean, "f32")[1], s[1] * 4 * U, "a NaN is left out of the maximum")


def test_norm_tiny_blocks_keep_finite_scales():
    """Rows whose numbers are subnormal: the scale stops at 2^-126, its reciprocal stays finite."""
    H = 256
    x = torch.zeros((2, H))
    x[0, :128] = 1e-41
    x[1] = 3e-37
    for kind in ("f32", "e8m0"):
        q = torch.zeros((2, H), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        sc = torch.zeros((2, 2), dtype=torch.float32 if kind == "f32" else torch.uint8, device="cuda")
        B.axe_rows_dispatch(B.RowsDesc(2, 1, 2, H, B.AXE_F32, B.AXE_FP8_E4M3, scale_dtype=int(kind == "e8m0")), x.cuda(), None, q, scales=sc)
        check_quantised(q, sc, kind, f64(x), 4 * U)


def test_norm_in_place():
    T, H = 70, 1030
    for dtype in ("bf16", "f32"):
        x, r, w, _ = norm_inputs(T, H, dtype, 4, True, False)
        d = B.RmsNormDesc(T, H, CODE[dtype], CODE[dtype], eps=EPS)
        y, s = torch.zeros_like(x).cuda(), torch.zeros_like(x).cuda()
        B.axe_rmsnorm(d, x.cuda(), w.cuda(), y, residual=r.cuda(), sum_out=s)
        x2, r2 = x.cuda(), r.cuda()
        B.axe_rmsnorm(d, x2, w.cuda(), x2, residual=r2, sum_out=r2)
        assert torch.equal(x2, y) and torch.equal(r2, s)


BACK_SHAPES = [(1, 1), (1, 2048), (3, 7), (65, 128), (2, 129), (300, 2048), (9, 1999), (2, 16384), (1, 32768), (5000, 64), (700, 768), (40, 5120), (2, 12345)]


def norm_backward(T, H, dtype, seed, with_dsum, pitched=False, ytype=None, wt="f32"):
    ytype = ytype or dtype
    h, dy = draw(seed, (T, H), dtype, 1.3), draw(seed + 1, (T, H), ytype)
    ds = draw(seed + 2, (T, H), dtype) if with_dsum else None
    w = (1.0 + 0.2 * draw(seed + 3, (H,), "f32")).to(TORCH[wt])
    pad = [(H + 8, 16), (H + 1, 3), (H + 24, 8), (H + 5, 0)] if pitched else [(None, 0)] * 4
    DY, Hm, DX = Mat(dy, *pad[0]), Mat(h, *pad[1]), Mat(torch.zeros_like(h), *pad[2])
    DS = Mat(ds, *pad[3]) if with_dsum else None
    d = B.RmsNormDesc(T, H, CODE[dtype], CODE[ytype], eps=EPS, weight_dtype=CODE[wt], x=DX.layout, sum=Hm.layout, y=DY.layout, residual=DS and DS.layout, x_elems=DX.buf.numel(),
                      sum_elems=Hm.buf.numel(), y_elems=DY.buf.numel(), residual_elems=DS.buf.numel() if DS else None)
    dw = torch.full((H,), 9.0, device="cuda")
    words = B.axe_rmsnorm_workspace(d)
    ws = torch.full((words,), -1, dtype=torch.int32, device="cuda") if words else None
    B.axe_rmsnorm_backward(d, DY.buf, Hm.buf, w.cuda(), DX.buf, dsum=DS and DS.buf, dweight=dw, workspace=ws)
    return h, dy, ds, w, DX, dw


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,H", BACK_SHAPES)
@pytest.mark.parametrize("with_dsum,pitched", [(False, False), (True, True)])
def test_norm_backward_against_64_bits(T, H, dtype, with_dsum, pitched):
    h, dy, ds, w, DX, dw = norm_backward(T, H, dtype, T + 3 * H, with_dsum, pitched)
    a, g, wv, s = f64(h), f64(dy), f64(w), f64(ds) if with_dsum else None
    dx, dwv = R.rmsnorm_backward(g, a, wv, EPS, s)
    rho = 1 / np.sqrt((a * a).mean(1, keepdims=True) + EPS)
    mag = rho * np.abs(g * wv) + rho ** 3 * np.abs(a) * np.abs(g * wv * a).mean(1, keepdims=True) + (np.abs(s) if with_dsum else 0)
    within(f64(DX.get()), dx, rounding(dx, dtype) + 64 * U * mag, "dx")
    # dw: rows are summed in chains and trees of fp32; as many roundings as a chain is long, at most T
    within(f64(dw), dwv, (64 + min(T, 1024)) * U * (np.abs(g * a * rho)).sum(0), "dw")
    assert DX.rest_untouched()


def test_norm_backward_against_differences():
    """The formula's gradient, and the kernel's, against central differences of the norm itself in 64 bits."""
    T, H, step = 2, 24, 1e-5
    h, dy, _, w, DX, dw = norm_backward(T, H, "f32", 5, False)
    a, g, wv = f64(h), f64(dy), f64(w)
    loss = lambda hh, ww: (R.rmsnorm(hh, ww, EPS)[0] * g).sum()         # noqa: E731
    num = np.zeros_like(a)
    for t in range(T):
        for c in range(H):
            e = np.zeros_like(a)
            e[t, c] = step
            num[t, c] = (loss(a + e, wv) - loss(a - e, wv)) / (2 * step)
    numw = np.array([(loss(a, wv + step * (np.arange(H) == c)) - loss(a, wv - step * (np.arange(H) == c))) / (2 * step) for c in range(H)])
    # differences: step^2 of the third derivative (of order 10 here) and 2^-52 / step of the loss
    within(R.rmsnorm_backward(g, a, wv, EPS)[0], num, 1e-8)
    within(f64(DX.get()), num, 1e-8 + 64 * U * 8)
    within(f64(dw), numw, 1e-8 + 64 * U * 8)


def test_norm_backward_mixed_types_in_place_and_without_dweight():
    h, dy, ds, w, DX, dw = norm_backward(33, 1000, "f32", 8, True, ytype="bf16", wt="bf16")
    a, g, wv, s = f64(h), f64(dy), f64(w), f64(ds)
    dx, dwv = R.rmsnorm_backward(g, a, wv, EPS, s)
    within(f64(DX.get()), dx, 1e-4)
    within(f64(dw), dwv, 97 * U * np.abs(g * a).sum(0) * 2)
    d = B.RmsNormDesc(33, 1000, B.AXE_F32, B.AXE_F32, eps=EPS)
    dyc, dsc, wc, hc = dy.float().cuda(), ds.cuda(), w.float().cuda(), h.cuda()
    out = torch.zeros((33, 1000), device="cuda")
    B.axe_rmsnorm_backward(d, dyc, hc, wc, out, dsum=dsc)
    dx_on_ds = dsc.clone()
    B.axe_rmsnorm_backward(d, dyc, hc, wc, dx_on_ds, dsum=dx_on_ds)
    dx_on_dy = dyc.clone()
    words = B.axe_rmsnorm_workspace(d)
    ws = torch.zeros(max(words, 1), dtype=torch.int32, device="cuda")
    dw2 = torch.zeros(1000, device="cuda")
    B.axe_rmsnorm_backward(d, dx_on_dy, hc, wc, dx_on_dy, dsum=dsc, dweight=dw2, workspace=ws)
    assert torch.equal(out, dx_on_ds) and torch.equal(out, dx_on_dy)
    within(f64(dw2), dwv, 97 * U * np.abs(g * a).sum(0) * 2)
    # no rows: the weights' gradient is zero
    d0 = B.RmsNormDesc(0, 1000, B.AXE_F32, B.AXE_F32)
    B.axe_rmsnorm_backward(d0, None, None, wc, None, dweight=dw2, workspace=ws)
    assert (dw2 == 0).all()


# ---- routing ------------------------------------------------------------------------------------------------------------------------------------

def logits_apart(T, E, dtype, seed):
    """Logits any two of which in a row differ by far more than fp32 rounds scores, in an order of their own for every row."""
    g = torch.Generator().manual_seed(seed)
    order = torch.stack([torch.randperm(E, generator=g) for _ in range(T)])
    return ((order.double() - E / 2) * (6.0 / max(E, 6))).to(TORCH[dtype])


def run_route(logits, E, k, order=True, mat=None, **kw):
    T = logits.shape[0]
    bias = kw.pop("bias", None)
    dtype = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}[logits.dtype]
    m = Mat(logits, *(mat or (None, 0)))
    d = B.RouteDesc(T, E, k, CODE[dtype], bias=None if bias is None else bias.cuda(), logits=m.layout, logits_elems=m.buf.numel(), **kw)
    ids = torch.full((T, k), 77, dtype=torch.int32, device="cuda")
    w = torch.full((T, k), 7.0, device="cuda")
    rows = torch.full((E + 1,), 77, dtype=torch.int32, device="cuda") if order else None
    row_of = torch.full((T, k), 77, dtype=torch.int32, device="cuda") if order else None
    words = B.axe_route_workspace(d)
    ws = torch.full((words,), -1, dtype=torch.int32, device="cuda") if words and order else None
    B.axe_route(d, m.buf, ids, w, rows, row_of, ws)
    return ids, w, rows, row_of


def check_route(logits, E, k, got, bias=None, score="softmax", scale=1.0, **kw):
    ids, w, rows, row_of = got
    want_ids, want_w = R.route(f64(logits), k, score, None if bias is None else f64(bias), scale=scale, **kw)
    assert np.array_equal(ids.cpu().numpy(), want_ids)
    # weights: exp of a difference (2 U of the argument, itself up to a few tens), sums over E, a division
    within(f64(w), want_w, np.abs(want_w) * 96 * U + 2.0 ** -126, "weights")
    if rows is not None:
        gr, ro = R.experts_order(want_ids, E)
        assert np.array_equal(rows.cpu().numpy(), gr) and np.array_equal(row_of.cpu().numpy(), ro)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,E,k", [(1, 128, 8), (1, 1, 1), (2, 8, 8), (5, 7, 3), (64, 128, 8), (65, 60, 4), (300, 64, 6), (129, 256, 8), (3, 1024, 64), (40, 513, 10), (1000, 16, 2), (17, 100, 33)])
def test_route_against_64_bits(T, E, k, dtype):
    logits = logits_apart(T, E, dtype, 3 * T + E)
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            got = run_route(logits, E, k, score=int(score == "sigmoid"), renorm=renorm, scale=2.5)
            check_route(logits, E, k, got, score=score, renorm=renorm, scale=2.5)


@pytest.mark.parametrize("T,E,k,groups,kept", [(70, 256, 8, 8, 4), (33, 160, 6, 8, 3), (9, 64, 4, 64, 9), (130, 60, 8, 4, 2), (5, 1024, 16, 16, 5), (3, 12, 2, 6, 1), (2, 512, 8, 2, 2)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("top2", [False, True])
def test_route_with_groups_and_bias(T, E, k, groups, kept, score, top2):
    logits = logits_apart(T, E, "f32", T + E)
    bias = 0.3 * torch.randn(E, generator=torch.Generator().manual_seed(E))
    for b in (None, bias):
        got = run_route(logits, E, k, mat=(E + 3, 5), score=int(score == "sigmoid"), groups=groups, groups_kept=kept, group_score=int(top2), bias=b)
        check_route(logits, E, k, got, bias=b, score=score, groups=groups, kept=kept, top2=top2)


def test_route_ties_go_to_the_lowest_index():
    T, E, k = 130, 96, 10
    g = torch.Generator().manual_seed(1)
    logits = torch.randint(0, 4, (T, E), generator=g).float()
    logits[0] = 0.0
    for kw in ({}, {"score": 1}, {"groups": 8, "groups_kept": 3}, {"groups": 8, "groups_kept": 3, "group_score": 1, "score": 1}):
        ids, w, rows, row_of = run_route(logits, E, k, **kw)
        ref = dict(groups=kw.get("groups", 1), kept=kw.get("groups_kept", 1), top2=bool(kw.get("group_score", 0)))
        check_route(logits, E, k, (ids, w, rows, row_of), score="sigmoid" if kw.get("score") else "softmax", **ref)
    assert ids.cpu()[0].tolist() == list(range(k))


@pytest.mark.parametrize("T", [3, 64, 200, 5000])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_masked_experts_and_rows_that_leave_nothing(T, score):
    E, k = 40, 6
    logits = logits_apart(T, E, "f32", 9)
    inf = float("inf")
    logits[0] = -inf                                                   # a padding token
    logits[1, 3:] = -inf                                               # three experts left for six choices
    logits[1, 1] = float("nan")
    logits[2, 5] = float("nan")
    if T > 10:
        logits[5] = torch.finfo(torch.float32).min                     # the lowest value is no mask
        logits[6, :30] = torch.finfo(torch.float32).min
        logits[7, 9] = inf
        logits[7, 4] = inf
        logits[T // 2:] = -inf
        logits[T - 1] = logits_apart(1, E, "f32", 10)[0]
    for kw in ({}, {"renorm": False}, {"groups": 4, "groups_kept": 2}, {"groups": 4, "groups_kept": 2, "group_score": 1}):
        got = run_route(logits, E, k, score=int(score == "sigmoid"), **kw)
        ref = {("kept" if n == "groups_kept" else n): v for n, v in kw.items() if n != "group_score"}
        check_route(logits, E, k, got, score=score, top2=bool(kw.get("group_score", 0)), **ref)
    ids, w, rows, row_of = got
    assert (ids.cpu()[0] == -1).all() and (w.cpu()[0] == 0).all() and (row_of.cpu()[0] == -1).all()


def test_route_masks_by_bias_and_infinite_bias():
    T, E, k = 70, 32, 4
    logits = logits_apart(T, E, "bf16", 2)
    bias = torch.zeros(E)
    bias[3], bias[4], bias[5] = -float("inf"), float("nan"), float("inf")
    got = run_route(logits, E, k, bias=bias, score=1)
    check_route(logits, E, k, got, bias=bias, score="sigmoid")
    assert (got[0].cpu()[:, 0] == 5).all() and not bool(((got[0] == 3) | (got[0] == 4)).any())


def test_route_of_no_tokens_and_without_the_order():
    rows = torch.full((17,), 5, dtype=torch.int32, device="cuda")
    d = B.RouteDesc(0, 16, 2)
    B.axe_route(d, None, None, None, rows, torch.zeros(1, dtype=torch.int32, device="cuda"), None)
    assert (rows == 0).all()
    logits = logits_apart(500, 64, "f32", 4)
    with_order, without = run_route(logits, 64, 5), run_route(logits, 64, 5, order=False)
    assert torch.equal(with_order[0], without[0]) and torch.equal(with_order[1], without[1])


@pytest.mark.parametrize("T,E,k", [(16, 128, 8), (17, 128, 8), (63, 128, 8), (64, 128, 8), (65, 128, 8), (66, 128, 8), (48, 256, 8), (49, 256, 8), (64, 256, 8), (32, 512, 20), (33, 512, 20), (2048, 200, 8), (2049, 200, 8), (257, 8, 2), (1024, 1024, 8), (4096, 128, 8), (4097, 60, 4), (33333, 256, 8), (20000, 8, 1), (9000, 1000, 64)])
def test_experts_order_of_many_tokens(T, E, k):
    g = torch.Generator(device="cuda").manual_seed(T)
    logits = torch.randn((T, E), generator=g, device="cuda").to(torch.bfloat16).float()
    logits[T // 3:T // 3 + T // 7] = -float("inf")
    d = B.RouteDesc(T, E, k)
    ids, w = torch.zeros((T, k), dtype=torch.int32, device="cuda"), torch.zeros((T, k), device="cuda")
    rows, row_of = torch.full((E + 1,), 9, dtype=torch.int32, device="cuda"), torch.full((T, k), 9, dtype=torch.int32, device="cuda")
    words = B.axe_route_workspace(d)
    ws = torch.full((max(words, 1),), 0x7FFFFFFF, dtype=torch.int32, device="cuda")
    B.axe_route(d, logits, ids, w, rows, row_of, ws)
    first = [x.clone() for x in (ids, w, rows, row_of)]
    B.axe_route(d, logits, ids, w, rows, row_of, ws)
    assert all(torch.equal(a, b) for a, b in zip(first, (ids, w, rows, row_of)))
    top = logits.sort(dim=1, descending=True, stable=True).indices[:, :k].int()
    there = (logits > -float("inf")).any(1, keepdim=True)
    assert torch.equal(ids, torch.where(there, top, -1))
    flat = torch.where(ids >= 0, ids, E).reshape(-1)
    at = flat.sort(stable=True).indices
    want = torch.empty(T * k, dtype=torch.int32, device="cuda")
    want[at] = torch.arange(T * k, dtype=torch.int32, device="cuda")
    assert torch.equal(row_of.reshape(-1), torch.where(flat < E, want, -1))
    assert torch.equal(rows, torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), torch.bincount(flat.long(), minlength=E + 1)[:E].cumsum(0)]).int())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T,E,k", [(1, 128, 8), (70, 60, 4), (5, 1024, 64), (300, 8, 2), (3, 7, 7), (130, 513, 3)])
def test_route_backward_against_64_bits(T, E, k, renorm, score, dtype):
    logits = logits_apart(T, E, dtype, T + E)
    if T > 60:
        logits[2] = -float("inf")
        logits[3, E // 2:] = -float("inf")
    ids = torch.from_numpy(R.route(f64(logits), k, score)[0]).int()
    g = draw(4, (T, k), "f32")
    m = Mat(logits, E + 5, 3)
    out = Mat(torch.zeros_like(logits), E + 5, 3)
    d = B.RouteDesc(T, E, k, CODE[dtype], score=int(score == "sigmoid"), renorm=renorm, scale=1.5, logits=m.layout, logits_elems=m.buf.numel())
    B.axe_route_backward(d, m.buf, ids.cuda(), g.cuda(), out.buf)
    want = R.route_backward(f64(logits), ids.numpy(), f64(g), score, renorm, 1.5)
    s = R.scores(f64(logits), score)
    chosen = np.where(ids.numpy() >= 0, np.take_along_axis(s, np.maximum(ids.numpy(), 0), 1), 0)
    total = chosen.sum(1, keepdims=True)
    mag = s * 2 * 1.5 * np.abs(f64(g)).max() / (np.where(total > 0, total, 1) if renorm else 1)
    within(f64(out.get()), want, rounding(want, dtype) + 96 * U * mag + 2.0 ** -126, "dlogits")
    assert out.rest_untouched()
    B.axe_route_backward(d, m.buf, ids.cuda(), g.cuda(), m.buf)
    assert torch.equal(m.get().view(torch.uint8), out.get().view(torch.uint8))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_route_backward_against_differences(renorm, score):
    T, E, k, step = 3, 10, 4, 1e-5
    logits = draw(3, (T, E), "f32")
    a = f64(logits)
    ids = R.route(a, k, score)[0]
    g = draw(4, (T, k), "f32")
    out = torch.zeros((T, E), device="cuda")
    d = B.RouteDesc(T, E, k, score=int(score == "sigmoid"), renorm=renorm)
    B.axe_route_backward(d, logits.cuda(), torch.from_numpy(ids).int().cuda(), g.cuda(), out)
    loss = lambda l: (R.route_weights(l, ids, score, renorm, 1.0) * f64(g)).sum()      # noqa: E731
    num = np.zeros_like(a)
    for t in range(T):
        for e in range(E):
            x = np.zeros_like(a)
            x[t, e] = step
            num[t, e] = (loss(a + x) - loss(a - x)) / (2 * step)
    within(f64(out), num, 1e-8 + 96 * U * 8)


# ---- rows ---------------------------------------------------------------------------------------------------------------------------------------

def some_order(T, k, M, seed, holes=True):
    """Every pair a row of its own among M, some of them none."""
    g = torch.Generator().manual_seed(seed)
    row_of = torch.randperm(M, generator=g)[:T * k].reshape(T, k).int()
    if holes and T * k > 2:
        row_of.view(-1)[::5] = -1
        row_of.view(-1)[1] = M + 3                                     # beyond the rows: none
    return row_of


ROWS_SHAPES = [(1, 8, 8, 2048), (5, 1, 9, 1), (64, 8, 512, 2048), (3, 2, 6, 129), (7, 64, 500, 40), (33, 6, 200, 1999), (300, 4, 1200, 768), (2, 3, 7, 12345), (1, 1, 1, 8), (20, 8, 170, 136)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,k,M,H", ROWS_SHAPES)
@pytest.mark.parametrize("pitched", [False, True])
def test_dispatch_copies(T, k, M, H, dtype, pitched):
    x = draw(T + H, (T, H), dtype)
    row_of = some_order(T, k, M, H)
    X = Mat(x, *((H + 3, 5) if pitched else (None, 0)))
    A = Mat(torch.full((M, H), 3.0).to(TORCH[dtype]), *((H + 8, 8) if pitched else (None, 0)))
    d = B.RowsDesc(T, k, M, H, CODE[dtype], CODE[dtype], tokens=X.layout, rows=A.layout, tokens_elems=X.buf.numel(), rows_elems=A.buf.numel())
    B.axe_rows_dispatch(d, X.buf, row_of.cuda(), A.buf)
    assert np.array_equal(f64(A.get()), R.dispatch(f64(x), row_of.numpy(), M, fill=3.0)) and A.rest_untouched()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("T,k,M,H", ROWS_SHAPES)
def test_dispatch_quantises_and_copies_quantised_rows(T, k, M, H, dtype, kind):
    x = draw(T + H, (T, H), dtype, 2.0)
    row_of, nb = some_order(T, k, M, H), -(-H // 128)
    st, sd = (B.AXE_SCALE_E8M0, torch.uint8) if kind == "e8m0" else (B.AXE_SCALE_F32, torch.float32)

    def rows():
        return torch.full((M, H), 0x21, dtype=torch.uint8, device="cuda"), torch.full((M, nb), 3, dtype=sd, device="cuda")

    A, sa = rows()
    B.axe_rows_dispatch(B.RowsDesc(T, k, M, H, CODE[dtype], B.AXE_FP8_E4M3, scale_dtype=st), x.cuda(), row_of.cuda(), A, scales=sa)
    # the same by quantising first: rows in order, then bytes and scales copied
    q, sq = torch.zeros((T, H), dtype=torch.uint8, device="cuda"), torch.zeros((T, nb), dtype=sd, device="cuda")
    B.axe_rows_dispatch(B.RowsDesc(T, 1, T, H, CODE[dtype], B.AXE_FP8_E4M3, scale_dtype=st), x.cuda(), None, q, scales=sq)
    check_quantised(q.view(torch.float8_e4m3fn), sq, kind, f64(x), 4 * U)
    A2, sa2 = rows()
    B.axe_rows_dispatch(B.RowsDesc(T, k, M, H, B.AXE_FP8_E4M3, B.AXE_FP8_E4M3, scale_dtype=st), q, row_of.cuda(), A2, token_scales=sq, scales=sa2)
    assert torch.equal(A, A2) and torch.equal(sa, sa2)
    ro = row_of.numpy()
    want, wants = R.dispatch(q.cpu().numpy().astype(float), ro, M, fill=0x21), R.dispatch(sq.cpu().numpy().astype(float), ro, M, fill=3)
    assert np.array_equal(A.cpu().numpy(), want) and np.array_equal(sa.cpu().numpy().astype(float), wants)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,k,M,H", ROWS_SHAPES)
@pytest.mark.parametrize("pitched", [False, True])
def test_combine_against_64_bits(T, k, M, H, dtype, pitched):
    rows, add = draw(T + H, (M, H), dtype), draw(7, (T, H), dtype)
    row_of, w = some_order(T, k, M, H), draw(8, (T, k), "f32")
    C, O = Mat(rows, *((H + 1, 3) if pitched else (None, 0))), Mat(torch.zeros((T, H)).to(TORCH[dtype]), *((H + 8, 16) if pitched else (None, 0)))
    A = Mat(add, *((H + 8, 16) if pitched else (None, 0)))
    d = B.RowsDesc(T, k, M, H, CODE[dtype], CODE[dtype], tokens=O.layout, rows=C.layout, tokens_elems=O.buf.numel(), rows_elems=C.buf.numel())
    a, r, ro, wv = f64(add), f64(rows), row_of.numpy(), f64(w)
    for use_w, use_add in ((True, False), (False, True), (True, True)):
        B.axe_rows_combine(d, C.buf, row_of.cuda(), w.cuda() if use_w else None, O.buf, add=A.buf if use_add else None)
        ww = wv if use_w else np.ones_like(wv)
        want = R.combine(r, ro, ww, a if use_add else None)
        mag = R.combine(np.abs(r), ro, np.abs(ww), np.abs(a) if use_add else None)
        within(f64(O.get()), want, rounding(want, dtype) + (k + 2) * U * mag)
    B.axe_rows_combine(d, C.buf, row_of.cuda(), w.cuda(), A.buf, add=A.buf)                # in place
    assert torch.equal(A.get(), O.get()) and O.rest_untouched()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,k,M,H", ROWS_SHAPES)
@pytest.mark.parametrize("pitched", [False, True])
def test_combine_backward_against_64_bits(T, k, M, H, dtype, pitched):
    rows, do = draw(T + H, (M, H), dtype), draw(7, (T, H), dtype)
    row_of, w = some_order(T, k, M, H), draw(8, (T, k), "f32")
    C, DO = Mat(rows, *((H + 1, 3) if pitched else (None, 0))), Mat(do, *((H + 8, 16) if pitched else (None, 0)))
    D = Mat(torch.full((M, H), 3.0).to(TORCH[dtype]), *((H + 1, 3) if pitched else (None, 0)))
    d = B.RowsDesc(T, k, M, H, CODE[dtype], CODE[dtype], tokens=DO.layout, rows=C.layout, tokens_elems=DO.buf.numel(), rows_elems=C.buf.numel())
    dw = torch.full((T, k), 7.0, device="cuda")
    B.axe_rows_combine_backward(d, DO.buf, C.buf, row_of.cuda(), w.cuda(), D.buf, dw)
    r, g, ro, wv = f64(rows), f64(do), row_of.numpy(), f64(w)
    want, wantw = R.combine_backward(g, r, ro, wv, fill=3.0)
    within(f64(D.get()), want, rounding(want, dtype) + 2 * U * np.abs(want), "drows")
    _, magw = R.combine_backward(np.abs(g), np.abs(r), ro, wv)
    within(f64(dw), wantw, 64 * U * magw, "dweights")
    assert D.rest_untouched()
    only = torch.full((T, k), 7.0, device="cuda")                      # either alone, the rows in place, no weights
    B.axe_rows_combine_backward(d, DO.buf, C.buf, row_of.cuda(), w.cuda(), None, only)
    assert torch.equal(only, dw)
    B.axe_rows_combine_backward(d, DO.buf, None, row_of.cuda(), None, D.buf, None)
    ones, _ = R.combine_backward(g, r, ro, np.ones_like(wv), fill=3.0)
    assert np.array_equal(f64(D.get()), ones)
    B.axe_rows_combine_backward(d, DO.buf, C.buf, row_of.cuda(), w.cuda(), C.buf, only)
    assert torch.equal(only, dw)


def test_dispatch_and_combine_are_each_others_gradient():
    """<dispatch(x), y> = <x, combine(y)> where the rows are exact: small integers."""
    T, k, H = 50, 4, 72
    M = T * k
    row_of = some_order(T, k, M, 3, holes=False).cuda()
    g = torch.Generator().manual_seed(0)
    x, y = torch.randint(-3, 4, (T, H), generator=g).float().cuda(), torch.randint(-3, 4, (M, H), generator=g).float().cuda()
    d = B.RowsDesc(T, k, M, H, B.AXE_F32, B.AXE_F32)
    A, c = torch.zeros((M, H), device="cuda"), torch.zeros((T, H), device="cuda")
    B.axe_rows_dispatch(d, x, row_of, A)
    B.axe_rows_combine(d, y, row_of, None, c)
    assert (A.double() * y.double()).sum().item() == (x.double() * c.double()).sum().item()


def test_calls_follow_their_stream_and_replay_from_a_graph():
    """All of it captured once and replayed on other inputs, eager work and synchronisation in between."""
    T, E, k, H = 130, 64, 4, 512
    M = T * k
    g = torch.Generator(device="cuda").manual_seed(3)
    x, r, w = torch.randn((T, H), generator=g, device="cuda"), torch.randn((T, H), generator=g, device="cuda"), torch.rand(H, generator=g, device="cuda")
    logits = torch.randn((T, E), generator=g, device="cuda")
    nd, rd = B.RmsNormDesc(T, H, B.AXE_F32, B.AXE_F32), B.RouteDesc(T, E, k)
    wd = B.RowsDesc(T, k, M, H, B.AXE_F32, B.AXE_F32)
    nw, rw = B.axe_rmsnorm_workspace(nd), B.axe_route_workspace(rd)
    ws_n, ws_r = torch.zeros(max(nw, 1), dtype=torch.int32, device="cuda"), torch.zeros(max(rw, 1), dtype=torch.int32, device="cuda")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")   # noqa: E731
    f32 = lambda *s: torch.zeros(s, device="cuda")                      # noqa: E731

    def buffers():
        return dict(y=f32(T, H), s=f32(T, H), ids=i32(T, k), wt=f32(T, k), rows=i32(E + 1), ro=i32(T, k), a=f32(M, H), o=f32(T, H), da=f32(M, H), dwt=f32(T, k),
                    dl=f32(T, E), dx=f32(T, H), dw=f32(H))

    def all_of_it(b):
        B.axe_rmsnorm(nd, x, w, b["y"], residual=r, sum_out=b["s"])
        B.axe_route(rd, logits, b["ids"], b["wt"], b["rows"], b["ro"], ws_r)
        B.axe_rows_dispatch(wd, b["y"], b["ro"], b["a"])
        B.axe_rows_combine(wd, b["a"], b["ro"], b["wt"], b["o"], add=b["s"])
        B.axe_rows_combine_backward(wd, b["o"], b["a"], b["ro"], b["wt"], b["da"], b["dwt"])
        B.axe_route_backward(rd, logits, b["ids"], b["dwt"], b["dl"])
        B.axe_rmsnorm_backward(nd, b["o"], b["s"], w, b["dx"], dsum=b["y"], dweight=b["dw"], workspace=ws_n)

    eager, graphed = buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        all_of_it(graphed)                                             # warm-up on a stream of its own
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        all_of_it(graphed)
    for step in range(4):
        x.copy_(torch.randn((T, H), generator=g, device="cuda"))
        logits.copy_(torch.randn((T, E), generator=g, device="cuda"))
        all_of_it(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in eager:
            assert torch.equal(eager[name], graphed[name]), (step, name)
