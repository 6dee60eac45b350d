"""What stands around the experts' products at the sizes from which kernels of their own are taken: operands past the caches (96, 128 and 256 MiB a call), few lanes a token in the gradient of
the logits (more than 8192 tokens).  Against the same in 64 bits on the device, in pieces.

Tolerances.  U = 2^-24; a result in 16 bits is off by half a step, 2^-8 (bf16) or 2^-11 (fp16) of it at most and 2^-25 where fp16 is subnormal, and by what fp32 does on the way, as derived for
the smaller sizes: 64 U of the magnitudes that enter for a row's sums, one more for every addition in a chain."""
import pytest
import torch

from paper_2601_19092_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
MIB = 1 << 20
CODE = {"bf16": B.AXE_BF16, "f16": B.AXE_F16, "f32": B.AXE_F32}
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF_ULP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": U}
SMALL = {"bf16": 0.0, "f16": 2.0 ** -25, "f32": 0.0}
PIECE = 1 << 24                                                        # elements that are compared at once


def normal(g, shape, dtype, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g).to(TORCH[dtype])


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def all_within(got, want, tol):
    return bool(((got.double() - want).abs() <= tol).all())


def pieces(T, per_row):
    n = max(1, PIECE // per_row)
    return [slice(t, min(T, t + n)) for t in range(0, T, n)]


# ---- the norm's gradient: from 128 MiB ----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("T,H,dtype,ytype,with_dsum", [
    (60000, 509, "bf16", "bf16", True), (50000, 1000, "f16", "f16", False), (9000, 2047, "f32", "bf16", True), (5000, 4099, "f32", "f32", False), (4100, 8191, "bf16", "bf16", True),
    (2601, 4095, "f32", "f16", True), (3000, 12001, "f16", "f16", False), (1500, 20001, "bf16", "bf16", True)])
def test_norm_backward_past_the_caches(T, H, dtype, ytype, with_dsum):
    eb, yb = TORCH[dtype].itemsize, TORCH[ytype].itemsize
    assert T * H * (yb + eb * (3 if with_dsum else 2)) >= 128 * MIB
    g = gen(T + H)
    h, dy, w = normal(g, (T, H), dtype, 1.3), normal(g, (T, H), ytype), 1.0 + 0.2 * torch.randn(H, generator=g, device="cuda")
    ds = normal(g, (T, H), dtype) if with_dsum else None
    d = B.RmsNormDesc(T, H, CODE[dtype], CODE[ytype], eps=1e-6)
    words = B.axe_rmsnorm_workspace(d)
    dx, dw, ws = torch.zeros_like(h), torch.full((H,), 9.0, device="cuda"), torch.full((words,), -1, dtype=torch.int32, device="cuda")
    B.axe_rmsnorm_backward(d, dy, h, w, dx, dsum=ds, dweight=dw, workspace=ws)
    want_dw, mag_dw = torch.zeros(H, dtype=torch.float64, device="cuda"), torch.zeros(H, dtype=torch.float64, device="cuda")
    for p in pieces(T, H):
        a, y = h[p].double(), dy[p].double()
        rho = (a.square().mean(1, keepdim=True) + 1e-6).rsqrt()
        u = y * w.double()
        want = rho * u - rho ** 3 * a * (u * a).mean(1, keepdim=True)
        mag = rho * u.abs() + rho ** 3 * a.abs() * (u * a).abs().mean(1, keepdim=True)
        if with_dsum:
            want, mag = want + ds[p].double(), mag + ds[p].double().abs()
        assert all_within(dx[p], want, want.abs() * HALF_ULP[dtype] + SMALL[dtype] + 64 * U * mag)
        part = y * a * rho
        want_dw += part.sum(0)
        mag_dw += part.abs().sum(0)
    # dw: a thread's chain over its rows (T / 512 at most), the rows of a workgroup (up to 8), 512 / 128 in a chain, trees of 8 and 16
    assert all_within(dw, want_dw, (64 + T // 512 + 48) * U * mag_dw)
    again, dw2 = torch.zeros_like(dx), torch.zeros_like(dw)
    B.axe_rmsnorm_backward(d, dy, h, w, again, dsum=ds, dweight=dw2, workspace=ws)
    assert torch.equal(again, dx) and torch.equal(dw2, dw)
    if with_dsum:                                                      # in place
        B.axe_rmsnorm_backward(d, dy, h, w, ds, dsum=ds, dweight=dw2, workspace=ws)
        assert torch.equal(ds, dx)


# ---- rows back to the tokens, and its gradient ----------------------------------------------------------------------------------------------------------

def order(T, k, M, g, holes):
    row_of = torch.randperm(M, generator=g, device="cuda")[:T * k].int().reshape(T, k)
    if holes:
        row_of.view(-1)[::5] = -1
        row_of.view(-1)[1] = M + 3
    return row_of


def named(row_of, M):
    """(rows to read: none as row 0, whether there is one)."""
    on = (row_of >= 0) & (row_of < M)
    return torch.where(on, row_of, 0).long(), on


@pytest.mark.parametrize("T,k,H,dtype,use_w,use_add,holes", [
    (4001, 8, 2049, "bf16", True, True, True), (13000, 3, 1024, "f16", True, False, True), (60000, 1, 513, "f32", True, True, False), (22000, 2, 1000, "bf16", False, True, True),
    (1300, 10, 2049, "f32", True, False, True), (8200, 4, 1999, "f16", True, True, False), (200001, 8, 40, "bf16", True, False, True), (1000, 64, 1024, "bf16", True, True, True)])
def test_combine_past_the_caches(T, k, H, dtype, use_w, use_add, holes):
    M = T * k + 3
    assert T * H * TORCH[dtype].itemsize * (k + 1 + use_add) >= 96 * MIB
    g = gen(T + H)
    rows, w, row_of = normal(g, (M, H), dtype), torch.randn((T, k), generator=g, device="cuda"), order(T, k, M, g, holes)
    if holes:
        rows[0] = float("nan")                                         # (read in place of a row that is none, if it is not named itself)
        row_of = torch.where(row_of == 0, -1, row_of)
    add = normal(g, (T, H), dtype) if use_add else None
    out = torch.zeros((T, H), dtype=TORCH[dtype], device="cuda")
    d = B.RowsDesc(T, k, M, H, CODE[dtype], CODE[dtype])
    B.axe_rows_combine(d, rows, row_of, w if use_w else None, out, add=add)
    at, on = named(row_of, M)
    for p in pieces(T, H):
        want = add[p].double() if use_add else torch.zeros((out[p].shape[0], H), dtype=torch.float64, device="cuda")
        mag = want.abs()
        for j in range(k):
            c = torch.where(on[p][:, j:j + 1], rows[at[p][:, j]].double(), 0.0)
            if use_w:
                c = c * w[p][:, j:j + 1].double()
            want, mag = want + c, mag + c.abs()
        assert all_within(out[p], want, want.abs() * HALF_ULP[dtype] + SMALL[dtype] + (k + 2) * U * mag)
    if use_add:                                                        # in place
        B.axe_rows_combine(d, rows, row_of, w if use_w else None, add, add=add)
        assert torch.equal(add, out)


# (T, k, H): 96 MiB and more but less than 256 with drows and dweights (stores past the caches), 256 and more (loads, too); one, two and four runs of a lane
BACK_SIZES = [(1600, 8, 2049, "bf16"), (3000, 8, 1024, "f16"), (6500, 8, 513, "bf16"), (2600, 10, 500, "f32"), (4200, 8, 2049, "f16"), (4100, 8, 1023, "f32"), (40000, 8, 509, "bf16"), (900, 64, 1100, "f32")]


@pytest.mark.parametrize("T,k,H,dtype", BACK_SIZES)
@pytest.mark.parametrize("holes", [False, True])
def test_combine_backward_past_the_caches(T, k, H, dtype, holes):
    M = T * k + 3
    assert T * H * TORCH[dtype].itemsize * (2 * k + 1) >= 96 * MIB
    g = gen(T + H)
    rows, dout, w, row_of = normal(g, (M, H), dtype), normal(g, (T, H), dtype), torch.randn((T, k), generator=g, device="cuda"), order(T, k, M, g, holes)
    d = B.RowsDesc(T, k, M, H, CODE[dtype], CODE[dtype])
    drows, dw = torch.full((M, H), 3.0, dtype=TORCH[dtype], device="cuda"), torch.full((T, k), 7.0, device="cuda")
    B.axe_rows_combine_backward(d, dout, rows, row_of, w, drows, dw)
    at, on = named(row_of, M)
    touched = torch.zeros(M, dtype=torch.bool, device="cuda")
    touched[at[on]] = True
    assert bool((drows[~touched] == 3.0).all())
    for p in pieces(T, H):
        do = dout[p]
        for j in range(k):
            there, a = on[p][:, j], at[p][:, j]
            # one product in fp32, rounded once: the same bits
            assert torch.equal(drows[a[there]], (do.float() * w[p][:, j:j + 1]).to(TORCH[dtype])[there])
            prod = rows[a].double() * do.double()
            want, mag = prod.sum(1), prod.abs().sum(1)
            assert all_within(dw[p][:, j], torch.where(there, want, 0.0), torch.where(there, 64 * U * mag, 0.0))
    only = torch.full((T, k), 7.0, device="cuda")
    B.axe_rows_combine_backward(d, dout, rows, row_of, w, None, only)
    assert torch.equal(only, dw)
    ones = torch.full((M, H), 3.0, dtype=TORCH[dtype], device="cuda")  # no weights, no dot product
    B.axe_rows_combine_backward(d, dout, None, row_of, None, ones, None)
    for j in range(k):
        there, a = on[:, j], at[:, j]
        assert torch.equal(ones[a[there]], dout[there])
    assert bool((ones[~touched] == 3.0).all())
    kept = rows[~touched].clone()                                      # in place
    B.axe_rows_combine_backward(d, dout, rows, row_of, w, rows, only)
    assert torch.equal(only, dw) and torch.equal(rows[touched], drows[touched]) and torch.equal(rows[~touched], kept)


# ---- the gradient of the logits: 16 and 32 lanes a token above 8192 tokens ------------------------------------------------------------------------------

def scores64(logits, score):
    x = logits.double()
    return torch.sigmoid(x) if score else torch.nan_to_num(torch.softmax(x, 1), nan=0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("E,k", [(60, 4), (128, 8), (128, 20), (200, 8), (256, 32), (200, 40), (512, 3), (9, 9)])
@pytest.mark.parametrize("T", [8193, 8200])
def test_route_backward_of_many_tokens(T, E, k, dtype):
    g = gen(E + k)
    logits = normal(g, (T, E), dtype)
    logits[5::97] = -float("inf")                                      # rows that leave nothing, and rows with a part masked
    logits[7::89, E // 2:] = -float("inf")
    gw = torch.randn((T, k), generator=g, device="cuda")
    masked = torch.isneginf(logits.double())
    top = logits.double().sort(dim=1, descending=True, stable=True)
    ids = torch.where(top.values[:, :k] > -float("inf"), top.indices[:, :k], -1)
    ids[3::101, 0] = E + 1                                             # no choice either
    on = (ids >= 0) & (ids < E)
    at = torch.where(on, ids, 0)
    for score in (0, 1):
        s = torch.where(masked, 0.0, scores64(logits, score))
        c = torch.where(on, s.gather(1, at), 0.0)
        for renorm in (True, False):
            gv = torch.where(on, 1.5 * gw.double(), 0.0)
            total = c.sum(1, keepdim=True)
            total = torch.where(total > 0, total, 1.0)
            if renorm:
                gv = torch.where(on, (gv - (gv * c).sum(1, keepdim=True) / total) / total, 0.0)
            ds = torch.zeros_like(s).scatter_add_(1, at, gv)
            want = s * (1 - s) * ds if score else s * (ds - (s * ds).sum(1, keepdim=True))
            out = torch.full((T, E), 7.0, dtype=TORCH[dtype], device="cuda")
            d = B.RouteDesc(T, E, k, CODE[dtype], score=score, renorm=renorm, scale=1.5)
            B.axe_route_backward(d, logits, ids.int(), gw, out)
            mag = s * 2 * 1.5 * gw.abs().amax().double() / (total if renorm else 1.0)
            assert all_within(out, want, want.abs() * HALF_ULP[dtype] + SMALL[dtype] + 96 * U * mag + 2.0 ** -126), (score, renorm)
            inplace = logits.clone()
            B.axe_route_backward(d, inplace, ids.int(), gw, inplace)
            assert torch.equal(inplace, out)
