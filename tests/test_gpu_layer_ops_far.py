"""What stands around the experts' products at the far ends: rows more than 2^32 bytes apart, calls of more rows than one launch holds, groups of experts of every kind of size."""
import numpy as np
import pytest
import torch

from oracle import layer_ref as R
from paper_2601_19092_amd import binding as B
from paper_2601_19092_amd import workloads as W

pytestmark = pytest.mark.gpu

FAR = (1 << 30) + 24                                                   # elements between rows: 2 GiB and more in 16 bits


def far_rows(values, offset=0):
    """A matrix at that pitch (the rest of the buffer is not touched, here or by the calls): (layout, buffer, view)."""
    rows, cols = values.shape
    n = (rows - 1) * FAR + cols + offset
    buf = torch.empty(n, dtype=values.dtype, device="cuda")
    view = torch.as_strided(buf, (rows, cols), (FAR, 1), offset)
    view.copy_(values)
    return B.Layout(W.spec([(rows, FAR, "m"), (cols, 1, "m")], O={"m": offset}), ["m"]), buf, view


def test_rows_further_apart_than_32_bits_reach():
    T, k, M, H = 2, 2, 4, 136
    g = torch.Generator().manual_seed(1)
    x = torch.randn((T, H), generator=g).bfloat16()
    row_of = torch.tensor([[3, 0], [2, 1]], dtype=torch.int32, device="cuda")
    w = torch.tensor([[0.5, 2.0], [1.0, -1.0]], device="cuda")
    La, A, Av = far_rows(torch.zeros((M, H)).bfloat16(), 8)
    d = B.RowsDesc(T, k, M, H, B.AXE_BF16, B.AXE_BF16, rows=La, rows_elems=A.numel())
    B.axe_rows_dispatch(d, x.cuda(), row_of, A)
    assert torch.equal(Av.cpu(), x[[0, 1, 1, 0]])
    out = torch.zeros((T, H), dtype=torch.bfloat16, device="cuda")
    B.axe_rows_combine(d, A, row_of, None, out)                        # twice each row: exact
    assert torch.equal(out.cpu(), (2 * x.float()).bfloat16())
    dw = torch.zeros((T, k), device="cuda")
    B.axe_rows_combine_backward(d, x.cuda(), A, row_of, w, A, dw)
    want = [x[0].float() * 2.0, x[1].float() * -1.0, x[1].float(), x[0].float() * 0.5]
    assert torch.equal(Av.cpu(), torch.stack(want).bfloat16())
    sq = x.double().square().sum(1)
    assert torch.allclose(dw.cpu().double(), torch.stack([sq, sq], 1), rtol=64 * 2.0 ** -24)
    q = torch.zeros((T, H), dtype=torch.uint8, device="cuda")
    sc = torch.zeros((T, 2), device="cuda")
    Lt, X, _ = far_rows(x)
    B.axe_rows_dispatch(B.RowsDesc(T, 1, T, H, B.AXE_BF16, B.AXE_FP8_E4M3, tokens=Lt, tokens_elems=X.numel()), X, None, q, scales=sc)
    q2, sc2 = torch.zeros_like(q), torch.zeros_like(sc)
    B.axe_rows_dispatch(B.RowsDesc(T, 1, T, H, B.AXE_BF16, B.AXE_FP8_E4M3), x.cuda(), None, q2, scales=sc2)
    assert torch.equal(q, q2) and torch.equal(sc, sc2)


def test_norm_and_routing_of_rows_further_apart_than_32_bits_reach():
    T, H, E, k = 3, 520, 24, 3
    g = torch.Generator().manual_seed(2)
    x, w = torch.randn((T, H), generator=g).bfloat16(), torch.randn(H, generator=g).cuda()
    y, dx, dw, dw2 = (torch.zeros(s, dtype=t, device="cuda") for s, t in (((T, H), torch.bfloat16),) * 2 + ((H, torch.float32),) * 2)
    near = B.RmsNormDesc(T, H, B.AXE_BF16, B.AXE_BF16)
    B.axe_rmsnorm(near, x.cuda(), w, y)
    ws = torch.zeros(max(1, B.axe_rmsnorm_workspace(near)), dtype=torch.int32, device="cuda")
    B.axe_rmsnorm_backward(near, y, x.cuda(), w, dx, dweight=dw, workspace=ws)
    Lx, X, _ = far_rows(x)
    Ly, Y, Yv = far_rows(torch.zeros((T, H)).bfloat16(), 3)
    far = B.RmsNormDesc(T, H, B.AXE_BF16, B.AXE_BF16, x=Lx, y=Ly, sum=Lx, x_elems=X.numel(), y_elems=Y.numel(), sum_elems=X.numel())
    B.axe_rmsnorm(far, X, w, Y)
    assert torch.equal(Yv, y)
    back = B.RmsNormDesc(T, H, B.AXE_BF16, B.AXE_BF16, y=Ly, sum=Lx, y_elems=Y.numel(), sum_elems=X.numel())
    dx2 = torch.zeros_like(dx)
    B.axe_rmsnorm_backward(back, Y, X, w, dx2, dweight=dw2, workspace=ws)
    assert torch.equal(dx2, dx) and torch.equal(dw2, dw)
    del X, Y, Yv
    logits = torch.randn((T, E), generator=g).half()
    Ll, L, Lv = far_rows(logits)
    d = B.RouteDesc(T, E, k, B.AXE_F16, logits=Ll, logits_elems=L.numel())
    ids, wt = torch.zeros((T, k), dtype=torch.int32, device="cuda"), torch.zeros((T, k), device="cuda")
    B.axe_route(d, L, ids, wt)
    assert np.array_equal(ids.cpu().numpy(), R.route(logits.double().numpy(), k)[0])
    want = torch.zeros((T, E), dtype=torch.float16, device="cuda")
    B.axe_route_backward(B.RouteDesc(T, E, k, B.AXE_F16), logits.cuda(), ids, wt, want)
    B.axe_route_backward(d, L, ids, wt, L)
    assert torch.equal(Lv, want)


def test_more_rows_than_one_launch_holds():
    # the norm: launches of 2^21 rows; every row the same few numbers times its own power of two
    T, H = (1 << 21) + 3, 8
    p = torch.exp2((torch.arange(T, device="cuda") % 7).float())[:, None]
    x = (torch.arange(1, H + 1, device="cuda").float()[None] * p).bfloat16()
    y = torch.zeros_like(x)
    B.axe_rmsnorm(B.RmsNormDesc(T, H, B.AXE_BF16, B.AXE_BF16, eps=0.0), x, None, y)
    assert torch.equal(y, y[:1].expand(T, H))                          # powers of two go out exactly
    assert torch.allclose(y[0].float(), torch.arange(1, H + 1, device="cuda").float() / 25.5 ** 0.5, rtol=2 ** -8)
    del x, y, p
    # the rows: launches of 2^25 waves
    T, k, H = (1 << 19) + 3, 64, 8
    M = T * k
    row_of = (M - 1 - torch.arange(M, dtype=torch.int32, device="cuda")).reshape(T, k)
    rows = (torch.arange(M, device="cuda") % 5).to(torch.float16)[:, None].expand(M, H).contiguous()
    do = (torch.arange(T, device="cuda") % 3).to(torch.float16)[:, None].expand(T, H).contiguous()
    d, dw = torch.zeros_like(rows), torch.zeros((T, k), device="cuda")
    B.axe_rows_combine_backward(B.RowsDesc(T, k, M, H, B.AXE_F16, B.AXE_F16), do, rows, row_of, None, d, dw)
    assert torch.equal(d, do.repeat_interleave(k, 0).flip(0))
    assert torch.equal(dw, (H * do[:, :1] * rows[:, 0].flip(0).reshape(T, k)).float())
    del row_of, rows, do, d, dw
    T = (1 << 25) + 5
    x = (torch.arange(T, device="cuda") % 3).to(torch.float16)[:, None].expand(T, H).contiguous()
    q, sc = torch.zeros((T, H), dtype=torch.uint8, device="cuda"), torch.zeros((T, 1), dtype=torch.uint8, device="cuda")
    B.axe_rows_dispatch(B.RowsDesc(T, 1, T, H, B.AXE_F16, B.AXE_FP8_E4M3, scale_dtype=B.AXE_SCALE_E8M0), x, None, q, scales=sc)
    code = torch.tensor([127, 119, 120], dtype=torch.uint8, device="cuda")          # of 0, 1 / 448 and 2 / 448: 2^0, 2^-8, 2^-7
    which = torch.arange(T, device="cuda") % 3
    assert torch.equal(sc[:, 0], code[which])
    byte = torch.tensor([0.0, 256.0, 256.0], device="cuda").to(torch.float8_e4m3fn).view(torch.uint8)
    assert torch.equal(q, byte[which][:, None].expand(T, H))


@pytest.mark.parametrize("E,groups,kept,k", [(6, 2, 1, 2), (7, 7, 3, 3), (8, 2, 1, 4), (40, 5, 2, 3), (64, 32, 4, 8), (64, 2, 1, 20), (128, 64, 10, 12), (128, 2, 1, 8), (256, 2, 1, 40), (256, 32, 3, 24), (512, 4, 1, 8),
                                             (512, 64, 5, 33), (1024, 2, 1, 8), (1000, 8, 3, 16), (1024, 64, 64, 8)])
@pytest.mark.parametrize("T", [1, 20, 70])
def test_groups_of_every_kind_of_size(E, groups, kept, k, T):
    """Groups that are part of a lane, whole lanes, half of a token's lanes; judged in registers or through LDS; by one or two choices; scores or logits."""
    g = torch.Generator().manual_seed(E + T)
    order = torch.stack([torch.randperm(E, generator=g) for _ in range(T)])
    logits = (order.float() - E / 2) * (6.0 / max(E, 6))
    bias = 0.2 * torch.randn(E, generator=g)
    for score, b, top2 in ((0, None, 0), (0, None, 1), (1, None, 1), (1, bias, 0), (0, bias, 1)):
        d = B.RouteDesc(T, E, k, score=score, groups=groups, groups_kept=kept, group_score=top2, bias=None if b is None else b.cuda())
        ids, w = torch.zeros((T, k), dtype=torch.int32, device="cuda"), torch.zeros((T, k), device="cuda")
        B.axe_route(d, logits.cuda(), ids, w)
        want, ww = R.route(logits.double().numpy(), k, "sigmoid" if score else "softmax", None if b is None else b.double().numpy(), groups, kept, bool(top2))
        assert np.array_equal(ids.cpu().numpy(), want), (score, top2)
        assert (np.abs(w.cpu().double().numpy() - ww) <= 96 * 2.0 ** -24 * ww).all()
