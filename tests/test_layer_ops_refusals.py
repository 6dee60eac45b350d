"""What the entry points around the experts' products refuse, without a GPU: bad sizes, types, layouts, buffers and workspaces are error codes before
anything is launched."""
import ctypes as C

import pytest

from paper_2601_19092_amd import binding as B
from paper_2601_19092_amd import workloads as W

P = [0x100000 * (i + 1) for i in range(12)]                            # addresses far from each other; never touched


def norm_rc(T=4, H=64, xt=B.AXE_BF16, yt=B.AXE_BF16, x=P[0], r=P[1], w=P[2], s=P[3], y=P[4], sc=None, **kw):
    d = B.RmsNormDesc(T, H, xt, yt, **kw)
    return B.lib().axe_rmsnorm(d.ref, x, r, w, s, y, sc, None)


def test_norm_refusals():
    assert norm_rc(xt=9) == B.AXE_EINVAL and norm_rc(yt=9) == B.AXE_EINVAL and norm_rc(weight_dtype=B.AXE_FP8_E4M3) == B.AXE_EINVAL
    assert norm_rc(xt=B.AXE_FP8_E4M3) == B.AXE_EINVAL
    assert norm_rc(xt=B.AXE_BF16, yt=B.AXE_F16) == B.AXE_EUNSUPPORTED and norm_rc(xt=B.AXE_F16, yt=B.AXE_F32) == B.AXE_EUNSUPPORTED
    assert norm_rc(eps=-1.0) == B.AXE_EINVAL and norm_rc(eps=float("nan")) == B.AXE_EINVAL
    assert norm_rc(scale_dtype=3) == B.AXE_EINVAL
    assert norm_rc(H=32769, T=1) == B.AXE_EUNSUPPORTED
    for name in ("x", "y"):
        assert norm_rc(**{name: None}) == B.AXE_EINVAL
    assert norm_rc(x=P[0] + 1) == B.AXE_EINVAL and norm_rc(y=P[4] + 1) == B.AXE_EINVAL and norm_rc(w=P[2] + 2) == B.AXE_EINVAL
    assert norm_rc(yt=B.AXE_FP8_E4M3) == B.AXE_EINVAL                  # no scales
    assert norm_rc(sc=P[5]) == B.AXE_EINVAL                            # scales of a y that has none
    # outputs on top of inputs, half way
    assert norm_rc(y=P[0] + 64) == B.AXE_EINVAL and norm_rc(s=P[1] + 64) == B.AXE_EINVAL and norm_rc(y=P[3]) == B.AXE_EINVAL
    assert norm_rc(y=P[2]) == B.AXE_EINVAL
    # in place at another pitch is not in place
    other = B.Layout(W.spec([(4, 72, "m"), (64, 1, "m")]))
    d = B.RmsNormDesc(4, 64, B.AXE_BF16, B.AXE_BF16, y=other)
    assert B.lib().axe_rmsnorm(d.ref, P[0], None, P[2], None, P[0], None, None) == B.AXE_EINVAL
    # sum on x while the residual overlaps it
    assert norm_rc(r=P[0] + 2, s=P[0]) == B.AXE_EINVAL
    # layouts: outside the buffer, columns not side by side, not the shape, sharded over GPUs
    for bad, rc in ((W.spec([(4, 64, "m"), (64, 1, "m")], O={"m": 1}), B.AXE_ERANGE), (W.spec([(4, 1, "m"), (64, 4, "m")]), B.AXE_EUNSUPPORTED),
                    (W.spec([(4, 64, "m"), (32, 1, "m")]), B.AXE_ESHAPE), (W.spec([(4, 64, "m"), (64, 1, "m")], R=[(2, 256, "m")]), B.AXE_EUNSUPPORTED)):
        L = B.Layout(bad)
        for which in ("x", "residual", "sum", "y"):
            d = B.RmsNormDesc(4, 64, B.AXE_BF16, B.AXE_BF16, **{which: L, which + "_elems": 256 if rc != B.AXE_EUNSUPPORTED else 4096})
            assert B.lib().axe_rmsnorm(d.ref, P[0], P[1], P[2], P[3], P[4], None, None) == rc, (bad, which)
    assert B.lib().axe_rmsnorm(None, *P[:6], None) == B.AXE_EINVAL
    assert b"NULL" in B.lib().axe_last_error()
    # no rows: nothing to do, nothing looked at
    assert norm_rc(T=0, x=None, r=None, w=None, s=None, y=None) == B.AXE_OK


def test_norm_negative_and_empty_sizes():
    d = B.RmsNormDesc(4, 64, B.AXE_BF16, B.AXE_BF16)
    for field, v in (("T", -1), ("H", 0), ("H", -5)):
        old = getattr(d.c, field)
        setattr(d.c, field, v)
        assert B.lib().axe_rmsnorm(d.ref, P[0], None, None, None, P[4], None, None) == B.AXE_EINVAL
        assert B.lib().axe_rmsnorm_workspace(d.ref) == B.AXE_EINVAL
        setattr(d.c, field, old)


def back_rc(T=4, H=64, xt=B.AXE_BF16, yt=B.AXE_BF16, dy=P[0], h=P[1], w=P[2], ds=P[3], dx=P[4], dw=P[5], ws=P[6], n=None, **kw):
    d = B.RmsNormDesc(T, H, xt, yt, **kw)
    words = B.lib().axe_rmsnorm_workspace(d.ref)
    return B.lib().axe_rmsnorm_backward(d.ref, dy, h, w, ds, dx, dw, ws, words if n is None else n, None)


def test_norm_backward_refusals():
    assert back_rc(yt=B.AXE_FP8_E4M3) == B.AXE_EUNSUPPORTED
    assert back_rc(xt=B.AXE_F16, yt=B.AXE_BF16) == B.AXE_EUNSUPPORTED
    for name in ("dy", "h", "dx"):
        assert back_rc(**{name: None}) == B.AXE_EINVAL
    assert back_rc(dx=P[1]) == B.AXE_EINVAL                            # dx on the normed rows
    assert back_rc(dx=P[0] + 16) == B.AXE_EINVAL and back_rc(dw=P[0]) == B.AXE_EINVAL and back_rc(dw=P[5] + 2) == B.AXE_EINVAL
    assert back_rc(dx=P[0], ds=P[0]) == B.AXE_EINVAL                   # dy, dsum and dx all one
    if B.lib().axe_rmsnorm_workspace(B.RmsNormDesc(4, 64, B.AXE_BF16, B.AXE_BF16).ref) > 0:
        assert back_rc(n=0) == B.AXE_EINVAL and back_rc(ws=None) == B.AXE_EINVAL and back_rc(ws=P[4]) == B.AXE_EINVAL
    assert back_rc(T=0, dw=None) == B.AXE_OK


def route_rc(T=4, E=32, k=4, lt=B.AXE_F32, l=P[0], ids=P[1], w=P[2], rows=P[3], ro=P[4], ws=P[5], n=None, bias=None, set_=None, **kw):
    d = B.RouteDesc(T, E, k, lt, **kw)
    d.c.d_bias = bias
    for f, v in (set_ or {}).items():
        setattr(d.c, f, v)
    words = B.lib().axe_route_workspace(d.ref)
    return B.lib().axe_route(d.ref, l, ids, w, rows, ro, ws, max(words, 0) if n is None else n, None)


def test_route_refusals():
    for f, v in (("T", -1), ("E", 0), ("k", 0), ("k", 33), ("score", 2), ("group_score", -1), ("groups", 0), ("groups", 5), ("groups_kept", 0), ("groups_kept", 2),
                 ("logit_dtype", B.AXE_FP8_E4M3), ("scale", float("inf"))):
        assert route_rc(set_={f: v}) == B.AXE_EINVAL, (f, v)
    assert route_rc(groups=16, groups_kept=1) == B.AXE_EINVAL          # four choices of two experts
    assert route_rc(E=1025) == B.AXE_EUNSUPPORTED and route_rc(E=128, k=65) == B.AXE_EUNSUPPORTED and route_rc(E=128, groups=128, groups_kept=64) == B.AXE_EUNSUPPORTED
    assert route_rc(T=1 << 30, k=2) == B.AXE_EUNSUPPORTED
    for name in ("l", "ids", "w", "rows", "ro"):
        assert route_rc(**{name: None}) == B.AXE_EINVAL, name
    assert route_rc(bias=0x1001) == B.AXE_EINVAL
    assert route_rc(ids=P[0]) == B.AXE_EINVAL and route_rc(w=P[1]) == B.AXE_EINVAL and route_rc(ro=P[3] + 4) == B.AXE_EINVAL and route_rc(ids=P[1] + 2) == B.AXE_EINVAL
    d = B.RouteDesc(5000, 32, 4)
    if B.lib().axe_route_workspace(d.ref) > 0:
        assert route_rc(T=5000, n=1) == B.AXE_EINVAL and route_rc(T=5000, ws=None) == B.AXE_EINVAL
    bad = B.Layout(W.spec([(4, 32, "m"), (32, 1, "m")], O={"m": 4}))
    assert route_rc(logits=bad, logits_elems=128) == B.AXE_ERANGE
    d = B.RouteDesc(4, 32, 4)
    for args in ((None, P[1], P[2], P[3]), (P[0], None, P[2], P[3]), (P[0], P[1], None, P[3]), (P[0], P[1], P[2], None), (P[0], P[1], P[2], P[0] + 4)):
        assert B.lib().axe_route_backward(d.ref, *args, None) == B.AXE_EINVAL, args
    assert B.lib().axe_route_workspace(None) == B.AXE_EINVAL


def rows_rc(fn, T=4, k=2, M=8, H=64, tt=B.AXE_BF16, rt=B.AXE_BF16, args=None, set_=None, **kw):
    d = B.RowsDesc(T, k, M, H, tt, rt, **kw)
    for f, v in (set_ or {}).items():
        setattr(d.c, f, v)
    return getattr(B.lib(), fn)(d.ref, *args, None)


DISPATCH = (P[0], None, P[1], P[2], None)
COMBINE = (P[0], P[1], P[2], P[3], P[4])
BACK = (P[0], P[1], P[2], P[3], P[4], P[5])


def but(args, i, v):
    return args[:i] + (v,) + args[i + 1:]


@pytest.mark.parametrize("fn,args", [("axe_rows_dispatch", DISPATCH), ("axe_rows_combine", COMBINE), ("axe_rows_combine_backward", BACK)])
def test_rows_refusals(fn, args):
    for f, v in (("T", -1), ("M", -1), ("H", 0), ("k", 0), ("tokens_dtype", 7), ("rows_dtype", 0), ("scale_dtype", 2)):
        assert rows_rc(fn, args=args, set_={f: v}) == B.AXE_EINVAL, (f, v)
    assert rows_rc(fn, args=args, set_={"k": 65}) == B.AXE_EUNSUPPORTED
    assert rows_rc(fn, args=args, tt=B.AXE_BF16, rt=B.AXE_F16) == B.AXE_EUNSUPPORTED
    assert rows_rc(fn, args=args, tt=B.AXE_FP8_E4M3, rt=B.AXE_BF16) == B.AXE_EUNSUPPORTED
    if fn != "axe_rows_dispatch":
        assert rows_rc(fn, args=args, tt=B.AXE_FP8_E4M3, rt=B.AXE_FP8_E4M3) == B.AXE_EUNSUPPORTED
    assert rows_rc(fn, args=args, rows=B.Layout(W.spec([(8, 64, "m"), (64, 1, "m")], O={"m": 1})), rows_elems=512) == B.AXE_ERANGE
    assert rows_rc(fn, args=args, T=0) == B.AXE_OK


def test_rows_buffers():
    for i in (0, 3):
        assert rows_rc("axe_rows_dispatch", args=but(DISPATCH, i, None)) == B.AXE_EINVAL
    assert rows_rc("axe_rows_dispatch", args=but(DISPATCH, 2, None)) == B.AXE_EINVAL       # no order with two choices
    assert rows_rc("axe_rows_dispatch", args=but(DISPATCH, 4, P[5])) == B.AXE_EINVAL       # scales of bf16 rows
    assert rows_rc("axe_rows_dispatch", rt=B.AXE_FP8_E4M3, args=DISPATCH) == B.AXE_EINVAL  # none of e4m3 rows
    assert rows_rc("axe_rows_dispatch", tt=B.AXE_FP8_E4M3, rt=B.AXE_FP8_E4M3, args=but(DISPATCH, 4, P[5])) == B.AXE_EINVAL
    assert rows_rc("axe_rows_dispatch", args=but(DISPATCH, 3, P[0] + 128)) == B.AXE_EINVAL
    for i in (0, 1, 4):
        assert rows_rc("axe_rows_combine", args=but(COMBINE, i, None)) == B.AXE_EINVAL
    assert rows_rc("axe_rows_combine", args=but(COMBINE, 4, P[0])) == B.AXE_EINVAL and rows_rc("axe_rows_combine", args=but(COMBINE, 4, P[3] + 64)) == B.AXE_EINVAL
    for i in (0, 2):
        assert rows_rc("axe_rows_combine_backward", args=but(BACK, i, None)) == B.AXE_EINVAL
    assert rows_rc("axe_rows_combine_backward", args=but(BACK, 1, None)) == B.AXE_EINVAL   # dweights without the rows
    assert rows_rc("axe_rows_combine_backward", args=but(BACK, 4, P[0])) == B.AXE_EINVAL
    assert rows_rc("axe_rows_combine_backward", args=(P[0], P[1], P[2], P[3], None, None)) == B.AXE_OK


def test_descriptors_of_the_binding_match_the_header():
    """Sizes of the structures: every field of the header is there (a missing one would shift what follows)."""
    lay = C.sizeof(B.axe_layout_t)
    assert C.sizeof(B.axe_rmsnorm_desc_t) == 16 + 24 + 4 * lay + 32
    assert C.sizeof(B.axe_route_desc_t) == 8 + 40 + lay + 16
    assert C.sizeof(B.axe_rows_desc_t) == 24 + 24 + 2 * lay + 16
