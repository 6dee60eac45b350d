"""What the binding refuses of the operands of the entry points around the experts' products: elements of another size than the descriptor says (the library would read or write past the end),
views that are not contiguous where there is no layout, tensors that hold too little.  Without a GPU: stand-ins for device tensors, and a library that only counts its calls."""
import pytest
import torch

from paper_2601_19092_amd import binding as B
from paper_2601_19092_amd import workloads as W

T, H, E, K, M = 4, 256, 32, 2, 8


class OnDevice:
    """A CPU tensor that says it is on the GPU."""

    def __init__(self, t):
        self.t = t
        self.is_cuda, self.dtype, self.itemsize, self.shape, self.nbytes = True, t.dtype, t.itemsize, t.shape, t.nbytes
        for n in ("numel", "is_contiguous", "stride", "data_ptr", "element_size", "storage_offset", "untyped_storage", "size"):
            setattr(self, n, getattr(t, n))


class Counting:
    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*args):
            self.calls += 1
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    L = Counting()
    monkeypatch.setattr(B, "_lib", L)
    monkeypatch.setattr(B, "_stream_ptr", lambda s: 0)
    return L


def dev(shape, dtype=torch.bfloat16):
    return OnDevice(torch.zeros(shape, dtype=dtype))


f32, i32 = torch.float32, torch.int32


def calls(fp8=False, e8m0=False):
    """(entry point, descriptor, its operands by name)."""
    yt, scale = (B.AXE_FP8_E4M3, dev((T, 2), torch.uint8 if e8m0 else f32)) if fp8 else (B.AXE_BF16, None)
    nd = B.RmsNormDesc(T, H, B.AXE_BF16, yt, scale_dtype=int(e8m0))
    rd = B.RowsDesc(T, K, M, H, B.AXE_BF16, yt, scale_dtype=int(e8m0))
    y = dev((T, H), torch.uint8) if fp8 else dev((T, H))
    rows = dev((M, H), torch.uint8) if fp8 else dev((M, H))
    out = [(B.axe_rmsnorm, nd, dict(x=dev((T, H)), weight=dev(H, f32), y=y, residual=dev((T, H)), sum_out=dev((T, H)), scales=scale)),
           (B.axe_rows_dispatch, rd, dict(tokens=dev((T, H)), row_of=dev((T, K), i32), rows=rows, scales=dev((M, 2), scale.dtype) if fp8 else None))]
    if fp8:
        copy = B.RowsDesc(T, K, M, H, B.AXE_FP8_E4M3, B.AXE_FP8_E4M3, scale_dtype=int(e8m0))
        out.append((B.axe_rows_dispatch, copy, dict(tokens=dev((T, H), torch.uint8), row_of=dev((T, K), i32), rows=rows, token_scales=scale, scales=dev((M, 2), scale.dtype))))
    else:
        out += [(B.axe_rmsnorm_backward, nd, dict(dy=dev((T, H)), sum=dev((T, H)), weight=dev(H, f32), dx=dev((T, H)), dsum=dev((T, H)), dweight=dev(H, f32), workspace=dev(64, i32))),
                (B.axe_route, B.RouteDesc(T, E, K, B.AXE_BF16), dict(logits=dev((T, E)), ids=dev((T, K), i32), weights=dev((T, K), f32), group_rows=dev(E + 1, i32), row_of=dev((T, K), i32))),
                (B.axe_route_backward, B.RouteDesc(T, E, K, B.AXE_BF16), dict(logits=dev((T, E)), ids=dev((T, K), i32), dweights=dev((T, K), f32), dlogits=dev((T, E)))),
                (B.axe_rows_combine, rd, dict(rows=rows, row_of=dev((T, K), i32), weights=dev((T, K), f32), tokens=dev((T, H)), add=dev((T, H)))),
                (B.axe_rows_combine_backward, rd, dict(dtokens=dev((T, H)), rows=rows, row_of=dev((T, K), i32), weights=dev((T, K), f32), drows=dev((M, H)), dweights=dev((T, K), f32)))]
    return out


ALL = [(a, i) for a, n in ((dict(), 7), (dict(fp8=True), 3), (dict(fp8=True, e8m0=True), 3)) for i in range(n)]


@pytest.mark.parametrize("kind,which", ALL)
def test_operands_as_described_are_taken(library, kind, which):
    f, d, ops = calls(**kind)[which]
    f(d, **ops)
    assert library.calls == 1


@pytest.mark.parametrize("kind,which", ALL)
def test_elements_of_another_size_are_refused(library, kind, which):
    f, d, ops = calls(**kind)[which]
    for name, t in ops.items():
        if t is None:
            continue
        for other in (torch.uint8, torch.bfloat16, torch.float32, torch.float64):
            if other.itemsize != t.itemsize:
                # (as many elements, and many more: it is their size that is wrong)
                for n in (t.t.numel(), 16 * t.t.numel()):
                    with pytest.raises(AssertionError):
                        f(d, **{**ops, name: dev(n, other)})
    assert library.calls == 0


@pytest.mark.parametrize("kind,which", ALL)
def test_views_and_short_tensors_are_refused_where_there_is_no_layout(library, kind, which):
    f, d, ops = calls(**kind)[which]
    for name, t in ops.items():
        if t is None or name == "workspace":
            continue
        shape = tuple(t.shape)
        wide = torch.zeros(shape[:-1] + (2 * shape[-1],), dtype=t.dtype)
        for bad in (wide[..., ::2], torch.zeros(t.t.numel() - 1, dtype=t.dtype), torch.zeros(1, dtype=t.dtype).expand(shape)):
            with pytest.raises(AssertionError):
                f(d, **{**ops, name: OnDevice(bad)})
        if len(shape) == 2:
            with pytest.raises(AssertionError):
                f(d, **{**ops, name: OnDevice(wide[:, :shape[1]])})
    assert library.calls == 0


def test_a_layout_says_what_a_view_has_to_hold(library):
    pitch = H + 24
    L = B.Layout(W.spec([(T, pitch, "m"), (H, 1, "m")]), ["m"])
    d = B.RmsNormDesc(T, H, B.AXE_BF16, B.AXE_BF16, x=L)
    buf = torch.zeros((T, pitch), dtype=torch.bfloat16)
    w, y = dev(H, f32), dev((T, H))
    for x in (buf, buf.view(-1), buf[:, :H], buf.view(-1)[:(T - 1) * pitch + H]):
        B.axe_rmsnorm(d, OnDevice(x), w, y)
    assert library.calls == 4
    for x in (buf[:T - 1], buf.view(-1)[1:(T - 1) * pitch + H], buf[:T - 1, :H], buf[:1].expand(T, pitch), torch.zeros(1, dtype=torch.bfloat16).expand(T, pitch)):
        with pytest.raises(AssertionError):
            B.axe_rmsnorm(d, OnDevice(x), w, y)
    assert library.calls == 4
