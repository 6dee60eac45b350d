"""Appending keys and values to a paged cache on the GPU against the same in 64 bits.

Tolerances.  U = 2^-24, H = half a step of the 16-bit type relative to the value (2^-8 bf16, 2^-11 fp16).  A turned element is a cos - b sin in fp32, three roundings: 3 U (|a| + |b|); then its own rounding,
H of the value (fp16: no less than 2^-25).  What is not turned is copied: the same bits.  e4m3: the scale max / 448 is off by that of its largest element and one rounding; a code by half a step
of e4m3, 2^-4 of the value or half of the smallest step, 2^-10, and by what the element and the scale are off by, in units of the scale."""
import numpy as np
import pytest
import torch

from oracle import cache_ref as R
from paper_2601_19092_amd import binding as B
from paper_2601_19092_amd import workloads as W

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
CODE = {"bf16": B.AXE_BF16, "f16": B.AXE_F16, "fp8": B.AXE_FP8_E4M3}
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn}
HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def f64(t):
    return t.detach().cpu().to(torch.float32).double().numpy()


def angles(rows, rotary):
    a = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(0, rotary, 2) / max(rotary, 1))
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32))


class Append:
    """One call: rows of one product (queries, keys and values side by side, pitched), or separate tensors."""

    def __init__(self, lengths, new, Hq, Hkv, D, page, dtype="bf16", cache=None, rotary=None, style="halves", seed=0, shared=True, spare=2, extra_rows=0, std=1.0):
        g = torch.Generator().manual_seed(seed)
        cache = cache or dtype
        rotary = D if rotary is None else rotary
        S, need = len(lengths), [max(0, -(-n // page)) for n in lengths]
        self.__dict__.update(lengths=lengths, Hq=Hq, Hkv=Hkv, D=D, page=page, dtype=dtype, cache=cache, style=style, rotary=rotary, pages=sum(need) + spare, most=max(need + [1]))
        self.table = torch.full((S, self.most), -1, dtype=torch.int32)
        perm, at = torch.randperm(self.pages, generator=g).int(), 0
        for s, n in enumerate(need):
            self.table[s, :n] = perm[at:at + n]
            at += n
        self.seq_rows = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32)
        T = self.T = int(self.seq_rows[-1]) + extra_rows
        self.rotation = angles(self.most * page, rotary)
        pitch = (Hq + 2 * Hkv) * D + 24
        self.buf = (torch.randn(T * pitch + 40, generator=g) * std).to(TORCH[dtype])
        view = lambda o, h: torch.as_strided(self.buf, (T, h, D), (pitch, D, 1), o * D + 8)  # noqa: E731
        self.q, self.k, self.v = view(0, Hq), view(Hq, Hkv), view(Hq + Hkv, Hkv)
        of = lambda o, h: B.Layout(W.spec([(T, pitch, "m"), (h, D, "m"), (D, 1, "m")], O={"m": o * D + 8}), ["m"])  # noqa: E731
        kw = dict(q=of(0, Hq), k=of(Hq, Hkv), v=of(Hq + Hkv, Hkv))
        self.desc = B.CacheDesc(T, S, Hq, Hkv, D, self.pages, page, self.most, CODE[dtype], CODE[cache], rotary_dim=rotary,
                                rotary_style=B.AXE_ROTATE_PAIRS if style == "pairs" else B.AXE_ROTATE_HALVES, **(kw if shared else {}))
        self.shared = shared

    def run(self, with_q=True, in_place=False, stream=None):
        dev = [self.buf.cuda()] * 3 if self.shared else [x.contiguous().cuda() for x in (self.q, self.k, self.v)]
        shape = (self.pages, self.page, self.Hkv, self.D)
        kc, vc = (torch.full(shape, 0x55, dtype=torch.uint8, device="cuda") if self.cache == "fp8" else torch.full(shape, 3.0, dtype=TORCH[self.cache], device="cuda") for _ in range(2))
        sc = [torch.full(shape[:3], 5.0, device="cuda") for _ in range(2)] if self.cache == "fp8" else [None, None]
        out = torch.full((self.T, self.Hq, self.D), 7.0, dtype=TORCH[self.dtype], device="cuda")
        held = [c.view(torch.float8_e4m3fn) if self.cache == "fp8" else c for c in (kc, vc)]
        B.axe_cache_append(self.desc, dev[1], dev[2], held[0], held[1], self.seq_rows.cuda(), torch.tensor(self.lengths, dtype=torch.int32).cuda(), self.table.cuda(),
                           rotation=self.rotation.cuda() if self.rotary else None, q=dev[0] if with_q else None, q_out=out if with_q else None, k_scales=sc[0], v_scales=sc[1], stream=stream)
        torch.cuda.synchronize()
        return out, kc, vc, sc

    def check(self, got, with_q=True):
        out, kc, vc, sc = got
        q, k, v = f64(self.q), f64(self.k), f64(self.v)
        wq, wk, wv = R.append(q, k, v, self.rotation.double().numpy(), self.seq_rows.numpy(), self.lengths, self.table.numpy(), self.page, self.pages, self.style)
        out = f64(out)
        for t in range(self.T):
            if not with_q or t not in wq:
                assert (out[t] == 7.0).all(), t
                continue
            self.near(out[t], wq[t], 3 * U * size(q[t], self.rotary, self.style), ("q", t))
        for cache, scales, want, of in ((kc, sc[0], wk, k), (vc, sc[1], wv, v)):
            c = f64(cache.view(torch.float8_e4m3fn) if self.cache == "fp8" else cache)
            raw = cache.cpu()
            rows = {at: t for t, s, p in R.tokens(self.seq_rows.numpy(), self.lengths) for at in [R.place(self.table.numpy(), self.page, self.pages, s, p)] if at is not None}
            for pg in range(self.pages):
                for sl in range(self.page):
                    if (pg, sl) not in want:
                        assert (raw[pg, sl] == (0x55 if self.cache == "fp8" else 3.0)).all(), "places that no token has are left as they are"
                        assert self.cache != "fp8" or (scales[pg, sl] == 5.0).all()
                        continue
                    err = 3 * U * (size(of[rows[pg, sl]], self.rotary, self.style) if of is k else 0.0)
                    y = want[pg, sl]
                    if self.cache != "fp8":
                        self.near(c[pg, sl], y, err, (pg, sl))
                        continue
                    s = scales[pg, sl].cpu().double().numpy()
                    most = np.abs(y).max(1)
                    s64 = np.where(most > 0, np.maximum(most / 448.0, 2.0 ** -126), 1.0)
                    assert (np.abs(s - s64) <= s64 * 3 * U + np.max(err) / 448.0).all()
                    x = np.clip(y / s[:, None], -448, 448)
                    tol = np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** -10) + err / s[:, None] + np.abs(x) * 2 * U
                    assert (np.abs(c[pg, sl] - x) <= tol).all(), (pg, sl)
        return self

    def near(self, got, want, err, what):
        tol = np.abs(want) * HALF[self.dtype] + err * (1 + HALF[self.dtype]) + (2.0 ** -25 if self.dtype == "f16" else 0)
        assert (np.abs(got - want) <= tol).all(), (what, got[np.abs(got - want) > tol][:4], want[np.abs(got - want) > tol][:4])


def size(x, rotary, style):
    """|a| + |b| of every element's pair; 0 where nothing is turned."""
    y, h = np.zeros_like(x), rotary // 2
    a, b = (np.arange(h), np.arange(h) + h) if style == "halves" else (2 * np.arange(h), 2 * np.arange(h) + 1)
    y[:, a] = y[:, b] = np.abs(x[:, a]) + np.abs(x[:, b])
    return y


@pytest.mark.parametrize("dtype, cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "fp8"), ("f16", "fp8")])
@pytest.mark.parametrize("style", ["halves", "pairs"])
@pytest.mark.parametrize("D, rotary", [(128, 128), (128, 64), (64, 40), (80, 80), (80, 10), (8, 8), (8, 2), (256, 256), (256, 254), (136, 0), (144, 48)])
def test_types_columns_rotations(dtype, cache, style, D, rotary):
    if cache == "fp8" and D % 16:
        with pytest.raises(B.AxeError, match="head_dim"):
            Append([70], [20], 4, 2, D, 16, dtype, cache, rotary, style).run()
        return
    a = Append([70, 3, 33], [20, 3, 1], 4, 2, D, 16, dtype, cache, rotary, style, seed=D + rotary)
    a.check(a.run())


@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (32, 4), (7, 7), (128, 1), (40, 8)])
def test_heads(Hq, Hkv):
    for shared in (True, False):
        a = Append([50, 9], [5, 9], Hq, Hkv, 64, 24, seed=Hq, shared=shared)
        a.check(a.run())
        a.check(a.run(with_q=False), with_q=False)


@pytest.mark.parametrize("page", [1, 5, 16, 64])
def test_pages_and_batches(page):
    a = Append([70, 3, 33, 64, 65, 1], [20, 3, 1, 64, 2, 1], 2, 1, 64, page, seed=page, extra_rows=3)   # (rows behind the last sequence)
    a.check(a.run())


@pytest.mark.parametrize("sequences", [65, 300, 5000])
def test_many_sequences(sequences):
    a = Append([1 + s % 7 for s in range(sequences)], [s % 3 if s % 7 else min(1, s % 3) for s in range(sequences)], 1, 1, 8, 4, seed=sequences, spare=0)
    a.check(a.run())


def test_many_rows_a_lane():
    """Enough tokens to fill the chip: up to three rows a lane, with rows left over."""
    for Hq, Hkv, D in ((6, 2, 128), (32, 8, 64), (3, 1, 256), (39, 3, 80)):
        n = 2100
        a = Append([n], [n], Hq, Hkv, D, 64, seed=Hq, spare=0)
        out, kc, vc, _ = a.run()
        q, k, v = (x.float().cuda() for x in (a.q, a.k, a.v))
        cos, sin = a.rotation[:n, :D // 2].cuda()[:, None], a.rotation[:n, D // 2:].cuda()[:, None]
        turn = lambda x: torch.cat([x[..., :D // 2].double() * cos - x[..., D // 2:].double() * sin, x[..., D // 2:].double() * cos + x[..., :D // 2].double() * sin], -1)  # noqa: E731
        at = a.table[0].long().cuda()[torch.arange(n, device="cuda") // 64] * 64 + torch.arange(n, device="cuda") % 64
        for got, x in ((out, q), (kc.reshape(-1, Hkv, D)[at], k)):
            want, size = turn(x), torch.cat([x[..., :D // 2].abs() + x[..., D // 2:].abs()] * 2, -1)
            assert ((got.double() - want).abs() <= want.abs() * HALF["bf16"] + 3 * U * size * (1 + HALF["bf16"])).all()
        assert torch.equal(vc.reshape(-1, Hkv, D)[at], a.v.cuda())


@pytest.mark.parametrize("lengths", [[-4, 5, 0], [2, 10 ** 6, 1], [2 ** 31 - 1, -(2 ** 31), 3]])
@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_positions_and_pages_that_are_none(lengths, cache):
    a = Append([40, 33, 20], [8, 7, 5], 2, 2, 64, 16, cache=cache, seed=3)
    a.lengths = lengths
    a.check(a.run())
    a.lengths = [40, 33, 20]
    a.table[0, 2], a.table[1, 1], a.table[2, 0] = -1, a.pages, 2 ** 31 - 1
    a.check(a.run())


@pytest.mark.parametrize("style", ["halves", "pairs"])
@pytest.mark.parametrize("rotary", [64, 40, 6, 0])
def test_what_is_not_turned_is_copied(style, rotary):
    """Columns past the turned ones, with what is not finite among them, come out as they are."""
    a = Append([30], [30], 2, 1, 64, 16, rotary=rotary, style=style, seed=rotary)
    for x in (a.q, a.k):
        if rotary < 64:
            x[3, :, rotary:] = float("nan")
            x[5, :, rotary + 1::2] = float("inf")
    out, kc, _, _ = a.run()
    assert torch.equal(out[..., rotary:].cpu().view(torch.int16), a.q[..., rotary:].contiguous().view(torch.int16))
    got = torch.stack([kc[int(a.table[0, p // 16]), p % 16] for p in range(30)]).cpu()
    assert torch.equal(got[..., rotary:].contiguous().view(torch.int16), a.k[..., rotary:].contiguous().view(torch.int16))
    assert torch.isfinite(out[..., :rotary]).all() and torch.isfinite(got[..., :rotary]).all()


def test_rows_of_zeros_and_of_what_is_not_finite_in_e4m3():
    a = Append([20], [20], 1, 1, 64, 16, cache="fp8", rotary=0, seed=5)
    a.v[2] = 0
    a.v[4, 0, 3], a.v[6, 0, 5], a.v[8, 0, 7] = float("nan"), float("inf"), float("-inf")
    _, _, vc, sc = a.run(with_q=False)
    at = [(int(a.table[0, p // 16]), p % 16) for p in range(20)]
    rows = [vc[x].view(torch.float8_e4m3fn).float().cpu()[0] for x in at]
    assert float(sc[1][at[2]]) == 1.0 and (rows[2] == 0).all()
    assert torch.isnan(rows[4][3]) and torch.isfinite(rows[4][torch.arange(64) != 3]).all() and torch.isfinite(sc[1][at[4]]).all()
    assert rows[6][5] == 448 and rows[8][7] == -448 and torch.isfinite(rows[6]).all() and torch.isfinite(sc[1][at[6]]).all()


@pytest.mark.parametrize("style", ["halves", "pairs"])
@pytest.mark.parametrize("D, rotary", [(128, 128), (64, 40), (256, 192)])
@pytest.mark.parametrize("tokens", [7, 1500])
def test_queries_turned_where_they_lie(style, D, rotary, tokens):
    """In place among the keys and values of one product: the bits of the call that is not in place, and nothing else of the rows changes."""
    Hq, Hkv, page = 6, 2, 16
    a = Append([tokens + 3], [tokens], Hq, Hkv, D, page, rotary=rotary, style=style, seed=D)
    out, kc, vc, _ = a.run()
    T, pitch = a.T, (Hq + 2 * Hkv) * D + 24
    of = lambda o, h: B.Layout(W.spec([(T, pitch, "m"), (h, D, "m"), (D, 1, "m")], O={"m": o * D + 8}), ["m"])  # noqa: E731
    d = B.CacheDesc(T, 1, Hq, Hkv, D, a.pages, page, a.most, B.AXE_BF16, rotary_dim=rotary, rotary_style=B.AXE_ROTATE_PAIRS if style == "pairs" else B.AXE_ROTATE_HALVES,
                    q=of(0, Hq), k=of(Hq, Hkv), v=of(Hq + Hkv, Hkv), out=of(0, Hq))
    buf = a.buf.cuda()
    kc2, vc2 = torch.full_like(kc, 3.0), torch.full_like(vc, 3.0)
    B.axe_cache_append(d, buf, buf, kc2, vc2, a.seq_rows.cuda(), torch.tensor(a.lengths, dtype=torch.int32).cuda(), a.table.cuda(), rotation=a.rotation.cuda(), q=buf, q_out=buf)
    view = torch.as_strided(buf, (T, Hq, D), (pitch, D, 1), 8)
    assert torch.equal(view, out) and torch.equal(kc, kc2) and torch.equal(vc, vc2)
    view.copy_(a.q.cuda())
    assert torch.equal(buf, a.buf.cuda())


def test_both_caches_in_one_buffer_of_any_order():
    """[page][K, V][head][slot][column], a gap behind every head: what lies between stays."""
    Hkv, D, page, gap = 3, 64, 16, 8
    a = Append([45, 20], [30, 20], 3, Hkv, D, page, seed=9, shared=False)
    head = page * D + gap
    L = lambda o: B.Layout(W.spec([(a.pages, 2 * Hkv * head, "m"), (page, D, "m"), (Hkv, head, "m"), (D, 1, "m")], O={"m": o}), ["m"])  # noqa: E731
    n = a.pages * 2 * Hkv * head
    d = B.CacheDesc(a.T, 2, 3, Hkv, D, a.pages, page, a.most, B.AXE_BF16, rotary_dim=a.rotary, k_cache=L(0), v_cache=L(Hkv * head), k_cache_elems=n, v_cache_elems=n)
    buf = torch.full((n,), 3.0, dtype=torch.bfloat16, device="cuda")
    out = torch.full((a.T, 3, D), 7.0, dtype=torch.bfloat16, device="cuda")
    q, k, v = (x.contiguous().cuda() for x in (a.q, a.k, a.v))
    B.axe_cache_append(d, k, v, buf, buf, a.seq_rows.cuda(), torch.tensor(a.lengths, dtype=torch.int32).cuda(), a.table.cuda(), rotation=a.rotation.cuda(), q=q, q_out=out)
    kc, vc = (torch.as_strided(buf, (a.pages, page, Hkv, D), (2 * Hkv * head, D, head, 1), o) for o in (0, Hkv * head))
    a.check((out, kc, vc, [None, None]))
    kc.fill_(3.0), vc.fill_(3.0)
    assert (buf == 3.0).all()


def test_places_past_2_to_the_31_bytes():
    a = Append([30], [30], 2, 1, 64, 16, seed=11, shared=False, spare=0)
    far = 3 * 2 ** 30 // 2
    L = B.Layout(W.spec([(a.pages, far, "m"), (16, 64, "m"), (64, 1, "m")]), ["m"])
    d = B.CacheDesc(a.T, 1, 2, 1, 64, a.pages, 16, a.most, B.AXE_BF16, rotary_dim=64, k_cache=L, v_cache=L)
    bufs = [torch.empty(far + 1024, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for x in bufs:
        x[:1024], x[far:] = 3.0, 3.0
    out = torch.full((a.T, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    q, k, v = (x.contiguous().cuda() for x in (a.q, a.k, a.v))
    B.axe_cache_append(d, k, v, bufs[0], bufs[1], a.seq_rows.cuda(), torch.tensor([30], dtype=torch.int32).cuda(), a.table.cuda(), rotation=a.rotation.cuda(), q=q, q_out=out)
    kc, vc = (torch.stack([x[:1024], x[far:]]).reshape(2, 16, 1, 64) for x in bufs)
    a.check((out, kc, vc, [None, None]))


def test_captured_and_replayed_with_other_tables():
    a = Append([60, 50], [4, 3], 4, 2, 64, 16, cache="fp8", seed=13)
    rows, lens, table, rot, buf = a.seq_rows.cuda(), torch.tensor(a.lengths, dtype=torch.int32).cuda(), a.table.cuda(), a.rotation.cuda(), a.buf.cuda()
    shape = (a.pages, 16, 2, 64)
    kc, vc = (torch.zeros(shape, dtype=torch.uint8, device="cuda") for _ in range(2))
    sc = [torch.zeros(shape[:3], device="cuda") for _ in range(2)]
    out = torch.zeros((a.T, 4, 64), dtype=torch.bfloat16, device="cuda")
    run = lambda: B.axe_cache_append(a.desc, buf, buf, kc.view(torch.float8_e4m3fn), vc.view(torch.float8_e4m3fn), rows, lens, table, rotation=rot, q=buf, q_out=out, k_scales=sc[0], v_scales=sc[1])  # noqa: E731
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        run()
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        run()
    for turn in range(4):
        a.lengths = [60 - 13 * turn, 50 - 9 * turn]
        lens.copy_(torch.tensor(a.lengths, dtype=torch.int32))
        kc.fill_(0x55), vc.fill_(0x55), out.fill_(7.0)
        for x in sc:
            x.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        a.check((out, kc, vc, sc))
