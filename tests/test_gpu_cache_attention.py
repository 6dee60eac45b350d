"""Attention over a paged cache on the GPU against the same in 64 bits.

Tolerances.  U = 2^-24, H = half a step of the 16-bit type relative to the value (2^-8 bf16, 2^-11 fp16).  With w_j the softmax's weights and A = sum_j w_j |v_j|:
  the result's own rounding                                H |o|
  the weights' rounding for the product with V             H A
  the scores: D products summed in fp32, the scaling, the exponential: each weight is off by a factor of at most e^(2 E), E = (D + 8) U reach + 4 U, reach = scale max_j sum_d |q_d k_jd|
  the sums over n keys, numerator and denominator          2 (n + 64) U A
  fp16's smallest steps: a term is held as at least w 2^9, w relative to the largest (e4m3 caches: times a scale that is more than half a power of two), so off by 2^-34 (2^-33): n 2^-32 max |v|
"""
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


WIDE = (66, 2)                                                         # 33 query heads to a head of the cache: tiles of 128 rows, whatever the batch; three tokens each


def f64(t):
    return t.detach().cpu().to(torch.float32).double().numpy()


class Batch:
    """Sequences of `lengths` tokens, the last `new` of them new, in shuffled pages."""

    def __init__(self, lengths, new, Hq, Hkv, D, page, dtype="bf16", cache=None, seed=0, std=1.0, spare=2, order="pshd", gap=0, garbage=None):
        g = torch.Generator().manual_seed(seed)
        self.lengths, self.new, self.Hq, self.Hkv, self.D, self.page, self.dtype, self.cache = lengths, new, Hq, Hkv, D, page, dtype, cache or dtype
        S, need = len(lengths), [-(-n // page) for n in lengths]
        self.pages, self.most = sum(need) + spare, max(need + [1])
        self.table = torch.full((S, self.most), -1, dtype=torch.int32)
        perm, at = torch.randperm(self.pages, generator=g).int(), 0
        for s, n in enumerate(need):
            self.table[s, :n] = perm[at:at + n]
            at += n
        self.seq_rows = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32)
        self.T = int(self.seq_rows[-1])
        self.q = (torch.randn((self.T, Hq, D), generator=g) * std).to(TORCH[dtype])
        # the caches in memory: axes in the given order, `gap` elements between neighbours of the third
        dims = {"p": self.pages, "s": page, "h": Hkv}
        step, strides = D + gap, {}
        for ax in reversed(order[:-1]):
            strides[ax] = step
            step *= dims[ax]
        self.strides = (strides["p"], strides["s"], strides["h"], 1)
        self.layout = B.Layout(W.spec([(self.pages, strides["p"], "m"), (page, strides["s"], "m"), (Hkv, strides["h"], "m"), (D, 1, "m")], O={"m": 16}), ["m"])
        self.kv, self.scales, self.values = [], [], []
        for _ in range(2):
            x = torch.randn((self.pages, page, Hkv, D), generator=g)
            if garbage is not None:                                    # everything that no sequence holds
                held = torch.zeros((self.pages, page), dtype=torch.bool)
                for s, n in enumerate(lengths):
                    for p in range(n):
                        held[self.table[s, p // page], p % page] = True
                x[~held] = garbage
            sc = None
            if self.cache == "fp8":
                sc = torch.nan_to_num(x.abs().amax(3), nan=1.0).clamp(1e-3, 1e3) / 448.0
                sc = sc * torch.exp(torch.randn(sc.shape, generator=g)) ** 0.2 * 1.3
                x = (x / sc[..., None]).clamp(-448, 448)
            x = x.to(TORCH[self.cache])
            self.values.append(f64(x) * (1.0 if sc is None else f64(sc)[..., None]))
            buf = torch.zeros(16 + step + 64, dtype=TORCH[self.cache])
            (torch.as_strided(buf.view(torch.uint8), x.shape, self.strides, 16).copy_(x.view(torch.uint8)) if self.cache == "fp8" else torch.as_strided(buf, x.shape, self.strides, 16).copy_(x))
            self.kv.append(buf.cuda())
            self.scales.append(None if sc is None else sc.contiguous().cuda())

    def desc(self, **kw):
        return B.CacheDesc(self.T, len(self.lengths), self.Hq, self.Hkv, self.D, self.pages, self.page, self.most, CODE[self.dtype], CODE[self.cache], k_cache=self.layout, v_cache=self.layout, **kw)

    def run(self, q=None, out=None, seq_rows=None, lengths=None, table=None, stream=None, desc=None, **kw):
        d = desc or self.desc(**kw)
        out = torch.full((self.T, self.Hq, self.D), 7.0, dtype=TORCH[self.dtype], device="cuda") if out is None else out
        words = B.axe_cache_attention_workspace(d)
        ws = torch.full((words,), -1, dtype=torch.int32, device="cuda") if words else None
        dev = lambda x, y: (y if x is None else x).cuda()  # noqa: E731
        B.axe_cache_attention(d, self.q.cuda() if q is None else q, self.kv[0], self.kv[1], dev(seq_rows, self.seq_rows), dev(lengths, torch.tensor(self.lengths, dtype=torch.int32)),
                              dev(table, self.table), out, k_scales=self.scales[0], v_scales=self.scales[1], workspace=ws, stream=stream)
        torch.cuda.synchronize()
        return out

    def check(self, out, causal=True, window=0, scale=None, lengths=None, table=None, seq_rows=None):
        rows = (self.seq_rows if seq_rows is None else seq_rows).numpy()
        want, spread, reach, seen = R.attention(f64(self.q), *self.values, rows, self.lengths if lengths is None else lengths, (self.table if table is None else table).numpy(),
                                                self.D ** -0.5 if scale is None else scale, causal, window)
        H, n = HALF[self.dtype], seen[:, None, None]
        E = (self.D + 8) * U * reach[..., None] + 4 * U
        most = max(np.nanmax(np.abs(np.where(np.isfinite(v), v, np.nan))) for v in self.values[1:])
        tol = H * np.abs(want) + (H + np.expm1(2 * E) + 2 * (n + 64) * U) * spread + (n * 2.0 ** -32 * most + 2.0 ** -25 if self.dtype == "f16" else 0.0)
        got = f64(out)
        none = np.isnan(want[:, 0, 0])
        assert (got[none] == 7.0).all(), "rows of no sequence are left as they are"
        bad = ~(np.abs(got - want) <= tol) & ~none[:, None, None]
        assert not bad.any(), f"{bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}, allowed {tol[bad][0]}"


@pytest.mark.parametrize("dtype, cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "fp8"), ("f16", "fp8")])
@pytest.mark.parametrize("D", [64, 128, 256, 16, 80, 8, 136])
@pytest.mark.parametrize("new, heads", [([1, 1, 1], (4, 2)), ([9, 8, 7], (4, 2)), ([3, 1, 70], (4, 2)), ([1, 2, 9], WIDE), ([3, 1, 20], (48, 48))])   # tiles of 16, 32, 32, 128 and 128 rows
def test_types_and_columns(dtype, cache, D, new, heads):
    if cache == "fp8" and D % 16:
        with pytest.raises(B.AxeError, match="head_dim"):
            Batch([130, 9, 77], new, *heads, D, 16, dtype, cache, seed=D).run()
        return
    b = Batch([530, 9, 77], new, *heads, D, 16, dtype, cache, seed=D)
    b.check(b.run())


@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (8, 1), (6, 2), (5, 5), (32, 4), (128, 1), (35, 7)])
def test_heads(Hq, Hkv):
    b = Batch([100, 33], [40, 1], Hq, Hkv, 64, 16, seed=Hq)
    b.check(b.run())


@pytest.mark.parametrize("page", [1, 3, 16, 24, 64, 100, 1000])
@pytest.mark.parametrize("new, heads", [(1, (4, 2)), (50, (4, 2)), (5, WIDE)])
def test_pages(page, new, heads):
    b = Batch([200, 63, 64, 65], [new] * 4, *heads, 128, page, seed=page)
    b.check(b.run())


@pytest.mark.parametrize("causal, window", [(False, 0), (True, 1), (True, 5), (True, 64), (True, 70), (True, 1000)])
@pytest.mark.parametrize("lengths, new, heads", [([300], [1], (4, 2)), ([300, 20, 150], [150, 20, 3], (4, 2)), ([300, 20, 150], [20, 7, 1], WIDE), ([300, 20, 150], [15, 20, 1], (48, 48))])
def test_masks(causal, window, lengths, new, heads):
    b = Batch(lengths, new, *heads, 64, 16, seed=window)
    b.check(b.run(causal=causal, window=window), causal, window)


@pytest.mark.parametrize("order, gap", [("pshd", 8), ("phsd", 0), ("hpsd", 16), ("sphd", 0)])
@pytest.mark.parametrize("page", [16, 24])
@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_layouts_of_the_cache(order, gap, page, cache):
    if cache == "fp8":
        gap = gap // 16 * 16
    for new, heads in (([1, 1] if gap else [20, 30], (4, 2)), ([4, 3], WIDE)):
        b = Batch([150, 40], new, *heads, 128, page, "bf16", cache, seed=gap, order=order, gap=gap)
        b.check(b.run())


@pytest.mark.parametrize("new", [[1, 1], [30, 40]])
def test_layouts_of_rows(new):
    b = Batch([150, 60], new, 6, 2, 80, 16, seed=3)
    T = b.T
    buf = torch.randn(T * 700 + 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    at = (700, 84, 1)
    torch.as_strided(buf, b.q.shape, at, 3).copy_(b.q)
    out = torch.full((T * 900 + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    before = out.clone()
    of = lambda p, h, o: B.Layout(W.spec([(T, p, "m"), (6, h, "m"), (80, 1, "m")], O={"m": o}), ["m"])  # noqa: E731
    d = b.desc(q=of(700, 84, 3), out=of(900, 81, 5), q_elems=buf.numel(), out_elems=out.numel())
    b.run(q=buf.cuda(), out=out, desc=d)
    view = torch.as_strided(out, (T, 6, 80), (900, 81, 1), 5)
    b.check(view)
    view.fill_(7.0)
    assert torch.equal(out, before), "what lies between the rows is left as it was"


@pytest.mark.parametrize("heads", [(4, 2), WIDE])
@pytest.mark.parametrize("new", [[0, 3, 0, 1, 5, 0], [0, 40, 0, 30, 5, 0], [0, 0, 0, 0, 0, 0]])
def test_sequences_without_new_tokens_without_keys_and_rows_of_none(new, heads):
    b = Batch([70, 80, 0, 90, 33, 1], new, *heads, 64, 16, seed=5)
    if b.T == 0:                                                       # rows, but none of a sequence's
        b.T, b.q = 3, torch.randn(3, heads[0], 64).to(torch.bfloat16)
    lengths = [70, 80, 0, 0, 2, 1]                                     # more new tokens than tokens: the first are at negative positions and see nothing
    b.check(b.run(lengths=torch.tensor(lengths, dtype=torch.int32)), lengths=lengths)
    b.check(b.run(lengths=torch.tensor(lengths, dtype=torch.int32), causal=False), causal=False, lengths=lengths)
    # rows behind the last sequence, and before the first
    if sum(new):
        rows = torch.clamp(b.seq_rows + 2, max=b.T - 1)
        b.check(b.run(seq_rows=rows, lengths=torch.tensor(lengths, dtype=torch.int32)), seq_rows=rows, lengths=lengths)


@pytest.mark.parametrize("page", [16, 7])
@pytest.mark.parametrize("new, heads", [([1, 1], (4, 2)), ([50, 60], (4, 2)), ([4, 5], WIDE)])
@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_pages_that_are_none_and_lengths_past_the_table(page, new, heads, cache):
    b = Batch([200, 150], new, *heads, 64, page, "bf16", cache, seed=7)
    table = b.table.clone()
    table[0, 1], table[0, 3], table[1, 0] = -1, b.pages, 2 ** 31 - 1
    table[1, 2:4] = -(2 ** 31)
    b.check(b.run(table=table), table=table)
    lengths = [100000, 2 ** 31 - 1]
    got = b.run(table=table, lengths=torch.tensor(lengths, dtype=torch.int32))
    b.check(got, lengths=lengths, table=table)
    lengths = [-5, -(2 ** 31)]
    b.check(b.run(lengths=torch.tensor(lengths, dtype=torch.int32)), lengths=lengths)


@pytest.mark.parametrize("garbage", [float("nan"), float("inf")])
@pytest.mark.parametrize("new, heads", [([1, 1], (4, 2)), ([9, 9], (4, 2)), ([60, 64], (4, 2)), ([4, 3], WIDE), ([10, 20], (48, 48))])
@pytest.mark.parametrize("dtype, cache, D, page", [("bf16", "bf16", 128, 16), ("f16", "f16", 80, 16), ("bf16", "bf16", 64, 10), ("bf16", "fp8", 128, 16)])
def test_what_no_sequence_holds_has_no_part(garbage, new, heads, dtype, cache, D, page):
    if cache == "fp8" and garbage == float("inf"):
        garbage = float("nan")                                         # (e4m3 has no infinities)
    b = Batch([100, 65], new, *heads, D, page, dtype, cache, seed=9, garbage=garbage)
    b.check(b.run())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("length, new, Hq, Hkv, D, window", [(90, 40, 4, 1, 128, 0), (90, 8, 2, 1, 64, 0), (300, 200, 1, 1, 64, 0), (700, 130, 8, 2, 256, 0), (90, 40, 4, 1, 128, 20), (100, 12, 2, 1, 128, 30),
                                                                (90, 9, *WIDE, 128, 0), (90, 9, *WIDE, 64, 12), (300, 140, 48, 48, 64, 0), (700, 9, *WIDE, 256, 0), (2000, 9, *WIDE, 128, 0)])
def test_values_that_are_not_finite_reach_those_that_see_them_alone(bad, length, new, Hq, Hkv, D, window):
    """A value that is not finite at one new token's place (and, with a window, at an old one): the tokens before it (behind the window) come out as if it were not there, the others not finite."""
    b = Batch([length], [new], Hq, Hkv, D, 16, seed=11)
    at = [length - new // 2] + ([length - new - window + 4] if window else [])   # (the old one is out of sight from the fifth new token on)
    marked = torch.zeros(length, dtype=torch.bool)
    for p in at:
        pg, sl = int(b.table[0, p // 16]), p % 16
        torch.as_strided(b.kv[1], (b.pages, 16, Hkv, D), b.strides, 16)[pg, sl] = bad
        marked[p] = True
        b.values[1][pg, sl] = bad
    out = b.run(window=window)
    sees = [any(marked[max(0, p - window + 1) if window else 0:p + 1]) for p in range(length - new, length)]
    rows = torch.tensor(sees)
    assert rows.any() and not rows.all()
    got = out.float().cpu()
    assert not torch.isfinite(got[rows]).any()
    clean = [np.where(np.isfinite(v), v, 0.0) for v in b.values]
    want, spread, reach, seen = R.attention(f64(b.q), *clean, b.seq_rows.numpy(), b.lengths, b.table.numpy(), D ** -0.5, True, window)
    keep = ~rows.numpy()
    E = (D + 8) * U * reach[..., None] + 4 * U
    tol = HALF["bf16"] * np.abs(want) + (HALF["bf16"] + np.expm1(2 * E) + 2 * (seen[:, None, None] + 64) * U) * spread
    assert (np.abs(f64(out) - want)[keep] <= tol[keep]).all()


def test_keys_that_are_not_finite_where_masked():
    b = Batch([90], [40], 4, 1, 64, 16, seed=13)
    p = 80
    pg, sl = int(b.table[0, p // 16]), p % 16
    torch.as_strided(b.kv[0], (b.pages, 16, 1, 64), b.strides, 16)[pg, sl] = float("nan")
    out = b.run().float().cpu()
    want = R.attention(f64(b.q), *b.values, b.seq_rows.numpy(), b.lengths, b.table.numpy(), 64 ** -0.5)[0]
    assert torch.isfinite(out[:30]).all() and not torch.isfinite(out[30:]).any()
    assert np.allclose(out[:30].numpy(), want[:30], atol=0.05)


@pytest.mark.parametrize("std, scale", [(30.0, None), (1e-3, None), (1.0, 1e-6), (4.0, 3.0), (1.0, 2.0 ** -100)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new, heads", [(1, (4, 2)), (40, (4, 2)), (5, WIDE)])
def test_sizes_of_scores(std, scale, dtype, new, heads):
    b = Batch([500], [new], *heads, 64, 16, dtype, seed=15, std=std)
    b.check(b.run(scale=scale), scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new, heads", [(1, (4, 2)), (40, (4, 2)), (5, WIDE)])
def test_scales_of_an_e4m3_cache_far_apart(dtype, new, heads):
    """Zeros, tiny and large ones side by side: terms times scales stay inside fp16's range."""
    b = Batch([300], [new], *heads, 64, 16, dtype, "fp8", seed=17)
    g = torch.Generator().manual_seed(2)
    sc = 2.0 ** torch.randint(-12, 8 if dtype == "f16" else 14, b.scales[1].shape, generator=g).float()
    sc[torch.rand(sc.shape, generator=g) < 0.2] = 0.0
    b.values[1] = b.values[1] / f64(b.scales[1])[..., None] * f64(sc)[..., None]
    b.values[1] = np.clip(b.values[1], -6e4, 6e4) if dtype == "f16" else b.values[1]
    codes = torch.as_strided(b.kv[1].view(torch.uint8), (b.pages, 16, 2, 64), b.strides, 16).view(torch.float8_e4m3fn).float().cpu()
    assert (np.abs(f64(codes) * f64(sc)[..., None]) <= 6e4).all() or dtype == "bf16"
    b.scales[1] = sc.cuda()
    out = f64(b.run())
    want, spread, reach, seen = R.attention(f64(b.q), *b.values, b.seq_rows.numpy(), b.lengths, b.table.numpy(), 8.0 ** -1)
    n, most = seen[:, None, None], np.abs(b.values[1]).max()
    E = (64 + 8) * U * reach[..., None] + 4 * U
    # (a term is rounded twice as it enters the sum: 2 H; what it counts there differs from the term itself by H at most)
    tol = HALF[dtype] * np.abs(want) + (2 * HALF[dtype] + np.expm1(2 * E) + 2 * (n + 64) * U) * spread + HALF[dtype] * np.abs(want) + (n * 2.0 ** -31 * most + 2.0 ** -25 if dtype == "f16" else 0.0)
    assert (np.abs(out - want) <= tol).all()


def dense(b, lengths, new, D, causal=True, window=0):
    """R.attention for long sequences, on the device in 64 bits."""
    Hq, Hkv, page = b.Hq, b.Hkv, b.page
    want, spread, reach, seen = (np.zeros((b.T, Hq, D)), np.zeros((b.T, Hq, D)), np.zeros((b.T, Hq)), np.zeros(b.T, dtype=np.int64))
    t0 = 0
    for s, (n, m) in enumerate(zip(lengths, new)):
        pages = b.table[s, :-(-n // page)].long()
        K, V = (torch.from_numpy(x)[pages].reshape(-1, Hkv, D)[:n].cuda() for x in b.values)
        q = b.q[t0:t0 + m].double().cuda()
        at, key = torch.arange(n - m, n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
        hidden = ((key > at) if causal else torch.zeros((m, n), dtype=torch.bool, device="cuda")) | ((key <= at - window) if window else False)
        for h in range(Hq):
            k, v = K[:, h // (Hq // Hkv)].contiguous(), V[:, h // (Hq // Hkv)].contiguous()
            x = (q[:, h].contiguous() @ k.t().contiguous()) * D ** -0.5
            w = torch.softmax(x.masked_fill(hidden, -torch.inf), 1)
            want[t0:t0 + m, h], spread[t0:t0 + m, h] = (w @ v).cpu().numpy(), (w @ v.abs()).cpu().numpy()
            reach[t0:t0 + m, h] = ((q[:, h].abs().contiguous() @ k.abs().t().contiguous()).amax(1) * D ** -0.5).cpu().numpy()
        seen[t0:t0 + m] = (~hidden).sum(1).cpu().numpy()
        t0 += m
    return want, spread, reach, seen


@pytest.mark.parametrize("lengths, new, Hq, Hkv, D, page, dtype, cache, window", [
    ([20000], [1], 8, 1, 128, 64, "bf16", "bf16", 0), ([9000, 3, 700], [1, 1, 1], 4, 4, 64, 16, "f16", "f16", 0), ([30000], [1], 4, 2, 64, 16, "bf16", "fp8", 0), ([5000, 900], [3, 1], 8, 1, 128, 24, "bf16", "bf16", 0),
    ([2500], [700], 4, 1, 128, 16, "bf16", "bf16", 0), ([3000, 40, 1800], [260, 40, 1], 8, 2, 64, 7, "f16", "f16", 0), ([2000, 1500], [500, 900], 2, 2, 256, 32, "bf16", "bf16", 0),
    ([4000], [400], 4, 1, 128, 16, "bf16", "fp8", 0), ([6000, 5000], [300, 1], 4, 1, 64, 16, "f16", "fp8", 1100), ([1200] * 3, [1200, 600, 1], 16, 16, 64, 16, "bf16", "bf16", 0),
    ([5000], [5000], 2, 2, 64, 64, "f16", "f16", 0), ([150] * 70, [2] * 70, 16, 16, 64, 16, "bf16", "bf16", 0), ([700] * 80, [1] * 80, 2, 1, 64, 16, "bf16", "bf16", 0), ([600] * 70, [9] * 70, 4, 1, 64, 16, "bf16", "bf16", 0),
    ([3000, 700], [9, 200], *WIDE, 128, 16, "bf16", "bf16", 0), ([3000, 40], [60, 1], 48, 48, 64, 24, "f16", "fp8", 0), ([2000, 900], [40, 3], *WIDE, 256, 16, "bf16", "fp8", 0), ([1700] * 70, [2] * 70, 33, 1, 64, 16, "bf16", "bf16", 0)])
def test_long_and_many(lengths, new, Hq, Hkv, D, page, dtype, cache, window):
    """Keys split among workgroups and not, cuts inside tiles, batches above 64 sequences; and the same bits a second time."""
    b = Batch(lengths, new, Hq, Hkv, D, page, dtype, cache, seed=19)
    out = b.run(window=window)
    want, spread, reach, seen = dense(b, lengths, new, D, window=window)
    E = (D + 8) * U * reach[..., None] + 4 * U
    n, most = seen[:, None, None], max(np.abs(v).max() for v in b.values)
    tol = HALF[dtype] * np.abs(want) + (HALF[dtype] + np.expm1(2 * E) + 2 * (n + 64) * U) * spread + (n * 2.0 ** -32 * most + 2.0 ** -25 if dtype == "f16" else 0.0)
    bad = ~(np.abs(f64(out) - want) <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}"
    assert torch.equal(out, b.run(window=window))


def test_more_sequences_than_a_workgroup_surveys():
    S = 4200
    b = Batch([3 + s % 40 for s in range(S)], [s % 3 for s in range(S)], 2, 1, 16, 16, seed=21, spare=0)
    b.check(b.run())
    b = Batch([3 + s % 40 for s in range(300)], [max(0, s % 8 - 3) for s in range(300)], 4, 1, 64, 16, seed=22, spare=0)   # tiles of 16 rows, most sequences with one or none
    b.check(b.run())
    rows = b.seq_rows.clone()                                          # a padded batch: the last 100 sequences' rows are nobody's
    rows[201:] = rows[200]
    b.check(b.run(seq_rows=rows), seq_rows=rows)


def test_a_cache_past_2_to_the_31_bytes():
    """Pages far apart: places whose offsets 32 bits do not hold, in pages of 16 tokens and of 24."""
    for page, new, heads in ((16, 1, 4), (24, 1, 4), (16, 20, 4), (24, 20, 4), (16, 20, 33), (24, 20, 33)):
        Hkv, D, far = 1, 64, 3 * 2 ** 30 // 2                           # elements between pages: 3 GiB
        small = Batch([2 * page - 3], [new], heads, Hkv, D, page, seed=23, spare=0)
        bufs = []
        for i in range(2):
            x = torch.from_numpy(small.values[i]).to(torch.bfloat16)
            buf = torch.empty(far + page * D, dtype=torch.bfloat16, device="cuda")
            for p in range(2):
                buf[p * far:p * far + page * D] = x[p].reshape(-1).cuda()
            bufs.append(buf)
        small.kv = bufs
        small.layout = B.Layout(W.spec([(2, far, "m"), (page, D, "m"), (D, 1, "m")]), ["m"])
        small.check(small.run())
        del bufs, buf, small
        torch.cuda.empty_cache()


@pytest.mark.parametrize("page", [16, 24])
@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("new, heads", [([1, 1], (4, 2)), ([9, 40], (4, 2)), ([9, 40], WIDE)])
def test_keys_and_values_laid_out_differently(new, heads, cache, page):
    b = Batch([900, 333], new, *heads, 128, page, "bf16", cache, seed=31)
    shape, step = (b.pages, page, heads[1], 128), page * 144                # values: head by head, then by pages, 16 elements between neighbouring tokens
    strides = (step, 144, b.pages * step, 1)
    x = torch.as_strided(b.kv[1].view(torch.uint8) if cache == "fp8" else b.kv[1], shape, b.strides, 16)
    buf = torch.zeros(heads[1] * b.pages * step, dtype=x.dtype, device="cuda")
    torch.as_strided(buf, shape, strides).copy_(x)
    b.kv[1] = buf.view(b.kv[1].dtype)
    other = B.Layout(W.spec([(n, s, "m") for n, s in zip(shape, strides)]), ["m"])
    b.check(b.run(desc=B.CacheDesc(b.T, 2, *heads, 128, b.pages, page, b.most, CODE["bf16"], CODE[cache], k_cache=b.layout, v_cache=other)))


def graph_of(f):
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        f()
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        f()
    return g


def test_captured_and_replayed_with_other_tables():
    """Three graphs of different shapes, each with its workspace, which lives as long as the graph; lengths, pages and rows change between the replays, eager calls run in between."""
    cases = []
    for lengths, new, Hq, Hkv, seed in (([900, 400, 700], [1, 1, 1], 8, 2, 25), ([600, 800], [70, 60], 4, 2, 26), ([1900, 800], [7, 9], 66, 2, 27)):
        b = Batch(lengths, new, Hq, Hkv, 128, 16, seed=seed)
        d = b.desc()
        dev = dict(q=b.q.cuda(), out=torch.zeros((b.T, Hq, 128), dtype=torch.bfloat16, device="cuda"), seq_rows=b.seq_rows.cuda(), lengths=torch.tensor(lengths, dtype=torch.int32).cuda(), table=b.table.cuda())
        ws = torch.zeros(max(1, B.axe_cache_attention_workspace(d)), dtype=torch.int32, device="cuda")
        run = lambda b=b, d=d, dev=dev, ws=ws: B.axe_cache_attention(d, dev["q"], b.kv[0], b.kv[1], dev["seq_rows"], dev["lengths"], dev["table"], dev["out"], workspace=ws)  # noqa: E731
        cases.append((b, dev, graph_of(run), ws))
    for turn in range(4):
        for b, dev, g, _ in cases:
            lengths = [max(1, n - 137 * turn) for n in b.lengths]
            table = b.table.roll(turn, 1)
            dev["lengths"].copy_(torch.tensor(lengths, dtype=torch.int32))
            dev["table"].copy_(table)
            g.replay()
        torch.cuda.synchronize()
        for b, dev, g, _ in cases:
            lengths = [max(1, n - 137 * turn) for n in b.lengths]
            table = b.table.roll(turn, 1)
            eager = b.run(lengths=torch.tensor(lengths, dtype=torch.int32), table=table)
            assert torch.equal(dev["out"], eager)
            b.check(eager, lengths=lengths, table=table)


def test_two_calls_on_two_streams():
    a, b = Batch([3000, 500], [1, 1], 8, 2, 128, 16, seed=27), Batch([700, 2900], [20, 10], 66, 2, 128, 16, seed=28)
    alone = [x.run() for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    sets = []
    for x in (a, b):
        d = x.desc()
        sets.append((d, x.q.cuda(), x.seq_rows.cuda(), torch.tensor(x.lengths, dtype=torch.int32).cuda(), x.table.cuda(), torch.zeros((x.T, x.Hq, 128), dtype=torch.bfloat16, device="cuda"),
                     torch.zeros(max(1, B.axe_cache_attention_workspace(d)), dtype=torch.int32, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(10):
        for x, s, (d, q, rows, lens, table, out, ws) in zip((a, b), streams, sets):
            B.axe_cache_attention(d, q, x.kv[0], x.kv[1], rows, lens, table, out, workspace=ws, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(sets[0][5], alone[0]) and torch.equal(sets[1][5], alone[1])
