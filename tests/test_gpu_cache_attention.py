"""Attention over a paged cache on the GPU against the same in 64 bits.

Tolerances.  U = 2^-24, H = half a step of the 16-bit type relative to the value (2^-8 bf16, 2^-11 fp16).  With w_j the softmax's weights and A = sum_j w_j |v_j|:
  the result's own rounding                                H |o|
  the weights' rounding for the product with V             H A
  the scores: D products summed in fp32, the scaling, the exponential: each weight is off by a factor of at most e^(2 E), E = (D + 8) U reach + 4 U, reach = scale max_j sum_d |q_d k_jd|
  the sums over n keys, numerator and denominator          2 (n + 64) U A
  fp16's smallest steps: a term is held as w 2^15 (e4m3 caches: w 2^8 times a scale that is at most 1 of the largest's power of two): n 2^-32 max |v|
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
@pytest.mark.parametrize("new", [[3, 1, 70], [1, 1, 1], [9, 8, 7]])    # tiles of 128, 16 and 32 rows
def test_types_and_columns(dtype, cache, D, new):
    if cache == "fp8" and D % 16:
        with pytest.raises(B.AxeError, match="head_dim"):
            Batch([130, 8, 77], new, 4, 2, D, 16, dtype, cache, seed=D).run()
        return
    b = Batch([530, 8, 77], new, 4, 2, D, 16, dtype, cache, seed=D)
    b.check(b.run())


@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (8, 1), (6, 2), (5, 5), (32, 4), (128, 1), (35, 7)])
def test_heads(Hq, Hkv):
    b = Batch([100, 33], [40, 1], Hq, Hkv, 64, 16, seed=Hq)
    b.check(b.run())


@pytest.mark.parametrize("page", [1, 3, 16, 24, 64, 100, 1000])
@pytest.mark.parametrize("new", [1, 50])
def test_pages(page, new):
    b = Batch([200, 63, 64, 65], [new] * 4, 4, 2, 128, page, seed=page)
    b.check(b.run())


@pytest.mark.parametrize("causal, window", [(False, 0), (True, 1), (True, 5), (True, 64), (True, 70), (True, 1000)])
@pytest.mark.parametrize("lengths, new", [([300], [1]), ([300, 20, 150], [150, 20, 3])])
def test_masks(causal, window, lengths, new):
    b = Batch(lengths, new, 4, 2, 64, 16, seed=window)
    b.check(b.run(causal=causal, window=window), causal, window)
