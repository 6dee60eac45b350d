"""Attention over an e4m3 cache whose values have small scales, or scales far apart: what a key weighs does not depend on the size of its value, and a value's size matters to those that see it alone.

Tolerances, with the names of tests/test_gpu_cache_attention.py: the result's own rounding H |o|; the terms' rounding for the product with V, H A; tiles that count in the sum what that rounding changed are off
by H |o| once more; scores (e^(2 E) - 1) A; sums 2 (n + 64) U A.  fp16's smallest steps: a term, its weight w relative to the row's largest, is held as at least w 2^9 times its scale over a power of
two that is at most twice the largest scale s that the row sees, so it is off by 2^-25 at most, its value by 2^-34 2 s 448: n 2^-33 448 s for all; and 2^-25 of the result itself."""
import numpy as np
import pytest
import torch

from oracle import cache_ref as R
from test_gpu_cache_attention import HALF, U, WIDE, Batch, f64

pytestmark = pytest.mark.gpu

D, PAGE = 64, 16
SHAPES = [([1], (4, 2)), ([9], (4, 2)), ([40], (4, 2)), ([5], WIDE), ([70], (48, 48))]   # tiles of 16, 32, 32, 128 and 128 rows


def batch(length, new, heads, dtype, score, scale, seed=0):
    """A sequence whose key j has the score score[j], in every head, and a value of codes from 224 to 448 times scale[j]."""
    b = Batch([length], new, *heads, D, PAGE, dtype, "fp8", seed=seed)
    g = torch.Generator().manual_seed(seed)
    b.q = torch.ones_like(b.q)
    codes = [torch.ones((b.pages, PAGE, heads[1], D)), torch.rand((b.pages, PAGE, heads[1], D), generator=g) * 224 + 224]
    k_scales, v_scales = torch.zeros((b.pages, PAGE, heads[1])), torch.zeros((b.pages, PAGE, heads[1]))
    for j in range(length):
        at = int(b.table[0, j // PAGE]), j % PAGE
        k_scales[at], v_scales[at] = score[j] * D ** 0.5 / D, scale[j]
    for i, (c, sc) in enumerate(zip(codes, (k_scales, v_scales))):
        c = c.to(torch.float8_e4m3fn)
        torch.as_strided(b.kv[i].view(torch.uint8), c.shape, b.strides, 16).copy_(c.view(torch.uint8).cuda())
        b.scales[i] = sc.cuda()
        b.values[i] = f64(c) * f64(sc)[..., None]
    return b, np.asarray(scale, dtype=np.float64)


def check(b, scale, window=0):
    out, (n,), new = f64(b.run(window=window)), b.lengths, b.T
    want, spread, reach, seen = R.attention(f64(b.q), *b.values, b.seq_rows.numpy(), b.lengths, b.table.numpy(), D ** -0.5, True, window)
    H, count, E = HALF[b.dtype], seen[:, None, None], (D + 8) * U * reach[..., None] + 4 * U
    most = np.array([scale[max(0, p - window + 1) if window else 0:p + 1].max() for p in range(n - new, n)])[:, None, None]
    tol = 2 * H * np.abs(want) + (H + np.expm1(2 * E) + 2 * (count + 64) * U) * spread + (count * 2.0 ** -33 * 448 * most + 2.0 ** -25 if b.dtype == "f16" else 0.0)
    bad = ~(np.abs(out - want) <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {out[bad][0]} for {want[bad][0]}, allowed {tol[bad][0]}"


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new, heads", SHAPES)
@pytest.mark.parametrize("size", [1e-3, 1.0, 3e-6])
def test_many_light_keys_beside_one_that_has_nearly_all_the_weight(dtype, new, heads, size):
    """1023 keys of 2^-15.3 each: 2.5 parts in a hundred."""
    score = np.full(1024, 16.0 - 15.3 * np.log(2.0))
    score[100] = 16.0
    check(*batch(1024, new, heads, dtype, score, np.full(1024, size / 448)))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new, heads", SHAPES)
@pytest.mark.parametrize("small, large, gap", [(3e-11, 3e-3, 6.0), (2.0 ** -40, 0.25, 3.0), (2.0 ** -90, 2.0 ** -8, 8.0), (0.0, 1e-2, 4.0)])
@pytest.mark.parametrize("heavy_first", [True, False])
def test_a_heavy_key_whose_value_is_next_to_nothing(dtype, new, heads, small, large, gap, heavy_first):
    score, scale = np.full(200, 10.0 - gap), np.full(200, large)
    at = 3 if heavy_first else 200 - max(new)
    score[at], scale[at] = 10.0, small
    check(*batch(200, new, heads, dtype, score, scale))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new, heads", SHAPES[1:])
@pytest.mark.parametrize("window", [0, 30])
def test_a_large_value_that_only_the_last_tokens_see(dtype, new, heads, window):
    """The tokens before it come out as exactly as without it; with a window, also those behind it that do not see the old large ones."""
    n, m = 150, new[0]
    rng = np.random.default_rng(1)
    score, scale = rng.uniform(0, 4, n), rng.uniform(0.5, 1, n) * 2.0 ** -20
    scale[n - 2:] = 2.0 ** 6
    if window:
        scale[n - m - window + 2] = 2.0 ** 6                           # (seen by the first two new tokens)
    check(*batch(n, new, heads, dtype, score, scale), window=window)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new, heads", SHAPES)
def test_tiny_scales(dtype, new, heads):
    """Down to the smallest normal number, and zeros."""
    rng = np.random.default_rng(2)
    for scale in (np.full(90, 2.0 ** -126), np.zeros(90), 2.0 ** rng.integers(-126, -60, 90).astype(np.float64)):
        check(*batch(90, new, heads, dtype, rng.uniform(0, 4, 90), scale))
