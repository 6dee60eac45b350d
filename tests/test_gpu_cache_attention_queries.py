"""Queries that are not finite among those of a batch: their rows come out as NaN, in one launch and in split calls, where a part of the keys may hold no score that is a number, and no other row does.
Tolerances: those of tests/test_gpu_cache_attention.py, and H |o| once more for tiles that count terms of e4m3 caches as rounded."""
import numpy as np
import pytest
import torch

from oracle import cache_ref as R
from test_gpu_cache_attention import HALF, U, WIDE, Batch, f64

pytestmark = pytest.mark.gpu

PAGE = 16
NAN, INF = float("nan"), float("inf")
SHAPES = [(90, 1, (4, 2)), (90, 8, (4, 2)), (300, 40, (4, 2)), (90, 9, WIDE), (400, 140, (48, 48)), (2500, 1, (4, 2)), (2500, 30, (4, 2)), (2000, 9, WIDE)]   # tiles of 16, 32 and 128 rows; the last three are split


@pytest.mark.parametrize("length, new, heads", SHAPES)
@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("bad", [NAN, INF])
def test_queries_that_are_not_finite(length, new, heads, cache, bad):
    """A query's rows are lost, and no others."""
    b = Batch([length], [new], *heads, 64, PAGE, "bf16", cache, seed=64)
    b.q[new // 2, 1] = bad
    out = b.run()
    assert torch.isnan(out[new // 2, 1]).all()
    out[new // 2, 1] = 0
    b.q[new // 2, 1] = 0
    keep = np.ones(out.shape[:2], dtype=bool)
    keep[new // 2, 1] = False
    want, spread, reach, seen = R.attention(f64(b.q), *b.values, b.seq_rows.numpy(), b.lengths, b.table.numpy(), 64 ** -0.5)
    E = (64 + 8) * U * reach[..., None] + 4 * U
    tol = 2 * HALF["bf16"] * np.abs(want) + (HALF["bf16"] + np.expm1(2 * E) + 2 * (seen[:, None, None] + 64) * U) * spread
    assert (np.abs(f64(out) - want) <= tol)[keep].all()
