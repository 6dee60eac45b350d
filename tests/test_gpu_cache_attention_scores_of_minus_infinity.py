"""Scores of -inf: such keys have the weight 0, and a token that has no other is zeros.  Tolerances: those of tests/test_gpu_cache_attention.py."""
import numpy as np
import pytest
import torch

from test_gpu_cache_attention import WIDE, Batch

pytestmark = pytest.mark.gpu

PAGE = 16


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("length, new, heads", [(90, 1, (4, 2)), (90, 8, (4, 2)), (300, 40, (4, 2)), (90, 9, WIDE), (400, 140, (48, 48)), (2500, 1, (4, 2)), (2500, 30, (4, 2)), (2000, 9, WIDE)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("all_of_them", [False, True])
def test_keys_of_minus_infinity(dtype, length, new, heads, causal, all_of_them):
    b = Batch([length], [new], *heads, 64, PAGE, dtype, seed=71)
    b.q[..., 5] = b.q[..., 5].abs() + 1                                # what the keys' -inf is multiplied with
    out = b.run(causal=causal)
    b.check(out, causal=causal)
    k = torch.as_strided(b.kv[0], (b.pages, PAGE, heads[1], 64), b.strides, 16)
    keys = range(length) if all_of_them else range(0, length, 3)
    for j in keys:
        k[int(b.table[0, j // PAGE]), j % PAGE, :, 5] = -float("inf")
        b.values[0][int(b.table[0, j // PAGE]), j % PAGE, :, 5] = -np.inf
    out = b.run(causal=causal)
    if all_of_them:
        assert (out == 0).all()
        return
    # the oracle without these keys: pages of one token each, of which theirs are none
    pages, table = b.pages * PAGE, torch.full((1, length), -1, dtype=torch.int32)
    for j in range(length):
        if j not in keys:
            table[0, j] = int(b.table[0, j // PAGE]) * PAGE + j % PAGE
    b.values = [np.where(np.isfinite(v), v, 0.0).reshape(pages, 1, heads[1], 64) for v in b.values]
    b.check(out, causal=causal, table=table)
