"""Attention whose scores are so large that fp32 numbers of their size are whole numbers apart, up to 2^100: one key has all the weight.

The oracle's row counts where its best key is further ahead of the second than 100 and what D products summed in fp32 and the scaling can be off by, 2 (D + 8) U reach (names of
tests/test_gpu_cache_attention.py): the others' weights are below e^-100, and the result is the best key's value, off by its own rounding H |v| and by that of the one term, H |v|; fp16: 2^-25."""
import numpy as np
import pytest
import torch

from test_gpu_cache_attention import HALF, U, WIDE, Batch, f64

pytestmark = pytest.mark.gpu

D, PAGE = 64, 16


@pytest.mark.parametrize("dtype, cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "fp8"), ("f16", "fp8")])
@pytest.mark.parametrize("length, new, heads", [(500, 1, (4, 2)), (500, 9, (4, 2)), (500, 40, (4, 2)), (500, 5, WIDE), (500, 70, (48, 48)), (9000, 1, (4, 2)), (3000, 9, WIDE)])   # tiles of 16, 32, 32, 128 and 128 rows; split
@pytest.mark.parametrize("std, scale", [(1.0, 2.0 ** 17), (1.0, 2.0 ** 24), (1.0, 2.0 ** 29), (1.0, 2.0 ** 60), (1.0, 2.0 ** 100), (9000.0, 1024.0)])
def test_one_key_has_all_the_weight(dtype, cache, length, new, heads, std, scale):
    b = Batch([length], [new], *heads, D, PAGE, dtype, cache, seed=51, std=std)
    out = f64(b.run(scale=scale))
    pages = b.table[0, :-(-length // PAGE)].long().numpy()
    K, V = (x[pages].reshape(-1, heads[1], D)[:length] for x in b.values)
    q, G, counted = f64(b.q), heads[0] // heads[1], 0
    for t in range(new):
        n = length - new + t + 1
        for h in range(heads[0]):
            x, reach = K[:n, h // G] @ q[t, h] * scale, (np.abs(K[:n, h // G]) @ np.abs(q[t, h])).max() * scale
            second, best = np.sort(x)[-2:]
            if best - second <= 100 + 2 * (D + 8) * U * reach:
                continue
            counted += 1
            v = V[int(x.argmax()), h // G]
            assert (np.abs(out[t, h] - v) <= 2 * HALF[dtype] * np.abs(v) * (1 + HALF[dtype]) + (2.0 ** -25 if dtype == "f16" else 0)).all(), (t, h)
    assert counted > new * heads[0] * 0.9 and np.isfinite(out).all()
