"""Values that are not finite among those of a batch: by column what comes out is not finite exactly where a seen value is not, everything else is what it would be without them, and the
call takes no more than a few times as long as without them.  Tolerances: those of tests/test_gpu_cache_attention.py, and H |o| once more for tiles that count terms of e4m3 caches as rounded."""
import numpy as np
import pytest
import torch

from oracle import cache_ref as R
from test_gpu_cache_attention import HALF, U, WIDE, Batch, f64

pytestmark = pytest.mark.gpu

PAGE = 16
NAN, INF = float("nan"), float("inf")


def put(b, j, columns, bad, sequence=0):
    """Position j's value, in the given columns of every head, becomes `bad` (e4m3: its codes NaN, or with columns None its scale `bad`)."""
    at = int(b.table[sequence, j // PAGE]), j % PAGE
    v = torch.as_strided(b.kv[1].view(torch.uint8) if b.cache == "fp8" else b.kv[1], (b.pages, PAGE, b.Hkv, b.D), b.strides, 16)
    if b.cache == "fp8" and columns is None:
        b.scales[1][at] = bad
        b.values[1][at] = np.nan
    elif b.cache == "fp8":
        v[at][:, columns] = 0x7f
        b.values[1][at][:, columns] = np.nan
    else:
        v[at][:, slice(None) if columns is None else columns] = bad
        b.values[1][at][:, slice(None) if columns is None else columns] = bad


def check(b, out, window=0, causal=True):
    """Every element against the oracle's from the finite values, or not finite."""
    marked = ~np.isfinite(b.values[1])
    clean = [b.values[0], np.where(marked, 0.0, b.values[1])]
    want, spread, reach, seen = R.attention(f64(b.q), *clean, b.seq_rows.numpy(), b.lengths, b.table.numpy(), b.D ** -0.5, causal, window)
    H, E = HALF[b.dtype], (b.D + 8) * U * reach[..., None] + 4 * U
    scale = max(np.abs(clean[1]).max(), 0 if b.scales[1] is None else 448 * float(torch.nan_to_num(b.scales[1], 0, 0, 0).abs().max()))
    tol = 2 * H * np.abs(want) + (H + np.expm1(2 * E) + 2 * (seen[:, None, None] + 64) * U) * spread + (seen[:, None, None] * 2.0 ** -32 * scale + 2.0 ** -25 if b.dtype == "f16" else 0.0)
    got, G = f64(out), b.Hq // b.Hkv
    lost = np.zeros(got.shape, dtype=bool)
    for t, s, p in R.tokens(b.seq_rows.numpy(), b.lengths):
        for j in range(max(0, p - window + 1) if window else 0, p + 1 if causal else b.lengths[s]):
            at = R.place(b.table.numpy(), PAGE, b.pages, s, j)
            if at is not None and marked[at].any():
                lost[t] |= np.repeat(marked[at], G, axis=0)
    assert not np.isfinite(got[lost]).any()
    bad = ~(np.abs(got - want) <= tol) & ~lost
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}"
    return lost


SHAPES = [(90, 8, (4, 2)), (300, 40, (4, 2)), (90, 9, WIDE), (400, 140, (48, 48)), (2500, 30, (4, 2)), (2000, 9, WIDE)]   # tiles of 16, 32, 128 and 128 rows; the last two are split


@pytest.mark.parametrize("dtype, cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "fp8"), ("f16", "fp8")])
@pytest.mark.parametrize("length, new, heads", SHAPES)
@pytest.mark.parametrize("window", [0, 3, 20])
def test_single_elements_of_several_values(dtype, cache, length, new, heads, window):
    """New tokens' and old ones', each in columns of its own."""
    b = Batch([length], [new], *heads, 64, PAGE, dtype, cache, seed=61)
    first = length - new
    for i, j in enumerate(sorted({first, first + 1, first + new // 2, length - 2, first - 5, max(0, first - 17)})):
        put(b, j, [3 + i, 40 + i], [NAN, INF, -INF][i % 3])
    lost = check(b, b.run(window=window), window)
    assert lost.any() and not lost.all()


@pytest.mark.parametrize("dtype, cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "fp8"), ("f16", "fp8")])
@pytest.mark.parametrize("length, new, heads", SHAPES)
@pytest.mark.parametrize("window", [0, 3])
@pytest.mark.parametrize("bad", [NAN, INF])
def test_whole_values(dtype, cache, length, new, heads, window, bad):
    """Rows that are nothing but NaN (in e4m3: by their scale) among rows that have one such element."""
    b = Batch([length], [new], *heads, 64, PAGE, dtype, cache, seed=62)
    first = length - new
    put(b, first + new // 2, None, bad), put(b, first + new // 3, [5], bad), put(b, length - 1, [6], NAN), put(b, first + 1, [7], NAN)
    lost = check(b, b.run(window=window), window)
    assert lost.any() and not lost.all()


@pytest.mark.parametrize("dtype, cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "fp8"), ("f16", "fp8")])
@pytest.mark.parametrize("length, new, heads", SHAPES)
@pytest.mark.parametrize("causal", [True, False])
def test_old_values_that_all_see(dtype, cache, length, new, heads, causal):
    b = Batch([length, 50], [new, 2], *heads, 64, PAGE, dtype, cache, seed=63)
    put(b, 2, [1, 63], NAN), put(b, 30, [2], INF)
    check(b, b.run(causal=causal), causal=causal)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("length, new, heads", SHAPES)
@pytest.mark.parametrize("page_of_none", [False, True])
def test_a_scale_at_the_end_of_fp32_that_the_last_token_sees(dtype, length, new, heads, page_of_none):
    """In fp16, relative to the scales that the others see, it is an infinity.  (page_of_none: the page it is in is none, and nobody sees it.)"""
    b = Batch([length], [new], *heads, 64, PAGE, dtype, "fp8", seed=66)
    b.scales[1] /= 1024
    b.values[1] /= 1024
    j = length - 1
    b.scales[1][int(b.table[0, j // PAGE]), j % PAGE] = 2.0 ** 127
    if page_of_none:
        b.table[0, j // PAGE] = b.pages
    out = f64(b.run())
    clean = b.values[1].copy()
    if not page_of_none:
        clean[int(b.table[0, j // PAGE]), j % PAGE] = 0
    want, spread, reach, seen = R.attention(f64(b.q), b.values[0], clean, b.seq_rows.numpy(), b.lengths, b.table.numpy(), 64 ** -0.5)
    rows = slice(0, new if page_of_none else new - 1)
    H, E, n = HALF[dtype], (64 + 8) * U * reach[..., None] + 4 * U, seen[:, None, None]
    tol = 2 * H * np.abs(want) + (H + np.expm1(2 * E) + 2 * (n + 64) * U) * spread + (n * 2.0 ** -32 * np.abs(clean).max() * 2 + 2.0 ** -25 if dtype == "f16" else 0.0)
    assert (np.abs(out - want) <= tol)[rows].all()


def microseconds(b, window):
    a, z = torch.cuda.Event(True), torch.cuda.Event(True)
    from paper_2601_19092_amd import binding as B
    d = b.desc(window=window)
    q, out, rows, lens, table = b.q.cuda(), torch.zeros_like(b.q).cuda(), b.seq_rows.cuda(), torch.tensor(b.lengths, dtype=torch.int32).cuda(), b.table.cuda()
    ws, best = torch.zeros(max(1, B.axe_cache_attention_workspace(d)), dtype=torch.int32, device="cuda"), 1e9
    for _ in range(7):
        a.record()
        for _ in range(3):
            B.axe_cache_attention(d, q, b.kv[0], b.kv[1], rows, lens, table, out, k_scales=b.scales[0], v_scales=b.scales[1], workspace=ws)
        z.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(z) / 3 * 1e3)
    return best


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("length, new, heads, window", [(12000, 128, (48, 48), 0), (12000, 16, (2, 2), 0), (12000, 128, (48, 48), 9000)])   # tiles of 128 tokens, of 16
@pytest.mark.parametrize("what", ["a query", "an old value", "one new value", "all new values"])
def test_what_is_not_finite_does_not_take_a_pass_a_token(cache, length, new, heads, window, what):
    """A tile of 128 (16) tokens, with something that is not finite in each of its heads: at most 6 times as long as without it.  (A pass a token would be 100 times, 12 times.)"""
    b = Batch([length], [new], *heads, 64, PAGE, "bf16", cache, seed=65)
    clean = microseconds(b, window)
    if what == "a query":
        b.q[new // 2] = NAN
    elif what == "an old value":
        put(b, 7000, [5], INF)
    elif what == "one new value":
        put(b, length - new // 2, [5], INF)
    else:
        for j in range(length - new, length):
            put(b, j, None, NAN)
    us = microseconds(b, window)
    assert us <= 6 * clean, (us, clean)
