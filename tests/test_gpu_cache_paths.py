"""Paths of the paged cache's kernels by the size of a call: rows of e4m3 caches, two and three a lane; e4m3 caches past 2^31 bytes; tables much wider than the sequences are long, as a program has them that
makes its descriptor once.  Tolerances: those of tests/test_gpu_cache_append.py and tests/test_gpu_cache_attention.py."""
import pytest
import torch

from paper_2601_19092_amd import binding as B
from paper_2601_19092_amd import workloads as W
from test_gpu_cache_append import Append
from test_gpu_cache_attention import WIDE, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, cache", [("bf16", "fp8"), ("f16", "fp8"), ("f16", "f16")])
@pytest.mark.parametrize("style", ["halves", "pairs"])
@pytest.mark.parametrize("Hq, Hkv, D, rotary", [(32, 8, 64, 64), (40, 4, 128, 64), (39, 3, 80, 20), (20, 4, 256, 256), (13, 1, 192, 0)])
def test_rows_a_lane(dtype, cache, style, Hq, Hkv, D, rotary):
    """More than 2048 workgroups at a row a lane: two rows, three, with rows left over."""
    a = Append([1130, 7], [1100, 6], Hq, Hkv, D, 48, dtype, cache, rotary, style, seed=Hq, extra_rows=2)
    a.check(a.run())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("page, new, heads", [(16, 1, 4), (24, 1, 4), (16, 20, 4), (24, 20, 4), (16, 20, 33), (24, 20, 33)])
def test_an_e4m3_cache_past_2_to_the_31_bytes(dtype, page, new, heads):
    D, far = 64, 3 * 2 ** 30
    b = Batch([2 * page - 3], [new], heads, 1, D, page, dtype, "fp8", seed=23, spare=0)
    for i in range(2):
        codes = torch.as_strided(b.kv[i].view(torch.uint8), (2, page, 1, D), b.strides, 16)
        buf = torch.empty(far + page * D, dtype=torch.uint8, device="cuda")
        for p in range(2):
            buf[p * far:p * far + page * D] = codes[p].reshape(-1)
        b.kv[i] = buf.view(torch.float8_e4m3fn)
    b.layout = B.Layout(W.spec([(2, far, "m"), (page, D, "m"), (D, 1, "m")]), ["m"])
    b.check(b.run())
    del buf
    b.kv.clear()
    torch.cuda.empty_cache()


def test_an_append_in_e4m3_past_2_to_the_31_bytes():
    a = Append([30], [30], 2, 1, 64, 16, cache="fp8", seed=11, shared=False, spare=0)
    far = 3 * 2 ** 30
    L = B.Layout(W.spec([(a.pages, far, "m"), (16, 64, "m"), (64, 1, "m")]), ["m"])
    d = B.CacheDesc(a.T, 1, 2, 1, 64, a.pages, 16, a.most, B.AXE_BF16, B.AXE_FP8_E4M3, rotary_dim=64, k_cache=L, v_cache=L)
    bufs = [torch.empty(far + 1024, dtype=torch.uint8, device="cuda") for _ in range(2)]
    for x in bufs:
        x[:1024], x[far:] = 0x55, 0x55
    out = torch.full((a.T, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    sc = [torch.full((a.pages, 16, 1), 5.0, device="cuda") for _ in range(2)]
    q, k, v = (x.contiguous().cuda() for x in (a.q, a.k, a.v))
    B.axe_cache_append(d, k, v, *(x.view(torch.float8_e4m3fn) for x in bufs), a.seq_rows.cuda(), torch.tensor([30], dtype=torch.int32).cuda(), a.table.cuda(), rotation=a.rotation.cuda(), q=q, q_out=out,
                       k_scales=sc[0], v_scales=sc[1])
    kc, vc = (torch.stack([x[:1024], x[far:]]).reshape(2, 16, 1, 64) for x in bufs)
    a.check((out, kc, vc, sc))


@pytest.mark.parametrize("width", [1, 40, 100, 600, 8192])
@pytest.mark.parametrize("dtype, cache", [("bf16", "bf16"), ("f16", "fp8")])
@pytest.mark.parametrize("lengths, new, heads, window", [([500], [1], (4, 2), 0), ([100] * 20, [9] * 20, (4, 2), 0), ([300], [300], (8, 8), 0), ([130, 9, 40], [70, 9, 1], WIDE, 0), ([300, 20], [200, 3], (48, 48), 100), ([90] * 70, [1] * 70, (16, 2), 30)])
def test_tables_wider_than_the_sequences_are_long(width, dtype, cache, lengths, new, heads, window):
    """Pages behind a sequence's last one belong to others, and are not seen: in one launch and in calls that are split for the keys there could be."""
    b = Batch(lengths, new, *heads, 64, 16, dtype, cache, seed=81)
    g = torch.Generator().manual_seed(width)
    if width > b.most:
        wide = torch.randint(0, b.pages, (len(lengths), width), generator=g, dtype=torch.int32)
        wide[:, :b.most] = torch.where(b.table < 0, wide[:, :b.most], b.table)
        b.table, b.most = wide, width
    b.check(b.run(window=window), window=window)
