"""The e4m3 codes that axe_rmsnorm and axe_rows_dispatch write are those of the fp32 quotient y / s, to the bit: no tolerance.

On 16-bit rows y / s lies on a midpoint between two codes often (a run's largest magnitude is 448 s, and y and it have 8 or 11 bits), so the product with a rounded reciprocal is another code
once in some 2000 elements of bf16 rows: the tests here have a few hundred thousand."""
import pytest
import torch

from paper_2601_19092_amd import binding as B

pytestmark = pytest.mark.gpu

CODE = {"bf16": B.AXE_BF16, "f16": B.AXE_F16, "f32": B.AXE_F32}
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def codes(y, kind):
    """(e4m3 bytes, scales) of fp32 rows by the definition; every step is one fp32 operation (the CPU's are correctly rounded)."""
    T, H = y.shape
    nb = -(-H // 128)
    blocks = torch.nn.functional.pad(y, (0, nb * 128 - H)).reshape(T, nb, 128)
    most = blocks.abs().amax(2)
    if kind == "f32":
        s = torch.where(most == 0, torch.ones_like(most), torch.div(most, torch.full_like(most, 448.0)).clamp_min(2.0 ** -126))
        stored = s
    else:
        e = torch.ceil(torch.log2(most.double() / 448.0)).clamp_min(-126.0)
        s = torch.where(most == 0, 0.0, e).exp2().float()
        stored = torch.where(most == 0, 127.0, e + 127).to(torch.uint8)
    q = (blocks / s[:, :, None]).clamp(-448.0, 448.0).reshape(T, nb * 128)[:, :H]
    return q.to(torch.float8_e4m3fn).view(torch.uint8), stored


def same_codes(q, sc, y, kind):
    want, s = codes(y, kind)
    assert torch.equal(sc.cpu(), s), "scales"
    off = (q.cpu().view(torch.uint8) != want).sum().item()
    assert off == 0, f"{off} of {want.numel()} codes are not those of the quotient"


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("T,H", [(300, 2048), (257, 1999), (40, 5), (700, 768)])
def test_quantised_rows(T, H, kind, dtype):
    x = torch.randn((T, H), generator=torch.Generator().manual_seed(T)).to(TORCH[dtype])
    q = torch.zeros((T, H), dtype=torch.uint8, device="cuda")
    sc = torch.zeros((T, -(-H // 128)), dtype=torch.float32 if kind == "f32" else torch.uint8, device="cuda")
    B.axe_rows_dispatch(B.RowsDesc(T, 1, T, H, CODE[dtype], B.AXE_FP8_E4M3, scale_dtype=int(kind == "e8m0")), x.cuda(), None, q, scales=sc)
    same_codes(q, sc, x.float(), kind)


@pytest.mark.parametrize("kind", ["f32", "e8m0"])
@pytest.mark.parametrize("T,H", [(300, 2048), (257, 1999), (40, 5), (70, 8192), (9, 20000)])
def test_quantised_norm(T, H, kind):
    """The rows that the norm quantises are the rows that it writes in fp32 (one computation, two forms of the result)."""
    x, w = (torch.randn(s, generator=torch.Generator().manual_seed(H)).bfloat16().float().cuda() for s in ((T, H), (H,)))
    y, q = torch.zeros((T, H), device="cuda"), torch.zeros((T, H), dtype=torch.uint8, device="cuda")
    sc = torch.zeros((T, -(-H // 128)), dtype=torch.float32 if kind == "f32" else torch.uint8, device="cuda")
    B.axe_rmsnorm(B.RmsNormDesc(T, H, B.AXE_F32, B.AXE_F32), x, w, y)
    B.axe_rmsnorm(B.RmsNormDesc(T, H, B.AXE_F32, B.AXE_FP8_E4M3, scale_dtype=int(kind == "e8m0")), x, w, q, scales=sc)
    same_codes(q, sc, y.cpu(), kind)


def test_norm_of_rows_that_are_their_own_norm():
    """Mean square 1 and eps 0: y = x exactly, so 16-bit rows reach their midpoints in the norm as well."""
    T, H = 200, 1024
    g = torch.Generator().manual_seed(1)
    # runs of eight magnitudes m / 64, m of 7 bits, whose squares add up to 8: drawn, and kept where the last one comes out whole
    m = torch.randint(1, 128, (200000, 7), generator=g)
    last = 8 * 64 * 64 - (m * m).sum(1)
    root = last.clamp_min(0).double().sqrt().round().long()
    runs = torch.cat([m, root[:, None]], 1)[(root * root == last) & (root > 0) & (root < 128)]
    assert len(runs) > 100
    pick = runs[torch.randint(0, len(runs), (T * H // 8,), generator=g)].reshape(T, H).float() / 64
    x = (pick * (torch.randint(0, 2, (T, H), generator=g) * 2 - 1)).bfloat16()
    assert torch.equal(x.double().square().mean(1), torch.ones(T, dtype=torch.float64))
    q, sc = torch.zeros((T, H), dtype=torch.uint8, device="cuda"), torch.zeros((T, H // 128), device="cuda")
    B.axe_rmsnorm(B.RmsNormDesc(T, H, B.AXE_BF16, B.AXE_FP8_E4M3, eps=0.0), x.cuda(), None, q, scales=sc)
    same_codes(q, sc, x.float(), "f32")


@pytest.mark.parametrize("which", ["any", "few bits", "near multiples", "tiny", "huge"])
def test_rows_next_to_midpoints(which):
    """Every element of a run is m s, m a midpoint of two codes, or one of the fp32 numbers beside it, for scales of every kind of mantissa: few bits above a multiple of 2^-3 among them, where
    quotients lie closest to what decides between two codes."""
    g = torch.Generator().manual_seed(3)
    T, nb = 3000, 4
    n = T * nb
    m24 = torch.randint(1 << 23, 1 << 24, (n,), generator=g)           # mantissas of the largest magnitudes
    if which == "few bits":
        m24 = torch.randint(128, 256, (n,), generator=g) << 16
    elif which == "near multiples":                                    # of scales: the largest that has such a scale
        s24 = (torch.randint(8, 16, (n,), generator=g) << 20) + torch.randint(-20, 21, (n,), generator=g)
        m24 = (s24.clamp_min(1 << 23).double() * 448 / 512).round().long()
        m24 = torch.where(m24 < 1 << 23, (s24.clamp_min(1 << 23).double() * 448 / 256).round().long(), m24)
    e = torch.randint(-20, 20, (n,), generator=g)
    if which == "tiny":
        e = torch.randint(-116, -100, (n,), generator=g)
    if which == "huge":
        e = torch.randint(90, 103, (n,), generator=g)
    most = (m24.double() * torch.exp2(e.double())).float()
    s = most / 448.0
    mids = torch.tensor([(2 * j + 1) / 1024 for j in range(8)] + [2.0 ** e * (1 + (2 * j + 1) / 16) for e in range(-6, 9) for j in range(8)])
    mids = mids[mids < 440]
    pick = mids[torch.randint(0, len(mids), (n, 128), generator=g)]
    x = (pick.double() * s[:, None].double()).float()
    x = (x.view(torch.int32) + torch.randint(-2, 3, (n, 128), generator=g).int()).view(torch.float32)
    x = torch.minimum(x, most[:, None]) * (torch.randint(0, 2, (n, 128), generator=g) * 2 - 1)
    x[:, 17] = most
    x = x.reshape(T, nb * 128)
    q, sc = torch.zeros((T, nb * 128), dtype=torch.uint8, device="cuda"), torch.zeros((T, nb), device="cuda")
    B.axe_rows_dispatch(B.RowsDesc(T, 1, T, nb * 128, B.AXE_F32, B.AXE_FP8_E4M3), x.cuda(), None, q, scales=sc)
    same_codes(q, sc, x, "f32")
