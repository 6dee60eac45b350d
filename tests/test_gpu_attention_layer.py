"""An attention layer over a paged cache as a program runs it: prefill, then token by token, each stage against the same in 64 bits from what the stage before it left; with the experts behind it; as one
captured graph.

Tolerances: those of the stages' own tests (tests/test_gpu_cache_attention.py, tests/test_gpu_cache_append.py) and for the products, whose operands are what the layer holds, one rounding of the
result and K roundings of fp32 on the way."""
import numpy as np
import pytest
import torch

from oracle import cache_ref as R
from oracle import layer_ref as LR
from paper_2601_19092_amd import attention_layer as A
from paper_2601_19092_amd import binding as B
from paper_2601_19092_amd import moe_layer

pytestmark = pytest.mark.gpu

U, H16 = 2.0 ** -24, 2.0 ** -8
HIDDEN, HQ, HKV, D, PAGE = 256, 4, 2, 64, 16


def f64(t):
    return t.detach().cpu().to(torch.float32).double().numpy()


def layers(new, lengths, fp8, window=0, seed=1):
    """Layers of one set of weights and one cache for calls of the given numbers of new tokens."""
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s, std=1.0: (torch.randn(s, generator=g) * std).to(torch.bfloat16).cuda()  # noqa: E731
    S, most = len(lengths), max(-(-n // PAGE) for n in lengths)
    w = (1 + 0.1 * torch.randn(HIDDEN, generator=g)).cuda(), rnd((HQ + 2 * HKV) * D, HIDDEN, std=HIDDEN ** -0.5), rnd(HIDDEN, HQ * D, std=(HQ * D) ** -0.5)
    pages = S * most + 1
    table = torch.randperm(pages, generator=g)[:S * most].int().reshape(S, most).cuda()
    made = [A.AttentionLayer(T, S, *w, HQ, HKV, pages, PAGE, most, A.rotation_table(most * PAGE, D), fp8_cache=fp8, window=window) for T in new]
    for L in made[1:]:
        L.k_cache, L.v_cache, L.k_scales, L.v_scales = made[0].k_cache, made[0].v_cache, made[0].k_scales, made[0].v_scales
    return made, table, rnd


def held(L):
    out = []
    for c, s in ((L.k_cache, L.k_scales), (L.v_cache, L.v_scales)):
        out.append(f64(c) * (1.0 if s is None else f64(s)[..., None]))
    return out


def product_ok(got, x, w):
    want = x @ w.T
    assert (np.abs(got - want) <= H16 * np.abs(want) + (x.shape[1] + 8) * U * (np.abs(x) @ np.abs(w).T)).all()


def check(L, stream_in, x, stream, seq_rows, lengths, table, out, window, before):
    y64, _ = LR.rmsnorm(f64(stream_in) + f64(x), f64(L.norm_weight), 1e-6)
    assert (np.abs(f64(L.y) - y64) <= H16 * np.abs(y64) + 300 * U * np.abs(y64).max()).all()
    assert (np.abs(f64(stream) - (f64(stream_in) + f64(x))) <= H16 * np.abs(f64(stream))).all()
    T, no = L.qkv.shape[0], HQ * D
    qkv = f64(L.y) @ f64(L.w_qkv).T
    size = np.abs(f64(L.y)) @ np.abs(f64(L.w_qkv)).T
    # keys and values in the cache, and the turned queries, from the product in 64 bits: the product's rounding, H each of a pair, then their own
    q, k, v = (qkv[:, a:b].reshape(T, -1, D) for a, b in ((0, no), (no, no + HKV * D), (no + HKV * D, no + 2 * HKV * D)))
    worst = lambda m: 2 * (H16 * np.abs(m).max() + (HIDDEN + 8) * U * size.max())  # noqa: E731
    pages = L.k_cache.shape[0]
    wq, wk, wv = R.append(q, k, v, L.rotation.double().cpu().numpy(), seq_rows, lengths, table.cpu().numpy(), PAGE, pages, "halves")
    turned, (K, V) = f64(L.qkv[:, :no]).reshape(T, HQ, D), held(L)
    step = 2.0 ** -4 if L.k_scales is not None else H16
    for t in wq:
        assert (np.abs(turned[t] - wq[t]) <= 2 * worst(q) + H16 * np.abs(wq[t])).all()
    for got, want, m in ((K, wk, k), (V, wv, v)):
        for at in want:
            assert (np.abs(got[at] - want[at]) <= 2 * worst(m) + step * (np.abs(want[at]) + np.abs(want[at]).max() * 2.0 ** -5)).all()
    for got, old, want in ((K, before[0], wk), (V, before[1], wv)):
        for at in want:
            got, old = got.copy(), old.copy()
            got[at] = old[at] = 0
        assert (got == old).all(), "places of the other tokens are left as they are"
    o, spread, reach, seen = R.attention(turned, K, V, seq_rows, lengths, table.cpu().numpy(), D ** -0.5, True, window)
    E = (D + 8) * U * reach[..., None] + 4 * U
    tol = H16 * np.abs(o) + (H16 + np.expm1(2 * E) + 2 * (seen[:, None, None] + 64) * U) * spread
    assert (np.abs(f64(L.o).reshape(T, HQ, D) - o) <= tol).all()
    product_ok(f64(out), f64(L.o), f64(L.w_out))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("window", [0, 24])
def test_prefill_then_token_by_token(fp8, window):
    lengths = [40, 17, 29]
    (pre, one), table, rnd = layers([86, 3], [n + 6 for n in lengths], fp8, window)
    stream, x = rnd(86, HIDDEN), rnd(86, HIDDEN)
    rows = torch.tensor([0, 40, 57, 86], dtype=torch.int32).cuda()
    inp, before = stream.clone(), held(pre)
    out = pre.forward(stream, rows, torch.tensor(lengths, dtype=torch.int32).cuda(), table, x)
    check(pre, inp, x, stream, rows.cpu().numpy(), lengths, table, out, window, before)
    rows = torch.arange(4, dtype=torch.int32).cuda()
    for step in range(1, 6):
        now = [n + step for n in lengths]
        stream, x = rnd(3, HIDDEN), rnd(3, HIDDEN)
        inp, before = stream.clone(), held(one)
        out = one.forward(stream, rows, torch.tensor(now, dtype=torch.int32).cuda(), table, x)
        check(one, inp, x, stream, rows.cpu().numpy(), now, table, out, window, before)


def test_a_decoder_layer_captured():
    """Attention and experts behind one another as a graph: replayed with other streams and lengths, the bits of the eager calls; without x the stream stays, with `out` it is not written."""
    lengths = [33, 20]
    (one,), table, rnd = layers([2], [n + 8 for n in lengths], False, seed=3)
    E, inter = 8, 128
    experts = moe_layer.MoeLayer(2, 1 + 0.1 * rnd(HIDDEN).float(), rnd(E, HIDDEN, std=HIDDEN ** -0.5), rnd(E, 2 * inter, HIDDEN, std=HIDDEN ** -0.5), rnd(E, HIDDEN, inter, std=inter ** -0.5), 2)
    one.k_cache.copy_(rnd(*one.k_cache.shape)), one.v_cache.copy_(rnd(*one.v_cache.shape))
    stream, x, out = rnd(2, HIDDEN), rnd(2, HIDDEN), torch.zeros((2, HIDDEN), dtype=torch.bfloat16, device="cuda")
    rows, lens = torch.arange(3, dtype=torch.int32).cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()
    s = torch.cuda.Stream()
    keep = stream.clone()
    with torch.cuda.stream(s):
        A.decoder_layer(one, experts, stream, rows, lens, table, x, out=out)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        A.decoder_layer(one, experts, stream, rows, lens, table, x, out=out)
    for step in range(4):
        fresh, add = rnd(2, HIDDEN), rnd(2, HIDDEN)
        k0, v0 = one.k_cache.clone(), one.v_cache.clone()
        lens.copy_(torch.tensor([n + step for n in lengths], dtype=torch.int32))
        stream.copy_(fresh), x.copy_(add)
        g.replay()
        torch.cuda.synchronize()
        got, got_stream, k1 = out.clone(), stream.clone(), one.k_cache.clone()
        one.k_cache.copy_(k0), one.v_cache.copy_(v0)
        again, stream2 = torch.zeros_like(out), fresh.clone()
        A.decoder_layer(one, experts, stream2, rows, lens, table, add, out=again)
        torch.cuda.synchronize()
        assert torch.equal(got, again) and torch.equal(k1, one.k_cache) and torch.equal(got_stream, stream2)
        assert torch.isfinite(got).all()
    assert not torch.equal(keep, stream)
    before = stream.clone()
    one.forward(stream, rows, lens, table)
    torch.cuda.synchronize()
    assert torch.equal(before, stream)
