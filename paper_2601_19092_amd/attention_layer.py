"""An attention layer over a paged cache run with the library's entry points, one after the other on one stream; with a mixture-of-experts layer behind it (moe_layer.MoeLayer), a decoder layer
from the stream to the stream:

    stream' = stream + x;  y = norm(stream') w              axe_rmsnorm
    q, k, v = y Wqkv                                        axe_gemm, side by side in one row per token
    keys and values to the cache, q and k turned            axe_cache_append, q where it lies
    o = attention over the cache                            axe_cache_attention
    x' = o Wo                                               axe_gemm: what MoeLayer.forward(stream', x') adds to the stream

All buffers are made once for a number of rows and sequences; forward() allocates nothing, so it may be captured into a graph and replayed with other contents of seq_rows, lengths and the page table.

    python -m paper_2601_19092_amd.attention_layer [sequences ...]   times a decode step of it, alone and with the experts behind it, and a prefill
"""
from __future__ import annotations

from typing import Optional

from . import binding as B
from . import workloads as W


def rotation_table(positions: int, rotary_dim: int, base: float = 10000.0):
    """(positions, rotary_dim) fp32 on the device: cosines, then sines, of position / base^(2 i / rotary_dim), the angles computed in 64 bits."""
    import torch
    at = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, rotary_dim, 2, dtype=torch.float64) / max(rotary_dim, 1))
    return torch.cat([at.cos(), at.sin()], 1).float().cuda()


class AttentionLayer:
    """tokens: rows of a call (all sequences' new tokens), sequences: rows of the tables.  norm_weight (hidden) fp32; qkv ((q_heads + 2 kv_heads) head_dim, hidden) and out (hidden, q_heads head_dim)
    in bf16 or fp16; rotation: rotation_table of max_pages page_tokens positions.  fp8_cache: keys and values in e4m3."""

    def __init__(self, tokens: int, sequences: int, norm_weight, qkv, out, q_heads: int, kv_heads: int, pages: int, page_tokens: int, max_pages: int, rotation, fp8_cache: bool = False,
                 eps: float = 1e-6, window: int = 0, rotary_style: int = B.AXE_ROTATE_HALVES):
        import torch
        half = qkv.dtype
        dt = {torch.bfloat16: B.AXE_BF16, torch.float16: B.AXE_F16}[half]
        H, D = qkv.shape[1], qkv.shape[0] // (q_heads + 2 * kv_heads)
        self.norm_weight, self.w_qkv, self.w_out, self.rotation = norm_weight, qkv, out, rotation
        N, no = qkv.shape[0], q_heads * D

        def new(*shape, dtype=half):
            return torch.zeros(shape, dtype=dtype, device="cuda")

        self.y, self.qkv, self.o, self.x = new(tokens, H), new(tokens, N), new(tokens, no), new(tokens, H)
        place = (pages, page_tokens, kv_heads, D)
        self.k_cache, self.v_cache = ((new(*place, dtype=torch.uint8).view(torch.float8_e4m3fn) if fp8_cache else new(*place)) for _ in range(2))
        self.k_scales, self.v_scales = ((new(*place[:3], dtype=torch.float32) if fp8_cache else None) for _ in range(2))
        self.norm = B.RmsNormDesc(tokens, H, dt, dt, eps=eps)

        def product(n, k):
            return B.GemmDesc(tokens, n, k, dt, dt, B.Layout(W.row_major_spec(tokens, k)), B.Layout(W.col_major_spec(k, n)), B.Layout(W.row_major_spec(tokens, n)), tokens * k, n * k, tokens * n)

        self.first, self.last = product(N, H), product(H, no)
        of = lambda at, heads: B.Layout(W.spec([(tokens, N, "m"), (heads, D, "m"), (D, 1, "m")], O={"m": at}), ["m"])  # noqa: E731
        common = dict(cache_dtype=B.AXE_FP8_E4M3 if fp8_cache else dt, rotary_dim=rotation.shape[1], rotary_style=rotary_style, window=window, q=of(0, q_heads), k=of(no, kv_heads),
                      v=of(no + kv_heads * D, kv_heads))
        shape = (tokens, sequences, q_heads, kv_heads, D, pages, page_tokens, max_pages, dt)
        self.append = B.CacheDesc(*shape, out=of(0, q_heads), **common)
        self.attend = B.CacheDesc(*shape, **common)
        self.ws = new(max(1, B.axe_cache_attention_workspace(self.attend)), dtype=torch.int32)

    def forward(self, stream, seq_rows, lengths, page_table, x=None, on: Optional[object] = None):
        """stream (tokens, hidden) becomes stream + x (x None: stays); returns what the layer adds to it (the layer's own buffer).  on: the torch stream to run on."""
        B.axe_rmsnorm(self.norm, x if x is not None else stream, self.norm_weight, self.y, residual=stream if x is not None else None, sum_out=stream if x is not None else None, stream=on)
        B.axe_gemm(self.first, self.y, self.w_qkv, self.qkv, stream=on)
        B.axe_cache_append(self.append, self.qkv, self.qkv, self.k_cache, self.v_cache, seq_rows, lengths, page_table, rotation=self.rotation, q=self.qkv, q_out=self.qkv,
                           k_scales=self.k_scales, v_scales=self.v_scales, stream=on)
        B.axe_cache_attention(self.attend, self.qkv, self.k_cache, self.v_cache, seq_rows, lengths, page_table, self.o, k_scales=self.k_scales, v_scales=self.v_scales, workspace=self.ws, stream=on)
        B.axe_gemm(self.last, self.o, self.w_out, self.x, stream=on)
        return self.x


def decoder_layer(attention: AttentionLayer, experts, stream, seq_rows, lengths, page_table, x=None, out=None, on: Optional[object] = None):
    """Both halves of a decoder layer: stream + x (x None: stays), attention, experts (a moe_layer.MoeLayer for as many tokens).  Returns the stream behind it (out, or stream itself)."""
    return experts.forward(stream, attention.forward(stream, seq_rows, lengths, page_table, x, on), out=out, on=on)


def synthetic(sequences: int, new: int, longest: int, fp8_cache: bool = False, hidden: int = W.MOE_HIDDEN, q_heads: int = 32, kv_heads: int = 4, head_dim: int = 128, page_tokens: int = 64, seed: int = 1):
    """(layer, stream, (seq_rows, lengths, page_table)): `new` tokens of each sequence, the longest of `longest` tokens in all, the others from half of that on; random weights, rows and cache."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)

    lengths = [max(new, longest - s * longest // (2 * sequences)) for s in range(sequences)]
    most = -(-longest // page_tokens)
    pages = sequences * most
    table = torch.randperm(pages, generator=g, device="cuda").int().reshape(sequences, most)
    T, no = sequences * new, q_heads * head_dim
    layer = AttentionLayer(T, sequences, 1 + 0.1 * normal(hidden, dtype=torch.float32), normal(no + 2 * kv_heads * head_dim, hidden, std=hidden ** -0.5), normal(hidden, no, std=no ** -0.5), q_heads,
                           kv_heads, pages, page_tokens, most, rotation_table(most * page_tokens, head_dim), fp8_cache)
    for cache, scales in ((layer.k_cache, layer.k_scales), (layer.v_cache, layer.v_scales)):
        for page in range(0, pages, 1024):                             # (a part at a time: the numbers are drawn in fp32)
            part = cache[page:page + 1024]
            part.copy_(normal(*part.shape, std=100.0 if fp8_cache else 1.0, dtype=part.dtype))
        if fp8_cache:
            scales.fill_(0.01)
    return layer, normal(T, hidden), (torch.arange(0, T + 1, new, dtype=torch.int32, device="cuda"), torch.tensor(lengths, dtype=torch.int32, device="cuda"), table)


def main(argv) -> None:
    import torch

    from . import moe_layer

    def us(f, n=100):
        for _ in range(30):
            f()
        a, b = torch.cuda.Event(True), torch.cuda.Event(True)
        a.record()
        for _ in range(n):
            f()
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b) / n * 1e3

    def report(what, L, stream, tables, experts):
        zero, out = torch.zeros_like(stream), torch.zeros_like(stream)
        parts = {"norm": us(lambda: B.axe_rmsnorm(L.norm, zero, L.norm_weight, L.y, residual=stream, sum_out=stream)), "first product": us(lambda: B.axe_gemm(L.first, L.y, L.w_qkv, L.qkv)),
                 "append": us(lambda: B.axe_cache_append(L.append, L.qkv, L.qkv, L.k_cache, L.v_cache, *tables, rotation=L.rotation, q=L.qkv, q_out=L.qkv, k_scales=L.k_scales, v_scales=L.v_scales)),
                 "attention": us(lambda: B.axe_cache_attention(L.attend, L.qkv, L.k_cache, L.v_cache, *tables, L.o, k_scales=L.k_scales, v_scales=L.v_scales, workspace=L.ws)),
                 "last product": us(lambda: B.axe_gemm(L.last, L.o, L.w_out, L.x))}
        whole, both = us(lambda: L.forward(stream, *tables, zero)), us(lambda: decoder_layer(L, experts, stream, *tables, zero, out=out))
        print(f"{what}: {whole:.1f} us; " + ", ".join(f"{n} {t:.1f}" for n, t in parts.items()) + f"; with the experts behind it {both:.1f}", flush=True)

    for S in [int(s) for s in argv] or [1, 64]:
        for fp8 in (False, True):
            L, stream, tables = synthetic(S, 1, 4096, fp8)
            report(f"decode of {S} sequences up to 4096 tokens, cache in {'e4m3' if fp8 else 'bf16'}", L, stream, tables, moe_layer.synthetic(S, fp8)[0])
    L, stream, tables = synthetic(1, 4096, 4096)
    report("prefill of 4096 tokens", L, stream, tables, moe_layer.synthetic(4096, False)[0])


if __name__ == "__main__":
    import sys
    main(sys.argv[1:])
