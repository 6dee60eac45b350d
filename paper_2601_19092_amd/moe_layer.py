"""A mixture-of-experts layer run with the library's entry points, one after the other on one stream:

    stream' = stream + x;  y = norm(stream') w              axe_rmsnorm
    logits  = y Wr                                          axe_gemm (fp32 result)
    experts, weights, the experts' order                    axe_route
    the tokens' rows in that order                          axe_rows_dispatch (fp8: quantised on the way)
    both products of every expert, gate in between          axe_gemm_grouped_pair, or in fp8 two axe_gemm_grouped with
                                                            the rows between them quantised by axe_rows_dispatch
    stream'[t] + the weighted sum of the token's rows       axe_rows_combine

All buffers are made once for a number of tokens; forward() allocates nothing, so it may be captured into a graph.

    python -m paper_2601_19092_amd.moe_layer [tokens ...]   times it and its parts, 16 bit and fp8
"""
from __future__ import annotations

from typing import Optional

from . import binding as B
from . import workloads as W


def interleaved(w):
    """(experts, gate rows then up rows, k) -> rows of both in runs of 16, as the gated epilogue reads them (a weight is laid out once)."""
    import torch
    E, n, k = w.shape
    return w.view(torch.uint8).reshape(E, 2, n // 32, 16, -1).transpose(1, 2).contiguous().view(w.dtype).reshape(E, n, k)


class MoeLayer:
    """norm_weight (hidden) fp32; router (experts, hidden) in the rows' type; gate_up (experts, 2 inter, hidden): gate rows, then up rows; down (experts, hidden, inter).
    fp8: gate_up and down are e4m3, with fp32 scales per 128 x 128 block, scales1 (experts, 2 inter / 128, hidden / 128) and scales2 (experts, hidden / 128, inter / 128)."""

    def __init__(self, tokens: int, norm_weight, router, gate_up, down, topk: int, scales1=None, scales2=None, eps: float = 1e-6, score: int = B.AXE_ROUTE_SOFTMAX,
                 bias=None, renorm: bool = True):
        import torch
        self.torch, self.T, self.k = torch, tokens, topk
        E, N1, H = gate_up.shape
        inter, M, half = N1 // 2, tokens * topk, router.dtype
        dt = {torch.bfloat16: B.AXE_BF16, torch.float16: B.AXE_F16}[half]
        self.fp8 = gate_up.dtype == torch.float8_e4m3fn
        if self.fp8 and half != torch.bfloat16:
            raise ValueError("the fp8 products write bf16")
        self.norm_weight, self.router, self.gate_up, self.down = norm_weight, router, interleaved(gate_up), down

        def new(*shape, dtype=half):
            return torch.zeros(shape, dtype=dtype, device="cuda")

        self.y, self.logits = new(tokens, H), new(tokens, E, dtype=torch.float32)
        self.ids, self.weights = new(tokens, topk, dtype=torch.int32), new(tokens, topk, dtype=torch.float32)
        self.group_rows, self.row_of = new(E + 1, dtype=torch.int32), new(tokens, topk, dtype=torch.int32)
        self.h, self.c = new(M, inter), new(M, H)
        self.norm = B.RmsNormDesc(tokens, H, dt, dt, eps=eps)
        self.router_product = B.GemmDesc(tokens, E, H, dt, B.AXE_F32, B.Layout(W.row_major_spec(tokens, H)), B.Layout(W.col_major_spec(H, E)),
                                         B.Layout(W.row_major_spec(tokens, E)), tokens * H, E * H, tokens * E)
        self.routing = B.RouteDesc(tokens, E, topk, score=score, bias=bias, renorm=renorm)
        self.route_ws = new(max(1, B.axe_route_workspace(self.routing)), dtype=torch.int32)
        wide = dt if not self.fp8 else B.AXE_FP8_E4M3
        self.a = new(M, H) if not self.fp8 else new(M, H, dtype=torch.uint8).view(torch.float8_e4m3fn)
        self.to_experts = B.RowsDesc(tokens, topk, M, H, dt, wide)
        self.back = B.RowsDesc(tokens, topk, M, H, dt, dt)
        self.a_scales = self.h8 = self.h_scales = self.sync = None
        if self.fp8:
            self.a_scales, self.h_scales = new(M, -(-H // 128), dtype=torch.float32), new(M, -(-inter // 128), dtype=torch.float32)
            self.h8 = new(M, inter, dtype=torch.uint8).view(torch.float8_e4m3fn)
            self.between = B.RowsDesc(M, 1, M, inter, dt, B.AXE_FP8_E4M3)
        else:
            self.sync = new(M + 1, dtype=torch.int32)
        self.first = B.GroupedGemmDesc(M, N1, H, E, B.Layout(W.row_major_spec(M, H)), B.Layout(W.gated_b_spec(H, N1, E)), B.Layout(W.row_major_spec(M, inter)),
                                       M * H, E * N1 * H, M * inter, wide, dt, epilogue=B.AXE_EPI_SWIGLU, scale_a=self.a_scales, scale_b=scales1)
        self.second = B.GroupedGemmDesc(M, H, inter, E, B.Layout(W.row_major_spec(M, inter)), B.Layout(W.spec([(E, H * inter, "m"), (inter, 1, "m"), (H, inter, "m")])),
                                        B.Layout(W.row_major_spec(M, H)), M * inter, E * H * inter, M * H, wide, dt, scale_a=self.h_scales, scale_b=scales2)

    def forward(self, stream, x=None, out=None, on: Optional[object] = None):
        """stream (tokens, hidden) becomes stream + x (x None: stays) and out (None: stream itself) that plus the experts' sum.  on: the torch stream to run on."""
        out = stream if out is None else out
        B.axe_rmsnorm(self.norm, x if x is not None else stream, self.norm_weight, self.y, residual=stream if x is not None else None,
                      sum_out=stream if x is not None else None, stream=on)
        B.axe_gemm(self.router_product, self.y, self.router, self.logits, stream=on)
        B.axe_route(self.routing, self.logits, self.ids, self.weights, self.group_rows, self.row_of, self.route_ws, stream=on)
        B.axe_rows_dispatch(self.to_experts, self.y, self.row_of, self.a, scales=self.a_scales, stream=on)
        if self.fp8:
            B.axe_gemm_grouped(self.first, self.a, self.gate_up, self.h, self.group_rows, stream=on)
            B.axe_rows_dispatch(self.between, self.h, None, self.h8, scales=self.h_scales, stream=on)
            B.axe_gemm_grouped(self.second, self.h8, self.down, self.c, self.group_rows, stream=on)
        else:
            B.axe_gemm_grouped_pair(self.first, self.second, self.a, self.gate_up, self.h, self.down, self.c, self.group_rows, self.sync, stream=on)
        return B.axe_rows_combine(self.back, self.c, self.row_of, self.weights, out, add=stream, stream=on)


def synthetic(tokens: int, fp8: bool, hidden: int = W.MOE_HIDDEN, inter: int = W.MOE_INTER, experts: int = W.MOE_EXPERTS, topk: int = W.MOE_TOPK, seed: int = 1, **kw):
    """(layer, stream, x) with random weights and rows."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)

    wt = torch.float8_e4m3fn if fp8 else torch.bfloat16
    s1 = s2 = None
    if fp8:                                                            # e4m3 weights of unit variance, their size in the scales
        s1 = torch.full((experts, 2 * inter // 128, hidden // 128), hidden ** -0.5, device="cuda")
        s2 = torch.full((experts, hidden // 128, inter // 128), inter ** -0.5, device="cuda")
    layer = MoeLayer(tokens, 1 + 0.1 * normal(hidden, dtype=torch.float32), normal(experts, hidden, std=hidden ** -0.5), normal(experts, 2 * inter, hidden, std=1 if fp8 else hidden ** -0.5, dtype=wt),
                     normal(experts, hidden, inter, std=1 if fp8 else inter ** -0.5, dtype=wt), topk, s1, s2, **kw)
    return layer, normal(tokens, hidden), normal(tokens, hidden)


def main(argv) -> None:
    import torch

    def us(f, n=200):
        for _ in range(100):
            f()
        a, b = torch.cuda.Event(True), torch.cuda.Event(True)
        a.record()
        for _ in range(n):
            f()
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b) / n * 1e3

    for tokens in [int(t) for t in argv] or [1, 64, 1024, 4096]:
        for fp8 in (False, True):
            L, stream, x = synthetic(tokens, fp8)
            zero, out = torch.zeros_like(x), torch.zeros_like(x)       # (the stream stays as it is over the passes)
            whole = us(lambda: L.forward(stream, zero, out=out))
            parts = {"norm": us(lambda: B.axe_rmsnorm(L.norm, zero, L.norm_weight, L.y, residual=stream, sum_out=stream)),
                     "router product": us(lambda: B.axe_gemm(L.router_product, L.y, L.router, L.logits)),
                     "route": us(lambda: B.axe_route(L.routing, L.logits, L.ids, L.weights, L.group_rows, L.row_of, L.route_ws)),
                     "dispatch": us(lambda: B.axe_rows_dispatch(L.to_experts, L.y, L.row_of, L.a, scales=L.a_scales)),
                     "combine": us(lambda: B.axe_rows_combine(L.back, L.c, L.row_of, L.weights, out, add=stream))}
            print(f"{tokens} tokens, {'fp8' if fp8 else 'bf16'}: {whole:.1f} us; " + ", ".join(f"{n} {t:.1f}" for n, t in parts.items()), flush=True)


if __name__ == "__main__":
    import sys
    main(sys.argv[1:])
