"""Timing cases of what stands around the experts' products of a mixture-of-experts layer, over the sizes, types and directions it is used at.

Four kinds of case; for each `run` makes the calls a user's program makes of paper_2601_19092_amd.binding, or computes the same in
elementary torch operations (`own` false):

  norm      axe_rmsnorm: root-mean-square norm of a residual stream after an addition; the result in 16 bits, or in e4m3 with a scale (fp32 or
            E8M0) per row and 128 columns, as the products read it; "backward": its gradients
  route     axe_route: which experts a token goes to, with which weights, and the order of the (token, choice) pairs by expert that the grouped
            product reads; "backward": the gradient of the logits
  dispatch  axe_rows_dispatch: the tokens' rows in that order, copied or quantised; "rows": the intermediate rows between the two products, quantised in place of order
  combine   axe_rows_combine: the weighted sum of a token's rows; "backward": the gradients of the rows and of the weights

Inputs come from the seed alone and are made on the GPU.
"""
from __future__ import annotations

import math

import torch

own = False

# the layer of the repository's grouped cases: hidden size, intermediate size, experts, experts per token
HIDDEN, INTER, EXPERTS, TOPK = 2048, 768, 128, 8
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "fp8": torch.float8_e4m3fn}
EPS = 1e-6


def listed():
    return [
        # one token of a decode step before the fp8 layer: the smallest call, where launch and latency count
        {"name": "norm fp8 1 token", "kind": "norm", "dir": "forward", "dtype": "bf16", "out": "fp8", "scales": "e8m0", "residual": True, "T": 1, "H": 2048},
        # a prefill chunk before an fp8 product of K = 8192 with fp32 scales per row
        {"name": "norm fp8 1000 x 8192", "kind": "norm", "dir": "forward", "dtype": "bf16", "out": "fp8", "scales": "f32", "residual": True, "T": 1000, "H": 8192},
        # no residual, a width that no vector divides
        {"name": "norm f16 2000 x 1999", "kind": "norm", "dir": "forward", "dtype": "f16", "out": "f16", "scales": "none", "residual": False, "T": 2000, "H": 1999},
        # a training step's batch through the layer's norm
        {"name": "norm backward 4096 x 2048", "kind": "norm", "dir": "backward", "dtype": "bf16", "out": "bf16", "scales": "none", "residual": True, "T": 4096, "H": 2048},
        # a decode step of one token, and a prefill or training batch, through the router of the 128-expert layer
        {"name": "route 1 token", "kind": "route", "dir": "forward", "dtype": "f32", "score": "softmax", "bias": False, "groups": 1, "kept": 1, "top2": False, "renorm": True, "pad": False, "T": 1, "E": 128, "k": 8},
        {"name": "route 4096 tokens", "kind": "route", "dir": "forward", "dtype": "f32", "score": "softmax", "bias": False, "groups": 1, "kept": 1, "top2": False, "renorm": True, "pad": False, "T": 4096, "E": 128, "k": 8},
        # sigmoid scores, a bias for balance, four of eight groups; a batch that ends in padding, whose rows have every expert masked
        {"name": "route groups 1000 tokens", "kind": "route", "dir": "forward", "dtype": "bf16", "score": "sigmoid", "bias": True, "groups": 8, "kept": 4, "top2": True, "renorm": True, "pad": True, "T": 1000, "E": 256, "k": 8},
        # the training step's gradient of the logits, of weights that are not renormalised (every expert of a token has one)
        {"name": "route backward 4096", "kind": "route", "dir": "backward", "dtype": "f32", "score": "softmax", "bias": False, "groups": 1, "kept": 1, "top2": False, "renorm": False, "pad": False, "T": 4096, "E": 128, "k": 8},
        # the layer's rows in the experts' order at a prefill, quantised on the way for the fp8 products
        {"name": "dispatch fp8 1024 tokens", "kind": "dispatch", "dir": "forward", "dtype": "bf16", "out": "fp8", "scales": "f32", "T": 1024, "E": 128, "k": 8, "H": 2048},
        # a decode batch's copies in 16 bits
        {"name": "dispatch f16 64 tokens", "kind": "dispatch", "dir": "forward", "dtype": "f16", "out": "f16", "scales": "none", "T": 64, "E": 128, "k": 8, "H": 2048},
        # the way back at a prefill, and its gradients in a training step: the largest
        {"name": "combine f16 4096 tokens", "kind": "combine", "dir": "forward", "dtype": "f16", "add": False, "T": 4096, "E": 128, "k": 8, "H": 2048},
        {"name": "combine backward 4096", "kind": "combine", "dir": "backward", "dtype": "bf16", "add": False, "T": 4096, "E": 128, "k": 8, "H": 2048},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "route", "route", "dispatch", "combine"])
    back = rng.random() < 0.4
    T = _log(rng, 1, 4096)
    if kind == "route":
        E = rng.choice([8, 16, 60, 64, 128, 160, 256, 512])
        groups = rng.choice([g for g in (1, 1, 1, 4, 8) if E % g == 0])
        kept = groups if groups == 1 else groups // 2
        k = min(rng.choice([1, 2, 4, 6, 8]), E // groups * kept)
        return {"kind": kind, "dir": "backward" if back else "forward", "dtype": rng.choice(["f32", "bf16", "f16"]), "score": rng.choice(["softmax", "sigmoid"]),
                "bias": rng.random() < 0.5, "groups": groups, "kept": kept, "top2": groups > 1 and rng.random() < 0.5, "renorm": k > 1 and rng.random() < 0.5,  # (one choice, renormalised, has weight one)
                "pad": rng.random() < 0.3, "T": T, "E": E, "k": k}
    H = _log(rng, 256, 8191)
    H = rng.choice([rng.choice([256, 512, 768, 1024, 1536, 2048, 2560, 3584, 4096, 5120, 7168, 8192]), H // 16 * 16 + 8, H | 1])   # a model's widths, and others
    dtype = rng.choice(["bf16", "f16", "f32"])
    largest = 2 * 4096 * TOPK * HIDDEN * 2                             # bytes of the largest listed case
    eb = 4 if dtype == "f32" else 2
    if kind == "norm":
        T = min(T, largest // (4 * H * eb) - 1)
        out = rng.choice([dtype, "fp8"]) if not back else dtype
        return {"kind": kind, "dir": "backward" if back else "forward", "dtype": dtype, "out": out, "scales": rng.choice(["f32", "e8m0"]) if out == "fp8" else "none",
                "residual": rng.random() < 0.6, "T": T, "H": H}
    E, k = rng.choice([8, 60, 128, 256]), rng.choice([1, 2, 4, 6, 8])
    while T * (2 * k + 1) * H * eb > largest:
        H = H // 2 | (H & 1)
    if kind == "combine":
        return {"kind": kind, "dir": "backward" if back else "forward", "dtype": dtype, "add": not back and rng.random() < 0.5, "T": T, "E": E, "k": k, "H": H}
    form = rng.choice(["copy", "quantise", "quantise", "rows"])
    if form == "rows":                                                 # between the two products: the order is there already
        E = k = 1
    return {"kind": kind, "dir": "rows" if form == "rows" else "forward", "dtype": dtype, "out": dtype if form == "copy" else "fp8",
            "scales": "none" if form == "copy" else rng.choice(["f32", "e8m0"]), "T": T, "E": E, "k": k, "H": H}


# ---- inputs ---------------------------------------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, std, dtype):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g).to(TORCH[dtype])


def _stream(g, T, H, dtype):
    """Rows of a residual stream: every row of a size of its own, a few columns that stand out, as trained models have them."""
    x = torch.empty((T, H), dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=g)
    rows = torch.empty((T, 1), dtype=torch.float32, device="cuda").normal_(0.0, 0.5, generator=g).exp_()
    cols = torch.empty((1, H), dtype=torch.float32, device="cuda").normal_(0.0, 0.5, generator=g).exp_()
    return (x * rows * cols).to(TORCH[dtype])


def _choices64(c, logits, bias):
    """What the experts, and the groups, are chosen by, in 64 bits."""
    x = logits.double()
    s = torch.softmax(x, 1) if c["score"] == "softmax" else torch.sigmoid(x)
    ch = s if bias is None else s + bias.double()
    per = c["E"] // c["groups"]
    in_groups = ch.reshape(-1, c["groups"], per)
    gs = in_groups.topk(min(2, per), 2).values.sum(2) if c["top2"] else in_groups.amax(2)
    return s, ch, gs


def _close(sorted_values, upto):
    """Rows with neighbours among the first `upto` + 1 of the descending values that 32 bits may not tell apart (equal ones are: the lower index)."""
    v = sorted_values[:, :upto + 1]
    if v.shape[1] < 2:
        return torch.zeros(v.shape[0], dtype=torch.bool, device=v.device)
    gap = v[:, :-1] - v[:, 1:]
    return ((gap > 0) & (gap < 8e-6 * (v[:, :-1].abs() + v[:, 1:].abs()))).any(1)


def _route_inputs(c, seed):
    """Logits of a router over mildly unbalanced experts, and the bias against that.  A row whose choice the rounding of its scores would make is drawn again."""
    g = _gen(seed)
    T, E = c["T"], c["E"]
    pop = torch.empty(E, dtype=torch.float32, device="cuda").normal_(0.0, 0.5, generator=g)
    bias = -0.1 * pop + 0.01 * torch.empty(E, dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=g) if c["bias"] else None

    def some(n):
        return (pop + torch.empty((n, E), dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=g)).to(TORCH[c["dtype"]])

    logits = some(T)
    for _ in range(40):
        s, ch, gs = _choices64(c, logits, bias)
        again = torch.zeros(T, dtype=torch.bool, device="cuda")
        if c["groups"] > 1:
            order = gs.sort(dim=1, descending=True, stable=True)
            again |= _close(order.values[:, c["kept"] - 1:c["kept"] + 1], 1)
            keep = torch.zeros_like(gs).scatter_(1, order.indices[:, :c["kept"]], 1.0).repeat_interleave(E // c["groups"], 1)
            ch = torch.where(keep > 0, ch, -math.inf)
        again |= _close(ch.sort(1, descending=True).values, c["k"])
        at = again.nonzero()[:, 0]
        if at.numel() == 0:
            break
        logits[at] = some(at.numel())
    if c["pad"]:
        logits[max(1, T - T // 32 - 1):] = -math.inf
    return logits, bias


def _order_inputs(c, g):
    """row_of of a routing, made by sorting: k different experts for every token."""
    T, E, k = c["T"], c["E"], c["k"]
    pop = torch.empty(E, dtype=torch.float32, device="cuda").normal_(0.0, 0.5, generator=g)
    noise = torch.empty((T, E), dtype=torch.float32, device="cuda").exponential_(1.0, generator=g)
    pick = (pop - noise.log()).topk(k, dim=1).indices
    at = pick.reshape(-1).sort(stable=True).indices
    row_of = torch.empty(T * k, dtype=torch.int32, device="cuda")
    row_of[at] = torch.arange(T * k, dtype=torch.int32, device="cuda")
    return row_of.reshape(T, k)


def _zeros(shape, dtype):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def _scale_buffer(c, rows):
    nb = -(-c["H"] // 128)
    # (an array of one-byte codes is read in words: room up to a whole one)
    return None if c["scales"] == "none" else _zeros((rows, nb), torch.float32) if c["scales"] == "f32" else _zeros((rows * nb + 3) // 4 * 4, torch.uint8)[:rows * nb].reshape(rows, nb)


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    s = {"case": c, "plan": None}
    if c["kind"] == "norm":
        T, H, dt = c["T"], c["H"], TORCH[c["dtype"]]
        s["x"] = _stream(g, T, H, c["dtype"])
        s["w"] = torch.empty(H, dtype=torch.float32, device="cuda").normal_(1.0, 0.2, generator=g)
        s["r"] = _stream(g, T, H, c["dtype"]) if c["residual"] else None
        if c["dir"] == "backward":                                     # r: what arrives at the stream itself
            s["dy"] = _normal(g, (T, H), 1.0, c["dtype"])
            s["dx"], s["dw"] = _zeros((T, H), dt), _zeros(H, torch.float32)
        else:
            s["sum"] = _zeros((T, H), dt) if c["residual"] else None
            s["y"], s["scales"] = _zeros((T, H), TORCH[c["out"]]), _scale_buffer(c, T)
        return s
    if c["kind"] == "route":
        T, E, k = c["T"], c["E"], c["k"]
        s["logits"], s["bias"] = _route_inputs(c, seed)
        if c["dir"] == "backward":
            s["ids"] = _route_plain(c, s["logits"], s["bias"])[0]
            s["dw"] = torch.empty((T, k), dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=g)
            s["dlogits"] = _zeros((T, E), TORCH[c["dtype"]])
        else:
            s["ids"], s["w"] = _zeros((T, k), torch.int32), _zeros((T, k), torch.float32)
            s["group_rows"], s["row_of"] = _zeros(E + 1, torch.int32), _zeros((T, k), torch.int32)
        return s
    T, k, H, dt = c["T"], c["k"], c["H"], TORCH[c["dtype"]]
    M = T * k
    s["row_of"] = None if c["dir"] == "rows" else _order_inputs(c, g)
    if c["kind"] == "dispatch":
        s["x"] = _stream(g, T, H, c["dtype"])
        s["rows"], s["scales"] = _zeros((M, H), TORCH[c["out"]]), _scale_buffer(c, M)
        return s
    s["rows"] = _normal(g, (M, H), 1.0, c["dtype"])
    s["w"] = torch.softmax(torch.empty((T, k), dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=g), 1)
    if c["dir"] == "backward":
        s["dout"] = _normal(g, (T, H), 1.0, c["dtype"])
        s["drows"], s["dw"] = _zeros((M, H), dt), _zeros((T, k), torch.float32)
    else:
        s["add"] = _stream(g, T, H, c["dtype"]) if c["add"] else None
        s["out"] = _zeros((T, H), dt)
    return s


# ---- the plain forms --------------------------------------------------------------------------------------------------------------------------

def _quantised_plain(y, scales):
    """(e4m3, scales) of the rows of y, a scale for every 128 columns."""
    T, H = y.shape
    nb = -(-H // 128)
    blocks = torch.nn.functional.pad(y, (0, nb * 128 - H)).reshape(T, nb, 128)
    a = blocks.abs().amax(2)
    if scales == "f32":
        sc = torch.where(a > 0, a / 448.0, 1.0)
        stored = sc
    else:
        m, e = torch.frexp(a / 448.0)                                  # a / 448 = m 2^e, 0.5 <= m < 1
        code = torch.where(a > 0, (e - (m == 0.5).int() + 127).clamp(1, 254), 127)
        sc = torch.exp2((code - 127).float())
        stored = code.to(torch.uint8)
    q = (blocks / sc[:, :, None]).clamp(-448.0, 448.0).reshape(T, nb * 128)[:, :H]
    return q.to(torch.float8_e4m3fn), stored


def _norm_plain(s):
    c = s["case"]
    h = s["x"].float()
    if c["dir"] == "backward":
        u = s["dy"].float() * s["w"]
        rho = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
        dx = rho * (u - h * rho.square() * (u * h).mean(1, keepdim=True))
        if s["r"] is not None:
            dx = dx + s["r"].float()
        return dx.to(s["x"].dtype), (s["dy"].float() * h * rho).sum(0)
    if s["r"] is not None:
        h = h + s["r"].float()
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * s["w"]
    stream = None if s["r"] is None else h.to(s["x"].dtype)
    if c["out"] != "fp8":
        return y.to(s["y"].dtype), stream
    q, sc = _quantised_plain(y, c["scales"])
    return q, _scales_out(c, sc), stream


def _scores_plain(c, logits):
    x = logits.float()
    if c["score"] == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-x))
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    t = e.sum(1, keepdim=True)
    return e / torch.where(t > 0, t, 1.0)


def _route_plain(c, logits, bias):
    T, E, k = c["T"], c["E"], c["k"]
    sc = _scores_plain(c, logits)
    ch = sc if bias is None else sc + bias
    ch = torch.where(logits.float() > -math.inf, ch, -math.inf)
    if c["groups"] > 1:
        per = E // c["groups"]
        best = ch.reshape(T, c["groups"], per).sort(2, descending=True).values
        if c["top2"] and per > 1:
            gs = best[:, :, 0] + torch.where(best[:, :, 1] > -math.inf, best[:, :, 1], 0.0)
        else:
            gs = best[:, :, 0]
        kept = gs.sort(dim=1, descending=True, stable=True).indices[:, :c["kept"]]
        keep = torch.zeros_like(gs).scatter_(1, kept, 1.0).repeat_interleave(per, 1)
        ch = torch.where(keep > 0, ch, -math.inf)
    order = ch.sort(dim=1, descending=True, stable=True)                   # equal choices: the lower index first
    ids = order.indices[:, :k]
    there = order.values[:, :k] > -math.inf
    w = torch.where(there, sc.gather(1, ids), 0.0)
    if c["renorm"]:
        t = w.sum(1, keepdim=True)
        w = w / torch.where(t > 0, t, 1.0)
    return torch.where(there, ids, -1).int(), w


def _order_plain(c, ids):
    T, E, k = c["T"], c["E"], c["k"]
    flat = torch.where(ids >= 0, ids, E).reshape(-1)
    at = flat.sort(stable=True).indices
    row_of = torch.empty(T * k, dtype=torch.int32, device=ids.device)
    row_of[at] = torch.arange(T * k, dtype=torch.int32, device=ids.device)
    counts = (flat[:, None] == torch.arange(E, device=ids.device)).sum(0)
    return torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int(), torch.where(flat < E, row_of, -1).reshape(T, k)


def _route_backward_plain(s):
    c = s["case"]
    sc = _scores_plain(c, s["logits"])
    there = s["ids"] >= 0
    ids = torch.where(there, s["ids"], 0).long()
    w = torch.where(there, sc.gather(1, ids), 0.0)
    g = torch.where(there, s["dw"], 0.0)
    if c["renorm"]:
        t = w.sum(1, keepdim=True)
        t = torch.where(t > 0, t, 1.0)
        g = torch.where(there, (g - (g * w).sum(1, keepdim=True) / t) / t, 0.0)
    ds = torch.zeros_like(sc).scatter_add_(1, ids, g)
    if c["score"] == "softmax":
        d = sc * (ds - (ds * sc).sum(1, keepdim=True))
    else:
        d = sc * (1.0 - sc) * ds
    return d.to(s["logits"].dtype)


def _rows_plain(s):
    c = s["case"]
    T, k, H = c["T"], c["k"], c["H"]
    if c["kind"] == "dispatch":
        x = s["x"].float()
        if s["row_of"] is not None:
            by_row = torch.empty(T * k, dtype=torch.int64, device=x.device)
            by_row[s["row_of"].reshape(-1).long()] = torch.arange(T * k, device=x.device) // k
            x = x[by_row]
        if c["out"] != "fp8":
            return x.to(s["rows"].dtype)
        q, sc = _quantised_plain(x, c["scales"])
        return q, _scales_out(c, sc)
    at = s["row_of"].reshape(-1).long()
    rows = s["rows"][at].float().reshape(T, k, H)
    if c["dir"] == "backward":
        do = s["dout"].float()
        dw = (rows * do[:, None, :]).sum(2)
        d = torch.empty_like(s["rows"])
        d[at] = (s["w"][:, :, None] * do[:, None, :]).reshape(T * k, H).to(d.dtype)
        return d, dw
    out = (rows * s["w"][:, :, None]).sum(1)
    if s["add"] is not None:
        out = out + s["add"].float()
    return out.to(s["out"].dtype)


def _scales_out(c, sc):
    """Scales as the values they stand for."""
    return sc if sc is None or c["scales"] == "f32" else sc.view(torch.float8_e8m0fnu)


# ---- the framework's calls ----------------------------------------------------------------------------------------------------------------------

def _plan(s):
    """The descriptor and the workspace that a program makes once for its sizes."""
    from paper_2601_19092_amd import binding as B
    c = s["case"]
    code = {"bf16": B.AXE_BF16, "f16": B.AXE_F16, "f32": B.AXE_F32, "fp8": B.AXE_FP8_E4M3}
    st = B.AXE_SCALE_E8M0 if c.get("scales") == "e8m0" else B.AXE_SCALE_F32
    words = 0
    if c["kind"] == "norm":
        d = B.RmsNormDesc(c["T"], c["H"], code[c["dtype"]], code[c["out"]], eps=EPS, scale_dtype=st)
        words = B.axe_rmsnorm_workspace(d) if c["dir"] == "backward" else 0
    elif c["kind"] == "route":
        d = B.RouteDesc(c["T"], c["E"], c["k"], code[c["dtype"]], score=B.AXE_ROUTE_SIGMOID if c["score"] == "sigmoid" else B.AXE_ROUTE_SOFTMAX,
                        groups=c["groups"], groups_kept=c["kept"], group_score=B.AXE_ROUTE_GROUP_TOP2 if c["top2"] else B.AXE_ROUTE_GROUP_MAX,
                        renorm=c["renorm"], bias=s["bias"])
        words = B.axe_route_workspace(d) if c["dir"] == "forward" else 0
    else:
        d = B.RowsDesc(c["T"], c["k"], c["T"] * c["k"], c["H"], code[c["dtype"]], code[c.get("out", c["dtype"])], scale_dtype=st)
    s["plan"] = B, d, torch.zeros(words, dtype=torch.int32, device="cuda") if words else None
    return s["plan"]


def run(state):
    s = state
    c = s["case"]
    if not own:
        if c["kind"] == "norm":
            return _norm_plain(s)
        if c["kind"] == "route":
            if c["dir"] == "backward":
                return _route_backward_plain(s)
            ids, w = _route_plain(c, s["logits"], s["bias"])
            return (ids, w) + _order_plain(c, ids)
        return _rows_plain(s)
    B, d, ws = s["plan"] or _plan(s)
    if c["kind"] == "norm":
        if c["dir"] == "backward":
            B.axe_rmsnorm_backward(d, s["dy"], s["x"], s["w"], s["dx"], dsum=s["r"], dweight=s["dw"], workspace=ws)
            return s["dx"], s["dw"]
        B.axe_rmsnorm(d, s["x"], s["w"], s["y"], residual=s["r"], sum_out=s["sum"], scales=s["scales"])
        return (s["y"], s["sum"]) if c["out"] != "fp8" else (s["y"], _scales_out(c, s["scales"]), s["sum"])
    if c["kind"] == "route":
        if c["dir"] == "backward":
            return B.axe_route_backward(d, s["logits"], s["ids"], s["dw"], s["dlogits"])
        B.axe_route(d, s["logits"], s["ids"], s["w"], s["group_rows"], s["row_of"], ws)
        return s["ids"], s["w"], s["group_rows"], s["row_of"]
    if c["kind"] == "dispatch":
        B.axe_rows_dispatch(d, s["x"], s["row_of"], s["rows"], scales=s["scales"])
        return s["rows"] if c["out"] != "fp8" else (s["rows"], _scales_out(c, s["scales"]))
    if c["dir"] == "backward":
        B.axe_rows_combine_backward(d, s["dout"], s["rows"], s["row_of"], s["w"], s["drows"], s["dw"])
        return s["drows"], s["dw"]
    return B.axe_rows_combine(d, s["rows"], s["row_of"], s["w"], s["out"], add=s["add"])


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------------------------------

def work(case):
    c = case
    width = {"bf16": 2, "f16": 2, "f32": 4, "fp8": 1}
    eb, T = width[c["dtype"]], c["T"]
    if c["kind"] == "route":
        E, k = c["E"], c["k"]
        if c["dir"] == "backward":                                     # the other experts' logits count where the scores are normalised over them
            read = T * (E if c["score"] == "softmax" and not c["renorm"] else k) * eb
            return {"bytes": read + T * k * 8 + T * E * eb, "flops": 6 * T * E}
        return {"bytes": T * E * eb + T * k * 12 + (E + 1) * 4 + (E * 4 if c["bias"] else 0), "flops": T * E * (4 + k)}
    H, k = c["H"], c.get("k", 1)
    ob = width[c.get("out", c["dtype"])]
    scale = {"none": 0, "f32": 4, "e8m0": 1}[c.get("scales", "none")] * -(-H // 128)
    if c["kind"] == "norm":
        if c["dir"] == "backward":
            return {"bytes": T * H * eb * (4 if c["residual"] else 3) + 8 * H, "flops": 12 * T * H}
        return {"bytes": T * H * (eb * (3 if c["residual"] else 1) + ob) + T * scale + 4 * H, "flops": 6 * T * H}
    order = 0 if c["dir"] == "rows" else T * k * 4
    if c["kind"] == "dispatch":
        return {"bytes": T * H * eb + T * k * (H * ob + scale) + order, "flops": 3 * T * H if scale else 0}
    if c["dir"] == "backward":
        return {"bytes": T * H * eb + 2 * T * k * H * eb + order + T * k * 8, "flops": 3 * T * k * H}
    return {"bytes": T * H * eb * (2 if c["add"] else 1) + T * k * H * eb + order + T * k * 4, "flops": 2 * T * k * H}


# ---- the same in 64 bits, from the definitions --------------------------------------------------------------------------------------------------------

def _blocks64(y, scales):
    """(y / s, s), s the scale of y's run of 128 columns."""
    q, s = torch.empty_like(y), []
    for b in range(0, y.shape[1], 128):
        part = y[:, b:b + 128]
        most = part.abs().max(1).values
        one = most / 448.0 if scales == "f32" else 2.0 ** torch.ceil(torch.log2(most / 448.0)).clamp(-126, 127)
        one = torch.where(most == 0, torch.ones_like(one), one)
        q[:, b:b + 128] = part / one[:, None]
        s.append(one)
    return q, torch.stack(s, 1)


def _exact_norm(c, s):
    x, w = s["x"].double(), s["w"].double()
    n = x.shape[1]
    if c["dir"] == "forward":
        h = x if s["r"] is None else x + s["r"].double()
        y = h / torch.sqrt((h * h).sum(1) / n + EPS)[:, None] * w[None, :]
        stream = None if s["r"] is None else h
        return (y, stream) if c["out"] != "fp8" else (*_blocks64(y, c["scales"]), stream)
    dy = s["dy"].double()
    rms = torch.sqrt((x * x).sum(1) / n + EPS)[:, None]
    unit = x / rms                                                     # d unit / d x = (1 - unit unit' / n) / rms
    du = dy * w[None, :]
    dx = (du - unit * ((du * unit).sum(1) / n)[:, None]) / rms
    return dx if s["r"] is None else dx + s["r"].double(), (dy * unit).sum(0)


def _exact_route(c, s):
    T, k = c["T"], c["k"]
    sc, ch, gs = _choices64(c, s["logits"], s["bias"])
    masked = torch.isneginf(s["logits"].double())
    sc = torch.where(masked, 0.0, sc)
    if c["dir"] == "backward":
        # of L = sum_j g_j w_j: the gradient by the scores, then through them
        ids = s["ids"].long()
        on = torch.zeros_like(sc)
        gd = torch.zeros_like(sc)
        t, j = (ids >= 0).nonzero(as_tuple=True)
        on[t, ids[t, j]] = 1.0
        gd[t, ids[t, j]] = s["dw"].double()[t, j]
        if c["renorm"]:
            total = (sc * on).sum(1, keepdim=True).clamp_min(1e-300)
            gd = on * (gd - (gd * sc).sum(1, keepdim=True) / total) / total
        return sc * (gd - (sc * gd).sum(1, keepdim=True)) if c["score"] == "softmax" else sc * (1 - sc) * gd
    left = torch.where(masked, -math.inf, ch)
    if c["groups"] > 1:
        per = c["E"] // c["groups"]
        out = gs.argsort(dim=1, descending=True, stable=True)[:, c["kept"]:]
        left.view(T, c["groups"], per)[torch.arange(T, device=out.device)[:, None], out] = -math.inf
    ids = torch.empty((T, k), dtype=torch.int64, device="cuda")
    for j in range(k):                                                 # the largest that is left, the first of equals
        top = left.max(1, keepdim=True).values
        first = (left == top).int().argmax(1)
        ids[:, j] = torch.where(top[:, 0] > -math.inf, first, -1)
        left[torch.arange(T, device="cuda"), first] = -math.inf
    w = torch.where(ids >= 0, sc.gather(1, ids.clamp_min(0)), 0.0)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
    return ids.int(), w, None, None


def _exact_rows(c, s):
    T, k = c["T"], c["k"]
    if c["kind"] == "dispatch":
        x = s["x"].double()
        rows = x if s["row_of"] is None else torch.empty((T * k, x.shape[1]), dtype=torch.float64, device="cuda")
        if s["row_of"] is not None:
            for j in range(k):
                rows[s["row_of"][:, j].long()] = x
        return rows if c["out"] != "fp8" else _blocks64(rows, c["scales"])
    if c["dir"] == "forward":
        out = torch.zeros((T, c["H"]), dtype=torch.float64, device="cuda") if s["add"] is None else s["add"].double()
        for j in range(k):
            out = out + s["w"][:, j:j + 1].double() * s["rows"][s["row_of"][:, j].long()].double()
        return out
    do = s["dout"].double()
    d, dw = torch.empty((T * k, c["H"]), dtype=torch.float64, device="cuda"), torch.empty((T, k), dtype=torch.float64, device="cuda")
    for j in range(k):
        at = s["row_of"][:, j].long()
        d[at] = s["w"][:, j:j + 1].double() * do
        dw[:, j] = (s["rows"][at].double() * do).sum(1)
    return d, dw


def exact(case, seed):
    c, s = case, prepare(case, seed)
    return (_exact_norm if c["kind"] == "norm" else _exact_route if c["kind"] == "route" else _exact_rows)(c, s)
