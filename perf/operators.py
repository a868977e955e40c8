"""Cases of the operators around the experts of an MoE layer, each in its plain form and as the library's call.

The operators: the root-mean-square norm that takes in the residual's addition and can answer in 8 bits with scales,
its gradient, token rows sorted by expert, the rows brought back to their tokens with the router's weights (without
weights this is the gradient of the sort), and the gradient of the weighted return.

`run` computes the plain form (elementary torch operations in 32 bits, rounded once at the end) while `own` is false
and calls the library where it is true.  `exact` gives the same outputs from the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0
AMAX_FLOOR = 2.0 ** -100      # an all-zero group of columns still gets a positive scale
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1, "none": 0}
NO_QUANT = -1                 # "group" of a norm case without 8-bit output; 0 is one scale per row


# ---- cases -----------------------------------------------------------------------------------------------------
def _norm(rows, d, dtype, add, wdtype, group, out=True):
    return dict(op="norm", rows=rows, d=d, dtype=dtype, add=add, wdtype=wdtype, group=group, out=out)


def _norm_grad(rows, d, dtype, wdtype, dsum):
    return dict(op="norm_grad", rows=rows, d=d, dtype=dtype, wdtype=wdtype, dsum=dsum)


def _dispatch(layers, tokens, k, experts, d, dtype, group, masked):
    return dict(op="dispatch", layers=layers, tokens=tokens, k=k, experts=experts, d=d, dtype=dtype, group=group,
                masked=masked)


def _combine(layers, tokens, k, experts, d, dtype, out_dtype, weights, add, masked):
    return dict(op="combine", layers=layers, tokens=tokens, k=k, experts=experts, d=d, dtype=dtype,
                out_dtype=out_dtype, weights=weights, add=add, masked=masked)


def _combine_grad(layers, tokens, k, experts, d, dtype, out_dtype, masked):
    return dict(op="combine_grad", layers=layers, tokens=tokens, k=k, experts=experts, d=d, dtype=dtype,
                out_dtype=out_dtype, masked=masked)


def listed():
    return [
        # the norm between two layers of the chained decode step when a single stream is served (latency)
        dict(_norm(1, 2048, "bf16", "f32", "f32", NO_QUANT), name="norm one stream"),
        # the same for a step of 512 streams whose experts read 8-bit rows: the router keeps its bf16 row
        dict(_norm(512, 2048, "bf16", "f32", "f32", 128), name="norm to 8 bits 512 streams"),
        # the norm of a training or prompt batch at the widest model of this repository
        dict(_norm(16384, 4096, "bf16", "bf16", "bf16", NO_QUANT), name="norm batch 16384x4096"),
        # its gradient where the residual stream brings a gradient of its own
        dict(_norm_grad(16384, 2048, "bf16", "bf16", True), name="norm grad 16384x2048"),
        # an odd width and a ragged batch in fp32
        dict(_norm_grad(1001, 1411, "f32", "f32", False), name="norm grad 1001x1411 f32"),
        # one decode step of all layers at once (60 experts, 4 selected, 256 streams, 24 layers)
        dict(_dispatch(24, 256, 4, 60, 2048, "bf16", 0, 0.0), name="dispatch decode 24 layers"),
        # a packed prompt batch of 8-bit rows with their scales; a tenth of the pairs is padding
        dict(_dispatch(1, 16384, 8, 64, 2048, "e4m3", 128, 0.1), name="dispatch prompt 8 bits"),
        # expert outputs of one stream back to its hidden row, 16 layers at once (latency)
        dict(_combine(16, 1, 8, 64, 2048, "f32", "f32", True, False, 0.0), name="combine one stream"),
        # expert outputs of a batch back to the residual stream, some pairs dropped
        dict(_combine(1, 16384, 6, 64, 2048, "bf16", "bf16", True, True, 0.1), name="combine batch"),
        # the gradient of the sort: the sum of a token's rows, without weights; a ragged batch, wide rows, 8 experts
        dict(_combine(1, 4099, 2, 8, 4096, "bf16", "bf16", False, False, 0.0), name="dispatch grad ragged"),
        # the gradient of the weighted return on a training batch
        dict(_combine_grad(1, 16384, 8, 64, 2048, "bf16", "bf16", 0.0), name="combine grad batch"),
        # the same on a small ragged batch in fp32 whose rows are no multiple of 16 bytes, many pairs dropped
        dict(_combine_grad(1, 777, 3, 10, 1002, "f32", "f32", 0.3), name="combine grad ragged f32"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng):
    """Mostly model widths (a multiple of 64), sometimes any number."""
    d = _spread(rng, 64, 8192)
    return d if rng.random() < 0.3 else max(64, d // 64 * 64)


def draw(rng):
    limit = 500e6    # bytes: below the largest listed case
    while True:
        op = rng.choice(["norm", "norm_grad", "dispatch", "combine", "combine_grad"])
        d, dtype = _width(rng), rng.choice(["bf16", "bf16", "f32"])
        if op == "norm":
            group = rng.choice([NO_QUANT, NO_QUANT, 0, 32, 64, 128])
            c = _norm(_spread(rng, 1, 20000), d, dtype, rng.choice(["none", "f32", dtype]), rng.choice(["f32", dtype]),
                      group, group == NO_QUANT or rng.random() < 0.5)
        elif op == "norm_grad":
            c = _norm_grad(_spread(rng, 1, 20000), d, dtype, rng.choice(["f32", dtype]), rng.random() < 0.5)
        else:
            experts = _spread(rng, 4, 256)
            k = rng.randint(1, min(8, experts))
            layers = 1 if rng.random() < 0.6 else _spread(rng, 2, 32)
            tokens = _spread(rng, 1, 20000 if layers == 1 else 512)
            masked = rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.5), 3)])
            if op == "dispatch":
                rows = rng.choice(["bf16", "f32", "e4m3"])
                c = _dispatch(layers, tokens, k, experts, d, rows, rng.choice([0, 32, 128]) if rows == "e4m3" else 0,
                              masked)
            elif op == "combine":
                weights = rng.random() < 0.7
                c = _combine(layers, tokens, k, experts, d, dtype, rng.choice(["f32", dtype]), weights,
                             weights and rng.random() < 0.5, masked)
            else:
                c = _combine_grad(layers, tokens, k, experts, d, dtype, rng.choice(["f32", dtype]), masked)
        if work(c)["bytes"] <= limit:
            return c


def _scale_cols(c):
    if c["op"] == "dispatch" and c["dtype"] != "e4m3":
        return 0
    return -(-c["d"] // c["group"]) if c["group"] else 1


def work(case):
    c = case
    d = c["d"]
    if c["op"] == "norm":
        n = c["rows"] * d
        b = n * (BYTES[c["dtype"]] * (1 + (c["add"] != "none") + c["out"]) + BYTES[c["add"]]) + d * BYTES[c["wdtype"]]
        if c["group"] != NO_QUANT:
            b += n + c["rows"] * _scale_cols(c) * 4
        return {"bytes": b, "flops": n * (5 + 3 * (c["group"] != NO_QUANT))}
    if c["op"] == "norm_grad":
        n = c["rows"] * d
        return {"bytes": n * BYTES[c["dtype"]] * (3 + c["dsum"]) + d * (BYTES[c["wdtype"]] + 4), "flops": 11 * n}
    tokens = c["layers"] * c["tokens"]
    pairs = tokens * c["k"]
    kept = round(pairs * (1 - c["masked"]))
    row, wide = d * BYTES[c["dtype"]], d * BYTES[c.get("out_dtype", "none")]
    if c["op"] == "dispatch":
        row += 4 * _scale_cols(c)
        return {"bytes": (tokens + kept) * row + pairs * 8 + kept * 4 + c["layers"] * (c["experts"] + 1) * 4,
                "flops": pairs}
    if c["op"] == "combine":
        return {"bytes": kept * row + tokens * wide * (1 + c["add"]) + pairs * 4 * (1 + c["weights"]),
                "flops": 2 * kept * d}
    return {"bytes": 2 * kept * row + tokens * wide + pairs * 12, "flops": 3 * kept * d}


# ---- inputs ----------------------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def _routing(c, gen):
    """Selected experts [L,T,K]: distinct per token, some experts more popular than others; masked pairs hold -1."""
    L, T, E, K = c["layers"], c["tokens"], c["experts"], c["k"]
    score = _normal(gen, L, T, E) + 0.7 * _normal(gen, L, 1, E)
    sel = torch.topk(score, K, dim=-1).indices.to(torch.int32)
    if c["masked"]:
        sel[torch.rand(L, T, K, device="cuda", generator=gen) < c["masked"]] = -1
    return sel


def _sorted_order(sel, E):
    """offsets [L,E+1], order [L,T*K] (pairs by expert, masked ones last) and the position of every pair, -1 masked
    (in the shape of sel)."""
    L, P = sel.shape[0], sel[0].numel()
    e = sel.reshape(L, P).long()
    e = torch.where((e >= 0) & (e < E), e, torch.full_like(e, E))
    order = torch.argsort(e, dim=1, stable=True)
    count = torch.zeros(L, E + 1, dtype=torch.long, device=sel.device).scatter_add_(1, e, torch.ones_like(e))
    offsets = torch.cat([torch.zeros_like(count[:, :1]), count[:, :E].cumsum(1)], 1)
    place = torch.empty_like(order).scatter_(1, order, torch.arange(P, device=sel.device).expand(L, P).contiguous())
    place = torch.where(e < E, place, torch.full_like(place, -1))
    return offsets.to(torch.int32), order.to(torch.int32), place.to(torch.int32).view_as(sel)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    d = c["d"]
    s = {"c": c}
    dt = DTYPES[c["dtype"]]
    if c["op"] in ("norm", "norm_grad"):
        R = c["rows"]
        # a residual stream has a few channels that are much larger than the others
        channel = 1.0 + 8.0 * (torch.rand(d, device="cuda", generator=gen) < 0.01)
        s["x"] = (_normal(gen, R, d) * channel).to(dt)
        s["weight"] = (1.0 + 0.1 * _normal(gen, d)).to(DTYPES[c["wdtype"]])
        if c["op"] == "norm":
            s["add"] = None if c["add"] == "none" else (0.5 * _normal(gen, R, d)).to(DTYPES[c["add"]])
            s["sum"] = None if c["add"] == "none" else torch.empty_like(s["x"])
            s["out"] = torch.empty_like(s["x"]) if c["out"] else None
            s["q"] = s["scales"] = None
            if c["group"] != NO_QUANT:
                s["q"] = torch.empty(R, d, dtype=torch.float8_e4m3fn, device="cuda")
                s["scales"] = torch.empty(R, _scale_cols(c), device="cuda")
        else:
            s["dout"] = _normal(gen, R, d).to(dt)
            s["dsum"] = _normal(gen, R, d).to(dt) if c["dsum"] else None
            s["dx"] = torch.empty_like(s["x"])
            s["dweight"] = torch.empty(d, device="cuda")
        return s
    L, T, K = c["layers"], c["tokens"], c["k"]
    P = T * K
    sel = _routing(c, gen)
    if c["op"] == "dispatch":
        s["sel"] = sel
        s["x"] = _normal(gen, L, T, d).to(dt)
        n = _scale_cols(c)
        s["scales"] = torch.rand(L, T, n, device="cuda", generator=gen) + 0.1 if n else None
        # what lies behind a layer's last sorted row is left as it was
        s["offsets"] = torch.zeros(L, c["experts"] + 1, dtype=torch.int32, device="cuda")
        s["perm"] = torch.full((L, P), -1, dtype=torch.int32, device="cuda")
        s["inv"] = torch.empty_like(sel)
        s["rows"] = torch.zeros(L, P, d, device="cuda", dtype=torch.uint8 if dt.itemsize == 1 else dt).view(dt)
        s["row_scales"] = torch.zeros(L, P, n, device="cuda") if n else None
        return s
    _, _, s["inv"] = _sorted_order(sel, c["experts"])
    wide = DTYPES[c["out_dtype"]]
    s["rows"] = _normal(gen, L, P, d).to(dt)
    s["w"] = torch.softmax(_normal(gen, L, T, K), -1)
    if c["op"] == "combine":
        s["w"] = s["w"] if c["weights"] else None
        s["add"] = _normal(gen, L, T, d).to(wide) if c["add"] else None
        s["y"] = torch.empty(L, T, d, dtype=wide, device="cuda")
    else:
        s["dy"] = _normal(gen, L, T, d).to(wide)
        s["drows"] = torch.zeros(L, P, d, dtype=dt, device="cuda")
        s["dw"] = torch.empty(L, T, K, device="cuda")
    return s


# ---- the library's calls ---------------------------------------------------------------------------------------
def _own(s):
    from paper_2412_00099_b200 import binding as mb
    c = s["c"]
    if c["op"] == "norm":
        r = mb.rmsnorm(s["x"], s["weight"], EPS, add=s["add"],
                       quant_group=None if c["group"] == NO_QUANT else c["group"],
                       out=mb.NormOut(s["out"], s["sum"], s["q"], s["scales"]))
        return [r.sum, r.out, r.q, r.scales]
    if c["op"] == "norm_grad":
        return mb.rmsnorm_backward(s["dout"], s["x"], s["weight"], EPS, dsum=s["dsum"], out=(s["dx"], s["dweight"]))
    if c["op"] == "dispatch":
        r = mb.dispatch(s["sel"], c["experts"], s["x"], scales=s["scales"],
                        out=mb.Dispatched(s["offsets"], s["perm"], s["inv"], s["rows"], s["row_scales"]))
        return [r.offsets, r.perm, r.inv, r.rows, r.scales]
    if c["op"] == "combine":
        return mb.combine(s["rows"], s["inv"], s["w"], add=s["add"], out=s["y"])
    return mb.combine_backward(s["dy"], s["rows"], s["inv"], s["w"], out=(s["drows"], s["dw"]))


# ---- plain forms -----------------------------------------------------------------------------------------------
def _plain_norm(s):
    c, x = s["c"], s["x"].float()
    total = None
    if s["add"] is not None:
        total = (x + s["add"].float()).to(s["x"].dtype)
        x = total.float()
    n = x * (1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)) * s["weight"].float()
    q = scales = None
    if c["group"] != NO_QUANT:
        R, d, cols = c["rows"], c["d"], _scale_cols(c)
        g = c["group"] or d
        padded = torch.nn.functional.pad(n, (0, cols * g - d)).view(R, cols, g)
        scales = padded.abs().amax(2).clamp_min(AMAX_FLOOR) / E4M3_MAX
        q = (padded / scales.unsqueeze(2)).clamp(-E4M3_MAX, E4M3_MAX).view(R, cols * g)[:, :d].to(torch.float8_e4m3fn)
    return [total, n.to(s["x"].dtype) if c["out"] else None, q, scales]


def _plain_norm_grad(s):
    h, g, w = s["x"].float(), s["dout"].float(), s["weight"].float()
    inv = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    gw = g * w
    dx = inv * gw - h * (inv * inv * inv * (gw * h).mean(1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return [dx.to(s["x"].dtype), (g * (h * inv)).sum(0)]


def _plain_take(there, token, x, into):
    """Row `token` of x [L,T,d] at every sorted position that is `there`, the row of `into` [L,P,d] elsewhere."""
    dtype = x.dtype
    if dtype.itemsize == 1:                                # 8-bit rows are moved as bytes
        x, into = x.view(torch.uint8), into.view(torch.uint8)
    layer = torch.arange(x.shape[0], device=x.device).unsqueeze(1)
    return torch.where(there.unsqueeze(2), x[layer, token], into).view(dtype)


def _plain_dispatch(s):
    c = s["c"]
    offsets, order, place = _sorted_order(s["sel"], c["experts"])
    there = torch.arange(order.shape[1], device="cuda") < offsets[:, -1:]
    token = order.long() // c["k"]
    scales = None if s["scales"] is None else _plain_take(there, token, s["scales"], s["row_scales"])
    return [offsets, torch.where(there, order, s["perm"]), place, _plain_take(there, token, s["x"], s["rows"]), scales]


def _plain_gather(s):
    """Rows of every pair [L,T,K,d] in 32 bits, zero where the pair is masked."""
    L = s["c"]["layers"]
    layer = torch.arange(L, device="cuda").view(L, 1, 1)
    rows = s["rows"][layer, s["inv"].long().clamp_min(0)].float()
    return torch.where((s["inv"] >= 0).unsqueeze(3), rows, torch.zeros_like(rows))


def _plain_combine(s):
    rows = _plain_gather(s)
    y = (rows * s["w"].unsqueeze(3) if s["w"] is not None else rows).sum(2)
    if s["add"] is not None:
        y = y + s["add"].float()
    return y.to(s["y"].dtype)


def _plain_combine_grad(s):
    c = s["c"]
    dy = s["dy"].float()
    dw = (_plain_gather(s) * dy.unsqueeze(2)).sum(3)
    L, P = c["layers"], c["tokens"] * c["k"]
    # the pair at every sorted position; masked pairs go to a position behind the last one
    place = s["inv"].view(L, P).long()
    place = torch.where(place >= 0, place, torch.full_like(place, P))
    pair = torch.full((L, P + 1), -1, device="cuda").scatter_(1, place, torch.arange(P, device="cuda").expand(L, P))
    pair = pair[:, :P]
    layer = torch.arange(L, device="cuda").unsqueeze(1)
    drows = s["w"].view(L, P)[layer, pair.clamp_min(0)].unsqueeze(2) * dy[layer, pair.clamp_min(0) // c["k"]]
    return [torch.where((pair >= 0).unsqueeze(2), drows.to(s["rows"].dtype), s["drows"]), dw]


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "dispatch": _plain_dispatch,
            "combine": _plain_combine, "combine_grad": _plain_combine_grad}[state["c"]["op"]](state)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------
def _e4m3(v):
    """Nearest value with 4 significant bits, exponents from -6 (below it a fixed step of 2^-9), ties to even."""
    _, e = torch.frexp(v)                                  # |v| in [2^(e-1), 2^e)
    step = torch.ldexp(torch.ones_like(v), (e - 4).clamp_min(-9))
    return torch.round(v / step) * step


def _exact_norm(s):
    c = s["c"]
    h = s["x"].double()
    total = None
    if s["add"] is not None:
        total = h + s["add"].double()
        h = total.to(s["x"].dtype).double()                # the norm is defined on the stored residual stream
    rms = (h.square().sum(1) / c["d"] + EPS).sqrt()
    n = h / rms[:, None] * s["weight"].double()
    if c["group"] == NO_QUANT:
        return [total, n if c["out"] else None, None, None]
    g = c["group"] or c["d"]
    col = torch.arange(c["d"], device="cuda") // g
    top = torch.zeros(c["rows"], _scale_cols(c), dtype=torch.float64, device="cuda")
    top.scatter_reduce_(1, col.expand(c["rows"], -1), n.abs(), "amax")
    scales = top.clamp_min(AMAX_FLOOR) / E4M3_MAX
    return [total, n if c["out"] else None, _e4m3(n / scales[:, col]), scales]


def _exact_norm_grad(s):
    h, g, w = s["x"].double(), s["dout"].double(), s["weight"].double()
    d = s["c"]["d"]
    rms = (h.square().sum(1, keepdim=True) / d + EPS).sqrt()
    unit = h / rms
    dunit = g * w
    dx = (dunit - unit * (unit * dunit).sum(1, keepdim=True) / d) / rms
    return [dx if s["dsum"] is None else dx + s["dsum"].double(), torch.einsum("rd,rd->d", g, unit)]


def _exact_dispatch(s):
    c = s["c"]
    L, E, K = c["layers"], c["experts"], c["k"]
    sel = s["sel"].reshape(L, -1).cpu().numpy()
    perm, inv = np.full(sel.shape, -1, np.int32), np.full(sel.shape, -1, np.int32)
    offsets = np.zeros((L, E + 1), np.int32)
    rows = torch.zeros(s["rows"].shape, dtype=torch.float64, device="cuda")
    scales = None if s["scales"] is None else torch.zeros(s["row_scales"].shape, dtype=torch.float64, device="cuda")
    for l in range(L):
        buckets = [np.flatnonzero(sel[l] == e) for e in range(E)]
        flat = np.concatenate(buckets).astype(np.int32)
        offsets[l, 1:] = np.cumsum([len(b) for b in buckets])
        perm[l, : len(flat)] = flat
        inv[l, flat] = np.arange(len(flat), dtype=np.int32)
        src = torch.from_numpy(flat // K).long().cuda()
        rows[l, : len(flat)] = s["x"][l].double()[src]
        if scales is not None:
            scales[l, : len(flat)] = s["scales"][l].double()[src]
    return [torch.from_numpy(offsets), torch.from_numpy(perm), torch.from_numpy(inv.reshape(s["sel"].shape)), rows, scales]


def _exact_combine(s):
    c = s["c"]
    y = s["add"].double() if s["add"] is not None else torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
    inv = s["inv"]
    for l in range(c["layers"]):
        rows = s["rows"][l].double()
        for k in range(c["k"]):
            t = (inv[l, :, k] >= 0).nonzero()[:, 0]
            part = rows[inv[l, t, k].long()]
            y[l, t] += part if s["w"] is None else part * s["w"][l, t, k, None].double()
    return y


def _exact_combine_grad(s):
    c = s["c"]
    inv = s["inv"]
    drows = torch.zeros(s["rows"].shape, dtype=torch.float64, device="cuda")
    dw = torch.zeros(s["w"].shape, dtype=torch.float64, device="cuda")
    for l in range(c["layers"]):
        rows, dyl = s["rows"][l].double(), s["dy"][l].double()
        for k in range(c["k"]):
            t = (inv[l, :, k] >= 0).nonzero()[:, 0]
            at = inv[l, t, k].long()
            drows[l, at] = dyl[t] * s["w"][l, t, k, None].double()
            dw[l, t, k] = torch.einsum("td,td->t", rows[at], dyl[t])
    return [drows, dw]


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "norm_grad": _exact_norm_grad, "dispatch": _exact_dispatch,
            "combine": _exact_combine, "combine_grad": _exact_combine_grad}[case["op"]](s)
