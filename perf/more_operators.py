"""Cases of the experts' own products on rows sorted by expert, each in its plain form and as the library's call.

The operators: a layer of every expert (with bias, activation and an added tensor, or gated: two projections, the activation
and the product of both), which can keep its pre-activations for the backward pass, in 8 bits too; its gradient with respect to
the rows, which can go through the activation of the layer below; its gradient with respect to weights and bias, from rows or
from their 8-bit checkpoint; and the checkpoint itself, into 8 bits and back.

Rows lie sorted by (layer, expert): group (l, e) is rows offsets[l][e] .. offsets[l][e + 1] of layer l.  Rows behind the last group
belong to nobody and are left as they were.

`run` computes the plain form (elementary torch operations in 32 bits, rounded once at the end) while `own` is false and calls
the library where it is true.  `exact` gives the same outputs from the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1 + 1 / 32, "none": 0}
E4M3_MAX = 448.0
BLOCK = 32                    # columns that share a power-of-two scale
SCALE_LOW = -127              # exponent of the smallest scale


# ---- cases -----------------------------------------------------------------------------------------------------
def _linear(layers, tokens, topk, experts, k, n, dtype, gated, act, bias, add, save, out_dtype, masked):
    return dict(op="linear", layers=layers, tokens=tokens, topk=topk, experts=experts, k=k, n=n, dtype=dtype, gated=gated,
                act=act, bias=bias, add=add, save=save, out_dtype=out_dtype, masked=masked)


def _backward(layers, tokens, topk, experts, k, n, dtype, gated, below, act, saved, add, masked):
    return dict(op="backward", layers=layers, tokens=tokens, topk=topk, experts=experts, k=k, n=n, dtype=dtype, gated=gated,
                below=below, act=act, saved=saved, add=add, masked=masked)


def _dweight(layers, tokens, topk, experts, k, n, dtype, gated, x, bias, dw_dtype, accumulate, masked):
    return dict(op="dweight", layers=layers, tokens=tokens, topk=topk, experts=experts, k=k, n=n, dtype=dtype, gated=gated,
                x=x, bias=bias, dw_dtype=dw_dtype, accumulate=accumulate, masked=masked)


def _pack(rows, d, dtype):
    return dict(op="pack", rows=rows, d=d, dtype=dtype)


def _unpack(rows, d, dtype):
    return dict(op="unpack", rows=rows, d=d, dtype=dtype)


def listed():
    return [
        # gate and up projection of the experts that one token selected (latency; 60 experts, 4 selected)
        dict(_linear(1, 1, 4, 60, 2048, 1408, "bf16", True, "silu", False, False, "none", "bf16", 0.0), name="gated one token"),
        # the same for one decode step of 256 streams, two layers at once: every expert's weights are read for some 17 rows
        dict(_linear(2, 256, 4, 60, 2048, 1408, "bf16", True, "silu", False, False, "none", "bf16", 0.0), name="gated decode 256 streams"),
        # gate and up projection of a training batch that keeps its pre-activations in 8 bits; some rows are padding
        dict(_linear(1, 4096, 8, 64, 2048, 1024, "bf16", True, "silu", False, False, "e4m3", "bf16", 0.03), name="gated training 8-bit checkpoint"),
        # the down projection of one expert that sees every token (a shared expert), onto the residual stream
        dict(_linear(1, 8192, 1, 1, 14336, 4096, "bf16", False, "none", False, True, "none", "bf16", 0.0), name="down prompt dense"),
        # a two-layer expert's first layer with bias, odd widths, fp32, some rows dropped
        dict(_linear(1, 333, 3, 10, 1002, 515, "f32", False, "gelu", True, False, "f32", "f32", 0.1), name="first layer ragged f32"),
        # the gradient of the down projection and of the gate in one: from dy to the gradients of both projections and h again
        dict(_backward(1, 4096, 8, 64, 1024, 2048, "bf16", False, "gated", "silu", "e4m3", False, 0.03), name="gate gradient training"),
        # on to the rows: both projections' gradients times their weights
        dict(_backward(1, 4096, 4, 60, 2048, 1408, "bf16", True, "none", "none", "none", False, 0.0), name="row gradient training"),
        # the gradient through one biased layer with an odd number of rows, fp32
        dict(_backward(1, 99, 2, 6, 515, 259, "f32", False, "plain", "gelu", "f32", False, 0.0), name="row gradient ragged f32"),
        # weight gradients of both projections from rows that were kept in 8 bits
        dict(_dweight(1, 4096, 8, 64, 2048, 1024, "bf16", True, "e4m3", False, "bf16", False, 0.03), name="weight gradient 8-bit rows"),
        # weight and bias gradient of a small batch, added to what earlier batches left in fp32
        dict(_dweight(1, 257, 3, 12, 640, 1000, "bf16", False, "bf16", True, "f32", True, 0.0), name="weight gradient small accumulate"),
        # the rows of a training batch into their 8-bit checkpoint
        dict(_pack(16384, 4096, "bf16"), name="pack 16384x4096"),
        # and back, an odd width
        dict(_unpack(5001, 1411, "f32"), name="unpack 5001x1411 f32"),
    ]


MOST_FLOPS, MOST_BYTES, MOST_FLOPS_F32 = 400e9, 1.2e9, 20e9


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, most):
    """Mostly model widths (a multiple of 64), now and then a multiple of 8, sometimes any number."""
    d, p = _spread(rng, 64, most), rng.random()
    return d if p < 0.15 else max(8, d // 8 * 8) if p < 0.4 else max(64, d // 64 * 64)


def draw(rng):
    while True:
        op = rng.choice(["linear", "linear", "backward", "backward", "dweight", "dweight", "pack", "unpack"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        if op in ("pack", "unpack"):
            c = dict(op=op, rows=_spread(rng, 1, 20000), d=_width(rng, 8192), dtype=dtype)
        else:
            experts = 1 if rng.random() < 0.15 else _spread(rng, 2, 128)
            layers = 1 if rng.random() < 0.8 else rng.randint(2, 4)
            head = dict(layers=layers, tokens=_spread(rng, 1, 8192 if layers == 1 else 512), topk=rng.randint(1, min(8, experts)),
                        experts=experts, k=_width(rng, 4096), n=_width(rng, 4096), dtype=dtype,
                        masked=rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.4), 3)]))
            kept = rng.choice(["none", dtype, "e4m3"])
            act = rng.choice(["silu", "silu", "gelu"])
            if op == "linear":
                gated = rng.random() < 0.5
                c = _linear(gated=gated, act=act if gated or rng.random() < 0.6 else "none", bias=rng.random() < 0.4,
                            add=rng.random() < 0.3, save=kept, out_dtype=rng.choice(["f32", dtype, dtype]), **head)
            elif op == "backward":
                below = rng.choice(["none", "plain", "gated"])
                c = _backward(gated=rng.random() < 0.4, below=below, act="none" if below == "none" else act,
                              saved="none" if below == "none" else rng.choice([dtype, "e4m3"]),
                              add=below == "none" and rng.random() < 0.4, **head)
            else:
                c = _dweight(gated=rng.random() < 0.4, x=rng.choice([dtype, "e4m3"]), bias=rng.random() < 0.5,
                             dw_dtype=rng.choice(["f32", dtype]), accumulate=rng.random() < 0.4, **head)
        w = work(c)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= (MOST_FLOPS_F32 if dtype == "f32" else MOST_FLOPS):
            return c


def work(case):
    c = case
    if c["op"] in ("pack", "unpack"):
        n = c["rows"] * c["d"]
        return {"bytes": n * (BYTES[c["dtype"]] + 1) + c["rows"] * -(-c["d"] // BLOCK), "flops": 2 * n}
    two = 1 + c["gated"]
    rows = c["layers"] * c["tokens"] * c["topk"] * (1 - c["masked"])
    groups = c["layers"] * c["experts"]
    touched = groups * (1 - (1 - c["topk"] * (1 - c["masked"]) / c["experts"]) ** c["tokens"]) if c["experts"] > 1 else groups
    e, n, k = BYTES[c["dtype"]], c["n"] * two, c["k"]
    flops = 2 * rows * n * k
    if c["op"] == "linear":
        out = rows * c["n"]
        return {"bytes": touched * n * k * e + rows * k * e + out * BYTES[c["out_dtype"]] * (1 + c["add"]) + rows * n * BYTES[c["save"]]
                + c["bias"] * touched * n * 4, "flops": flops}
    if c["op"] == "backward":
        wide = {"none": 1, "plain": 1, "gated": 2}[c["below"]]
        return {"bytes": touched * n * k * e + rows * n * e + rows * k * (wide * e + wide * BYTES[c["saved"]] + (c["below"] != "none") * e
                + c["add"] * e), "flops": flops}
    return {"bytes": groups * n * (k + c["bias"] * 2) * BYTES[c["dw_dtype"]] * (1 + c["accumulate"]) + rows * n * e + rows * k * BYTES[c["x"]],
            "flops": flops}


# ---- inputs ----------------------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def _weights(gen, c, dt):
    """[L,E,n,k] of a trained layer's size, made layer by layer."""
    w = torch.empty(c["layers"], c["experts"], c["n"], c["k"], dtype=dt, device="cuda")
    w.normal_(0.0, c["k"] ** -0.5, generator=gen)
    return w


def _groups(c, gen):
    """offsets [L,E+1] of the rows that a router leaves: distinct experts per token, some more popular than others, dropped pairs."""
    L, T, E, K = c["layers"], c["tokens"], c["experts"], c["topk"]
    score = _normal(gen, L, T, E) + 0.3 * _normal(gen, L, 1, E)
    sel = torch.topk(score, K, dim=-1).indices
    kept = torch.rand(L, T, K, device="cuda", generator=gen) >= c["masked"]
    count = torch.zeros(L, E, dtype=torch.long, device="cuda").scatter_add_(1, sel.view(L, -1), kept.view(L, -1).long())
    return torch.cat([torch.zeros_like(count[:, :1]), count.cumsum(1)], 1).to(torch.int32), int(count.max())


def _to_blocks(v):
    """Columns in blocks of 32, zeros behind the last."""
    blocks = -(-v.shape[-1] // BLOCK)
    return torch.nn.functional.pad(v, (0, blocks * BLOCK - v.shape[-1])).unflatten(-1, (blocks, BLOCK))


def _pack8(v):
    """e4m3 values and e8m0 scales of fp32 columns: the smallest power of two that brings a block's largest value to 448 at most."""
    b = _to_blocks(v)
    m, e = torch.frexp(b.abs().amax(-1) / E4M3_MAX)
    e = torch.where(m == 0, torch.full_like(e, SCALE_LOW), torch.where(m == 0.5, e - 1, e)).clamp_min(SCALE_LOW)
    q = torch.ldexp(b, -e.unsqueeze(-1)).flatten(-2)[..., : v.shape[-1]]
    return q.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _halves(v, pack):
    """pack applied to the two halves of the columns [gate | up], whose blocks do not mix."""
    a, b = (pack(h) for h in v.chunk(2, -1))
    return tuple(torch.cat([p.view(torch.uint8), q.view(torch.uint8)], -1).view(p.dtype) for p, q in zip(a, b))


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s, dt = {"c": c}, DTYPES[c["dtype"]]
    if c["op"] in ("pack", "unpack"):
        # activations: a few channels much larger than the others
        x = _normal(gen, c["rows"], c["d"]) * (1.0 + 8.0 * (torch.rand(c["d"], device="cuda", generator=gen) < 0.01))
        blocks = -(-c["d"] // BLOCK)
        if c["op"] == "pack":
            s["x"] = x.to(dt)
            s["q"] = torch.empty(c["rows"], c["d"], dtype=torch.float8_e4m3fn, device="cuda")
            s["scales"] = torch.empty(c["rows"], blocks, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
        else:
            s["q"], s["scales"] = _pack8(x.to(dt).float())
            s["x"] = torch.empty(c["rows"], c["d"], dtype=dt, device="cuda")
        return s
    L, R, n, k = c["layers"], c["tokens"] * c["topk"], c["n"], c["k"]
    two = 1 + c["gated"]
    s["offsets"], s["most"] = _groups(c, gen)
    if c["op"] == "linear":
        s["x"] = _normal(gen, L, R, k).to(dt)
        s["w"], s["w_up"] = _weights(gen, c, dt), _weights(gen, c, dt) if c["gated"] else None
        s["bias"] = 0.1 * _normal(gen, L, c["experts"], n) if c["bias"] else None
        s["bias_up"] = 0.1 * _normal(gen, L, c["experts"], n) if c["bias"] and c["gated"] else None
        out = DTYPES[c["out_dtype"]]
        s["add"] = _normal(gen, L, R, n).to(out) if c["add"] else None
        # rows that belong to no expert keep what they hold
        s["out"] = torch.zeros(L, R, n, dtype=out, device="cuda")
        s["saved"] = s["scales"] = None
        if c["save"] == "e4m3":
            s["saved"] = torch.zeros(L, R, two * n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
            s["scales"] = torch.zeros(L, R, two * -(-n // BLOCK), dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
        elif c["save"] != "none":
            s["saved"] = torch.zeros(L, R, two * n, dtype=dt, device="cuda")
        return s
    s["dout"] = _normal(gen, L, R, two * n).to(dt)
    if c["op"] == "backward":
        s["w"], s["w_up"] = _weights(gen, c, dt), _weights(gen, c, dt) if c["gated"] else None
        s["add"] = _normal(gen, L, R, k).to(dt) if c["add"] else None
        wide = 2 * k if c["below"] == "gated" else k
        s["saved"] = s["scales"] = s["h"] = None
        if c["below"] != "none":
            z = 1.5 * _normal(gen, L, R, wide)
            s["saved"] = z.to(dt)
            if c["saved"] == "e4m3":
                s["saved"], s["scales"] = _halves(z, _pack8) if c["below"] == "gated" else _pack8(z)
            s["h"] = torch.zeros(L, R, k, dtype=dt, device="cuda")
        s["dx"] = torch.zeros(L, R, wide, dtype=dt, device="cuda")
        return s
    s["x"], s["scales"] = _normal(gen, L, R, k).to(dt), None
    if c["x"] == "e4m3":
        s["x"], s["scales"] = _pack8(s["x"].float())
    dw, E = DTYPES[c["dw_dtype"]], c["experts"]

    shapes = [(L, E, n, k), (L, E, n, k) if c["gated"] else None, (L, E, n) if c["bias"] else None,
              (L, E, n) if c["bias"] and c["gated"] else None]
    s["into"] = [None if d is None else torch.empty(d, dtype=dw, device="cuda") for d in shapes]
    # what earlier batches left: a training step passes the buffers of `into` themselves, here they are apart so that passes are alike
    s["before"] = [None if d is None else _normal(gen, *d).to(dw) for d in shapes] if c["accumulate"] else None
    return s


# ---- the library's calls ---------------------------------------------------------------------------------------
def _name(act):
    return None if act == "none" else act


def _own(s):
    from paper_2412_00099_b200 import binding as mb
    c = s["c"]
    if c["op"] == "pack":
        return mb.checkpoint_pack(s["x"], out=mb.Checkpoint(s["q"], s["scales"]))
    if c["op"] == "unpack":
        return mb.checkpoint_unpack(s["q"], s["scales"], out=s["x"])
    if c["op"] == "linear":
        return mb.expert_linear(s["x"], s["offsets"], s["w"], w_up=s["w_up"], bias=s["bias"], bias_up=s["bias_up"], act=_name(c["act"]),
                                add=s["add"], out=mb.LinearOut(s["out"], s["saved"], s["scales"]))
    if c["op"] == "backward":
        return mb.expert_linear_backward(s["dout"], s["offsets"], s["w"], w_up=s["w_up"], saved=s["saved"], scales=s["scales"],
                                         act=_name(c["act"]), add=s["add"], out=mb.LinearGrad(s["dx"], s["h"]))
    return mb.expert_linear_dweight(s["dout"], s["x"], s["offsets"], scales=s["scales"], out=mb.WeightGrad(*s["into"]),
                                    add=None if s["before"] is None else mb.WeightGrad(*s["before"]))


# ---- plain forms -----------------------------------------------------------------------------------------------
def _unpack8(q, scales):
    return (_to_blocks(q.float()) * scales.float().unsqueeze(-1)).flatten(-2)[..., : q.shape[-1]]


def _unpack8_halves(q, scales):
    d, b = q.shape[-1] // 2, scales.shape[-1] // 2
    return torch.cat([_unpack8(q[..., :d], scales[..., :b]), _unpack8(q[..., d:], scales[..., b:])], -1)


def _act(z, act):
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_grad(z, act):
    if act == "silu":
        g = 1.0 / (1.0 + torch.exp(-z))
        return g * (1.0 + z * (1.0 - g))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    return torch.ones_like(z)


def _plain_places(s):
    """Every group's rows side by side: row numbers [G,most] in the flattened rows, L*R where a group has no more."""
    c, off = s["c"], s["offsets"].long()
    R = c["tokens"] * c["topk"]
    start = off + R * torch.arange(c["layers"], device="cuda").unsqueeze(1)
    first, last = start[:, :-1].reshape(-1, 1), start[:, 1:].reshape(-1, 1)
    row = first + torch.arange(s["most"], device="cuda")
    return torch.where(row < last, row, torch.full_like(row, c["layers"] * R))


def _take(rows, at):
    """Rows [L,R,d] at [G,most], a row of zeros at the end for places that hold none."""
    flat = rows.flatten(0, 1).float()
    return torch.cat([flat, flat.new_zeros(1, flat.shape[1])])[at]


def _put(grouped, at, into):
    """The reverse, into a copy of `into` and in its type."""
    flat = torch.cat([into.flatten(0, 1), into.new_zeros(1, into.shape[-1])])
    flat[at.reshape(-1)] = grouped.flatten(0, 1).to(into.dtype)
    return flat[:-1].view_as(into)


def _plain_linear(s):
    c, at = s["c"], _plain_places(s)
    x = _take(s["x"], at)

    def project(w, bias):
        z = torch.bmm(x, w.flatten(0, 1).float().transpose(1, 2))
        return z if bias is None else z + bias.flatten(0, 1).unsqueeze(1)
    z = project(s["w"], s["bias"])
    out = _act(z, c["act"])
    if c["gated"]:
        up = project(s["w_up"], s["bias_up"])
        out, z = out * up, torch.cat([z, up], -1)
    if s["add"] is not None:
        out = out + _take(s["add"], at)
    out = _put(out, at, s["out"])
    if c["save"] == "e4m3":
        q, scales = _halves(z, _pack8) if c["gated"] else _pack8(z)
        return [out] + [_put(v.view(torch.uint8), at, o.view(torch.uint8)).view(o.dtype) for v, o in ((q, s["saved"]), (scales, s["scales"]))]
    return [out, None if c["save"] == "none" else _put(z, at, s["saved"]), None]


def _plain_backward(s):
    c, at = s["c"], _plain_places(s)
    dout, n = _take(s["dout"], at), c["n"]
    t = torch.bmm(dout[..., :n], s["w"].flatten(0, 1).float())
    if c["gated"]:
        t = t + torch.bmm(dout[..., n:], s["w_up"].flatten(0, 1).float())
    if c["below"] == "none":
        return [_put(t if s["add"] is None else t + _take(s["add"], at), at, s["dx"]), None]
    z = s["saved"]
    if c["saved"] == "e4m3":
        z = _unpack8_halves(z, s["scales"]) if c["below"] == "gated" else _unpack8(z, s["scales"])
    z = _take(z, at)
    if c["below"] == "plain":
        return [_put(t * _act_grad(z, c["act"]), at, s["dx"]), _put(_act(z, c["act"]), at, s["h"])]
    g, up = z.chunk(2, -1)
    a = _act(g, c["act"])
    return [_put(torch.cat([t * up * _act_grad(g, c["act"]), t * a], -1), at, s["dx"]), _put(a * up, at, s["h"])]


def _plain_dweight(s):
    c, at = s["c"], _plain_places(s)
    dout = _take(s["dout"], at)
    x = _take(s["x"] if s["scales"] is None else _unpack8(s["x"], s["scales"]), at)

    def whole(grad, into, before):
        if into is None:
            return None
        grad = grad.view(into.shape)
        return (grad if before is None else grad + before.float()).to(into.dtype)
    parts = dout.chunk(1 + c["gated"], -1)
    dw = [torch.bmm(d.transpose(1, 2), x) for d in parts] + [None] * (1 - c["gated"])
    db = [d.sum(1) for d in parts] + [None] * (1 - c["gated"])
    return [whole(g, i, b) for g, i, b in zip(dw + db, s["into"], s["before"] or [None] * 4)]


def run(state):
    if own:
        return list(_own(state)) if state["c"]["op"] != "unpack" else _own(state)
    op = state["c"]["op"]
    if op == "pack":
        return list(_pack8(state["x"].float()))
    if op == "unpack":
        return _unpack8(state["q"], state["scales"]).to(state["x"].dtype)
    return {"linear": _plain_linear, "backward": _plain_backward, "dweight": _plain_dweight}[op](state)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------
def _e4m3(v):
    """Nearest value with 4 significant bits, exponents from -6 (below it a fixed step of 2^-9), ties to even."""
    _, e = torch.frexp(v)                                  # |v| in [2^(e-1), 2^e)
    step = torch.ldexp(torch.ones_like(v), (e - 4).clamp_min(-9))
    return torch.round(v / step) * step


def _exact_scales(v):
    """Scale of every block: the power of two s with largest / 448 <= s < largest / 224."""
    cols = v.shape[-1]
    blocks = -(-cols // BLOCK)
    top = torch.zeros(v.shape[:-1] + (blocks,), dtype=torch.float64, device="cuda")
    top.scatter_reduce_(-1, (torch.arange(cols, device="cuda") // BLOCK).expand(v.shape), v.abs(), "amax")
    s = torch.exp2(torch.round(torch.log2(top / E4M3_MAX)).clamp(SCALE_LOW, 127))
    s = torch.where(s * E4M3_MAX < top, 2 * s, s)          # the logarithm is rounded: the two borders decide
    return torch.where(s * E4M3_MAX / 2 >= top, s / 2, s).clamp_min(2.0 ** SCALE_LOW)


def _exact_wide(scales, cols):
    return scales.repeat_interleave(BLOCK, -1)[..., :cols]


def _exact_pack(v):
    scales = _exact_scales(v)
    return _e4m3(v / _exact_wide(scales, v.shape[-1])), scales


def _exact_act(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    return z


def _exact_slope(z, act):
    if act == "silu":
        g = torch.sigmoid(z)
        return g + z * g * torch.sigmoid(-z)
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / (2 * math.pi) ** 0.5
    return torch.ones_like(z)


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "pack":
        return list(_exact_pack(s["x"].double()))
    if c["op"] == "unpack":
        return s["q"].double() * _exact_wide(s["scales"].double(), c["d"])
    n, k, off = c["n"], c["k"], s["offsets"].tolist()
    double = dict(dtype=torch.float64, device="cuda")

    def halves(v, f, two):
        return torch.cat([f(h) for h in v.chunk(2, -1)], -1) if two else f(v)

    def saved_rows(l, a, b):
        z = s["saved"][l, a:b].double()
        if s["scales"] is None:
            return z
        scale = s["scales"][l, a:b].double()
        return z * halves(scale, lambda h: _exact_wide(h, k), c["below"] == "gated")

    if c["op"] == "linear":
        res = [torch.zeros(s["out"].shape, **double), None if s["saved"] is None else torch.zeros(s["saved"].shape, **double),
               None if s["scales"] is None else torch.zeros(s["scales"].shape, **double)]
        if res[2] is not None:
            res[2] += 2.0 ** SCALE_LOW                     # a byte of zero stands for the smallest scale
    elif c["op"] == "backward":
        res = [torch.zeros(s["dx"].shape, **double), None if s["h"] is None else torch.zeros(s["h"].shape, **double)]
    else:
        res = [None if i is None else torch.zeros(i.shape, **double) if b is None else b.double()
               for i, b in zip(s["into"], s["before"] or [None] * 4)]
    for l in range(c["layers"]):
        for e in range(c["experts"]):
            a, b = off[l][e], off[l][e + 1]
            if a == b:
                continue
            if c["op"] == "linear":
                x = s["x"][l, a:b].double()
                z = x @ s["w"][l, e].double().T + (0 if s["bias"] is None else s["bias"][l, e].double())
                y = _exact_act(z, c["act"])
                if c["gated"]:
                    up = x @ s["w_up"][l, e].double().T + (0 if s["bias_up"] is None else s["bias_up"][l, e].double())
                    y, z = y * up, torch.cat([z, up], -1)
                res[0][l, a:b] = y if s["add"] is None else y + s["add"][l, a:b].double()
                if c["save"] == "e4m3":
                    res[1][l, a:b] = halves(z, lambda h: _exact_pack(h)[0], c["gated"])
                    res[2][l, a:b] = halves(z, lambda h: _exact_pack(h)[1], c["gated"])
                elif c["save"] != "none":
                    res[1][l, a:b] = z
            elif c["op"] == "backward":
                dout = s["dout"][l, a:b].double()
                t = dout[:, :n] @ s["w"][l, e].double()
                if c["gated"]:
                    t += dout[:, n:] @ s["w_up"][l, e].double()
                if c["below"] == "none":
                    res[0][l, a:b] = t if s["add"] is None else t + s["add"][l, a:b].double()
                    continue
                z = saved_rows(l, a, b)
                y, slope = _exact_act(z[:, :k], c["act"]), _exact_slope(z[:, :k], c["act"])
                if c["below"] == "plain":
                    res[0][l, a:b], res[1][l, a:b] = t * slope, y
                else:
                    res[0][l, a:b, :k], res[0][l, a:b, k:] = t * z[:, k:] * slope, t * y
                    res[1][l, a:b] = y * z[:, k:]
            else:
                dout, x = s["dout"][l, a:b].double(), s["x"][l, a:b].double()
                if s["scales"] is not None:
                    x = x * _exact_wide(s["scales"][l, a:b].double(), k)
                for i in range(1 + c["gated"]):
                    d = dout[:, i * n:(i + 1) * n]
                    res[i][l, e] += d.T @ x
                    if c["bias"]:
                        res[2 + i][l, e] += d.sum(0)
    return res
