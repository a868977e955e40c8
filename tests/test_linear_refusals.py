"""What the experts' products (mcce_expert_linear and its gradients) and the 8-bit checkpoints refuse: every check is on the host and comes before any
launch, so the calls here use addresses that nothing ever reads."""
import ctypes as C

import pytest

from paper_2412_00099_b200 import binding as mb
from paper_2412_00099_b200 import build as mbuild

EINVAL, ENOSPC = -1, -2
P = [C.c_void_p(0x1000000 * (i + 1)) for i in range(20)]     # distinct, 16 MB apart, never dereferenced
ODD = C.c_void_p(0x999001)


@pytest.fixture(scope="module")
def lib():
    mbuild.build()
    return mb.load()


def at(p, nbytes):
    return C.c_void_p(p.value + nbytes)


def lin(**kw):
    """2 layers of 3 experts, 10 rows each, 32 -> 64, bf16, gated, 8-bit kept values."""
    f = dict(n_layers=2, n_experts=3, rows=10, n=64, k=32, dtype=mb.BF16, out_dtype=mb.F32, bias_dtype=mb.F32, saved_dtype=mb.E4M3, act=1,
             gated=1, below=2, ld_x=0, ld_y=0, ld_add=0, ld_saved=0, ld_h=0, ld_w=0, step_w=0)
    f.update(kw)
    return mb.Linear(**f)


def forward(lib, p=None, x=P[0], off=P[1], w=P[2], wu=P[3], b=P[4], bu=P[5], add=P[6], out=P[7], saved=P[8], sc=P[9], ws=None, nbytes=0):
    p = lin() if p is None else p
    return lib.mcce_expert_linear(C.byref(p), x, off, w, wu, b, bu, add, out, saved, sc, ws, nbytes, None)


def backward(lib, p=None, g=P[0], off=P[1], w=P[2], wu=P[3], add=None, saved=P[4], sc=P[5], dx=P[6], h=P[7], ws=None, nbytes=0):
    p = lin() if p is None else p
    return lib.mcce_expert_linear_backward(C.byref(p), g, off, w, wu, add, saved, sc, dx, h, ws, nbytes, None)


def dweight(lib, p=None, g=P[0], x=P[1], sc=P[2], off=P[3], aw=P[4], awu=P[5], ab=P[6], abu=P[7], dw=P[8], dwu=P[9], db=P[10], dbu=P[11],
            ws=P[12], nbytes=1 << 20):
    p = lin() if p is None else p
    return lib.mcce_expert_linear_dweight(C.byref(p), g, x, sc, off, aw, awu, ab, abu, dw, dwu, db, dbu, ws, nbytes, None)


BAD = [dict(n_layers=0), dict(n_experts=0), dict(n_layers=65, n_experts=64), dict(rows=-1), dict(rows=1 << 31), dict(n_layers=4, rows=1 << 30),
       dict(n=0), dict(k=0), dict(n=(1 << 20) + 1), dict(k=(1 << 20) + 1), dict(dtype=mb.E4M3), dict(dtype=5), dict(gated=2), dict(gated=-1), dict(ld_w=31),
       dict(ld_w=-32), dict(step_w=64 * 32 - 1), dict(step_w=-1), dict(ld_w=1 << 41), dict(ld_x=31)]


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_descriptor(lib, bad):
    p = lin(**bad)
    assert forward(lib, p) == EINVAL and dweight(lib, p) == EINVAL
    p.below, p.act = (1, 1)                                                       # ld_x: rows of dx
    assert backward(lib, p) == EINVAL
    if "ld_x" not in bad:
        assert lib.mcce_expert_linear_dweight_workspace_bytes(C.byref(p), P[0], P[1]) == 0


def test_types_and_strides(lib):
    for bad in (dict(out_dtype=mb.E4M3), dict(out_dtype=9), dict(dtype=mb.F32, out_dtype=mb.BF16), dict(bias_dtype=mb.E4M3), dict(saved_dtype=7),
                dict(dtype=mb.F32, saved_dtype=mb.BF16), dict(act=3), dict(act=-1), dict(ld_y=63), dict(ld_add=63), dict(ld_saved=127)):
        assert forward(lib, lin(**bad)) == EINVAL, bad
    for bad in (dict(below=3), dict(below=-1), dict(act=9), dict(ld_y=127), dict(ld_x=63), dict(ld_saved=63), dict(ld_h=31), dict(saved_dtype=mb.F32)):
        assert backward(lib, lin(**bad)) == EINVAL, bad
    for bad in (dict(out_dtype=mb.E4M3), dict(dtype=mb.F32, out_dtype=mb.BF16), dict(saved_dtype=mb.F32), dict(ld_y=127), dict(ld_x=31)):
        assert dweight(lib, lin(**bad)) == EINVAL, bad


def test_missing_and_misaligned(lib):
    assert lib.mcce_expert_linear(None, *P[:11], 0, None) == EINVAL and lib.mcce_expert_linear_backward(None, *P[:10], 0, None) == EINVAL
    assert lib.mcce_expert_linear_dweight_workspace_bytes(None, None, None) == 0
    for name in ("x", "off", "w", "wu", "bu", "out", "sc"):
        assert forward(lib, **{name: None}) == EINVAL, name
    assert forward(lib, saved=None) == EINVAL                                     # scales without anything kept
    assert forward(lib, b=None) == EINVAL                                         # the second bias without the first
    assert forward(lib, lin(gated=0)) == EINVAL and forward(lib, lin(gated=0), wu=None) == EINVAL       # a second matrix, a second bias
    assert forward(lib, lin(saved_dtype=mb.BF16)) == EINVAL                       # scales without 8 bits
    for name in ("x", "off", "w", "wu", "b", "bu", "add", "out"):
        assert forward(lib, **{name: ODD}) == EINVAL, name
    for name in ("g", "off", "w", "wu", "saved", "sc", "dx"):
        assert backward(lib, **{name: None}) == EINVAL, name
    assert backward(lib, add=P[9]) == EINVAL                                      # nothing is added behind an activation
    plain = lin(below=0, act=0)
    assert backward(lib, plain, saved=None, sc=None) == EINVAL                    # h without a layer below
    assert backward(lib, lin(below=0), saved=None, sc=None, h=None) == EINVAL     # an activation without one
    for name in ("g", "off", "w", "wu", "dx", "h"):
        assert backward(lib, **{name: ODD}) == EINVAL, name
    for name in ("g", "x", "sc", "off", "dw", "dwu", "dbu", "awu", "abu", "ws"):
        assert dweight(lib, **{name: None}) == EINVAL, name
    assert dweight(lib, db=None, dbu=None) == EINVAL                              # something to add to a bias that is not wanted
    for name in ("g", "off", "aw", "awu", "ab", "abu", "dw", "dwu", "db", "dbu", "ws"):
        assert dweight(lib, **{name: ODD}) == EINVAL, name
    need = lib.mcce_expert_linear_dweight_workspace_bytes(C.byref(lin()), P[0], P[1])
    assert need == 2 * 10 * 32 * 2 and dweight(lib, nbytes=need - 1) == ENOSPC
    assert lib.mcce_expert_linear_dweight_workspace_bytes(C.byref(lin(saved_dtype=mb.BF16)), P[0], P[1]) == 0
    long = lin(n_layers=1, n_experts=1, rows=100000, saved_dtype=mb.BF16)
    assert lib.mcce_expert_linear_dweight_workspace_bytes(C.byref(long), P[0], P[1]) % (2 * 64 * 4) == 0     # parts of the bias's gradient


def test_workspace_for_copies(lib):
    """bf16 rows that are not aligned to 16 bytes need a workspace where copying them pays, and only there."""
    big = dict(n_layers=1, n_experts=2, rows=4096, gated=0, below=0, act=0, saved_dtype=mb.BF16)
    fwd, bwd, dw = lib.mcce_expert_linear_workspace_bytes, lib.mcce_expert_linear_backward_workspace_bytes, lib.mcce_expert_linear_dweight_workspace_bytes
    even, odd, small = lin(n=512, k=512, **big), lin(n=511, k=515, **big), lin(n=511, k=515, **dict(big, rows=16))
    bias = 4 * 2 * 512 * 4                               # parts of the bias's gradient: four chunks of rows
    for p in (even, small):
        assert fwd(C.byref(p), P[0], P[1], None) == bwd(C.byref(p), P[0], P[1], None) == 0 and dw(C.byref(p), P[0], P[1]) == (bias if p is even else 0)
    rows_x, rows_y, weights = 4096 * 520 * 2, 4096 * 512 * 2, (2 * 511 * 520 * 2 + 255) // 256 * 256
    assert fwd(C.byref(odd), P[0], P[1], None) == rows_x + weights and dw(C.byref(odd), P[0], P[1]) == rows_x + rows_y + bias
    assert bwd(C.byref(odd), P[0], P[1], None) == rows_y + weights
    assert fwd(C.byref(even), at(P[0], 2), P[1], None) == 4096 * 512 * 2 and fwd(C.byref(lin(n=511, k=515, **dict(big, dtype=mb.F32, saved_dtype=mb.F32))), P[0], P[1], None) == 0
    assert fwd(None, P[0], P[1], None) == bwd(None, P[0], P[1], None) == 0
    need = rows_x + weights
    a = dict(wu=None, b=None, bu=None, add=None, saved=None, sc=None)
    assert forward(lib, odd, ws=None, nbytes=need, **a) == EINVAL and forward(lib, odd, ws=at(P[15], 8), nbytes=need, **a) == EINVAL
    assert forward(lib, odd, ws=P[15], nbytes=need - 1, **a) == ENOSPC
    for other in (P[0], P[2], P[7]):
        assert forward(lib, odd, ws=at(other, 16), nbytes=need, **a) == EINVAL
    a = dict(wu=None, saved=None, sc=None, h=None)
    assert backward(lib, odd, ws=P[15], nbytes=rows_y + weights - 1, **a) == ENOSPC and backward(lib, odd, nbytes=1 << 30, **a) == EINVAL
    for other in (P[0], P[2], P[6]):
        assert backward(lib, odd, ws=at(other, 16), nbytes=need, **a) == EINVAL


def test_nothing_to_do(lib):
    assert forward(lib, lin(rows=0), x=None, off=None, w=None, out=None) == 0
    assert backward(lib, lin(rows=0), g=None, off=None, w=None, dx=None) == 0
    assert lib.mcce_checkpoint_pack(None, mb.BF16, 0, 8, 0, 0, None, None, None) == 0
    assert lib.mcce_checkpoint_unpack(None, None, mb.F32, 0, 8, 0, 0, None, None) == 0


def refused_pairs(call, names, allowed):
    """Every pair of arguments at one address, or one 16 bytes into the other, that is not allowed: outputs last after "|"."""
    ins, outs = [n.split() for n in names.split("|")]
    address = {n: P[i] for i, n in enumerate(ins + outs)}
    for i, o in enumerate(outs):
        for other in ins + outs[:i]:
            if (o, other) not in allowed:
                assert call(**dict(address, **{o: address[other]})) == EINVAL, (o, other)
            assert call(**dict(address, **{o: at(address[other], 16)})) == EINVAL, (o, other)


def test_outputs_that_share_memory(lib):
    refused_pairs(lambda **k: forward(lib, **k), "x off w wu b bu add | out saved sc", {("out", "add")})
    refused_pairs(lambda **k: backward(lib, **k), "g off w wu saved sc | dx h", set())
    same = lin(saved_dtype=mb.BF16)
    refused_pairs(lambda **k: backward(lib, same, sc=None, **k), "g off w wu saved | dx h", {("dx", "saved")})
    plain = lin(below=0, act=0)
    refused_pairs(lambda **k: backward(lib, plain, saved=None, sc=None, h=None, **k), "g off w wu add | dx", {("dx", "add")})
    refused_pairs(lambda **k: dweight(lib, **k), "g x sc off aw awu ab abu | dw dwu db dbu",
                  {("dw", "aw"), ("dwu", "awu"), ("db", "ab"), ("dbu", "abu")})
    names = dict(g=P[0], x=P[1], sc=P[2], off=P[3], aw=P[4], awu=P[5], ab=P[6], abu=P[7], dw=P[8], dwu=P[9], db=P[10], dbu=P[11])
    for p in names.values():
        assert dweight(lib, **dict(names, ws=p)) == EINVAL and dweight(lib, **dict(names, ws=at(p, -16))) == EINVAL
    assert forward(lib, lin(ld_y=80), add=P[7]) == EINVAL and backward(lib, lin(saved_dtype=mb.BF16, ld_x=80), sc=None, dx=P[4]) == EINVAL   # other strides


def pack(lib, x=P[0], dtype=mb.BF16, rows=4, d=96, ld_x=0, ld_q=0, q=P[1], sc=P[2]):
    return lib.mcce_checkpoint_pack(x, dtype, rows, d, ld_x, ld_q, q, sc, None)


def unpack(lib, x=P[0], dtype=mb.BF16, rows=4, d=96, ld_x=0, ld_q=0, q=P[1], sc=P[2]):
    return lib.mcce_checkpoint_unpack(q, sc, dtype, rows, d, ld_x, ld_q, x, None)


@pytest.mark.parametrize("call", [pack, unpack])
def test_checkpoint(lib, call):
    for bad in (dict(x=None), dict(q=None), dict(sc=None), dict(x=ODD), dict(dtype=mb.E4M3), dict(dtype=4), dict(rows=-1), dict(rows=1 << 31), dict(d=0),
                dict(d=(1 << 20) + 1), dict(ld_x=95), dict(ld_q=95), dict(ld_x=-96)):
        assert call(lib, **bad) == EINVAL, bad
    for o in (dict(q=P[0]), dict(sc=P[0]), dict(sc=P[1]), dict(q=at(P[0], 4 * 96 * 2 - 1)), dict(sc=at(P[1], 4 * 96 - 1))):
        if call is pack or "x" in o or o.get("sc") is not P[1] and o.get("sc") is None:
            assert call(lib, **o) == EINVAL, o
    assert unpack(lib, x=at(P[1], 2)) == EINVAL and unpack(lib, x=at(P[2], 2)) == EINVAL


def test_binding(lib):
    import torch
    x, off, w = torch.zeros(4, 8), torch.zeros(3, dtype=torch.int32), torch.zeros(2, 6, 8)
    g = torch.zeros(4, 6)
    for call in (lambda: mb.expert_linear(x, off, w), lambda: mb.expert_linear_backward(g, off, w), lambda: mb.expert_linear_dweight(g, x, off),
                 lambda: mb.checkpoint_pack(x), lambda: mb.checkpoint_unpack(x.to(torch.float8_e4m3fn), x)):
        with pytest.raises(mb.McceError, match="no CPU path"):
            call()
    out = mb.LinearOut(torch.zeros(4, 6))
    for act in ("relu", 1, ""):
        with pytest.raises(mb.McceError, match="act"):
            mb.expert_linear(x, off, w, act=act, out=out)
    leaf = torch.zeros(4, 8, requires_grad=True)
    with pytest.raises(mb.McceError, match="requires grad"):
        mb.expert_linear(leaf, off, w, out=out)
    with pytest.raises(mb.McceError, match="requires grad"):
        mb.expert_linear_dweight(g, leaf, off, out=mb.WeightGrad(torch.zeros(2, 6, 8)))
    with pytest.raises(mb.McceError, match="requires grad"):
        mb.expert_linear_backward(g, off, w, out=mb.LinearGrad(leaf))
    with pytest.raises(mb.McceError, match="requires grad"):
        mb.checkpoint_pack(leaf, out=mb.Checkpoint(x.to(torch.float8_e4m3fn), torch.zeros(4, 1).to(mb.E8M0)))
