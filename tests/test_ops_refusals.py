"""What the operators around the experts (mcce_rmsnorm, mcce_dispatch, mcce_combine and the gradients) refuse: every
check is on the host and comes before any launch, so the calls here use addresses that nothing ever reads."""
import ctypes as C

import pytest

from paper_2412_00099_b200 import binding as mb
from paper_2412_00099_b200 import build as mbuild

EINVAL, ENOSPC = -1, -2
P = [C.c_void_p(0x10000 * (i + 1)) for i in range(12)]     # distinct, 64 KB aligned, never dereferenced


@pytest.fixture(scope="module")
def lib():
    mbuild.build()
    return mb.load()


def norm(**kw):
    f = dict(rows=4, d=64, dtype=mb.BF16, add_dtype=mb.F32, weight_dtype=mb.F32, quant_group=32, eps=1e-6, ld_x=0,
             ld_add=0, ld_sum=0, ld_out=0, ld_q=0)
    f.update(kw)
    return mb.Norm(**f)


def rows(**kw):
    f = dict(n_layers=2, n_tokens=10, top_k=4, n_experts=8, d=64, dtype=mb.BF16, token_dtype=mb.F32, scale_cols=0,
             ld_token=0, ld_rows=0)
    f.update(kw)
    return mb.Rows(**f)


def call_norm(lib, n, x=P[0], add=P[1], w=P[2], s=P[3], o=P[4], q=P[5], sc=P[6]):
    return lib.mcce_rmsnorm(None if n is None else C.byref(n), x, add, w, s, o, q, sc, None)


BAD_NORM = [dict(rows=-1), dict(rows=1 << 31), dict(d=0), dict(d=16385), dict(d=-8), dict(dtype=mb.E4M3), dict(dtype=7),
            dict(weight_dtype=mb.E4M3), dict(dtype=mb.F32, weight_dtype=mb.BF16), dict(eps=-1e-6),
            dict(eps=float("nan")), dict(eps=float("inf")), dict(ld_x=63), dict(ld_add=-64), dict(ld_sum=1),
            dict(ld_out=63)]


@pytest.mark.parametrize("bad", BAD_NORM, ids=str)
def test_norm_descriptor(lib, bad):
    n = norm(**bad)
    assert call_norm(lib, n) == EINVAL
    assert lib.mcce_rmsnorm_backward_workspace_bytes(C.byref(n)) == 0
    assert lib.mcce_rmsnorm_backward(C.byref(n), P[0], P[1], P[2], P[3], P[4], P[5], P[6], 1 << 30, None) == EINVAL


@pytest.mark.parametrize("bad", [dict(quant_group=16), dict(quant_group=-1), dict(quant_group=256), dict(ld_q=63),
                                 dict(add_dtype=mb.E4M3), dict(dtype=mb.F32, add_dtype=mb.BF16)], ids=str)
def test_norm_forward_only_fields(lib, bad):
    assert call_norm(lib, norm(**bad)) == EINVAL


def test_norm_buffers(lib):
    n = norm()
    assert call_norm(lib, None) == EINVAL
    assert call_norm(lib, n, x=None) == EINVAL and call_norm(lib, n, w=None) == EINVAL
    assert call_norm(lib, n, s=None, o=None, q=None, sc=None) == EINVAL           # nothing to compute
    assert call_norm(lib, n, sc=None) == EINVAL and call_norm(lib, n, q=None) == EINVAL
    odd = C.c_void_p(0x10001)
    for name in ("x", "add", "w", "s", "o", "sc"):
        assert call_norm(lib, n, **{name: odd}) == EINVAL, name
    assert call_norm(lib, norm(ld_sum=128), s=P[0]) == EINVAL                      # in place with another stride
    assert call_norm(lib, norm(rows=0), x=None, w=None) == 0                       # no rows: nothing to do


def test_norm_backward_buffers(lib):
    n = norm()
    need = lib.mcce_rmsnorm_backward_workspace_bytes(C.byref(n))
    assert need > 0 and lib.mcce_rmsnorm_backward_workspace_bytes(None) == 0

    def call(dout=P[0], h=P[1], dsum=P[2], w=P[3], dx=P[4], dw=P[5], ws=P[6], nbytes=need, n=n):
        return lib.mcce_rmsnorm_backward(C.byref(n), dout, h, dsum, w, dx, dw, ws, nbytes, None)
    for name in ("dout", "h", "w", "dx", "ws"):
        assert call(**{name: None}) == EINVAL, name
    odd = C.c_void_p(0x10001)
    for name in ("dout", "h", "dsum", "w", "dx", "dw", "ws"):
        assert call(**{name: odd}) == EINVAL, name
    assert call(nbytes=need - 1) == ENOSPC
    assert call(dx=P[0], n=norm(ld_sum=128)) == EINVAL and call(dx=P[2], n=norm(ld_sum=128)) == EINVAL


BAD_ROWS = [dict(n_layers=0), dict(n_layers=65536), dict(n_tokens=-1), dict(top_k=0), dict(top_k=17), dict(d=0), dict(d=(1 << 24) + 1),
            dict(n_tokens=1 << 28, top_k=8), dict(ld_token=63), dict(ld_rows=1), dict(ld_rows=-64),
            dict(scale_cols=-1), dict(dtype=3), dict(dtype=-1)]


@pytest.mark.parametrize("bad", BAD_ROWS, ids=str)
def test_rows_descriptor(lib, bad):
    r = rows(**bad)
    assert lib.mcce_dispatch_workspace_bytes(C.byref(r)) == 0
    assert lib.mcce_dispatch(C.byref(r), P[0], P[1], None, P[2], P[3], P[4], P[5], None, P[6], 1 << 30, None) == EINVAL
    assert lib.mcce_combine(C.byref(r), P[0], P[1], P[2], P[3], P[4], None) == EINVAL
    assert lib.mcce_combine_backward(C.byref(r), P[0], P[1], P[2], P[3], P[4], P[5], None) == EINVAL


def test_dispatch_refusals(lib):
    def call(sel=P[0], x=P[1], sc=None, off=P[2], perm=P[3], inv=P[4], out=P[5], osc=None, ws=P[6], nbytes=1 << 30, **kw):
        r = rows(**kw)
        return lib.mcce_dispatch(C.byref(r), sel, x, sc, off, perm, inv, out, osc, ws, nbytes, None)
    assert lib.mcce_dispatch_workspace_bytes(None) == 0
    for name in ("sel", "x", "off", "inv", "out"):
        assert call(**{name: None}) == EINVAL, name
    assert call(n_experts=0) == EINVAL and call(n_experts=257) == EINVAL
    assert call(scale_cols=2) == EINVAL and call(scale_cols=2, sc=P[7]) == EINVAL and call(sc=P[7], osc=P[8]) == EINVAL
    odd = C.c_void_p(0x10001)
    for name in ("sel", "x", "off", "perm", "inv", "out"):
        assert call(**{name: odd}) == EINVAL, name
    big = dict(n_tokens=100000)
    need = lib.mcce_dispatch_workspace_bytes(C.byref(rows(**big)))
    assert need > 0
    assert call(ws=None, **big) == EINVAL and call(ws=C.c_void_p(0x10004), **big) == EINVAL
    assert call(nbytes=need - 1, **big) == ENOSPC


def test_combine_refusals(lib):
    odd = C.c_void_p(0x10001)

    def call(rows_=P[0], inv=P[1], w=P[2], add=P[3], y=P[4], **kw):
        return lib.mcce_combine(C.byref(rows(**kw)), rows_, inv, w, add, y, None)
    for name in ("rows_", "inv", "y"):
        assert call(**{name: None}) == EINVAL, name
    for name in ("rows_", "inv", "w", "add", "y"):
        assert call(**{name: odd}) == EINVAL, name
    for bad in (dict(dtype=mb.E4M3), dict(dtype=mb.F32, token_dtype=mb.BF16), dict(token_dtype=mb.E4M3)):
        assert call(**bad) == EINVAL
        assert lib.mcce_combine_backward(C.byref(rows(**bad)), P[0], P[1], P[2], P[3], P[4], P[5], None) == EINVAL
    assert call(n_tokens=0, rows_=None, inv=None, y=None) == 0                     # no tokens: nothing to do

    def back(dy=P[0], rows_=P[1], inv=P[2], w=P[3], dr=P[4], dw=P[5]):
        return lib.mcce_combine_backward(C.byref(rows()), dy, rows_, inv, w, dr, dw, None)
    for name in ("dy", "rows_", "inv", "dr"):
        assert back(**{name: None}) == EINVAL, name
    for name in ("dy", "rows_", "inv", "w", "dr", "dw"):
        assert back(**{name: odd}) == EINVAL, name
    assert lib.mcce_combine_backward(None, P[0], P[1], P[2], P[3], P[4], P[5], None) == EINVAL


def refused_pairs(call, names, allowed):
    """Every pair of arguments at one address that is not allowed: `names` are the arguments, outputs last after "|"."""
    ins, outs = [n.split() for n in names.split("|")]
    address = {n: P[i] for i, n in enumerate(ins + outs)}
    for i, o in enumerate(outs):
        for other in ins + outs[:i]:
            if (o, other) not in allowed:
                assert call(**dict(address, **{o: address[other]})) == EINVAL, (o, other)


def test_outputs_at_an_inputs_address(lib):
    refused_pairs(lambda **k: call_norm(lib, norm(), **k), "x add w | s o q sc", {("s", "x")})

    def norm_back(dout, h, dsum, w, dx, dw):
        return lib.mcce_rmsnorm_backward(C.byref(norm()), dout, h, dsum, w, dx, dw, P[11], 1 << 30, None)
    refused_pairs(norm_back, "dout h dsum w | dx dw", {("dx", "dout"), ("dx", "dsum")})

    def dispatch(sel, x, sc, off, perm, inv, out, osc):
        return lib.mcce_dispatch(C.byref(rows(scale_cols=2)), sel, x, sc, off, perm, inv, out, osc, P[11], 1 << 30, None)
    refused_pairs(dispatch, "sel x sc | off perm inv out osc", set())

    def combine(rows_, inv, w, add, y):
        return lib.mcce_combine(C.byref(rows()), rows_, inv, w, add, y, None)
    refused_pairs(combine, "rows_ inv w add | y", {("y", "add")})

    def combine_back(dy, rows_, inv, w, dr, dw):
        return lib.mcce_combine_backward(C.byref(rows()), dy, rows_, inv, w, dr, dw, None)
    refused_pairs(combine_back, "dy rows_ inv w | dr dw", {("dr", "rows_")})


def at(p, nbytes):
    return C.c_void_p(p.value + nbytes)


def test_outputs_that_reach_into_another_tensor(lib):
    """An output that starts one row into another tensor, or whose last row is another's first: refused like one at its address."""
    n = norm()                                       # 4 rows of 64: x 512 bytes (bf16), add 1024 (fp32), weight 256, q 256, scales 32
    row = dict(x=128, add=256, w=64, s=128, o=128, q=64, sc=8)
    size = dict(x=512, add=1024, w=256, s=512, o=512, q=256, sc=32)
    names = ["x", "add", "w", "s", "o", "q", "sc"]
    for i, out in enumerate(names):
        for other in names[:i]:
            if i >= 3:
                for place in (at(P[names.index(other)], size[other] - row[other]), at(P[names.index(other)], row[out] - size[out])):
                    assert call_norm(lib, n, **{out: place}) == EINVAL, (out, other)
    assert call_norm(lib, norm(rows=2, ld_x=256, ld_sum=192), s=at(P[0], 128)) == EINVAL      # row 1 of the sum is inside row 1 of x
    assert call_norm(lib, norm(rows=2), s=at(P[0], 128)) == EINVAL                             # in place, one row late

    def norm_back(dout=P[0], h=P[1], dsum=P[2], w=P[3], dx=P[4], dw=P[5], ws=P[6]):
        return lib.mcce_rmsnorm_backward(C.byref(n), dout, h, dsum, w, dx, dw, ws, 1 << 30, None)
    for i in range(4):
        step = 64 if i == 3 else 128
        assert norm_back(dx=at(P[i], step)) == EINVAL and norm_back(dx=at(P[i], -384)) == EINVAL
        assert norm_back(dw=at(P[i], step)) == EINVAL and norm_back(ws=at(P[i], 16)) == EINVAL and norm_back(ws=at(P[i], -16)) == EINVAL
    assert norm_back(dw=at(P[4], 256)) == EINVAL and norm_back(ws=at(P[4], 16)) == EINVAL and norm_back(ws=at(P[5], 16)) == EINVAL
    assert norm_back(ws=at(P[5], -1008)) == EINVAL

    def dispatch(place=(), **kw):                    # 2 layers of 10 tokens x 4, rows of 128 bytes, 2 scales
        r = rows(**dict(dict(scale_cols=2), **kw))
        a = dict(sel=P[0], x=P[1], sc=P[2], off=P[3], perm=P[4], inv=P[5], out=P[6], osc=P[7], ws=P[8])
        a.update(place)
        return lib.mcce_dispatch(C.byref(r), a["sel"], a["x"], a["sc"], a["off"], a["perm"], a["inv"], a["out"], a["osc"], a["ws"], 1 << 30, None)
    names = ["sel", "x", "sc", "off", "perm", "inv", "out", "osc"]
    for i, out in enumerate(names):
        for j, other in enumerate(names[:i]):
            if i >= 3:
                assert dispatch({out: at(P[j], 16)}) == EINVAL and dispatch({out: at(P[j], -16)}) == EINVAL, (out, other)
    # with a workspace: 4096 tokens, tensors 64 MB apart
    far = {n: C.c_void_p((i + 1) << 26) for i, n in enumerate(names + ["ws"])}
    for n_ in names:
        assert dispatch(dict(far, ws=at(far[n_], 16)), n_tokens=4096) == EINVAL, n_

    def combine(rows_=P[0], inv=P[1], w=P[2], add=P[3], y=P[4], **kw):
        return lib.mcce_combine(C.byref(rows(**kw)), rows_, inv, w, add, y, None)
    for i in range(4):
        assert combine(y=at(P[i], 16)) == EINVAL and combine(y=at(P[i], -16)) == EINVAL

    def combine_back(dy=P[0], rows_=P[1], inv=P[2], w=P[3], dr=P[4], dw=P[5]):
        return lib.mcce_combine_backward(C.byref(rows()), dy, rows_, inv, w, dr, dw, None)
    for i in range(4):
        for d in (16, -16):
            assert combine_back(dr=at(P[i], d)) == EINVAL and combine_back(dw=at(P[i], d)) == EINVAL
    assert combine_back(dw=at(P[4], 16)) == EINVAL and combine_back(dw=at(P[4], -16)) == EINVAL


def test_shared_memory_is_found_exactly(tmp_path):
    """The check itself (span.h, compiled here) against sets of bytes: rows side by side, between one another, with equal and
    unequal strides; sizes that would overflow 64 bits."""
    import os
    import random
    import subprocess
    src = tmp_path / "span.cpp"
    src.write_text('#include "span.h"\nextern "C" int apart3(long long p, long long r, long long s, long long w, long long p2, long long r2, '
                   'long long s2, long long w2) { return mcce::disjoint(mcce::span((void*)p, r, s, w), mcce::span((void*)p2, r2, s2, w2)); }\n'
                   'extern "C" int huge(long long n) { return mcce::disjoint(mcce::row_span((void*)4096, n, n, 64, 4), mcce::row_span((void*)8192, 3, n, 64, 4)); }\n')
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", mbuild.CSRC, str(src), "-o", str(tmp_path / "span.so")], check=True)
    so = C.CDLL(os.path.join(str(tmp_path), "span.so"))
    so.apart3.argtypes = [C.c_longlong] * 8
    so.huge.argtypes = [C.c_longlong]
    rng = random.Random(3)

    def touched(p, rows, step, width):
        return {p + i * step + j for i in range(rows) for j in range(width)}
    seen = [0, 0]
    for _ in range(20000):
        a, b = [(rng.randint(100, 160), rng.randint(1, 9), 0, rng.randint(1, 9)) for _ in range(2)]
        sa = a[3] + rng.randint(0, 12)
        sb = sa if rng.random() < 0.4 and sa >= b[3] else b[3] + rng.randint(0, 12)
        a, b = (a[0], a[1], sa, a[3]), (b[0], b[1], sb, b[3])
        want = not (touched(*a) & touched(*b))
        seen[want] += 1
        assert bool(so.apart3(*a, *b)) == want, (a, b)
    assert min(seen) > 4000
    for n in (1 << 62, (1 << 63) - 1):
        assert so.huge(n) in (0, 1)


def test_set_norm_needs_a_context(lib):
    assert lib.mcce_set_norm(None, P[0], 1e-6) == EINVAL


def test_set_norm_refuses_weights_that_are_not_on_its_device():
    """The kernels would read the address: an error on the host instead, before the library hears of it."""
    import torch
    calls = []

    class Lib:
        def mcce_set_norm(self, *a):
            calls.append(a)
            return 0
    eng = object.__new__(mb.Engine)
    eng.L, eng.d, eng.device, eng.lib, eng.ctx, eng._keep = 2, 16, torch.device("cuda", 0), Lib(), C.c_void_p(), []
    for weight in (torch.ones(2, 16), torch.ones(2, 16, device="meta")):
        with pytest.raises(mb.McceError, match="cuda:0"):
            eng.set_norm(weight)
    assert not calls and not eng._keep
    eng.set_norm(None)
    assert len(calls) == 1


def test_binding_refuses_cpu_tensors():
    import torch
    with pytest.raises(mb.McceError, match="no CPU path"):
        mb.rmsnorm(torch.zeros(2, 8), torch.ones(8))
    with pytest.raises(mb.McceError, match="no CPU path"):
        mb.rmsnorm_backward(torch.zeros(2, 8), torch.zeros(2, 8), torch.ones(8))
    with pytest.raises(mb.McceError, match="no CPU path"):
        mb.dispatch(torch.zeros(2, 2, dtype=torch.int32), 4)
    with pytest.raises(mb.McceError, match="no CPU path"):
        mb.combine(torch.zeros(4, 8), torch.zeros(2, 2, dtype=torch.int32))
    with pytest.raises(mb.McceError, match="no CPU path"):
        mb.combine_backward(torch.zeros(2, 8), torch.zeros(4, 8), torch.zeros(2, 2, dtype=torch.int32))


def test_binding_refuses_to_lose_a_gradient():
    """The calls record nothing for autograd: a tensor that needs a gradient is refused while autograd is recording.  (CPU tensors: what
    is not refused for its gradient is refused for its device.)"""
    import torch

    def leaf(*shape):
        return torch.zeros(*shape, requires_grad=True)
    x, w, i = torch.zeros(4, 8), torch.ones(8), torch.zeros(2, 2, dtype=torch.int32)
    pair = torch.zeros(2, 2)
    y, sorted_ = mb.NormOut(torch.zeros(4, 8), torch.zeros(4, 8)), mb.Dispatched(torch.zeros(5, dtype=torch.int32), None, i, x, x)
    calls = [(lambda x, w, a: mb.rmsnorm(x, w, add=a, out=y), (x, w, x)),
             (lambda g, h, w, s: mb.rmsnorm_backward(g, h, w, dsum=s, out=(x, w)), (x, x, w, x)),
             (lambda x, s: mb.dispatch(i, 4, x, scales=s, out=sorted_), (x[:2], x[:2])),
             (lambda r, w, a: mb.combine(r, i, w, add=a, out=x[:2]), (x, pair, x[:2])),
             (lambda g, r, w: mb.combine_backward(g, r, i, w, out=(x, pair)), (x[:2], x, pair))]
    for call, args in calls:
        for k, a in enumerate(args):
            some = [leaf(*b.shape) if j == k else b for j, b in enumerate(args)]
            with pytest.raises(mb.McceError, match="requires grad"):
                call(*some)
            with torch.no_grad(), pytest.raises(mb.McceError, match="CUDA"):
                call(*some)
    with pytest.raises(mb.McceError, match="requires grad"):                  # a result that needs one
        mb.rmsnorm(x, w, out=mb.NormOut(leaf(4, 8)))
