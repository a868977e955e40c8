"""The operators around the experts against plain implementations in 64 bits: root-mean-square norm with the residual's
addition and 8-bit output, its gradient, rows sorted by expert, their weighted return and its gradient.

Tolerances.  u = 2^-24 is half an fp32 step, U(T) half a step of the output type relative to the value (bf16 2^-8, fp32
2^-24).  A fp32 sum of n terms is off by at most (n - 1) u times the sum of the terms' magnitudes, whatever its order;
each multiplication or division adds u.  The norm's sum of squares has only positive terms and no thread adds more than 64 of
them in a row before the tree (10 levels at most), so it is off by 74 u relatively, its mean plus eps by 3 u more (1 / d is
rounded too) and r by half of that and the two units in the last place of the reciprocal square root (4 u): 43 u; h r weight
adds two: 45 u.  NORM_U = 64 u covers it with room for the two factors in the scales."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2412_00099_b200 import binding as mb

u = 2.0 ** -24
NORM_U = 64 * u
F32, BF16 = torch.float32, torch.bfloat16


def U(t):
    return torch.finfo(t).eps / 2


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, dtype=F32):
    return torch.randn(*shape, device="cuda", generator=g).to(dtype)


def within(got, want, tol, what=""):
    """|got - want| <= tol elementwise (NaN fails)."""
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), "%s: %d of %d off, worst %g over its tolerance" % (
        what, int(bad.sum()), bad.numel(), float(((got.double() - want).abs() / tol.clamp_min(1e-300))[bad].max()))


def e4m3(v):
    """Nearest e4m3 value of a float64 tensor, ties to even, saturating."""
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), (e - 4).clamp_min(-9))
    return (torch.round(v / step) * step).clamp(-448.0, 448.0)


# ---- norm ------------------------------------------------------------------------------------------------------
def check_norm(x, w, eps, add, group, r):
    """r = rmsnorm(...) against the definition on the h that it returned (or on x)."""
    d, T = x.shape[-1], x.dtype
    h = x.double()
    if add is not None:
        want = x.double() + add.double()
        if r.sum is not None:
            within(r.sum, want, want.abs() * (U(T) + 2 * u), "sum")
            h = r.sum.double()
        else:
            h = (x.float() + add.float()).to(T).double()      # the one fp32 addition and rounding of the definition
    n = h / (h.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
    if r.out is not None:
        within(r.out, n, n.abs() * (U(T) + NORM_U) * (1 + U(T)), "out")
    if r.q is not None:
        g = group or d
        col = torch.arange(d, device="cuda") // g
        top = torch.zeros(n.shape[:-1] + (r.scales.shape[-1],), dtype=torch.float64, device="cuda")
        top.scatter_reduce_(-1, col.expand(n.shape), n.abs(), "amax")
        scales = top.clamp_min(2.0 ** -100) / 448.0
        within(r.scales, scales, scales * NORM_U, "scales")
        # the quantised value is the rounding of something within n's and the scale's tolerance: rounding is monotone
        v = n / scales[..., col]
        lo, hi = e4m3(v - v.abs() * 3 * NORM_U), e4m3(v + v.abs() * 3 * NORM_U)
        q = r.q.double()
        assert ((q >= lo) & (q <= hi)).all()


NORM_SHAPES = [(1, 1), (1, 2048), (3, 7), (2, 64), (5, 100), (257, 96), (64, 130), (33, 1411), (512, 2048), (7, 4096),
               (19, 5076), (3, 8192), (2, 16384), (2, 16383), (1000, 72), (130, 1000), (4, 11111)]


@pytest.mark.parametrize("rows,d", NORM_SHAPES)
@pytest.mark.parametrize("T,A,W", [(BF16, None, F32), (BF16, F32, BF16), (BF16, BF16, F32), (F32, None, F32), (F32, F32, F32)])
def test_norm(rows, d, T, A, W):
    g = gen(rows * 31 + d)
    x = normal(g, rows, d, dtype=T) * 3
    w = (1 + 0.2 * normal(g, d)).to(W)
    add = None if A is None else normal(g, rows, d, dtype=A)
    for group in (None, 0, 32, 64, 128):
        r = mb.rmsnorm(x, w, 1e-5, add=add, quant_group=group)
        check_norm(x, w, 1e-5, add, group, r)
        again = mb.rmsnorm(x, w, 1e-5, add=add, quant_group=group)
        for a, b in zip(r, again):
            assert (a is None and b is None) or torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        if group is not None:                       # only the 8-bit rows: same bits
            q = mb.rmsnorm(x, w, 1e-5, add=add, quant_group=group, out=mb.NormOut(None, None, torch.empty_like(r.q), torch.empty_like(r.scales)))
            assert torch.equal(q.q.view(torch.uint8), r.q.view(torch.uint8)) and torch.equal(q.scales, r.scales)


@pytest.mark.parametrize("T", [BF16, F32])
@pytest.mark.parametrize("d,ld", [(64, 72), (100, 101), (2048, 2056), (2048, 2050), (96, 4096), (1002, 1004)])
def test_norm_strides_and_in_place(T, d, ld):
    """Rows further apart than their width, every tensor another stride; the sum in place; nothing between the rows touched."""
    g, R = gen(5), 37
    full = normal(g, R, ld, dtype=T)
    keep, x = full.clone(), full[:, :d]
    add = normal(g, R, ld + 3)[:, 2:d + 2]
    w = 1 + 0.1 * normal(g, d)
    o, q = torch.full((R, ld + 8), 7.0, device="cuda", dtype=T), torch.zeros(R, ld + 16, device="cuda", dtype=torch.uint8)
    sc = torch.empty(R, -(-d // 32), device="cuda")
    want = mb.rmsnorm(x.contiguous(), w, 1e-6, add=add.contiguous(), quant_group=32)
    r = mb.rmsnorm(x, w, 1e-6, add=add, quant_group=32,
                   out=mb.NormOut(o[:, 4:d + 4], x, q[:, 1:d + 1].view(torch.float8_e4m3fn), sc))
    check_norm(keep[:, :d], w, 1e-6, add, 32, r)
    assert torch.equal(r.sum, want.sum)
    assert torch.equal(full[:, d:], keep[:, d:]) and (o[:, :4] == 7).all() and (o[:, d + 4:] == 7).all()
    assert (q[:, 0] == 0).all() and (q[:, d + 1:] == 0).all()


def test_norm_small_large_and_special_rows():
    d = 256
    w = torch.ones(d, device="cuda")
    x = torch.zeros(6, d, device="cuda")
    x[1] = 1e-30                                    # squares vanish: r = 1 / sqrt(eps)
    x[2] = 1e18
    x[3, 5] = float("nan")
    x[4, 7] = float("inf")
    x[5] = 3e-45
    r = mb.rmsnorm(x, w, 1e-6, quant_group=64)
    assert (r.out[0] == 0).all() and (r.q[0].float() == 0).all()
    assert (r.scales[0] == np.float32(2.0 ** -100) / np.float32(448)).all()
    assert torch.allclose(r.out[1], torch.full((d,), 1e-27, device="cuda"), rtol=1e-5, atol=0)
    assert torch.allclose(r.out[2], torch.ones(d, device="cuda"), rtol=1e-5)
    assert r.out[3].isnan().all() and r.scales[3].isnan().all() and r.q[3].float().isnan().all()
    # an infinite entry: r = 0, every finite entry becomes 0, the infinite one 0 * inf
    assert r.out[4, 7].isnan() and (r.out[4, :7] == 0).all() and r.scales[4, 0].isnan() and (r.scales[4, 1:] < 1e-30).all()
    assert r.out[5].isfinite().all()
    # eps = 0 on a row of zeros: 1 / 0, then 0 * inf
    assert mb.rmsnorm(x[:1], w, 0.0).out.isnan().all()
    for T in (BF16, F32):                            # no rows
        e = mb.rmsnorm(torch.empty(0, 8, device="cuda", dtype=T), torch.ones(8, device="cuda"), add=torch.empty(0, 8, device="cuda"), quant_group=0)
        assert e.out.shape == (0, 8) and e.scales.shape == (0, 1)


@pytest.mark.parametrize("d", [128, 4096, 1411, 16384])
@pytest.mark.parametrize("T", [BF16, F32])
@pytest.mark.parametrize("alike", [True, False])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
def test_norm_to_8_bits_rounds_the_quotient(d, T, alike, group):
    """q is the e4m3 rounding of n / scale.  With x = 1, eps = 0 (r = 1) n is the weight itself, so what stays between n and q is the
    division that forms a group's factor and the multiplication by it: 2 u.  The weights lie a few u off the e4m3 ties of their
    group, whose largest values are arbitrary."""
    R, g = 3, gen(d + group)
    cols = -(-d // group) if group else 1
    top = 1 + torch.rand(cols, device="cuda", generator=g)
    top = top.repeat_interleave(group or d)[:d]
    tie = torch.randint(8, 16, (d,), device="cuda", generator=g).double() + 0.5        # halfway between two of 4 significant bits
    tie = tie * 2.0 ** torch.randint(-2, 5, (d,), device="cuda", generator=g).double()
    off = 1 + u * (torch.rand(d, device="cuda", generator=g).double() * 12 - 6)
    w = (tie * off * top.double() / 448.0).float()
    first = torch.arange(0, d, group or d, device="cuda")
    w[first] = top[first]
    x = torch.ones(R, d + 1, device="cuda", dtype=T)
    x = x[:, :d].contiguous() if alike else x[:, 1:]
    out = mb.NormOut(None, None, torch.empty(R, d, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(R, cols, device="cuda"))
    assert torch.equal(mb.rmsnorm(x, w, 0.0).out[0], w.to(T))        # r = 1
    r = mb.rmsnorm(x, w, 0.0, quant_group=group, out=out)
    v = w.double() * 448.0 / top.double()
    lo, hi = e4m3(v - v.abs() * 2.01 * u), e4m3(v + v.abs() * 2.01 * u)
    q = r.q.double()
    bad = (q < lo) | (q > hi)
    assert not bad.any(), "%d of %d" % (int(bad.sum()), bad.numel())
    scale = (top.double() / 448.0)[first]
    within(r.scales, scale.expand(R, cols), scale * 1.01 * u, "scales")


def check_gradient(g, h, w, eps, ds, dx, dw):
    """dx and dweight against the formulas in 64 bits."""
    R = h.shape[0]
    H, G, Wd = h.double(), g.double(), w.double()
    r = 1 / (H.square().mean(1, keepdim=True) + eps).sqrt()
    hg = H * G * Wd
    want = r * G * Wd - H * r ** 3 * hg.mean(1, keepdim=True) + (ds.double() if ds is not None else 0)
    # every term is off by its own roundings: three factors r at NORM_U, the mean of h g by 74 u of the magnitudes
    size = r * (G * Wd).abs() + 2 * H.abs() * r ** 3 * hg.abs().mean(1, keepdim=True) + (ds.double().abs() if ds is not None else 0)
    within(dx, want, want.abs() * U(h.dtype) * (1 + NORM_U) + 4 * NORM_U * size, "dx")
    terms = G * H * r
    within(dw, terms.sum(0), (R + 64 + 48) * u * terms.abs().sum(0), "dweight")


@pytest.mark.parametrize("R,d", [(1, 1), (1, 2048), (3, 7), (300, 64), (33, 1411), (700, 2048), (1201, 96), (5, 16384),
                                 (9, 4097), (2000, 250), (64, 4096), (13, 8192), (150, 5076)])
@pytest.mark.parametrize("T,W", [(BF16, F32), (BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("with_dsum", [True, False])
def test_norm_gradient(R, d, T, W, with_dsum):
    gn = gen(R + d)
    h, g = normal(gn, R, d, dtype=T) * 2, normal(gn, R, d, dtype=T)
    w = (1 + 0.2 * normal(gn, d)).to(W)
    ds = normal(gn, R, d, dtype=T) if with_dsum else None
    eps = 1e-5
    dx, dw = mb.rmsnorm_backward(g, h, w, eps, dsum=ds)
    check_gradient(g, h, w, eps, ds, dx, dw)
    dx2, dw2 = mb.rmsnorm_backward(g, h, w, eps, dsum=ds)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    dx3, none = mb.rmsnorm_backward(g, h, w, eps, dsum=ds, want_dweight=False)
    assert none is None and torch.equal(dx3, dx)
    if with_dsum:                                    # in place of the incoming gradients
        for target in (g.clone(), ds.clone()):
            a = [g, ds]
            a[0 if torch.equal(target, g) else 1] = target
            assert torch.equal(mb.rmsnorm_backward(a[0], h, w, eps, dsum=a[1], out=(target, None))[0], dx)


# rows for several turns of every CTA: three stages of the ring (aligned, more than eight turns), ragged rows whose threads keep their
# columns from row to row, with one to six CTAs per SM, the last turn with and without rows for every CTA
@pytest.mark.parametrize("R,d,T,W", [(5000, 2048, BF16, BF16), (7500, 1024, BF16, F32), (60000, 256, BF16, BF16), (1500, 4096, F32, F32),
                                     (2500, 2048, F32, F32), (9000, 520, F32, F32), (1001, 1411, F32, F32), (2500, 1411, BF16, BF16),
                                     (700, 4097, BF16, F32), (701, 2049, F32, F32), (3001, 515, F32, F32), (400, 9217, F32, F32),
                                     (451, 10003, BF16, BF16), (9000, 100, BF16, BF16), (1300, 8192, BF16, F32)])
@pytest.mark.parametrize("with_dsum", [True, False])
def test_norm_gradient_of_batches(R, d, T, W, with_dsum):
    gn = gen(R + d)
    h, g = normal(gn, R, d, dtype=T) * 2, normal(gn, R, d, dtype=T)
    w = (1 + 0.2 * normal(gn, d)).to(W)
    ds = normal(gn, R, d, dtype=T) if with_dsum else None
    dx, dw = mb.rmsnorm_backward(g, h, w, 1e-5, dsum=ds)
    check_gradient(g, h, w, 1e-5, ds, dx, dw)
    alone, none = mb.rmsnorm_backward(g, h, w, 1e-5, dsum=ds, want_dweight=False)
    assert none is None and torch.equal(alone, dx)
    if with_dsum:                                    # in place of what other rows are still to be fetched from
        t = ds.clone()
        got = mb.rmsnorm_backward(g, h, w, 1e-5, dsum=t, out=(t, torch.empty_like(dw)))
        assert torch.equal(t, dx) and torch.equal(got[1], dw)
    t = g.clone()
    got = mb.rmsnorm_backward(t, h, w, 1e-5, dsum=ds, out=(t, torch.empty_like(dw)))
    assert torch.equal(t, dx) and torch.equal(got[1], dw)


@pytest.mark.parametrize("T", [BF16, F32])
@pytest.mark.parametrize("d,layout", [(64, "aligned"), (61, "ragged"), (64, "unlike")])
@pytest.mark.parametrize("rms", [1e18, 1e15, 1e13, 1e-13, 1e-15, 3e-20])
def test_norm_gradient_of_large_and_small_rows(T, d, layout, rms):
    """r^2 and r^3 leave the range of fp32, the products that they stand in do not.  (The smallest squares are subnormal: each
    rounding of them and of the mean is off by 2^-150, 13 u of their sum together, which NORM_U's room covers.)"""
    gn, R = gen(d), 40
    pad = 1 if layout == "unlike" else 0
    h, g, ds = normal(gn, R, d + pad)[:, pad:], normal(gn, R, d, dtype=T), normal(gn, R, d, dtype=T) / rms
    h = (h * rms).to(T)
    if pad:
        h = torch.cat([h, h], 1)[:, pad:d + pad]
    w = 1 + 0.2 * normal(gn, d)
    check_gradient(g, h, w, 0.0, None, *mb.rmsnorm_backward(g, h, w, 0.0))
    check_gradient(g, h, w, 0.0, ds, *mb.rmsnorm_backward(g, h, w, 0.0, dsum=ds))


def test_norm_gradient_against_differences():
    """<gradient, direction> against central differences of the definition in 64 bits (truncation ~1e-10)."""
    R, d, eps = 7, 96, 1e-5
    gn = gen(11)
    x, add, g = normal(gn, R, d), normal(gn, R, d), normal(gn, R, d)
    w = 1 + 0.2 * normal(gn, d)
    s = normal(gn, R, d)                             # gradient of the sum past the norm
    h = mb.rmsnorm(x, w, eps, add=add).sum
    dx, dw = mb.rmsnorm_backward(g, h, w, eps, dsum=s)

    def loss(H, W):
        return ((H / (H.square().mean(1, keepdim=True) + eps).sqrt() * W) * g.double()).sum() + (H * s.double()).sum()
    for k in range(3):
        v, vw = normal(gn, R, d).double(), normal(gn, d).double()
        H, W, t = h.double(), w.double(), 1e-6
        num = (loss(H + t * v, W) - loss(H - t * v, W)) / (2 * t)
        size = (dx.double() * v).abs().sum()
        assert abs(num - (dx.double() * v).sum()) <= (4 * NORM_U + 1e-8) * 3 * size
        num = (loss(H, W + t * vw) - loss(H, W - t * vw)) / (2 * t)
        size = (dw.double() * vw).abs().sum() * 10   # dw sums terms of both signs
        assert abs(num - (dw.double() * vw).sum()) <= (NORM_U + 1e-8) * size


@pytest.mark.parametrize("R,d", [(1, 64), (3, 2048), (4, 1411), (16, 128), (20, 7), (33, 40)])
def test_norm_gradient_of_few_rows_into_an_unaligned_weight_gradient(R, d):
    gn = gen(R)
    h, g, w = normal(gn, R, d), normal(gn, R, d), 1 + 0.1 * normal(gn, d)
    for shift in (0, 1):
        dw = torch.full((d + 8,), 3.0, device="cuda")
        out = mb.rmsnorm_backward(g, h, w, out=(torch.empty_like(h), dw[shift:d + shift]))
        check_gradient(g, h, w, 1e-6, None, *out)
        assert (dw[:shift] == 3).all() and (dw[d + shift:] == 3).all()


def test_norm_gradient_strides_and_no_rows():
    gn, R, d = gen(3), 29, 200
    big = [normal(gn, R, d + 8 + 2 * i, dtype=BF16) for i in range(4)]
    h, g, ds, dx = [b[:, 2:d + 2] for b in big]
    w = 1 + 0.1 * normal(gn, d)
    edge = big[3].clone()
    got = mb.rmsnorm_backward(g, h, w, dsum=ds, out=(dx, torch.empty(d, device="cuda")))
    check_gradient(g, h, w, 1e-6, ds, *got)
    assert torch.equal(big[3][:, :2], edge[:, :2]) and torch.equal(big[3][:, d + 2:], edge[:, d + 2:])
    e = torch.empty(0, 16, device="cuda")
    dx0, dw0 = mb.rmsnorm_backward(e, e, torch.ones(16, device="cuda"))
    assert dx0.shape == (0, 16) and (dw0 == 0).all()


# ---- dispatch --------------------------------------------------------------------------------------------------
def routing(g, L, T, K, E, masked=0.0, skew=0.0):
    score = torch.rand(L, T, E, device="cuda", generator=g) + skew * torch.rand(L, 1, E, device="cuda", generator=g)
    sel = torch.topk(score, K, dim=-1).indices.to(torch.int32)
    if masked:
        sel[torch.rand(L, T, K, device="cuda", generator=g) < masked] = -1
    return sel


def sorted_by_hand(sel, E):
    """offsets, perm (-1 behind the end), inv with numpy, layer by layer."""
    L, T, K = sel.shape
    s = sel.reshape(L, -1).cpu().numpy()
    perm, inv, off = np.full(s.shape, -1, np.int32), np.full(s.shape, -1, np.int32), np.zeros((L, E + 1), np.int32)
    for l in range(L):
        flat = np.concatenate([np.flatnonzero(s[l] == e) for e in range(E)] or [[]]).astype(np.int32)
        off[l, 1:] = np.cumsum([(s[l] == e).sum() for e in range(E)])
        perm[l, :len(flat)] = flat
        inv[l, flat] = np.arange(len(flat))
    return off, perm, inv.reshape(sel.shape)


DISPATCH = [(1, 1, 1, 1, 8), (1, 1, 8, 64, 2048), (3, 5, 2, 8, 96), (24, 16, 4, 60, 128), (1, 300, 16, 256, 24), (2, 1000, 6, 64, 100),
            (1, 5000, 8, 64, 33), (1, 2049, 1, 7, 1), (5, 129, 3, 16, 250), (1, 20000, 2, 200, 16)]


@pytest.mark.parametrize("L,T,K,E,d", DISPATCH)
@pytest.mark.parametrize("masked", [0.0, 0.4, 1.0])
def test_dispatch(L, T, K, E, d, masked):
    g = gen(T + E)
    sel = routing(g, L, T, K, E, masked, skew=0.5)
    off, perm, inv = sorted_by_hand(sel, E)
    for T_ in (BF16, F32, torch.float8_e4m3fn):
        x = normal(g, L, T, d, dtype=T_)
        scales = torch.rand(L, T, 5, device="cuda", generator=g) if T_.itemsize == 1 else None
        raw = torch.int16 if T_ == BF16 else torch.int32 if T_ == F32 else torch.uint8
        out = mb.Dispatched(torch.full((L, E + 1), 9, device="cuda", dtype=torch.int32), torch.full((L, T * K), -7, device="cuda", dtype=torch.int32),
                            torch.full((L, T, K), -7, device="cuda", dtype=torch.int32), torch.full((L, T * K, d), 99, device="cuda", dtype=raw).view(T_),
                            None if scales is None else torch.full((L, T * K, 5), -3.0, device="cuda"))
        r = mb.dispatch(sel, E, x, scales=scales, out=out)
        assert np.array_equal(r.offsets.cpu().numpy(), off) and np.array_equal(r.inv.cpu().numpy(), inv)
        for l in range(L):
            n = off[l, E]
            p = torch.from_numpy(perm[l, :n]).long().cuda()
            assert torch.equal(r.perm[l, :n].long(), p) and (r.perm[l, n:] == -7).all()
            assert torch.equal(r.rows[l, :n].view(raw), x[l][p // K].view(raw)) and (r.rows[l, n:].view(raw) == 99).all()
            if scales is not None:
                assert torch.equal(r.scales[l, :n], scales[l][p // K]) and (r.scales[l, n:] == -3).all()
    alone = mb.dispatch(sel, E)                      # only the sort, fresh buffers
    assert np.array_equal(alone.offsets.cpu().numpy(), off) and np.array_equal(alone.inv.cpu().numpy(), inv) and alone.rows is None


@pytest.mark.parametrize("L,T,K,E,d,T_,cols", [(1, 70, 1, 4, 8192, F32, 100), (2, 33, 3, 9, 6152, BF16, 33), (1, 41, 16, 20, 1040, torch.float8_e4m3fn, 1),
                                               (1, 9, 2, 3, 60000, BF16, 7), (1, 600, 5, 11, 4112, F32, 64), (1, 3, 4, 4, 2064, BF16, 300)])
def test_dispatch_rows_of_many_pieces(L, T, K, E, d, T_, cols):
    """Rows that a warp moves in several pieces, the last one short; scale rows narrower and wider than a warp."""
    g = gen(d)
    sel = routing(g, L, T, K, E, 0.2)
    off, perm, _ = sorted_by_hand(sel, E)
    x, scales = normal(g, L, T, d, dtype=T_), torch.rand(L, T, cols, device="cuda", generator=g)
    r = mb.dispatch(sel, E, x, scales=scales)
    for l in range(L):
        n = off[l, E]
        p = torch.from_numpy(perm[l, :n]).long().cuda() // K
        assert torch.equal(r.rows[l, :n].view(torch.uint8), x[l].view(torch.uint8)[p]) and torch.equal(r.scales[l, :n], scales[l][p])


def test_dispatch_unusual_ids_and_layout():
    """The same expert twice for a token, ids outside [0, E) of every kind, one layer without the leading size, rows
    further apart than their width, no perm wanted, no tokens."""
    E, K, d = 5, 4, 40
    sel = torch.tensor([[2, 2, 0, 2], [-1, 5, 4, 4], [2147483647, -2147483648, 0, 256], [1, 1, 1, 1], [-1, -1, -1, -1]], device="cuda", dtype=torch.int32)
    off, perm, inv = sorted_by_hand(sel[None], E)
    g = gen(1)
    x = normal(g, 5, 64)[:, 3:3 + d]
    out = mb.Dispatched(torch.empty(E + 1, device="cuda", dtype=torch.int32), None, torch.empty(5, K, device="cuda", dtype=torch.int32),
                        torch.full((20, 48), 4.0, device="cuda")[:, 2:2 + d])
    r = mb.dispatch(sel, E, x, out=out)
    assert np.array_equal(r.offsets.cpu().numpy(), off[0]) and np.array_equal(r.inv.cpu().numpy(), inv[0])
    n = off[0, E]
    assert torch.equal(r.rows[:n], x[torch.from_numpy(perm[0, :n] // K).long().cuda()]) and (r.rows[n:] == 4).all()
    z = mb.dispatch(sel[:0], E, x[:0])
    assert (z.offsets == 0).all() and z.rows.shape == (0, d) and z.inv.shape == (0, K)


# ---- combine and its gradient ----------------------------------------------------------------------------------
def positions(g, L, T, K, masked):
    """Random distinct positions per layer, as a sort would give them; masked pairs -1, or out of range."""
    P = T * K
    inv = torch.stack([torch.randperm(P, device="cuda", generator=g) for _ in range(L)]).to(torch.int32).view(L, T, K)
    hole = torch.rand(L, T, K, device="cuda", generator=g) < masked
    inv[hole] = torch.where(torch.rand(int(hole.sum()), device="cuda", generator=g) < 0.5, -1, P).to(torch.int32)
    return inv, ~hole


COMBINE = [(1, 1, 1, 8), (1, 1, 8, 2048), (3, 5, 2, 96), (16, 1, 8, 2048), (1, 300, 16, 24), (2, 500, 6, 100), (1, 2049, 1, 1),
           (5, 129, 3, 250), (1, 777, 3, 1002), (2, 33, 4, 1411), (1, 64, 2, 4096), (1, 40, 5, 11111), (1, 9, 7, 20000)]


@pytest.mark.parametrize("L,T,K,d", COMBINE)
@pytest.mark.parametrize("R,Y", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("masked", [0.0, 0.5, 1.0])
def test_combine_and_gradient(L, T, K, d, R, Y, masked):
    g = gen(T * 7 + d)
    inv, kept = positions(g, L, T, K, masked)
    P = T * K
    rows = normal(g, L, P, d, dtype=R)
    w = torch.softmax(normal(g, L, T, K), -1)
    add, dy = normal(g, L, T, d, dtype=Y), normal(g, L, T, d, dtype=Y)
    # what a masked pair points at is never looked at: rows that no pair names, and the weights of masked pairs, are NaN
    named = torch.zeros(L, P, dtype=torch.bool, device="cuda")
    for l in range(L):
        named[l, inv[l][kept[l]].long()] = True
    rows[~named] = float("nan")
    w_ = torch.where(kept, w, torch.full_like(w, float("nan")))
    at = inv.long().clamp(0, P - 1)
    picked = torch.stack([rows[l][at[l]] for l in range(L)]).double()
    picked = torch.where(kept[..., None], picked, torch.zeros((), dtype=torch.float64, device="cuda"))
    for weight, a in ((w_, None), (w_, add), (None, None), (None, add)):
        wk = torch.where(kept, w.double() if weight is not None else torch.ones_like(w).double(), torch.zeros_like(w).double())[..., None]
        want = (wk * picked).sum(2) + (a.double() if a is not None else 0)
        size = (wk * picked).abs().sum(2) + (a.double().abs() if a is not None else 0)
        y = mb.combine(rows, inv, weight, add=a, out_dtype=Y)
        within(y, want, want.abs() * U(Y) + (K + 2) * u * size * (1 + U(Y)), "y")
        assert torch.equal(y, mb.combine(rows, inv, weight, add=a, out_dtype=Y))
        if a is not None:                           # in place
            b = a.clone()
            assert torch.equal(mb.combine(rows, inv, weight, add=b, out=b), y)
        drows = torch.full((L, P, d), 5.0, device="cuda", dtype=R)
        _, dw = mb.combine_backward(dy, rows, inv, weight, out=(drows, torch.full((L, T, K), 8.0, device="cuda")))
        terms = picked * dy.double()[:, :, None]
        within(dw, terms.sum(3), (d + 8) * u * terms.abs().sum(3), "dw")
        assert (dw[~kept] == 0).all()
        assert (drows[~named] == 5).all()
        for l in range(L):
            wantd = (wk[l] * dy[l].double()[:, None])[kept[l]]
            within(drows[l][inv[l][kept[l]].long()], wantd, wantd.abs() * (U(R) + 2 * u), "drows")
        alone, none = mb.combine_backward(dy, rows, inv, weight, want_dw=False, out=(torch.full_like(drows, 5.0), None))
        assert none is None and torch.equal(alone, drows)
        mine = rows.clone()                         # drows in place of rows: the products first
        got, dw2 = mb.combine_backward(dy, mine, inv, weight, out=(mine, torch.empty_like(dw)))
        assert torch.equal(dw2, dw) and torch.equal(got[named], drows[named]) and got[~named].isnan().all()


def test_combine_strides_and_empty():
    g, T, K, d = gen(2), 50, 3, 72
    inv, _ = positions(g, 1, T, K, 0.2)
    inv = inv[0]
    rows = normal(g, T * K, 80, dtype=BF16)[:, 4:4 + d]
    base = normal(g, T, 90)
    y, keep = base[:, 8:8 + d], base.clone()
    w = torch.rand(T, K, device="cuda", generator=g)
    want = mb.combine(rows.contiguous(), inv, w, out_dtype=F32)
    assert torch.equal(mb.combine(rows, inv, w, out=y), want)
    assert torch.equal(base[:, :8], keep[:, :8]) and torch.equal(base[:, 8 + d:], keep[:, 8 + d:])
    z = mb.combine(rows[:0], inv[:0], w[:0])
    assert z.shape == (0, d)
    dz = mb.combine_backward(z, rows[:0], inv[:0], w[:0])
    assert dz[0].shape == (0, d) and dz[1].shape == (0, K)


def test_combine_gradient_of_rows_apart():
    """Rows further apart than their width: a fresh drows gets the same strides."""
    g, T, K, d = gen(12), 40, 2, 56
    inv, _ = positions(g, 1, T, K, 0.0)
    base = normal(g, T * K, 64)
    rows, dy, w = base[:, :d], normal(g, T, d), torch.rand(T, K, device="cuda", generator=g)
    drows, dw = mb.combine_backward(dy, rows, inv[0], w)
    want = mb.combine_backward(dy, rows.contiguous(), inv[0], w)
    assert torch.equal(drows, want[0]) and torch.equal(dw, want[1])


def test_combine_gradient_against_differences():
    """The return of sorted rows and the sort are adjoint: differences of the definition in 64 bits in every input."""
    g, T, K, E, d = gen(4), 31, 3, 6, 48
    sel = routing(g, 1, T, K, E, masked=0.2)[0]
    x, w, dy = normal(g, T, d), torch.rand(T, K, device="cuda", generator=g), normal(g, T, d)
    r = mb.dispatch(sel, E, x)
    r.rows[int(r.offsets[-1]):] = 0
    drows, dw = mb.combine_backward(dy, r.rows, r.inv, w)
    drows[int(r.offsets[-1]):] = 0
    dx = mb.combine(drows, r.inv)
    kept = (sel >= 0).double()

    def loss(X, W):
        return ((W * kept).sum(1, keepdim=True) * X * dy.double()).sum()
    v, vw, t = normal(g, T, d).double(), normal(g, T, K).double(), 1e-6
    num = (loss(x.double() + t * v, w.double()) - loss(x.double() - t * v, w.double())) / (2 * t)
    assert abs(num - (dx.double() * v).sum()) <= ((K + 4) * u + 1e-8) * 4 * (dx.double() * v).abs().sum()
    num = (loss(x.double(), w.double() + t * vw) - loss(x.double(), w.double() - t * vw)) / (2 * t)
    size = ((x.double() * dy.double()).abs().sum(1, keepdim=True) * vw.abs()).sum()
    assert abs(num - (dw.double() * vw).sum()) <= ((d + 8) * u + 1e-8) * size


# ---- how they are used -----------------------------------------------------------------------------------------
def test_offsets_beyond_32_bits():
    """Sorted rows of more than 2^32 elements: the last rows land and come back where they belong."""
    g, T, K, E, d = gen(6), 65600, 8, 4, 8192
    sel = routing(g, 1, T, K, 64, 0.0)[0] % E
    x = normal(g, T, d, dtype=BF16)
    r = mb.dispatch(sel, E, x)
    assert r.rows.numel() > 2 ** 32 and int(r.offsets[-1]) == T * K
    for p in (0, T * K // 2, T * K - 2, T * K - 1):
        assert torch.equal(r.rows[p], x[int(r.perm[p]) // K])
    y = mb.combine(r.rows, r.inv)                    # K times x: bf16 sums of equal terms are exact up to one rounding
    for t in (0, T // 2, T - 1):
        within(y[t], K * x[t].double(), K * x[t].double().abs() * (U(BF16) + (K + 2) * u), "y")
    w = torch.rand(T, K, device="cuda", generator=g)
    _, dw = mb.combine_backward(x, r.rows, r.inv, w, out=(r.rows, torch.empty(T, K, device="cuda")))
    for t in (0, T - 1):
        sq = x[t].double().square().sum()
        within(dw[t], sq.expand(K), (d + 8) * u * sq.expand(K), "dw")
        p = int(r.inv[t, K - 1])
        within(r.rows[p], w[t, K - 1].double() * x[t].double(), (w[t, K - 1].double() * x[t].double()).abs() * (U(BF16) + 2 * u), "drows")


def block(x, add, w, sel, sel_w, E, experts, group=None):
    """norm with the residual's addition -> sort -> experts -> weighted return onto the residual stream."""
    n = mb.rmsnorm(x, w, 1e-6, add=add)
    s = mb.dispatch(sel, E, n.out)
    s.rows[int(s.offsets[-1]):] = 0
    o = experts(s)
    return n, s, o, mb.combine(o, s.inv, sel_w, add=n.sum)


def test_a_block_forward_and_backward():
    """A whole block with linear experts, forward and every gradient, against 64 bits.  fp32 throughout, so the only errors are the
    operators' own and those of the experts' products (d terms each)."""
    g, T, K, E, d = gen(8), 70, 3, 5, 64
    x, add = normal(g, T, d), normal(g, T, d)
    w = 1 + 0.1 * normal(g, d)
    We = normal(g, E, d, d) / math.sqrt(d)
    sel, sel_w = routing(g, 1, T, K, E, masked=0.15)[0], torch.rand(T, K, device="cuda", generator=g)
    dy = normal(g, T, d)
    Wd = We.double()

    def experts(s):
        off = s.offsets.tolist()
        return torch.cat([(s.rows[off[e]:off[e + 1]].double() @ Wd[e].T) for e in range(E)] + [s.rows[off[E]:].double() * 0]).float()
    n, s, o, y = block(x, add, w, sel, sel_w, E, experts)
    do, dsel_w = mb.combine_backward(dy, o, s.inv, sel_w)
    off = s.offsets.tolist()
    do[off[E]:] = 0
    drows = torch.cat([(do[off[e]:off[e + 1]].double() @ Wd[e]) for e in range(E)] + [do[off[E]:].double() * 0]).float()
    dn = mb.combine(drows, s.inv)
    dx, dw = mb.rmsnorm_backward(dn, n.sum, w, 1e-6, dsum=dy)
    # the same in 64 bits with automatic differentiation
    X, A, W, SW = (t.double().requires_grad_() for t in (x, add, w, sel_w))
    H = X + A
    N = H / (H.square().mean(1, keepdim=True) + 1e-6).sqrt() * W
    kept = sel >= 0
    part = torch.einsum("td,tkod->tko", N, Wd[sel.clamp_min(0).long()])
    Y = H + (torch.where(kept, SW, torch.zeros_like(SW))[..., None] * part).sum(1)
    (Y * dy.double()).sum().backward()
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    # relative errors in the 2-norm: a handful of fp32 roundings per value, 64 u at most from the norm
    for got, want in ((y, Y.detach()), (dx, X.grad), (dx, A.grad), (dw, W.grad), (dsel_w, SW.grad)):
        assert rel(got, want) <= 4 * NORM_U


def test_sort_and_return_reproduce_the_expert_forward():
    """dispatch has the grouping of the engine's own pass, and dispatch -> experts -> combine gives the engine's y."""
    from paper_2412_00099_b200 import synth
    import helpers as H
    wl = synth.QWEN.with_(L=2, S=72, E=20, K=4, C=10, d=256, I=128, n_shared=0)
    W = H.weights_for(wl)
    eng = mb.engine_for(wl, deterministic=True)
    eng.set_router(H.to_dev(wl.router()))
    Wd = {k: (None if v is None else H.to_dev(v)) for k, v in W.items()}
    eng.set_experts(**Wd)
    x = H.to_dev(next(iter(wl.hidden_trace(1))))
    sel, sel_w = (t[0] for t in eng.route_step(hidden=x[None]))
    y = eng.moe_forward(x, sel, sel_w)
    offsets, perm = eng.grouping()
    s = mb.dispatch(sel, wl.E, x)
    assert np.array_equal(s.offsets.cpu().numpy(), offsets) and np.array_equal(s.perm.cpu().numpy(), perm)
    o = torch.empty(wl.L, wl.S * wl.K, wl.d, device="cuda")
    for l in range(wl.L):
        for e in range(wl.E):
            a, b = offsets[l, e], offsets[l, e + 1]
            r = s.rows[l, a:b].double()
            hgate, hup = r @ Wd["Wg"][l, e].double().T, r @ Wd["Wu"][l, e].double().T
            act = (hgate * torch.sigmoid(hgate) * hup).to(BF16).double()
            o[l, a:b] = (act @ Wd["Wd"][l, e].double().T).float()
    H.ffn_close(y.cpu().numpy(), mb.combine(o, s.inv, sel_w).cpu().numpy())


def all_calls(x, add, w, sel, sel_w, E, dy):
    n = mb.rmsnorm(x, w, 1e-6, add=add, quant_group=32)
    s = mb.dispatch(sel, E, n.q, scales=n.scales)
    t = mb.dispatch(sel, E, n.out)
    y = mb.combine(t.rows, t.inv, sel_w, add=n.sum)
    do, dw = mb.combine_backward(dy, t.rows, t.inv, sel_w)
    dx, dweight = mb.rmsnorm_backward(mb.combine(do, t.inv), n.sum, w, 1e-6, dsum=dy)
    return [n.out, n.sum, n.q, n.scales, s.offsets, s.inv, s.rows, s.scales, t.rows, y, do, dw, dx, dweight]


@pytest.mark.parametrize("T,d", [(1, 64), (300, 256), (2500, 100)])
def test_streams_and_graphs(T, d):
    """On a side stream, captured and replayed on new inputs, two captured graphs replayed at the same time on two streams."""
    K, E = 4, 12

    def inputs(seed):
        g = gen(seed)
        return [normal(g, T, d, dtype=BF16), normal(g, T, d), 1 + 0.1 * normal(g, d), routing(g, 1, T, K, E)[0],
                torch.rand(T, K, device="cuda", generator=g), E, normal(g, T, d, dtype=BF16)]
    ins = [inputs(20), inputs(21), inputs(22)]
    want = [[t.clone() for t in all_calls(*i)] for i in ins]
    torch.cuda.synchronize()
    same = lambda a, b: all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(a, b))  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = all_calls(*ins[0])
    side.synchronize()
    assert same(got, want[0])
    graphs = []
    for k in (0, 1):
        static = [t.clone() if isinstance(t, torch.Tensor) else t for t in ins[k]]
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = all_calls(*static)
        graphs.append((gr, static, out))
    for s, new in zip(graphs[0][1], ins[2]):         # new inputs in the captured buffers
        if isinstance(s, torch.Tensor):
            s.copy_(new)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for (gr, _, _), st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
    torch.cuda.synchronize()
    assert same(graphs[0][2], want[2]) and same(graphs[1][2], want[1])


def test_results_count_as_changed():
    """A tensor that a backward pass has saved and a call then overwrites: the backward pass refuses."""
    x, w = torch.ones(4, 64, device="cuda"), torch.ones(64, device="cuda")
    leaf = torch.ones(4, 64, device="cuda", requires_grad=True)
    loss = (leaf * x).sum()
    mb.rmsnorm(x, w, add=x.clone(), out=mb.NormOut(sum=x))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    versions = dx._version, dw._version
    mb.rmsnorm_backward(x, x, w, out=(dx, dw))
    assert dx._version > versions[0] and dw._version > versions[1]
    with torch.inference_mode():
        y = mb.rmsnorm(torch.ones(4, 64, device="cuda"), w).out
    assert torch.isfinite(y).all()


def test_binding_refuses_what_does_not_fit():
    x, w = torch.zeros(4, 16, device="cuda"), torch.ones(16, device="cuda")
    bad = pytest.raises(mb.McceError)
    with bad:
        mb.rmsnorm(x.half(), w)
    with bad:
        mb.rmsnorm(x, w[:8])
    with bad:
        mb.rmsnorm(x, w, add=x[:2])
    with bad:
        mb.rmsnorm(x, w, add=x.bfloat16())           # neither fp32 nor the type of x ... x is fp32
    with bad:
        mb.rmsnorm(x[:1].expand(4, 16), w)           # rows overlap
    with bad:
        mb.rmsnorm(x.t()[:4, :4], w[:4])             # columns not contiguous
    with bad:
        mb.rmsnorm(x, w, quant_group=48)
    with bad:
        mb.rmsnorm(x, w, eps=-1.0)
    with bad:
        mb.rmsnorm_backward(x, x.bfloat16(), w)
    sel = torch.zeros(4, 2, device="cuda", dtype=torch.int32)
    with bad:
        mb.dispatch(sel.long(), 4, x)
    with bad:
        mb.dispatch(sel, 0, x)
    with bad:
        mb.dispatch(sel, 257, x)
    with bad:
        mb.dispatch(sel, 4, x[:3])
    with bad:
        mb.combine(x, sel)                           # 4 rows for 8 pairs
    with bad:
        mb.combine(torch.zeros(8, 16, device="cuda"), sel, torch.zeros(4, 2, device="cuda", dtype=BF16))
    with bad:
        mb.combine(torch.zeros(8, 16, device="cuda"), sel, out_dtype=BF16)
    with bad:
        mb.combine_backward(x[:3], torch.zeros(8, 16, device="cuda"), sel)


def test_chained_step_with_norms_equals_the_composition():
    """mcce_set_norm: layer l routes and runs its experts on the norm of the residual stream, which itself stays as it is.  Against
    single-layer engines joined by the operators (fp32-pipe experts, so every step is the same kernels: bit for bit), with
    one layer and several, and off again."""
    from paper_2412_00099_b200 import synth
    import helpers as H
    for wl in (synth.TINY.with_(L=3, S=6), synth.TINY.with_(L=1, S=5),
               synth.QWEN.with_(L=3, S=20, E=12, K=4, C=6, d=264, I=256, n_shared=1)):
        Wr, W = wl.router(), H.weights_for(wl)
        Wd = {k: (None if v is None else H.to_dev(v)) for k, v in W.items()}
        full = mb.engine_for(wl, ffn_impl=mb.FFN_SIMT)
        full.set_router(H.to_dev(Wr))
        full.set_experts(**Wd)
        plain = mb.engine_for(wl, ffn_impl=mb.FFN_SIMT)
        plain.set_router(H.to_dev(Wr))
        plain.set_experts(**Wd)
        singles = []
        for l in range(wl.L):
            e = mb.engine_for(wl.with_(L=1), ffn_impl=mb.FFN_SIMT)
            e.set_router(H.to_dev(Wr[l:l + 1]))
            e.set_experts(**{k: (None if v is None else v[l:l + 1].contiguous()) for k, v in Wd.items()})
            singles.append(e)
        nw = 1 + 0.3 * normal(gen(wl.L), wl.L, wl.d)
        full.set_norm(nw, 1e-5)
        for x0 in [H.to_dev(x)[0] for x in wl.with_(L=1).hidden_trace(4)]:
            keep = x0.clone()
            x_c, sel_c = full.decode_step_chained(x0, want_sel=True)
            assert torch.equal(x0, keep)
            x = x0
            for l, e in enumerate(singles):
                n = mb.rmsnorm(x, nw[l], 1e-5).out
                sel, w = e.route_step(hidden=n[None, None])
                y = e.moe_forward(n[None], sel[0], w[0])[0]
                assert torch.equal(sel[0, 0], sel_c[l])
                x = mb.rmsnorm(x, nw[l], 1e-5, add=y, want_out=False).sum
            assert torch.equal(x, x_c)
        full.set_norm(None)                          # off: the step of an engine that never had one
        full.reset()
        x0 = H.to_dev(next(iter(wl.with_(L=1).hidden_trace(1))))[0]
        assert torch.equal(full.decode_step_chained(x0), plain.decode_step_chained(x0))
        with pytest.raises(mb.McceError):
            full.set_norm(nw, -1.0)
        with pytest.raises(AssertionError):
            full.set_norm(nw[:, :8])
        for e in [full, plain, *singles]:
            e.close()


def test_norm_weights_live_as_long_as_the_engine():
    """Steps under way read the weight that was set when they were queued: replacing it frees nothing."""
    import weakref
    from paper_2412_00099_b200 import synth
    eng = mb.engine_for(synth.TINY)
    weights = [torch.ones(synth.TINY.L, synth.TINY.d, device="cuda") for _ in range(2)]
    alive = [weakref.ref(w) for w in weights]
    for w in weights:
        eng.set_norm(w)
    eng.set_norm(None)
    del weights, w
    assert all(a() is not None for a in alive)
    eng.close()


@pytest.mark.parametrize("S,d,n_shared", [(72, 256, 0), (130, 512, 1)])
def test_chained_step_with_norms_on_the_tensor_path(S, d, n_shared):
    """The normalised buffer as the tensor-core experts and the router GEMM read it, several layers and one: against single-layer
    engines joined by the operators (deterministic contexts add in a fixed order: bit for bit)."""
    from paper_2412_00099_b200 import synth
    import helpers as H
    for L in (3, 1):
        wl = synth.QWEN.with_(L=L, S=S, E=12, K=4, C=6, d=d, I=256, n_shared=n_shared)
        Wr, W = wl.router(), H.weights_for(wl)
        Wd = {k: (None if v is None else H.to_dev(v)) for k, v in W.items()}

        def engine(layers, wr, we):
            e = mb.engine_for(wl.with_(L=layers), ffn_impl=mb.FFN_TENSOR, deterministic=True)
            e.set_router(wr)
            e.set_experts(**we)
            assert e.uses_tensor_path()
            return e
        full = engine(L, H.to_dev(Wr), Wd)
        singles = [engine(1, H.to_dev(Wr[l:l + 1]), {k: (None if v is None else v[l:l + 1].contiguous()) for k, v in Wd.items()})
                   for l in range(L)]
        nw = 1 + 0.3 * normal(gen(L), L, d)
        full.set_norm(nw, 1e-5)
        for x0 in [H.to_dev(x)[0] for x in wl.with_(L=1).hidden_trace(4)]:
            x_c, sel_c = full.decode_step_chained(x0, want_sel=True)
            x = x0
            for l, e in enumerate(singles):
                n = mb.rmsnorm(x, nw[l], 1e-5).out
                sel, w = e.route_step(hidden=n[None, None])
                y = e.moe_forward(n[None], sel[0], w[0])[0]
                assert torch.equal(sel[0, 0], sel_c[l])
                x = mb.rmsnorm(x, nw[l], 1e-5, add=y, want_out=False).sum
            assert torch.equal(x, x_c)
        for e in [full, *singles]:
            e.close()


def test_columns_of_one_buffer_and_overlaps():
    """Tensors that are columns of one buffer share no memory and are taken; outputs that reach into an input are refused."""
    g, R, d = gen(31), 21, 64
    buf = normal(g, R, 4 * d, dtype=BF16)
    x, add, w = buf[:, :d], buf[:, d:2 * d], 1 + 0.1 * normal(g, d)
    want = mb.rmsnorm(x.clone(), w, 1e-6, add=add.clone())
    r = mb.rmsnorm(x, w, 1e-6, add=add, out=mb.NormOut(buf[:, 2 * d:3 * d], buf[:, 3 * d:]))
    assert torch.equal(r.out, want.out) and torch.equal(r.sum, want.sum)
    dx, dw = mb.rmsnorm_backward(x.clone(), add.clone(), w, dsum=x.clone())
    got = mb.rmsnorm_backward(x, add, w, dsum=x, out=(buf[:, 2 * d:3 * d], torch.empty_like(dw)))
    assert torch.equal(got[0], dx) and torch.equal(got[1], dw)
    with pytest.raises(mb.McceError):                # the sum one row late in x
        mb.rmsnorm(x[:-1], w, 1e-6, add=add[:-1], out=mb.NormOut(None, x[1:]))
    with pytest.raises(mb.McceError):
        mb.rmsnorm(x[:8], w, 1e-6, out=mb.NormOut(buf[4:12, d // 2:d // 2 + d]))
    T, K = 7, 3
    rows, inv = buf[:, :d], torch.randperm(T * K, device="cuda", generator=g).to(torch.int32).view(T, K)
    y = mb.combine(rows.clone(), inv)
    got = mb.combine(rows, inv, out=buf[:T, d:2 * d])
    assert torch.equal(got, y)
    with pytest.raises(mb.McceError):
        mb.combine(rows, inv, out=rows[2:2 + T])
    dy = normal(g, T, d, dtype=BF16)
    drows, dw = mb.combine_backward(dy, rows.clone(), inv)
    got = mb.combine_backward(dy, rows, inv, out=(buf[:, 2 * d:3 * d], torch.empty_like(dw)))
    assert torch.equal(got[0], drows) and torch.equal(got[1], dw)
    sel = torch.randint(0, 4, (R, 1), device="cuda", generator=g).to(torch.int32)
    want = mb.dispatch(sel, 4, rows.clone())
    out = want._replace(rows=buf[:, d:2 * d])
    assert torch.equal(mb.dispatch(sel, 4, rows, out=out).rows, mb.dispatch(sel, 4, rows.clone()).rows)
    with pytest.raises(mb.McceError):
        mb.dispatch(sel, 4, rows, out=want._replace(inv=want.perm.view(R, 1)))
    with pytest.raises(mb.McceError):
        mb.dispatch(sel, 4, rows, out=want._replace(rows=rows))


def test_inside_an_autograd_function():
    """The way to train with them: a Function of the two calls, parameters that require grad handed straight in."""
    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w):
            ctx.save_for_backward(x, w)
            return mb.rmsnorm(x, w, 1e-6).out

        @staticmethod
        def backward(ctx, g):
            x, w = ctx.saved_tensors
            return mb.rmsnorm_backward(g, x, w, 1e-6)
    gn = gen(40)
    x, w, g = normal(gn, 9, 96).requires_grad_(), (1 + 0.1 * normal(gn, 96)).requires_grad_(), normal(gn, 9, 96)
    Norm.apply(x, w).backward(g)
    check_gradient(g, x.detach(), w.detach(), 1e-6, None, x.grad, w.grad)
    with pytest.raises(mb.McceError, match="requires grad"):
        mb.rmsnorm(x, w)
    with torch.no_grad():
        assert torch.equal(mb.rmsnorm(x, w).out, Norm.apply(x, w))


# the layouts of batches: more tokens than fill the device with one unit per lane (2368), 16-byte units, two elements and one, one pair
# per token, two and more, rows of one warp and of several, both sides of the limit
@pytest.mark.parametrize("L,T,K,d", [(1, 2500, 8, 256), (1, 2367, 5, 256), (1, 2368, 5, 256), (3, 1200, 1, 520), (1, 3000, 2, 1032), (2, 1300, 3, 2048),
                                     (1, 2600, 6, 250), (1, 2600, 2, 250), (2, 1250, 4, 141), (1, 2500, 1, 333), (1, 2400, 3, 2050),
                                     (1, 2400, 2, 2307), (1, 5000, 16, 24)])
@pytest.mark.parametrize("R,Y", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("masked", [0.0, 0.3])
def test_combine_and_gradient_of_batches(L, T, K, d, R, Y, masked):
    g = gen(T * 7 + d)
    inv, kept = positions(g, L, T, K, masked)
    P = T * K
    rows = normal(g, L, P, d, dtype=R)
    named = torch.zeros(L, P, dtype=torch.bool, device="cuda")
    for l in range(L):
        named[l, inv[l][kept[l]].long()] = True
    rows[~named] = float("nan")
    w = torch.softmax(normal(g, L, T, K), -1)
    w_ = torch.where(kept, w, torch.full_like(w, float("nan")))
    add, dy = normal(g, L, T, d, dtype=Y), normal(g, L, T, d, dtype=Y)
    at = inv.long().clamp(0, P - 1)
    picked = torch.where(kept[..., None], torch.stack([rows[l][at[l]] for l in range(L)]).double(), torch.zeros((), dtype=torch.float64, device="cuda"))
    for weight, a in ((w_, add), (None, None)):
        wk = torch.where(kept, w.double() if weight is not None else torch.ones_like(w).double(), torch.zeros_like(w).double())[..., None]
        want = (wk * picked).sum(2) + (a.double() if a is not None else 0)
        size = (wk * picked).abs().sum(2) + (a.double().abs() if a is not None else 0)
        y = mb.combine(rows, inv, weight, add=a, out_dtype=Y)
        within(y, want, want.abs() * U(Y) + (K + 2) * u * size * (1 + U(Y)), "y")
        drows = torch.full((L, P, d), 5.0, device="cuda", dtype=R)
        _, dw = mb.combine_backward(dy, rows, inv, weight, out=(drows, torch.full((L, T, K), 8.0, device="cuda")))
        terms = picked * dy.double()[:, :, None]
        within(dw, terms.sum(3), (d + 8) * u * terms.abs().sum(3), "dw")
        assert (dw[~kept] == 0).all() and (drows[~named] == 5).all()
        for l in range(L):
            wantd = (wk[l] * dy[l].double()[:, None])[kept[l]]
            within(drows[l][inv[l][kept[l]].long()], wantd, wantd.abs() * (U(R) + 2 * u), "drows")
        alone, _ = mb.combine_backward(dy, rows, inv, weight, want_dw=False, out=(torch.full_like(drows, 5.0), None))
        assert torch.equal(alone, drows)
        mine = rows.clone()
        got, dw2 = mb.combine_backward(dy, mine, inv, weight, out=(mine, torch.empty_like(dw)))
        assert torch.equal(dw2, dw) and torch.equal(got[named], drows[named]) and got[~named].isnan().all()
