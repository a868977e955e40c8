"""The experts' products where several CTAs, maps or kernels could serve a call: what the rules choose for odd offsets, every way of sharing a reduction, strided
results.  Tolerances as in test_gpu_linear: u = 2^-24, U(T) half a step of T relative to the value; a sum of k products is within (k + 8) u of its terms'
magnitudes S."""
import pytest
import torch

import test_gpu_linear as base
from test_gpu_linear import BF16, F32, U, act, gen, inside, normal, offsets_of, slope, some_counts, sums, u, within

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2412_00099_b200 import binding as mb


@pytest.mark.parametrize("T", [BF16, F32])
@pytest.mark.parametrize("E,R,n,k", [(1, 30, 264, 4096), (4, 7, 136, 2048), (6, 120, 136, 2048), (4, 160, 136, 2048), (4, 400, 136, 1040), (4, 1200, 72, 64),
                                     (5, 3, 40, 64), (8, 900, 520, 136), (8, 320, 136, 2048), (6, 120, 2048, 136), (8, 320, 2048, 136), (4, 400, 2048, 136)])
@pytest.mark.parametrize("gated", [False, True])
def test_offsets_that_give_a_row_twice(T, E, R, n, k, gated):
    """[0, R, 0, R ..]: whatever those rows become, the calls end as always, without a wait that gives up, touch nothing outside them, and the weight gradients
    are those of the rows that every expert was given."""
    g, two = gen(R + n), 1 + gated
    off = torch.tensor([0, R] * ((E + 2) // 2), dtype=torch.int32, device="cuda")[:E + 1].contiguous()
    buf = torch.full((3 * R, two * max(n, k)), 7.0, device="cuda", dtype=T)
    x, dout = normal(g, R, k, dtype=T), normal(g, R, two * n, dtype=T)
    w, wu = normal(g, E, n, k, dtype=T, std=k ** -0.5), normal(g, E, n, k, dtype=T, std=k ** -0.5) if gated else None
    for _ in range(3):
        mb.expert_linear(x, off, w, w_up=wu, out=mb.LinearOut(buf[R:2 * R, :n]))
        mb.expert_linear_backward(dout, off, w, w_up=wu, out=mb.LinearGrad(buf[R:2 * R, :k]))
    mb.expert_linear_status()
    assert (buf[:R] == 7).all() and (buf[2 * R:] == 7).all() and (buf[:, max(n, k):] == 7).all()
    r = mb.expert_linear_dweight(dout, x, off, gated=gated, want_db=True, out_dtype=F32)
    for i in range(two):
        d = dout[:, i * n:(i + 1) * n].double()
        dw, S, db, Sb = d.T @ x.double(), d.abs().T @ x.double().abs(), d.sum(0), d.abs().sum(0)
        for e in range(E):
            on = 1 - e % 2
            within(r[i][e], on * dw, on * ((R + 8) * u * S + dw.abs() * 2 * u), "dw")
            within(r[2 + i][e], on * db, on * ((R + 8) * u * Sb + db.abs() * 2 * u), "db")
    mb.expert_linear_status()


def test_a_wait_that_gives_up_is_reported_once():
    """On the stream it happened on and on another, and the calls after it are whole."""
    g, R, n, k = gen(4), 300, 136, 72
    off, x, w = offsets_of([[100, 200]])[0], normal(g, R, k, dtype=BF16), normal(g, 2, n, k, dtype=BF16)
    want = mb.expert_linear(x, off, w).out
    mb.expert_linear_status()
    lib, side = mb.load(), torch.cuda.Stream()
    for stream in (torch.cuda.current_stream(), side):
        with torch.cuda.stream(stream):
            assert lib.mcce_selftest_expert_linear_timeout(1_000_000, stream.cuda_stream) == 0     # 1 ms
            with pytest.raises(mb.McceError, match="bounded wait"):
                mb.expert_linear_status()
            mb.expert_linear_status()
        assert torch.equal(mb.expert_linear(x, off, w).out, want)
        mb.expert_linear_status()


@pytest.mark.parametrize("T", [BF16, F32])
@pytest.mark.parametrize("E,R,n,k", [(1, 1, 200, 64), (2, 7, 200, 64), (1, 30, 200, 4096), (4, 160, 136, 2048), (1, 200, 136, 2048), (6, 120, 200, 64), (6, 360, 200, 64),
                                     (2, 900, 200, 64), (2, 100, 51, 33)])
@pytest.mark.parametrize("gated", [False, True])
def test_silu_in_fp32(T, E, R, n, k, gated):
    """fp32 results of bf16 rows are those of an fp32 activation.  A row of x has a single 1, so that z is a weight, exactly, from -80 to 80.  silu(z) = z / (1 + e^-z):
    two steps (4 u) each of the exponential and the division (what CUDA states for expf and, between 2^-126 and 2^126, __fdividef), a rounding (u) each of the sum
    and the product, one more times z_up: 11 u, 12 with their products."""
    g = gen(R + n)
    off = offsets_of(some_counts(1, E, R, g))[0]
    col = torch.randint(k, (R,), device="cuda", generator=g)
    x = torch.zeros(R, k, device="cuda", dtype=T)
    x[torch.arange(R, device="cuda"), col] = 1
    w, wu = (160 * torch.rand(E, n, k, device="cuda", generator=g) - 80).to(T), normal(g, E, n, k, dtype=T) if gated else None
    out = mb.expert_linear(x, off, w, w_up=wu, act="silu", out_dtype=F32).out
    owner = torch.bucketize(torch.arange(R, device="cuda"), off[1:].long(), right=True)
    z = w[owner, :, col].double()
    want = z * torch.sigmoid(z) * (wu[owner, :, col].double() if gated else 1)
    within(out, want, 12 * u * want.abs() + 2.0 ** -149, "silu")


@pytest.mark.parametrize("T,O", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("pad", [0, 8, 3])
@pytest.mark.parametrize("add", [False, True])
def test_gradients_into_one_buffer(T, O, pad, add):
    """dw and dw_up as the two halves of one buffer [E,2n,k] with padded rows (as a fused gate and up weight lies): those of separate tensors, bit for bit where the
    kernel is the same, nothing else touched; and the products that read weights from such a buffer."""
    g, E, R, n, k = gen(8), 5, 700, 72, 136
    off = offsets_of([[100, 0, 333, 17, 250]])[0]
    x, dout = normal(g, R, k, dtype=T), normal(g, R, 2 * n, dtype=T)
    buf = torch.full((E, 2 * n, k + pad), 9.0, device="cuda", dtype=O)
    halves = mb.WeightGrad(buf[:, :n, :k], buf[:, n:, :k])
    before = mb.WeightGrad(*[normal(g, E, n, k, dtype=O) for _ in range(2)]) if add else None
    if add:
        halves.dw.copy_(before.dw), halves.dw_up.copy_(before.dw_up)
    want = mb.expert_linear_dweight(dout, x, off, gated=True, add=before, out_dtype=O)
    mb.expert_linear_dweight(dout, x, off, gated=True, add=halves if add else None, out=halves)
    assert torch.equal(halves.dw, want.dw) and torch.equal(halves.dw_up, want.dw_up) and (buf[:, :, k:] == 9).all()
    w = buf.to(T)
    w, wu = w[:, :n, :k], w[:, n:, :k]
    for a, b in ((mb.expert_linear(x, off, w, w_up=wu, act="silu").out, mb.expert_linear(x, off, w.contiguous(), w_up=wu.contiguous(), act="silu").out),
                 (mb.expert_linear_backward(dout, off, w, w_up=wu).dx, mb.expert_linear_backward(dout, off, w.contiguous(), w_up=wu.contiguous()).dx)):
        # a start or stride that is no multiple of 16 bytes may take another kernel: two sums of at most 2 n or k products, and a rounding, per element
        assert torch.equal(a, b) or (pad == 3 and ((a.double() - b.double()).abs() <= 2 * (2 * n + k + 8) * u * 40 * b.double().abs().max() + 2 * U(T) * b.double().abs()).all())
    mb.expert_linear_status()


# Ways of sharing a reduction that tiles of 32, 64 and 128 rows have: two or four CTAs (rows per group, slabs of 64 products and tiles decide)
SPLIT_FORWARD = [(1, 1, 100, 136, 2048), (1, 4, 400, 136, 1040), (2, 1, 200, 264, 1024),        # 128 rows
                 (1, 1, 60, 136, 2048), (1, 3, 120, 72, 1024),                                  # 64 rows: four, two
                 (1, 2, 60, 520, 4096), (1, 1, 16, 136, 1024), (1, 2, 40, 72, 1088)]            # 32 rows: four, two
SPLIT_BACKWARD = [(1, 1, 100, 1024, 136), (1, 4, 400, 1040, 136), (2, 1, 200, 1088, 264), (1, 1, 60, 2048, 136), (1, 3, 120, 1024, 72), (1, 2, 100, 520, 136),
                  (1, 2, 60, 4096, 520), (1, 1, 16, 1024, 136), (1, 2, 40, 1088, 72), (1, 1, 16, 512, 136)]


@pytest.mark.parametrize("shape", SPLIT_FORWARD, ids=str)
@pytest.mark.parametrize("O", [BF16, F32])
@pytest.mark.parametrize("gated", [False, True])
def test_shared_reductions(shape, O, gated):
    base.test_linear(shape, BF16, O, gated)


@pytest.mark.parametrize("shape", SPLIT_BACKWARD, ids=str)
@pytest.mark.parametrize("gated", [False, True])
def test_shared_reductions_backward(shape, gated):
    base.test_linear_backward(shape, BF16, gated)


@pytest.mark.parametrize("L,E,R", [(1, 3, 7), (1, 3, 30), (1, 3, 150), (1, 3, 500), (2, 2, 700), (1, 1, 90)])
@pytest.mark.parametrize("n,k", [(136, 72), (200, 1088), (1088, 192)])
@pytest.mark.parametrize("gated", [False, True])
def test_weights_whose_step_is_no_multiple_of_a_row(L, E, R, n, k, gated):
    """Matrices of padded rows with something between them, so that they are not rows of one tall matrix: the same bits as packed ones, whatever lies between."""
    g, ld = gen(n + R), k + 8
    off = offsets_of(some_counts(L, E, R, g))
    x, dout = normal(g, L, R, k, dtype=BF16), normal(g, L, R, (1 + gated) * n, dtype=BF16)
    packed = [normal(g, L, E, n, k, dtype=BF16, std=k ** -0.5) for _ in range(1 + gated)] + [None] * (1 - gated)
    apart = []
    for w in packed:
        step = n * ld + 24
        buf = torch.full((L * E * step,), float("nan"), device="cuda", dtype=BF16)
        apart.append(w if w is None else torch.as_strided(buf, (L, E, n, k), (E * step, step, ld, 1)).copy_(w))
    there = inside(off, R)
    a, b = (mb.expert_linear(x, off, w, w_up=wu, act="gelu", save="same") for w, wu in (apart, packed))
    assert torch.equal(a.out[there], b.out[there]) and torch.equal(a.saved[there], b.saved[there]) and a.out[there].isfinite().all()
    a, b = (mb.expert_linear_backward(dout, off, w, w_up=wu).dx for w, wu in (apart, packed))
    assert torch.equal(a[there], b[there]) and a[there].isfinite().all()
    mb.expert_linear_status()


@pytest.mark.parametrize("pad,between", [(8, 0), (8, 32), (0, 64), (2, 0)])
@pytest.mark.parametrize("T,O", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("n,k", [(72, 136), (300, 264), (130, 520)])
def test_gradients_into_rows_further_apart(T, O, pad, between, n, k):
    """dw with padded rows and something between the matrices, without anything added (written by copies from shared memory where 16 bytes allow it)."""
    g, L, E, R = gen(n + pad), 2, 3, 333
    off = offsets_of([[100, 0, 200], [7, 128, 64]])
    x, dout = normal(g, L, R, k, dtype=T), normal(g, L, R, n, dtype=T)
    step = n * (k + pad) + between
    buf = torch.full((L * E * step,), 9.0, device="cuda", dtype=O)
    dw = torch.as_strided(buf, (L, E, n, k), (E * step, step, k + pad, 1))
    want = mb.expert_linear_dweight(dout, x, off, out_dtype=O).dw
    mb.expert_linear_dweight(dout, x, off, out=mb.WeightGrad(dw))
    assert torch.equal(dw, want)
    dw.fill_(9.0)
    assert (buf == 9).all()
    mb.expert_linear_status()


@pytest.mark.parametrize("save", ["same", "e4m3"])
@pytest.mark.parametrize("tokens,d,f", [(37, 64, 96), (150, 72, 40), (500, 128, 192), (900, 256, 136)])
def test_layer_and_its_gradients_in_bf16(tokens, d, f, save):
    """Norm, sort, gated experts, down projection with bias, weighted return onto the residual stream, and back, in bf16, against 64 bits, every tensor by its relative
    2-norm, which a missing or wrong part of a few percent exceeds.  A rounding is off by at most U = 2^-8 of a value, evenly spread, so U / sqrt(3) in the root mean
    square; at most 8 of them lie one behind the other, independent of one another: sqrt(8 / 3) U.  Products of random matrices keep relative norms,
    slopes and sums move them by less than 2: 2 sqrt(8 / 3) U = 0.0128.  What was kept in 8 bits (2^-4) is taken from what the forward call kept, one stage more
    of the 64-bit formula: the same tolerance."""
    E, K, T = 5, 2, BF16
    g = gen(tokens)
    x, wn = normal(g, tokens, d, dtype=T), 1 + 0.1 * normal(g, d)
    wg, wu, wd = (normal(g, E, *s, dtype=T, std=s[1] ** -0.5) for s in ((f, d), (f, d), (d, f)))
    bd = normal(g, E, d, std=0.1).to(T)
    sel = torch.stack([torch.randperm(E, generator=g, device="cuda")[:K] for _ in range(tokens)]).to(torch.int32)
    sel[3, 1] = -1
    sw, dy = torch.softmax(normal(g, tokens, K), -1), normal(g, tokens, d, dtype=T)
    h = mb.rmsnorm(x, wn, 1e-6).out
    s = mb.dispatch(sel, E, h)
    a = mb.expert_linear(s.rows, s.offsets, wg, w_up=wu, act="silu", save=save)
    o = mb.expert_linear(a.out, s.offsets, wd, bias=bd).out
    y = mb.combine(o, s.inv, sw, add=x)
    do, dsw = mb.combine_backward(dy, o, s.inv, sw)
    da = mb.expert_linear_backward(do, s.offsets, wd, saved=a.saved, scales=a.scales, act="silu")
    gd = mb.expert_linear_dweight(do, da.h, s.offsets, want_db=True)
    drows = mb.expert_linear_backward(da.dx, s.offsets, wg, w_up=wu).dx
    gu = mb.expert_linear_dweight(da.dx, s.rows, s.offsets, gated=True)
    dh = mb.combine(drows, s.inv)
    dx, dwn = mb.rmsnorm_backward(dh, x, wn, 1e-6, dsum=dy)

    # 64 bits, with the pre-activations that the backward pass gets where they were kept in 8 bits
    X, N, W = x.double(), wn.double(), [w.double() for w in (wg, wu, wd)]
    r = (X.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
    H = X * r * N
    Y, dH = X.clone(), torch.zeros_like(X)
    G = dict(wg=torch.zeros_like(W[0]), wu=torch.zeros_like(W[1]), wd=torch.zeros_like(W[2]), bd=torch.zeros_like(bd.double()), sw=torch.zeros_like(sw.double()))
    kept = None if save == "same" else base.unpacked(a.saved, a.scales, 2)
    for k in range(K):
        for e in range(E):
            t = (sel[:, k] == e).nonzero()[:, 0]
            z, up = H[t] @ W[0][e].T, H[t] @ W[1][e].T
            out = (act(z, "silu") * up) @ W[2][e].T + bd[e].double()
            Y[t] += sw[t, k, None].double() * out
            G["sw"][t, k] = (out * dy[t].double()).sum(-1)
            D = sw[t, k, None].double() * dy[t].double()
            if kept is not None:
                z, up = kept[s.inv[t, k].long()].chunk(2, -1)
            hidden = act(z, "silu") * up
            G["wd"][e] += D.T @ hidden
            G["bd"][e] += D.sum(0)
            back = D @ W[2][e]
            dz, du = back * up * slope(z, "silu"), back * act(z, "silu")
            G["wg"][e] += dz.T @ H[t]
            G["wu"][e] += du.T @ H[t]
            dH[t] += dz @ W[0][e] + du @ W[1][e]
    v = dH * N
    G["x"] = dy.double() + r * v - X * r ** 3 * (v * X).mean(-1, keepdim=True)
    G["wn"] = (dH * X * r).sum(0)
    ours = dict(x=dx, wn=dwn, wg=gu.dw, wu=gu.dw_up, wd=gd.dw, bd=gd.db, sw=dsw)
    for name, got, want in [("y", y, Y)] + [(n, ours[n], G[n]) for n in ours]:
        off = float((got.double() - want).norm() / want.norm())
        assert off <= 2 * (8 / 3) ** 0.5 * U(T), (name, off)
    mb.expert_linear_status()


IN_PLACE = [(1, 2, 3, 40, 64), (1, 3, 40, 72, 136), (1, 1, 30, 1088, 264), (1, 1, 60, 2048, 136), (1, 1, 100, 1024, 264), (1, 4, 200, 200, 136), (2, 3, 700, 136, 200), (1, 3, 300, 51, 77)]


@pytest.mark.parametrize("T", [BF16, F32])
@pytest.mark.parametrize("shape", IN_PLACE, ids=str)
@pytest.mark.parametrize("gated", [False, True])
def test_results_in_place_of_inputs(T, shape, gated):
    """out over add, dx over add and over the kept values, dw over what it is added to: the bits of results of their own, whatever shares the work."""
    L, E, R, n, k = shape
    g, two = gen(R + k), 1 + gated
    off = offsets_of(some_counts(L, E, R, g, full=False))
    x, dout = normal(g, L, R, k, dtype=T), normal(g, L, R, two * n, dtype=T)
    w = [normal(g, L, E, n, k, dtype=T, std=k ** -0.5) for _ in range(two)] + [None] * (2 - two)
    there = inside(off, R)

    def same(got, want, before):
        assert torch.equal(got[there], want[there]) and torch.equal(got[~there], before[~there])
    add = normal(g, L, R, n, dtype=T)
    want, got = mb.expert_linear(x, off, w[0], w_up=w[1], act="gelu", add=add).out, add.clone()
    mb.expert_linear(x, off, w[0], w_up=w[1], act="gelu", add=got, out=mb.LinearOut(got))
    same(got, want, add)
    add = normal(g, L, R, k, dtype=T)
    want, got = mb.expert_linear_backward(dout, off, w[0], w_up=w[1], add=add).dx, add.clone()
    mb.expert_linear_backward(dout, off, w[0], w_up=w[1], add=got, out=mb.LinearGrad(got))
    same(got, want, add)
    for below in (1, 2):
        z = normal(g, L, R, below * k, dtype=T)
        want, got = mb.expert_linear_backward(dout, off, w[0], w_up=w[1], saved=z, act="silu"), z.clone()
        r = mb.expert_linear_backward(dout, off, w[0], w_up=w[1], saved=got, act="silu", out=mb.LinearGrad(got, torch.empty_like(x)))
        same(got, want.dx, z)
        assert torch.equal(r.h[there], want.h[there])
    before = mb.WeightGrad(*[None if i >= two else normal(g, L, E, n, k, dtype=T) for i in range(2)], *[None if i >= two else normal(g, L, E, n, dtype=T) for i in range(2)])
    want = mb.expert_linear_dweight(dout, x, off, gated=gated, want_db=True, add=before)
    mb.expert_linear_dweight(dout, x, off, gated=gated, add=before, out=before)
    assert all(a is None or torch.equal(a, b) for a, b in zip(before, want))
    mb.expert_linear_status()


@pytest.mark.parametrize("T", [BF16, F32])
@pytest.mark.parametrize("E,R", [(4096, 3000), (4096, 30000), (700, 5), (1000, 40000), (577, 100000)])
def test_many_groups(T, E, R):
    """More groups than threads in any kernel's block, up to the limit; a third of them empty.  Small integers: every sum is exact."""
    g, n, k = gen(E + R), 16, 24
    c = torch.rand(E, device="cuda", generator=g) * (torch.rand(E, device="cuda", generator=g) > 0.33)
    c = (c / c.sum() * R).long()
    first = torch.randint(3, 90, (1,), generator=torch.Generator().manual_seed(E)).item() if R > 100 else 0        # rows in front of the first group are nobody's either
    c[E // 2] += (R - first - int(c.sum())) // 2
    off = torch.cat([torch.full((1,), first, device="cuda"), first + c.cumsum(0)]).to(torch.int32)
    end = int(off[-1])
    assert 0 <= first <= end <= R
    whole = lambda *s: torch.randint(-3, 4, s, device="cuda", generator=g).to(T)
    x, dout, w, wu = whole(R, k), whole(R, 2 * n), whole(E, n, k), whole(E, n, k)
    for t in (x, dout):
        t[:first], t[end:] = float("nan"), float("inf")
    owner = torch.bucketize(torch.arange(first, end, device="cuda"), off[1:].long(), right=True)
    xs, ds = x[first:end].double(), dout[first:end].double()
    out = torch.full((R, n), 7.0, device="cuda", dtype=F32)
    mb.expert_linear(x, off, w, out=mb.LinearOut(out))
    assert torch.equal(out[first:end].double(), torch.einsum("rk,rnk->rn", xs, w[owner].double())) and (out[:first] == 7).all() and (out[end:] == 7).all()
    dx = torch.full((R, k), 7.0, device="cuda", dtype=T)
    mb.expert_linear_backward(dout, off, w, w_up=wu, out=mb.LinearGrad(dx))
    want = torch.einsum("rn,rnk->rk", ds[:, :n], w[owner].double()) + torch.einsum("rn,rnk->rk", ds[:, n:], wu[owner].double())
    assert torch.equal(dx[first:end].double(), want.to(T).double()) and (dx[:first] == 7).all() and (dx[end:] == 7).all()
    r = mb.expert_linear_dweight(dout, x, off, gated=True, want_db=True, out_dtype=F32)
    for i in range(2):
        d = ds[:, i * n:(i + 1) * n]
        dw = torch.zeros(E, n, k, dtype=torch.float64, device="cuda").index_add_(0, owner, torch.einsum("rn,rk->rnk", d, xs))
        assert torch.equal(r[i].double(), dw) and torch.equal(r[2 + i].double(), torch.zeros(E, n, dtype=torch.float64, device="cuda").index_add_(0, owner, d))
    mb.expert_linear_status()
