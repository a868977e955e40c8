"""The experts' products on sorted rows (expert_linear, its gradients) and their 8-bit checkpoints against plain implementations in
64 bits.

Tolerances.  u = 2^-24 is half an fp32 step, U(T) half a step of the output type relative to the value (bf16 2^-8, fp32 2^-24).  A sum of k
products formed in fp32 is off by at most k u times the sum S of the terms' magnitudes when every addition is rounded; the tensor
cores truncate (2 u) once per 16 products (k u / 8) and once more where the 16 are brought to one exponent: (k + 8) u S covers both.  Adding a
bias or another tensor rounds once more.  The activations' slopes are below 1.13; the exponential, division and distribution function have
errors of a few u, the fast exponential |z| 2^-22 more: ACT_U = 128 u relative to the value for |z| <= 30."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2412_00099_b200 import binding as mb

u = 2.0 ** -24
ACT_U = 128 * u
F32, BF16, E4M3, E8M0 = torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu


def U(t):
    return torch.finfo(t).eps / 2


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, dtype=F32, std=1.0):
    return (torch.randn(*shape, device="cuda", generator=g) * std).to(dtype)


def within(got, want, tol, what=""):
    """|got - want| <= tol elementwise (NaN fails)."""
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), "%s: %d of %d off, worst %g over its tolerance" % (
        what, int(bad.sum()), bad.numel(), float(((got.double() - want).abs() / tol.clamp_min(1e-300))[bad].max()))


def offsets_of(counts):
    """[L,E+1] from rows per group [L][E]."""
    c = torch.tensor(counts, dtype=torch.int64)
    return torch.cat([torch.zeros_like(c[:, :1]), c.cumsum(1)], 1).to(torch.int32).cuda()


def ndtr(z):
    """The normal distribution; erfc keeps its relative precision where 1 + erf is 0 (below -8.3 in 64 bits)."""
    return 0.5 * torch.special.erfc(-z * math.sqrt(0.5))


def act(z, name):
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return z * ndtr(z)
    return z


def slope(z, name):
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    if name == "gelu":
        return ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def groups(off, R):
    """(group, layer, expert, first row among all, end) of every group."""
    o = off.cpu().tolist()
    for l, row in enumerate(o):
        for e in range(len(row) - 1):
            yield l * (len(row) - 1) + e, l, e, l * R + row[e], l * R + row[e + 1]


def sums(rows, w, off):
    """rows [L,R,k] times w[g]^T [n,k], in 64 bits, and the sums of the terms' magnitudes; rows of no group are 0."""
    L, R, k = rows.shape
    flat, wf = rows.double().flatten(0, 1), w.flatten(0, 1)
    z = torch.zeros(L * R, w.shape[-2], dtype=torch.float64, device="cuda")
    S = torch.zeros_like(z)
    for g, _, _, a, b in groups(off, R):
        z[a:b] = flat[a:b] @ wf[g].double().T
        S[a:b] = flat[a:b].abs() @ wf[g].double().abs().T
    return z.view(L, R, -1), S.view(L, R, -1)


def per_row(v, off, R):
    """v [L,E,n] for every row [L,R,n]."""
    out = torch.zeros(v.shape[0] * R, v.shape[-1], dtype=torch.float64, device="cuda")
    for g, _, _, a, b in groups(off, R):
        out[a:b] = v.flatten(0, 1)[g].double()
    return out.view(v.shape[0], R, -1)


def inside(off, R):
    m = torch.zeros(off.shape[0], R, dtype=torch.bool, device="cuda")
    for l, row in enumerate(off.cpu().tolist()):
        m[l, :row[-1]] = True
    return m


def blocks(v, pad=0.0):
    n = -(-v.shape[-1] // 32)
    return torch.nn.functional.pad(v, (0, n * 32 - v.shape[-1]), value=pad).unflatten(-1, (n, 32))


def block_scales(v):
    """The smallest power of two, 2^-127 at least, with the block's largest magnitude at most 448 times it; 64 bits."""
    m, e = torch.frexp(blocks(v).abs().amax(-1) / 448.0)
    e = torch.where(m == 0.5, e - 1, e)
    return torch.where(m == 0, torch.full_like(m, 2.0 ** -127), torch.ldexp(torch.ones_like(m), e.clamp_min(-127)))


def e4m3(v):
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), (e - 4).clamp_min(-9))
    return torch.round(v / step) * step


def wide(scales, cols):
    return scales.double().repeat_interleave(32, -1)[..., :cols]


def check_packed(q, scales, z, dz, what):
    """q, scales hold z, known to within dz."""
    lo, hi = block_scales((z.abs() - dz).clamp_min(0)), block_scales(z.abs() + dz)
    s = scales.double()
    assert ((s >= lo) & (s <= hi)).all(), what + ": scales"
    s = wide(scales, z.shape[-1])
    q = q.double()
    assert ((q >= e4m3((z - dz) / s)) & (q <= e4m3((z + dz) / s))).all(), what + ": values"


def some_counts(L, E, R, g, full=True):
    """Rows per group: uneven, some of them empty, all R rows or fewer."""
    out = []
    for _ in range(L):
        share = torch.rand(E, generator=g, device="cuda") * (torch.rand(E, generator=g, device="cuda") > 0.25)
        used = R if full else R * 2 // 3
        c = (share / share.sum().clamp_min(1e-6) * used).long()
        c[int(torch.randint(E, (1,), generator=g, device="cuda"))] += used - int(c.sum())
        out.append(c.clamp_min(0).tolist())
    return out


# (L, E, R, n, k): the tensor path needs strides that are multiples of 8 and starts of 16 bytes; the others take any
SHAPES = [(1, 1, 1, 1, 1), (1, 1, 1, 8, 8), (1, 4, 4, 64, 64), (1, 3, 40, 64, 128), (2, 5, 37, 72, 200), (1, 7, 300, 136, 264),
          (1, 2, 700, 320, 64), (1, 60, 64, 128, 256), (3, 4, 130, 40, 96), (1, 1, 517, 515, 259), (1, 6, 77, 33, 31),
          (1, 4, 1100, 192, 512), (1, 300, 500, 16, 24), (1, 1, 257, 1000, 1002), (1, 1, 16, 264, 4096), (1, 2, 40, 136, 2048), (1, 1, 60, 192, 1024),
          (1, 1, 3, 100, 2056), (2, 3, 5, 72, 520), (1, 2, 600, 520, 192), (1, 1, 30, 4096, 264), (1, 3, 65, 2048, 136), (1, 4, 1500, 515, 1003), (2, 2, 900, 777, 1026), (1, 3, 2100, 1001, 520)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("T,O", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("gated", [False, True])
def test_linear(shape, T, O, gated):
    L, E, R, n, k = shape
    g = gen(R * 7 + n)
    off = offsets_of(some_counts(L, E, R, g, full=R % 2 == 0))
    x = normal(g, L, R, k, dtype=T)
    w, wu = normal(g, L, E, n, k, dtype=T, std=k ** -0.5), normal(g, L, E, n, k, dtype=T, std=k ** -0.5) if gated else None
    z0, S = sums(x, w, off)
    zu0, Su = sums(x, wu, off) if gated else (None, None)
    there = inside(off, R)
    for name, bias, add, save in [(None, False, False, None), ("silu", True, False, "same"), ("gelu", False, True, "e4m3"), ("silu", True, True, "e4m3")]:
        b = normal(g, L, E, n, dtype=F32 if add else T) if bias else None
        bu = normal(g, L, E, n, dtype=F32 if add else T) if bias and gated else None
        a = normal(g, L, R, n, dtype=O) if add else None
        halves = 2 if gated else 1
        out = mb.LinearOut(torch.full((L, R, n), 7.0, device="cuda", dtype=O),
                           None if save is None else torch.full((L, R, halves * n), 3.0, device="cuda").to(T if save == "same" else E4M3),
                           torch.full((L, R, halves * -(-n // 32)), 2.0, device="cuda").to(E8M0) if save == "e4m3" else None)
        r = mb.expert_linear(x, off, w, w_up=wu, bias=b, bias_up=bu, act=name, add=a, out=out)
        z, dz = z0, (k + 8) * u * S
        if bias:
            z = z + per_row(b, off, R)
            dz = dz + z.abs() * 2 * u
        y, dy = act(z, name), 1.13 * dz
        dy = dy + y.abs() * ACT_U
        if gated:
            up, dup = zu0, (k + 8) * u * Su
            if bias:
                up = up + per_row(bu, off, R)
                dup = dup + up.abs() * 2 * u
            dy = y.abs() * dup + (up.abs() + dup) * dy
            y = y * up
        if add:
            y = y + a.double()
        dy = (dy + y.abs() * 4 * u) * (1 + U(O)) + y.abs() * U(O)
        within(r.out[there], y[there], dy[there], "out")
        assert (r.out[~there] == 7).all()
        if save == "same":
            want, tol = (torch.cat([z, up], -1), torch.cat([dz, dup], -1)) if gated else (z, dz)
            within(r.saved[there], want[there], (tol * (1 + U(T)) + want.abs() * U(T))[there], "saved")
            assert (r.saved[~there] == 3).all()
        if save == "e4m3":
            nb = -(-n // 32)
            check_packed(r.saved[there][:, :n], r.scales[there][:, :nb], z[there], dz[there], "saved")
            if gated:
                check_packed(r.saved[there][:, n:], r.scales[there][:, nb:], up[there], dup[there], "saved, second half")
            assert (r.saved[~there].float() == 3).all() and (r.scales[~there].float() == 2).all()
        again = mb.expert_linear(x, off, w, w_up=wu, bias=b, bias_up=bu, act=name, add=a, save=save, out_dtype=O)
        for p, q in zip(r, again):
            assert (p is None and q is None) or torch.equal(p[there].view(torch.uint8), q[there].view(torch.uint8))
    mb.expert_linear_status()


def unpacked(q, scales, halves):
    cols, nb = q.shape[-1] // halves, scales.shape[-1] // halves
    return torch.cat([q[..., i * cols:(i + 1) * cols].double() * wide(scales[..., i * nb:(i + 1) * nb], cols) for i in range(halves)], -1)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("T", [BF16, F32])
@pytest.mark.parametrize("gated", [False, True])
def test_linear_backward(shape, T, gated):
    L, E, R, n, k = shape
    g = gen(R * 5 + n)
    off = offsets_of(some_counts(L, E, R, g, full=R % 2 == 1))
    two = 2 if gated else 1
    dout = normal(g, L, R, two * n, dtype=T)
    w, wu = normal(g, L, E, n, k, dtype=T, std=n ** -0.5), normal(g, L, E, n, k, dtype=T, std=n ** -0.5) if gated else None
    t, S = sums(dout[..., :n], w.transpose(-1, -2), off)
    if gated:
        tu, Su = sums(dout[..., n:], wu.transpose(-1, -2), off)
        t, S = t + tu, S + Su
    dt = (two * n + 8) * u * S
    there = inside(off, R)
    for below, name, kind, add in [(0, None, None, False), (0, None, None, True), (1, "gelu", "same", False), (2, "silu", "same", False),
                                   (1, "silu", "e4m3", False), (2, "gelu", "e4m3", False), (2, None, "same", False)]:
        a = normal(g, L, R, k, dtype=T) if add else None
        saved = scales = None
        if below:
            z = normal(g, L, R, below * k, std=2.0)
            saved = z.to(T)
            if kind == "e4m3":
                parts = [mb.checkpoint_pack(z[..., i * k:(i + 1) * k].contiguous()) for i in range(below)]
                saved = torch.cat([p.q.view(torch.uint8) for p in parts], -1).view(E4M3)
                scales = torch.cat([p.scales.view(torch.uint8) for p in parts], -1).view(E8M0)
            z = saved.double() if scales is None else unpacked(saved, scales, below)
        out = mb.LinearGrad(torch.full((L, R, max(below, 1) * k), 7.0, device="cuda", dtype=T),
                            torch.full((L, R, k), 5.0, device="cuda", dtype=T) if below else None)
        r = mb.expert_linear_backward(dout, off, w, w_up=wu, saved=saved, scales=scales, act=name, add=a, out=out)
        if below == 0:
            want = t if a is None else t + a.double()
            tol = dt + want.abs() * 2 * u
        else:
            y, sl = act(z[..., :k], name), slope(z[..., :k], name)
            dsl = (sl.abs() + z[..., :k].abs() + 1) * ACT_U
            if below == 2:
                up = z[..., k:]
                want = torch.cat([t * up * sl, t * y], -1)
                tol = torch.cat([up.abs() * (dt * sl.abs() + t.abs() * dsl), dt * y.abs() + t.abs() * y.abs() * ACT_U], -1) + want.abs() * 4 * u
                h = y * up
            else:
                want, h = t * sl, y
                tol = dt * sl.abs() + t.abs() * dsl + want.abs() * 4 * u
            within(r.h[there], h[there], (h.abs() * (ACT_U + U(T)))[there] * (1 + U(T)), "h")
            assert (r.h[~there] == 5).all()
        within(r.dx[there], want[there], (tol * (1 + U(T)) + want.abs() * U(T))[there], "dx")
        assert (r.dx[~there] == 7).all()
        again = mb.expert_linear_backward(dout, off, w, w_up=wu, saved=saved, scales=scales, act=name, add=a)
        assert torch.equal(again.dx[there], r.dx[there])
    mb.expert_linear_status()


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("T,O", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("gated", [False, True])
def test_linear_dweight(shape, T, O, gated):
    L, E, R, n, k = shape
    g = gen(R * 3 + n)
    off = offsets_of(some_counts(L, E, R, g, full=R % 2 == 0))
    two = 2 if gated else 1
    dout, there = normal(g, L, R, two * n, dtype=T), inside(off, R)
    dout[~there] = float("nan")                     # rows of nobody hold anything
    for eight, add in [(False, False), (True, True), (False, True), (True, False)]:
        x, scales = normal(g, L, R, k, dtype=T), None
        xd = x.double()
        if eight:
            x, scales = mb.checkpoint_pack(x)
            xd = unpacked(x, scales, 1)
        else:
            x[~there] = float("inf")
        before = None
        if add:
            before = [normal(g, L, E, n, k, dtype=O) for _ in range(two)] + [None] * (2 - two)
            before = mb.WeightGrad(*before, *([normal(g, L, E, n, dtype=O) for _ in range(two)] + [None] * (2 - two)))
        r = mb.expert_linear_dweight(dout, x, off, scales=scales, gated=gated, want_db=True, add=before, out_dtype=O)
        for i in range(two):
            d = dout[..., i * n:(i + 1) * n].double().flatten(0, 1)
            for gi, l, e, a, b in groups(off, R):
                m = b - a
                xs = xd.flatten(0, 1)[a:b]
                dw, S = d[a:b].T @ xs, d[a:b].abs().T @ xs.abs()
                db, Sb = d[a:b].sum(0), d[a:b].abs().sum(0)
                if add:
                    dw, db = dw + before[i][l, e].double(), db + before[2 + i][l, e].double()
                within(r[i][l, e], dw, ((m + 8) * u * S + dw.abs() * 2 * u) * (1 + U(O)) + dw.abs() * U(O), "dw %d" % i)
                within(r[2 + i][l, e], db, ((m + 8) * u * Sb + db.abs() * 2 * u) * (1 + U(O)) + db.abs() * U(O), "db %d" % i)
        again = mb.expert_linear_dweight(dout, x, off, scales=scales, gated=gated, want_db=True, add=before, out_dtype=O)
        for p, q in zip(r, again):
            assert (p is None and q is None) or torch.equal(p, q)
    mb.expert_linear_status()


@pytest.mark.parametrize("T", [BF16, F32])
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 31), (5, 32), (7, 33), (64, 4096), (33, 1411), (257, 96), (1000, 40), (2, 8200), (0, 64)])
def test_checkpoint(rows, d, T):
    g = gen(rows + d)
    x = normal(g, rows, d, dtype=T) * torch.exp(3 * normal(g, rows, 1)).to(T)
    if rows > 2:
        x[0] = 0
        x[1, : d // 2] = 448 * 2.0 ** -9             # a largest value at the border of its scale
        x[2, d // 2] = 1e-38
    c = mb.checkpoint_pack(x)
    check_packed(c.q, c.scales, x.double(), torch.zeros_like(x.double()), "pack")
    for O in (BF16, F32):
        back = mb.checkpoint_unpack(c.q, c.scales, dtype=O)
        within(back, unpacked(c.q, c.scales, 1), torch.full(x.shape, 2.0 ** -134, dtype=torch.float64, device="cuda"), "unpack")
        within(back, x.double(), x.double().abs() * 2.0 ** -4 + wide(c.scales, d) * 2.0 ** -10, "round trip")


def test_checkpoint_special_blocks():
    x = torch.ones(4, 96, device="cuda")
    x[0, 5], x[1, 40], x[2, 90], x[3, 0] = float("nan"), float("inf"), float("-inf"), 3e38
    for T in (F32, BF16):
        c = mb.checkpoint_pack(x.to(T))
        back = mb.checkpoint_unpack(c.q, c.scales, dtype=F32)
        bad = torch.zeros(4, 96, dtype=torch.bool, device="cuda")
        bad[0, :32] = bad[1, 32:64] = bad[2, 64:] = True
        assert back[bad].isnan().all() and back[~bad].isfinite().all()
        assert (back[0, 32:] == 1).all() and abs(float(back[3, 0]) / 3e38 - 1) <= 2.0 ** -4


# ---- strides, places, streams, graphs --------------------------------------------------------------------------
def padded(t, right, left=0, fill=9.0):
    """The same values as columns of a wider buffer, and the buffer."""
    full = torch.full(t.shape[:-1] + (left + t.shape[-1] + right,), fill, device="cuda").to(t.dtype)
    view = full[..., left:left + t.shape[-1]]
    view.copy_(t)
    return view, full


@pytest.mark.parametrize("T", [BF16, F32])
@pytest.mark.parametrize("left,right", [(8, 24), (0, 8), (1, 2), (4, 4)])
def test_strides(T, left, right):
    """Every tensor another stride and start (aligned to what the copies want, or not): the results of contiguous ones, nothing beside them touched."""
    g, R, n, k, E = gen(7), 210, 72, 136, 3
    off = offsets_of([[100, 0, 90]])[0]
    x, w, wu, add = normal(g, R, k, dtype=T), normal(g, E, n, k, dtype=T, std=0.1), normal(g, E, n, k, dtype=T, std=0.1), normal(g, R, n, dtype=T)
    want = mb.expert_linear(x, off, w, w_up=wu, act="silu", add=add, save="same")
    xs, ws, wus, adds = padded(x, right, left)[0], padded(w, right, left)[0], padded(wu, right, left)[0], padded(add, right + 1, left)[0]
    out, full = padded(torch.zeros(R, n, device="cuda", dtype=T), right + 8, left)
    saved, full_saved = padded(torch.zeros(R, 2 * n, device="cuda", dtype=T), right + 16, left)
    r = mb.expert_linear(xs, off, ws, w_up=wus, act="silu", add=adds, out=mb.LinearOut(out, saved))
    tol = (k + 16) * u * 10 * (1 if T == F32 else 0) + (2 * U(T) if T == BF16 else 0)      # other kernels, other orders of summation
    close = lambda a, b: (a.double() - b.double()).abs().max() <= tol * b.double().abs().max()
    assert close(r.out[:190], want.out[:190]) and close(r.saved[:190], want.saved[:190])
    assert (full[:, :left] == 9).all() and (full[:, left + n:] == 9).all() and (full_saved[:, left + 2 * n:] == 9).all() and (out[190:] == 0).all()
    # gradients: both matrices in one buffer, dx over the kept values, dw into columns of a wider buffer, added in place
    both = torch.cat([w, wu], 1)
    dout = normal(g, R, 2 * n, dtype=T)
    z = normal(g, R, 2 * k, dtype=T)
    ref = mb.expert_linear_backward(dout, off, w, w_up=wu, saved=z, act="gelu")
    zs = padded(z, right, left)[0]
    got = mb.expert_linear_backward(padded(dout, right, left)[0], off, both[:, :n], w_up=both[:, n:], saved=zs, act="gelu",
                                    out=mb.LinearGrad(zs, torch.empty(R, k, device="cuda", dtype=T)))
    assert close(got.dx[:190], ref.dx[:190]) and close(got.h[:190], ref.h[:190]) and torch.equal(zs[190:], z[190:])
    dw = [padded(torch.ones(E, n, k, device="cuda", dtype=T), right, left) for _ in range(2)]
    ref = mb.expert_linear_dweight(dout, x, off, gated=True)
    into = mb.WeightGrad(dw[0][0], dw[1][0])
    got = mb.expert_linear_dweight(padded(dout, right, left)[0], xs, off, gated=True, add=into, out=into)
    for a, b, (_, whole) in zip(got[:2], ref[:2], dw):
        assert close(a, b + 1) and (whole[..., :left] == 9).all() and (whole[..., left + k:] == 9).all()


def test_rows_far_apart():
    """Offsets beyond 2^32 elements: rows, weights and results with strides of 2^27 and more."""
    g, R, n, k = gen(3), 36, 64, 64
    big = torch.empty(R * (1 << 27) + 4096, device="cuda", dtype=BF16)
    for T in (BF16, F32):
        buf = big if T == BF16 else big.view(F32)
        step = (1 << 27) if T == BF16 else (1 << 26)
        x, w, dout = normal(g, R, k, dtype=T), normal(g, 1, n, k, dtype=T), normal(g, R, n, dtype=T)
        off = offsets_of([[R]])[0]
        place = lambda at, cols: torch.as_strided(buf, (R, cols), (step, 1), at)
        xs, outs = place(0, k), place(1024, n)
        xs.copy_(x)
        want = mb.expert_linear(x, off, w).out
        r = mb.expert_linear(xs, off, w, out=mb.LinearOut(outs))
        assert torch.equal(r.out, want)
        xs.copy_(x)
        assert torch.equal(mb.expert_linear_dweight(dout, xs, off).dw, mb.expert_linear_dweight(dout, x, off).dw)
        c = mb.checkpoint_pack(x)
        assert torch.equal(mb.checkpoint_unpack(c.q, c.scales, out=outs), mb.checkpoint_unpack(c.q, c.scales, dtype=T))
    ws = torch.as_strided(big, (R, 16, 64), (1 << 27, 64, 1))
    ws.copy_(normal(g, R, 16, 64, dtype=BF16))
    off = offsets_of([[1] * R])[0]
    x = normal(g, R, 64, dtype=BF16)
    assert torch.equal(mb.expert_linear(x, off, ws).out, mb.expert_linear(x, off, ws.contiguous()).out)


@pytest.mark.parametrize("T", [BF16, F32])
@pytest.mark.parametrize("R,E", [(7, 3), (300, 4), (900, 2)])
def test_offsets_that_are_no_offsets(T, R, E):
    """What reaches outside [0, R] is cut off, a group that ends before it begins is empty: nothing outside the rows is touched."""
    g, n, k = gen(5), 72, 64
    buf = torch.full((R + 200, n), 7.0, device="cuda", dtype=T)
    x, w = normal(g, R, k, dtype=T), normal(g, E, n, k, dtype=T)
    for o in ([-5] + [R // 2] * (E - 1) + [R + 100000], [2 ** 31 - 1] * (E + 1), [-2 ** 31] * E + [3], [R] + [0] * E):
        off = torch.tensor(o, dtype=torch.int32, device="cuda")
        mb.expert_linear(x, off, w, out=mb.LinearOut(buf[100:100 + R]))
        mb.expert_linear_backward(buf[100:100 + R], off, w)
        mb.expert_linear_dweight(buf[100:100 + R], x, off, want_db=True)
        assert (buf[:100] == 7).all() and (buf[100 + R:] == 7).all()
    mb.expert_linear_status()


@pytest.mark.parametrize("T", [BF16, F32])
def test_one_experts_nan_stays_its_own(T):
    g, n, k, counts = gen(6), 136, 72, [37, 100, 0, 64, 300]
    off, E, R = offsets_of([counts])[0], 5, 501
    x, w, dout = normal(g, R, k, dtype=T), normal(g, E, n, k, dtype=T), normal(g, R, n, dtype=T)
    x[40], dout[41], w[1, 3] = float("nan"), float("inf"), float("-inf")
    bad = torch.zeros(R, dtype=torch.bool, device="cuda")
    bad[37:137] = True
    out = mb.expert_linear(x, off, w, act="silu").out
    assert out[~bad].isfinite().all() and not out[40].isfinite().any()
    dx = mb.expert_linear_backward(dout, off, w).dx
    assert dx[~bad].isfinite().all()
    r = mb.expert_linear_dweight(dout, x, off, want_db=True)
    others = [0, 2, 3, 4]
    assert r.dw[others].isfinite().all() and r.db[others].isfinite().all() and not r.dw[1].isfinite().all() and not r.db[1].isfinite().all()
    assert (r.dw[2] == 0).all() and (r.db[2] == 0).all()


@pytest.mark.parametrize("n,k", [(192, 136), (72, 320), (256, 256)])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("T", [BF16, F32])
def test_dweight_of_every_number_of_rows(T, gated, n, k):
    """Groups of 0 to 140 rows, every third full of NaN.  Small integers: the sums (below 9 * 140) are exact in fp32."""
    g = gen(n + k)
    counts = torch.randperm(141, generator=torch.Generator().manual_seed(k)).tolist()
    two, R, off = 1 + gated, sum(counts), offsets_of([counts])[0]
    dout = torch.randint(-3, 4, (R, two * n), device="cuda", generator=g).to(T)
    x = torch.randint(-3, 4, (R, k), device="cuda", generator=g).to(T)
    want = [torch.stack([dout[a:b, i * n:(i + 1) * n].double().T @ x[a:b].double() for a, b in zip(off.tolist(), off.tolist()[1:])]) for i in range(two)]
    bad = [e for e in range(141) if e % 3 == 1 and counts[e]]
    for e in bad:
        dout[off[e]:off[e + 1]], x[off[e]:off[e + 1]] = float("nan"), float("inf")
    ours = [e for e in range(141) if e not in bad]
    for O in ([F32, BF16] if T == BF16 else [F32]):
        r = mb.expert_linear_dweight(dout, x, off, gated=gated, out_dtype=O)
        for i in range(two):
            assert torch.equal(r[i][ours].double(), want[i][ours].to(O).double())
            assert r[i][bad].isnan().all()
    mb.expert_linear_status()


@pytest.mark.parametrize("T", [BF16, F32])
def test_nothing(T):
    """No rows at all, and rows that belong to nobody: nothing is read or written but the weights' gradients, 0 or what is added."""
    g, E, n, k = gen(2), 3, 40, 64
    w = normal(g, E, n, k, dtype=T)
    for R in (0, 50):
        off = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
        x, dout = normal(g, R, k, dtype=T), normal(g, R, n, dtype=T)
        out = torch.full((R, n), 7.0, device="cuda", dtype=T)
        assert (mb.expert_linear(x, off, w, out=mb.LinearOut(out)).out == 7).all()
        dx = torch.full((R, k), 7.0, device="cuda", dtype=T)
        assert (mb.expert_linear_backward(dout, off, w, out=mb.LinearGrad(dx)).dx == 7).all()
        before = mb.WeightGrad(normal(g, E, n, k, dtype=T), None, normal(g, E, n, dtype=T))
        for eight in (False, True):
            rows = mb.checkpoint_pack(x) if eight else (x, None)
            r = mb.expert_linear_dweight(dout, rows[0], off, scales=rows[1], want_db=True)
            assert (r.dw == 0).all() and (r.db == 0).all()
            r = mb.expert_linear_dweight(dout, rows[0], off, scales=rows[1], want_db=True, add=before)
            assert torch.equal(r.dw, before.dw) and torch.equal(r.db, before.db)


def test_streams_and_graphs():
    """On a stream of the caller's, captured and replayed on new values: the same bits as in order."""
    g = gen(9)
    L, E, R, n, k = 1, 6, 600, 192, 256
    off = offsets_of(some_counts(L, E, R, g))
    x, w, wu = normal(g, L, R, k, dtype=BF16), normal(g, L, E, n, k, dtype=BF16, std=0.1), normal(g, L, E, n, k, dtype=BF16, std=0.1)
    wd, dy = normal(g, L, E, k, n, dtype=BF16, std=0.1), normal(g, L, R, k, dtype=BF16)
    few = normal(g, 2, k, dtype=BF16)
    off_few = offsets_of([[1, 0, 0, 1, 0, 0]])[0]

    def step():
        a = mb.expert_linear(x, off, w, w_up=wu, act="silu", save="e4m3")
        y = mb.expert_linear(a.out, off, wd, add=x).out
        d = mb.expert_linear_backward(dy, off, wd, saved=a.saved, scales=a.scales, act="silu")
        dx = mb.expert_linear_backward(d.dx, off, w, w_up=wu, add=dy).dx
        c = mb.checkpoint_pack(x)
        dw = mb.expert_linear_dweight(d.dx, c.q, off, scales=c.scales, gated=True, want_db=True)
        dwd = mb.expert_linear_dweight(dy, d.h, off)
        return [a.out, y, d.dx, d.h, dx, *dw, dwd.dw, mb.expert_linear(few, off_few, w[0]).out]
    side = torch.cuda.Stream()
    want = step()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(2):
            got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        held = step()
    for seed in (1, 2):
        x.copy_(normal(gen(seed), L, R, k, dtype=BF16))
        off.copy_(offsets_of(some_counts(L, E, R, gen(seed))))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, step()))
    mb.expert_linear_status()


def test_two_calls_at_once():
    """Two streams with calls that wait inside for their own copies: each one's own results."""
    g = gen(10)
    off = offsets_of([[700, 300, 500, 548]])[0]
    data = [(normal(g, 2048, 512, dtype=BF16), normal(g, 4, 768, 512, dtype=BF16, std=0.05)) for _ in range(2)]
    want = [mb.expert_linear(x, off, w, act="gelu").out for x, w in data]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(mb.expert_linear(data[i][0], off, data[i][1], act="gelu").out)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in range(2) for o in got[i])
    mb.expert_linear_status()


# ---- a layer, forwards and backwards -----------------------------------------------------------------------------
@pytest.mark.parametrize("T", [F32, BF16])
@pytest.mark.parametrize("tokens,d,f", [(37, 64, 96), (150, 72, 40)])
def test_layer_and_its_gradients(T, tokens, d, f):
    """Norm, sort, gated experts, down projection with bias, weighted return onto the residual stream, and back to the gradients of everything; against the
    formulas in 64 bits (their gradients by autograd, and by differences).  Every value on the way is a sum of at most 2 f products or of d terms: 8 stages
    of (2 f + 8) u each, tenfold for cancellation, relative to the largest gradient of a tensor; in bf16 8 stages of a rounding each, tenfold too."""
    E, K = 5, 2
    g = gen(tokens)
    x, wn = normal(g, tokens, d, dtype=T), 1 + 0.1 * normal(g, d)
    wg, wu, wd = (normal(g, E, *s, dtype=T, std=s[1] ** -0.5) for s in ((f, d), (f, d), (d, f)))
    bd = normal(g, E, d, std=0.1).to(T)
    sel = torch.stack([torch.randperm(E, generator=g, device="cuda")[:K] for _ in range(tokens)]).to(torch.int32)
    sel[3, 1] = -1                                        # a dropped pair
    sw = torch.softmax(normal(g, tokens, K), -1)
    dy = normal(g, tokens, d, dtype=T)

    def ours():
        h = mb.rmsnorm(x, wn, 1e-6).out
        s = mb.dispatch(sel, E, h)
        a = mb.expert_linear(s.rows, s.offsets, wg, w_up=wu, act="silu", save="same")
        o = mb.expert_linear(a.out, s.offsets, wd, bias=bd).out
        y = mb.combine(o, s.inv, sw, add=x)
        do, dsw = mb.combine_backward(dy, o, s.inv, sw)
        da = mb.expert_linear_backward(do, s.offsets, wd, saved=a.saved, act="silu")
        gd = mb.expert_linear_dweight(do, da.h, s.offsets, want_db=True)
        drows = mb.expert_linear_backward(da.dx, s.offsets, wg, w_up=wu).dx
        gu = mb.expert_linear_dweight(da.dx, s.rows, s.offsets, gated=True)
        dh = mb.combine(drows, s.inv)
        dx, dwn = mb.rmsnorm_backward(dh, x, wn, 1e-6, dsum=dy)
        return y, dict(x=dx, wn=dwn, wg=gu.dw, wu=gu.dw_up, wd=gd.dw, bd=gd.db, sw=dsw)
    y, grads = ours()
    leaves = {k: v.double().requires_grad_() for k, v in dict(x=x, wn=wn, wg=wg, wu=wu, wd=wd, bd=bd, sw=sw).items()}

    def formula(v):
        h = v["x"] / (v["x"].square().mean(-1, keepdim=True) + 1e-6).sqrt() * v["wn"]
        out = v["x"]
        for k in range(K):
            e, on = sel[:, k].long().clamp_min(0), (sel[:, k] >= 0).double()
            gate, up = torch.einsum("td,tfd->tf", h, v["wg"][e]), torch.einsum("td,tfd->tf", h, v["wu"][e])
            r = torch.einsum("tf,tdf->td", act(gate, "silu") * up, v["wd"][e]) + v["bd"][e]
            out = out + (v["sw"][:, k] * on)[:, None] * r
        return out
    want = formula(leaves)
    loss = (want * dy.double()).sum()
    loss.backward()
    tol = 8 * 10 * ((2 * f + 8) * u + (U(T) if T == BF16 else 0))
    assert (y.double() - want).abs().max() <= tol * want.abs().max()
    for k, v in grads.items():
        ref = leaves[k].grad
        assert (v.double() - ref).abs().max() <= tol * ref.abs().max(), k
        # a difference of the formula along a random direction
        step = normal(gen(1), *ref.shape).double()
        eps = 1e-5
        moved = [dict({n: t.detach() for n, t in leaves.items()}, **{k: leaves[k].detach() + s * eps * step}) for s in (1, -1)]
        diff = sum(s * (formula(m) * dy.double()).sum() for s, m in zip((1, -1), moved)) / (2 * eps)
        assert abs(float(diff - (v.double() * step).sum())) <= tol * float((ref.abs() * step.abs()).sum()) + 1e-6 * float(diff.abs())
    again_y, again = ours()
    assert torch.equal(again_y, y) and all(torch.equal(again[k], grads[k]) for k in grads)
