"""The experts' products where several CTAs, maps or kernels could serve a call: what the rules choose for odd offsets, every way of sharing a reduction, strided
results.  Tolerances as in test_gpu_linear: u = 2^-24, U(T) half a step of T relative to the value; a sum of k products is within (k + 8) u of its terms'
magnitudes S."""
import pytest
import torch

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
