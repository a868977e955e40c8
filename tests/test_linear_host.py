"""Host side of the experts' products: what the self-test of their bounded waits refuses, and which products get a workspace for copies."""
import ctypes as C

from paper_2412_00099_b200 import binding as mb
from paper_2412_00099_b200 import build as mbuild


def test_limits():
    mbuild.build()
    lib = mb.load()
    for limit in (0, 1_000_000_001, 1 << 63):
        assert lib.mcce_selftest_expert_linear_timeout(limit, None) == -1


def test_copies_by_the_tiles_of_the_product():
    """A weight gradient's tiles are those of its weights, not of its rows: one expert's 65 x 65 from 4096 unaligned bf16 rows are 6 tiles of 32 x 64, so that eight CTAs
    share each and copying the rows first gains nothing (29.6 us without, 28.7 with); 511 x 515 are 144 and gain (121 against 38)."""
    lib = mb.load()

    def need(n, k):
        p = mb.Linear(n_layers=1, n_experts=1, rows=4096, n=n, k=k, dtype=mb.BF16, out_dtype=mb.BF16, bias_dtype=mb.F32, saved_dtype=mb.BF16)
        parts = 8 * n * 4 + 255 & ~255                   # of the bias's gradient: eight chunks of 512 rows
        return lib.mcce_expert_linear_dweight_workspace_bytes(C.byref(p), C.c_void_p(1 << 24), C.c_void_p(1 << 28)) - parts
    assert need(65, 65) == 0
    assert need(511, 515) == 4096 * (512 + 520) * 2
