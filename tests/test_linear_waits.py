"""What the self-test of the experts' products' bounded waits refuses (on the host, before any launch)."""
from paper_2412_00099_b200 import binding as mb
from paper_2412_00099_b200 import build as mbuild


def test_limits():
    mbuild.build()
    lib = mb.load()
    for limit in (0, 1_000_000_001, 1 << 63):
        assert lib.mcce_selftest_expert_linear_timeout(limit, None) == -1
