"""What the sources of the experts' products (csrc/linear*.cu, linear.cuh) have to keep to where no run can show it."""
import ctypes as C
import os
import re
import subprocess

from paper_2412_00099_b200 import build as mbuild


def code(name):
    """A source without its comments."""
    with open(os.path.join(mbuild.CSRC, name)) as f:
        text = f.read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


def sources():
    return [n for n in sorted(os.listdir(mbuild.CSRC)) if n.startswith("linear") and n.endswith((".cu", ".cuh"))]


def test_nothing_is_read_as_constant():
    """These kernels may take their place while the kernel that writes their inputs is still running, and wait for it then.  A load that promises
    that its memory does not change while the kernel lives (__ldg, .nc, const __restrict__) may be moved in front of that wait."""
    assert {"linear.cu", "linear.cuh", "linear_few.cu", "linear_tc.cu"} <= set(sources())
    for name in sources():
        assert not re.search(r"__ldg|\.nc\b|__restrict__", code(name)), name


def test_waits_that_last_as_long_as_a_reduction(tmp_path):
    """The sums of a tile, a group's last slab and the other CTAs' sums are waited for while whole reductions pass: up to 2^31 - 1 rows, 2^24 slabs of
    128 at 0.8 us each, are 13 s.  Their limits have to grow with the slabs; the plain 2 s would call a healthy launch dead."""
    src = tmp_path / "limit.cpp"
    src.write_text('#include "wait_limit.h"\nextern "C" unsigned long long limit(long long slabs) { return mcce::tc::reduction_limit_ns(slabs); }\n')
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", mbuild.CSRC, str(src), "-o", str(tmp_path / "limit.so")], check=True)
    limit = C.CDLL(str(tmp_path / "limit.so")).limit
    limit.argtypes, limit.restype = [C.c_longlong], C.c_ulonglong
    for slabs in (0, 1, 8, 1 << 20, 1 << 24, 4096 << 24):          # the last: of all groups together
        assert limit(slabs) >= 2_000_000_000 + 10 * 800 * slabs
    text = code("linear_tc.cu")
    for bar, what in (("bar_tfull", "to - from"), ("bar_tail", "since"), ("bar_parts", "to - from")):
        waits = re.findall(r"wait\w*\(%s[^;]*;" % bar, text)
        assert waits and all("reduction_limit_ns(%s)" % what in w for w in waits), bar
