"""What the sources of the experts' products (csrc/linear*.cu, linear.cuh) have to keep to where no run can show it."""
import os
import re

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
