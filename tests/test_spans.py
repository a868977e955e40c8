"""Which tensors share a byte (csrc/span.h), for stacks of matrices: several blocks of rows."""
import ctypes as C
import random
import subprocess

from paper_2412_00099_b200 import build as mbuild


def test_stacks_of_matrices(tmp_path):
    """Against sets of bytes: two halves of one buffer with padded rows, blocks between one another, rows of single tensors among them."""
    src = tmp_path / "stack.cpp"
    src.write_text('#include "span.h"\nusing namespace mcce;\n'
                   'static Span of(const long long* v) { return stack_span((void*)v[0], v[1], v[2], v[3], v[4], v[5], 1); }\n'
                   'extern "C" int apart2(const long long* a, const long long* b) { return disjoint(of(a), of(b)); }\n'
                   'extern "C" int same(const long long* a, const long long* b) { return same_or_apart(of(a), of(b)); }\n')
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-shared", "-fPIC", "-I", mbuild.CSRC, str(src), "-o", str(tmp_path / "stack.so")], check=True)
    so = C.CDLL(str(tmp_path / "stack.so"))

    def arg(v):
        return (C.c_longlong * 6)(*v)

    def touched(p, count, far, rows, step, width):
        return {p + c * far + i * step + j for c in range(count) for i in range(rows) for j in range(width)}
    rng, seen = random.Random(5), [0, 0]
    for _ in range(20000):
        v = []
        for _ in range(2):
            rows, width = rng.randint(1, 4), rng.randint(1, 6)
            step = width + rng.randint(0, 8)
            v.append([rng.randint(100, 200), rng.randint(1, 5), (rows - 1) * step + width + rng.randint(0, 30), rows, step, width])
        if rng.random() < 0.4:                              # the other half of the same buffer, or columns beside
            v[1][1:5] = v[0][1:5]
            v[1][5] = min(v[1][5], v[1][4])
            v[1][2] = v[0][2] = max(v[0][2], (v[1][3] - 1) * v[1][4] + v[1][5])
        a, b = v
        want = not (touched(*a) & touched(*b))
        seen[want] += 1
        assert bool(so.apart2(arg(a), arg(b))) == bool(so.apart2(arg(b), arg(a))) == want, (a, b)
        assert so.same(arg(a), arg(a))
        if not want:
            assert bool(so.same(arg(a), arg(b))) == (a[0] == b[0] and a[3:] == b[3:] and a[1] == b[1] and (a[1] == 1 or a[2] == b[2])) or a[3] == 1
    assert min(seen) > 4000
    halves = [(4096, 64, 2 * 40 * 80, 40, 80, 64), (4096 + 40 * 80, 64, 2 * 40 * 80, 40, 80, 64)]
    assert so.apart2(arg(halves[0]), arg(halves[1])) and not so.apart2(arg(halves[0]), arg((4096 + 39 * 80 + 63,) + halves[1][1:]))
    big = (4096, 4096, 1 << 50, 1 << 20, 1 << 41, 64)       # sizes that would overflow 64 bits
    assert so.apart2(arg(big), arg((8192, 3, 1 << 50, 5, 1 << 41, 64))) in (0, 1)
