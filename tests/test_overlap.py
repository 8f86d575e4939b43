"""Whether operands share memory (csrc/overlap.h), compiled for the host, against a
count of bytes (CPU only)."""
import ctypes
import itertools
import os
import subprocess

import numpy as np
import pytest

from paper_2609_34867_amd import build

PROGRAM = r'''
#include "overlap.h"
using namespace p4q;
static Rows at(long long p, long long rows, long long stride, long long width) {
    return rows_at(reinterpret_cast<void *>(p), rows, stride, width);
}
extern "C" int shared(long long p, long long pr, long long ps, long long pw, long long q, long long qr, long long qs, long long qw) {
    return share_memory(at(p, pr, ps, pw), at(q, qr, qs, qw));
}
'''


@pytest.fixture(scope="module")
def shared(tmp_path_factory):
    d = tmp_path_factory.mktemp("overlap")
    (d / "o.cpp").write_text(PROGRAM)
    lib = d / "o.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{build.CSRC}",
                    str(d / "o.cpp"), "-o", str(lib)], check=True)
    fn = ctypes.CDLL(os.fspath(lib)).shared
    fn.argtypes = [ctypes.c_longlong] * 8
    return lambda a, b: bool(fn(*a, *b))


def bytes_of(at, rows, stride, width):
    return {at + i * stride + j for i in range(rows) for j in range(width)}


# (rows, stride, width)
FORMS = [(1, 3, 3), (1, 40, 5), (2, 6, 4), (3, 6, 2), (4, 4, 4), (3, 6, 6), (5, 6, 1)]


def test_against_a_count_of_bytes(shared):
    """Exact where at most one operand has gaps or both have the same stride."""
    for f, g in itertools.product(FORMS, FORMS):
        for q in range(1, 90):
            a, b = (40, *f), (q, *g)
            want = bool(bytes_of(*a) & bytes_of(*b))
            assert shared(a, b) == want and shared(b, a) == want, (a, b)


def test_different_strides(shared):
    """Both with gaps: never said of operands that do not, always of those that begin together."""
    rng = np.random.default_rng(0)
    for _ in range(5000):
        a, b = ((int(p), int(r), int(w + g), int(w)) for p, r, w, g in zip(rng.integers(1, 60, 2), rng.integers(1, 6, 2),
                                                                           rng.integers(1, 9, 2), rng.integers(0, 9, 2)))
        if shared(a, b):
            assert bytes_of(*a) & bytes_of(*b)
        assert shared(a, (a[0], *b[1:]))


def test_none_and_far(shared):
    assert not shared((0, 4, 8, 8), (1, 4, 8, 8))
    # 2^20 rows, 2^23 apart
    big = (1 << 40, 1 << 20, 1 << 23, 1 << 22)
    last = (1 << 40) + ((1 << 20) - 1) * (1 << 23)
    assert shared(big, (last, 1, 16, 16)) and not shared(big, (last + (1 << 22), 1, 16, 16))
    assert shared(big, (last - 15, 1, 16, 16)) and not shared(big, (last - 16, 1, 16, 16))
