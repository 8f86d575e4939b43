"""Which kernel takes an MXFP4 product (csrc/mx4_choice.h), compiled for the host: the sizes
that the GPU tests run reach the kernels that they are meant for (CPU only)."""
import ctypes
import os
import subprocess

import pytest

import mx4_sizes as sizes
from paper_2609_34867_amd import build

PROGRAM = r'''
#include "mx4_choice.h"
using namespace p4q;
extern "C" int pick(int form, int M, int N, int K, int cus) { return mx4_kernel(static_cast<Epilogue>(form), M, N, K, cus); }
extern "C" int waves(long long groups, int cus) { return mx4_rows_waves(groups, cus); }
'''
NAMES = ["rows 16", "rows 32", "64x64", "64x64 parts", "64x128", "64x128 parts", "128x128", "128x192", "192x192", "192x256",
         "256x256"]
LISTS = [(0, sizes.LINEAR, sizes.SLOTS), (1, sizes.GATED, sizes.GATED_SLOTS), (2, sizes.QUANTIZED, sizes.GATED_SLOTS)]


@pytest.fixture(scope="module")
def choice(tmp_path_factory):
    d = tmp_path_factory.mktemp("choice")
    (d / "c.cpp").write_text(PROGRAM)
    lib = d / "c.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{build.CSRC}",
                    str(d / "c.cpp"), "-o", str(lib)], check=True)
    so = ctypes.CDLL(os.fspath(lib))
    so.waves.argtypes = [ctypes.c_longlong, ctypes.c_int]
    so.kernel = lambda form, M, N, K, cus=256: NAMES[so.pick(form, M, N, K, cus)]
    return so


@pytest.mark.parametrize("form,kernel,M,N,K", [(f, *c) for f, cases, _ in LISTS for c in cases])
def test_sizes_reach_their_kernel(choice, form, kernel, M, N, K):
    assert choice.kernel(form, M, N, K) == kernel
    rows, outputs = sizes.tile(kernel, form > 0)
    assert M > rows and (M % rows or N % outputs)


@pytest.mark.parametrize("form,cases,slots", LISTS)
def test_every_kernel_every_way(form, cases, slots):
    for kernel, room in slots.items():
        mine = [c[1:] for c in cases if c[0] == kernel]
        outputs = sizes.tile(kernel, form > 0)[1]
        assert any(N % 32 == 0 and N > outputs for _, N, _ in mine), f"{kernel}: whole tiles of rows at half lines"
        if form < 2:
            assert any(N % 32 for _, N, _ in mine), f"{kernel}: other rows"
        assert {-(-K // 256) % 2 for _, _, K in mine} == {0, 1}, f"{kernel}: stages"
        if kernel in ("128x128", "192x192", "192x256", "256x256"):
            assert any(sizes.tiles(kernel, form > 0, M, N) > room for M, N, _ in mine), f"{kernel}: a second tile"
    assert {c[0] for c in cases} == set(slots)


# the calls of a decoder: rows, outputs, k; linear, gated
@pytest.mark.parametrize("form,M,N,K,kernel", [
    (0, 1, 4096, 11008, "rows 16"), (0, 16, 12288, 4096, "rows 16"), (0, 384, 12288, 4096, "128x192"),
    (0, 704, 12288, 4096, "192x192"), (0, 704, 5120, 13824, "128x128"), (0, 11264, 4096, 11008, "256x256"),
    (1, 16, 11008, 4096, "rows 16"), (2, 704, 13824, 5120, "192x256"), (1, 11264, 11008, 4096, "256x256")])
def test_a_decoders_calls(choice, form, M, N, K, kernel):
    assert choice.kernel(form, M, N, K) == kernel


def test_limits(choice):
    """A kernel of the form's for every size up to the limits, whatever the number of CUs."""
    ends = (1, 16, 17, 1024, 1025, 1 << 20)
    for cus in (1, 256, 304):
        for M in ends:
            for N in (1, 32, 4096, 1 << 22):
                for K in (32, 288, 131072):
                    for form, slots in ((0, sizes.SLOTS), (1, sizes.GATED_SLOTS), (2, sizes.GATED_SLOTS)):
                        name = choice.kernel(form, M, N, K, cus)
                        assert name == "rows 16" if M <= 16 else name in slots or (name == "rows 32" and M <= 1024)
                        # one work-group a tile: the grid holds them
                        if "parts" in name:
                            assert sizes.tiles(name, False, M, N) * 512 < 2 ** 32


@pytest.mark.parametrize("groups,n", [(1, 4), (511, 4), (512, 2), (1 << 24, 2)])
def test_wavefronts_of_few_rows(choice, groups, n):
    assert choice.waves(groups, 256) == n
