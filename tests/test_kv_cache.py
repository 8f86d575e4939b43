"""The paged cache's address arithmetic (csrc/kv_cache.h), compiled for the host:
no table entry, length or list of packed rows, however wrong, gives an address
outside the cache or the rows (CPU only)."""
import ctypes
import os
import subprocess

import pytest

from paper_2609_34867_amd import build

PROGRAM = r'''
#include "kv_cache.h"
using namespace p4q;
extern "C" {
int shift_of(int page_size) { return page_shift(page_size); }
int page_of(int entry, int num_pages) { return valid_page(entry, num_pages); }
int column(long long key, int shift, int max_pages) { return page_column(key, shift, max_pages); }
int by(int n, int G) { const Magic g = magic_of(G); return magic_div(n, g.m, g.shift); }
int fetched(int key, int keys, int shift) { return fetch_column(key, keys, shift); }
long long row(int page, int Hk, int h, int shift, int slot, int D) { return page_row(page, Hk, h, shift, slot, D); }
int count(int len) { return key_count(len); }
int first(int b, int e, int n) { return packed_span(b, e, n).first; }
int last(int b, int e, int n) { return packed_span(b, e, n).last; }
}
'''
LOW, HIGH = -2 ** 31, 2 ** 31 - 1


@pytest.fixture(scope="module")
def kv(tmp_path_factory):
    d = tmp_path_factory.mktemp("kv")
    (d / "kv.cpp").write_text(PROGRAM)
    lib = d / "kv.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{build.CSRC}",
                    str(d / "kv.cpp"), "-o", str(lib)], check=True)
    so = ctypes.CDLL(os.fspath(lib))
    so.column.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    so.row.restype = ctypes.c_longlong
    return so


def test_page_sizes(kv):
    good = {1 << s: s for s in range(4, 13)}
    for n in list(range(-3, 5000)) + [8192, HIGH, LOW]:
        assert kv.shift_of(n) == good.get(n, -1)


@pytest.mark.parametrize("entry,page", [(0, 0), (6, 6), (7, -1), (-1, -1), (LOW, -1), (HIGH, -1)])
def test_table_entries(kv, entry, page):
    assert kv.page_of(entry, 7) == page


@pytest.mark.parametrize("key,col", [(0, 0), (31, 0), (32, 1), (95, 2), (96, -1), (-1, -1), (LOW, -1), (HIGH, -1),
                                     (2 ** 40, -1), (-2 ** 40, -1)])
def test_columns(kv, key, col):
    assert kv.column(key, 5, 3) == col


@pytest.mark.parametrize("keys", [1, 15, 16, 17, 63, 64, 65, 2 ** 30 - 1])
@pytest.mark.parametrize("shift", [4, 6, 12])
def test_entries_past_the_keys_are_not_fetched(kv, keys, shift):
    last = (keys - 1) >> shift
    for key in [*range(0, 200), keys - 1, keys, keys + 127, 2 ** 30 + 128]:
        assert kv.fetched(key, keys, shift) == (key >> shift if key < keys else last)


def test_nothing_is_fetched_without_keys(kv):
    assert [kv.fetched(key, 0, 4) for key in (0, 1, 64, 128, HIGH)] == [-1] * 5


def test_rows_pass_32_bits(kv):
    assert kv.row(0, 3, 2, 4, 5, 64) == (2 * 16 + 5) * 64
    assert kv.row(HIGH // 16, 1024, 1023, 12, 4095, 128) == (((HIGH // 16) * 1024 + 1023) * 4096 + 4095) * 128
    # rows of one page and head are contiguous, pages do not overlap
    seen = {kv.row(p, 3, h, 4, s, 64) for p in range(4) for h in range(3) for s in range(16)}
    assert seen == set(range(0, 4 * 3 * 16 * 64, 64))


def test_lengths_and_spans(kv):
    assert [kv.count(n) for n in (LOW, -1, 0, 1, HIGH)] == [0, 0, 0, 1, HIGH]
    ends = [LOW, -5, -1, 0, 1, 9, 10, 11, HIGH]
    for b in ends:
        for e in ends:
            f, l = kv.first(b, e, 10), kv.last(b, e, 10)
            assert 0 <= f <= l <= 10
            if 0 <= b <= e <= 10:
                assert (f, l) == (b, e)
            if e <= b:
                assert f == l


def test_division_by_multiplication(kv):
    """n / G for every group size, around multiples of G over the whole range of n."""
    for G in range(1, 1025):
        most = HIGH // G
        for m in {0, 1, 2, 127, 128, 1 << 20, most // 3, most - 1, most}:
            for n in {m * G - 1, m * G, m * G + 1, m * G + G - 1}:
                if 0 <= n <= HIGH:
                    assert kv.by(n, G) == n // G, (n, G)
        for n in (1 << 24, (1 << 24) - 1, 1 << 30, HIGH - 1, HIGH):
            assert kv.by(n, G) == n // G, (n, G)
