"""Which rows, positions and pages of a cache a call reaches (csrc/kv_range.h), walked on the host up to the ends of 32 bits: what a GPU
test cannot see, as a read outside a buffer mostly finds memory."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1705_09864_amd", "csrc")
SOURCE = """
#define __host__
#define __device__
#include "kv_range.h"
extern "C" void span_of(int begin, int end, int tokens, int rows, int max_new, int width, int* out) {
  const bmx::KvSpan s = bmx::kv_span_of(begin, end, tokens, rows, max_new, width);
  out[0] = s.row0, out[1] = s.count, out[2] = s.first, out[3] = s.length;
}
extern "C" int page_at(int low, int high, int at, int* out) { return bmx::kv_page_at(low, high, at, out, out + 1, out + 2); }
extern "C" int pages_to(int end) { return bmx::kv_pages_to(end); }
extern "C" int all_in(int t0, int n, int low, int high) { return bmx::kv_all_in(t0, n, low, high); }
extern "C" int64_t pages_of(int max_new) { return bmx::kv_pages_of(max_new); }
"""
TOP = 2**31 - 1


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("kv_range")
    src, so = str(d / "range.cpp"), str(d / "range.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-ftrapv", "-shared", "-fPIC", "-I", CSRC, src, "-o", so])
    L = ctypes.CDLL(so)
    L.pages_of.restype = ctypes.c_int64
    return L


NUMBERS = [-TOP - 1, -TOP, -100, -1, 0, 1, 5, 63, 64, 65, 128, 1000, TOP - 129, TOP - 65, TOP - 64, TOP - 63, TOP - 62, TOP - 1, TOP]


def test_spans(lib):
    """Rows inside [0, rows), no more than max_new of them, positions inside the table, whatever the numbers in device memory are."""
    out = (ctypes.c_int * 4)()
    for begin in NUMBERS:
        for end in NUMBERS:
            for tokens in NUMBERS:
                for rows, most, width in ((1, 1, 1), (240, 80, 2), (TOP, TOP, 1 << 25), (TOP, 7, TOP), (70, 70, 0)):
                    lib.span_of(begin, end, tokens, rows, most, width, out)
                    row0, count, first, length = out
                    assert 0 <= row0 <= row0 + count <= rows and 0 <= count <= most
                    assert first == max(tokens, 0) - count and length == min(max(tokens, 0), 64 * width)


def test_pages_of_positions(lib):
    """Every page that positions [low, high) lie in, its tokens, and none besides, at the ends of 32 bits as elsewhere."""
    out = (ctypes.c_int * 3)()
    for low in NUMBERS[1:] + list(range(-70, 70, 3)):
        for high in sorted({*NUMBERS[4:], *(min(low + n, TOP) for n in (1, 2, 3, 63, 64, 65, 66, 127, 200))}):
            count = high - low
            if count > TOP:  # (more than a call's rows can be)
                continue
            span = lib.pages_of(max(count, 0))
            places = range(min(span + 1, 6)) if span <= 6 else [0, 1, 2, span - 3, span - 2, span - 1]
            got = 0
            for at in places:
                if lib.page_at(low, high, at, out):
                    page, t0, t1 = out
                    assert page == low // 64 + at and 0 <= t0 < t1 <= 64
                    assert (page * 64 + t0, page * 64 + t1) == (max(low, page * 64), min(high, page * 64 + 64))
                    got += t1 - t0
                else:
                    assert (low // 64 + at) * 64 >= high or count <= 0
            if count <= 0:
                assert got == 0
            elif span <= 6:
                assert got == count  # (the launch's pages are enough)
            else:
                assert (low // 64 + span) * 64 >= high


def test_pages_of_a_launch(lib):
    for n in (0, 1, 2, 3, 63, 64, 65, 66, 67, TOP - 63, TOP - 62, TOP - 61, TOP):
        most = max((low + n - 1) // 64 - low // 64 + 1 for low in (0, 1, 31, 62, 63)) if n else 0
        assert most <= lib.pages_of(n) <= n // 64 + 2


def test_pages_and_places_that_a_row_sees(lib):
    for end in NUMBERS:
        assert lib.pages_to(end) == max(0, -(-end // 64))
    for t0 in [0, 64, 128, (TOP >> 6 << 6) - 64, TOP >> 6 << 6]:
        for low in NUMBERS[3:]:
            for high in NUMBERS:
                assert bool(lib.all_in(t0, 64, low, high)) == (t0 >= low and t0 + 64 <= high)
