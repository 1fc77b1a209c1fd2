"""The launch rule of attention over the row cache, compiled for the host."""
import ctypes as C
import os
import subprocess

import pytest

CODE = r"""
#include "attend_shape.h"
// ranks asked about go to *asked; clusters of up to `holds` blocks fit
extern "C" int shape(long long roots, int per_root, long long tiles, int sms, int holds, int* ranks, int* take, int* asked) {
  *asked = 0;
  const auto s = tgnn_history::choose_attend_shape(roots, per_root, tiles, sms, [&](int r) { *asked = r; return r <= holds; });
  *ranks = s.ranks;
  *take = s.take;
  return s.by_block;
}
"""


@pytest.fixture(scope="module")
def shape(tmp_path_factory):
    from paper_2608_16305_b200 import build
    d = tmp_path_factory.mktemp("shape")
    src, lib = os.path.join(d, "s.cpp"), os.path.join(d, "s.so")
    with open(src, "w") as f:
        f.write(CODE)
    subprocess.check_call([os.environ.get("CXX", "g++"), "-std=c++17", "-shared", "-fPIC", "-O1", "-Wall", "-Werror", "-I", build.CSRC, "-o", lib, src])
    fn = C.CDLL(lib).shape
    fn.argtypes = [C.c_longlong, C.c_int, C.c_longlong, C.c_int, C.c_int] + [C.POINTER(C.c_int)] * 3

    def call(roots, per_root, tiles, sms=148, holds=16):
        out = [C.c_int() for _ in range(3)]
        by_block = fn(roots, per_root, tiles, sms, holds, *map(C.byref, out))
        return (bool(by_block), out[0].value, out[1].value, out[2].value)
    return call


def test_clusters_of_sixteen_only_where_they_fit(shape):
    """Three roots over long windows: 16 blocks each where the device holds such a cluster, else the 8 that every device holds."""
    assert shape(3, 1, 2000) == (True, 16, 1, 16)
    assert shape(3, 1, 2000, holds=8) == (True, 8, 1, 16)
    assert shape(3, 1, 2000, holds=0) == (True, 8, 1, 16)
    assert shape(20, 1, 2000) == (True, 16, 1, 16)                 # 20 roots of 64 warps: 1280 of 1776
    for roots, tiles in ((3, 64), (30, 2000), (100, 2000)):        # smaller clusters are not asked about
        by_block, ranks, take, asked = shape(roots, 1, tiles)
        assert by_block and 1 <= ranks <= 8 and asked == 0


def test_work_is_shared_out_once(shape):
    """Every shape covers its units: blocks only where tiles are many, several units per warp only within a root."""
    for sms in (16, 132, 148):
        for roots in (1, 3, 100, 600, 1775, 1776, 3552, 10 ** 6):
            for per_root in (1, 2, 8):
                for tiles in (0, 1, 2, 3, 17, 200, 2 ** 26):
                    by_block, ranks, take, _ = shape(roots, per_root, tiles, sms)
                    assert ranks in (1, 2, 4, 8, 16) and take in (1, per_root)
                    assert (ranks == 1 or by_block) and (take == 1 or not by_block) and (take == 1 or tiles <= 1) and (not by_block or tiles > 2)
                    assert ranks == 1 or 4 * ranks <= tiles


def test_short_windows_of_many_units_go_by_warp(shape):
    """1700 roots of two heads over three tiles have a warp each (a block each took 22.7 us, a warp each 16.5); over long windows a block each up to
    twice as many units."""
    assert shape(1700, 2, 3)[0] is False and shape(1776, 1, 16)[0] is False
    assert shape(880, 2, 3)[0] is True and shape(1775, 1, 16)[0] is True
    assert shape(1776, 1, 17)[0] is True and shape(3551, 1, 125)[0] is True and shape(3552, 1, 125)[0] is False
