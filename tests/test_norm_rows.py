"""How the norm's rows are dealt out to blocks (no GPU needed): each row once, however they lie and however few blocks fit on the device."""
import ctypes
import os
import subprocess

import pytest

import paper_2511_12500_b200 as iris

CSRC = os.path.join(os.path.dirname(iris.__file__), "csrc")
SOURCE = """
#include "norm_rows.h"
#include <vector>
using namespace iris::rows;
// Rows that no group has, or more than one.
extern "C" int missed(int64_t rows, int64_t room, int groups, int at_once, int period) {
  const int64_t blocks = norm_grid(groups, at_once, rows, room);
  std::vector<int> seen(rows, 0);
  for (int64_t block = 0; block < blocks; ++block)
    for (int index = 0; index < groups; ++index) {
      const NormWalk w = norm_walk(block, blocks, index, groups, period, norm_set(block, period), at_once);
      for (int64_t r = w.first; r < rows; r += w.step)
        for (int q = 0; q < at_once; ++q)
          if (r + q * w.each < rows) ++seen[r + q * w.each];
    }
  int bad = 0;
  for (int n : seen) bad += n != 1;
  return bad;
}
extern "C" int64_t grid(int groups, int at_once, int64_t rows, int64_t room) { return norm_grid(groups, at_once, rows, room); }
"""


@pytest.fixture(scope="module")
def dealt(tmp_path_factory):
    at = tmp_path_factory.mktemp("norm_rows")
    (at / "dealt.cpp").write_text(SOURCE)
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-Wall", "-Werror", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(at / "dealt.cpp"), "-o", str(at / "dealt.so")])
    lib = ctypes.CDLL(str(at / "dealt.so"))
    i64, i32 = ctypes.c_int64, ctypes.c_int
    lib.missed.argtypes = [i64, i64, i32, i32, i32]
    lib.grid.argtypes, lib.grid.restype = [i32, i32, i64, i64], i64
    return lib


@pytest.mark.parametrize("period", [1, 2, 4, 8])
@pytest.mark.parametrize("room", [1, 2, 3, 5, 7, 8, 15, 33, 148])
def test_each_row_once(dealt, room, period):
    for groups in (1, 2, 3, 4, 12):
        for at_once in (1, 2, 4):
            for rows in [*range(1, 70), 127, 1000, 5003]:
                assert dealt.missed(rows, room, groups, at_once, period) == 0, (rows, groups, at_once)


def test_no_more_blocks_than_fit_but_for_the_places_where_rows_begin(dealt):
    assert dealt.grid(4, 1, 100000, 15) == 15 and dealt.grid(4, 2, 100000, 148) == 148 and dealt.grid(1, 1, 20, 148) == 20
    assert [dealt.grid(2, 1, 1000, room) for room in (1, 7, 8, 9)] == [8, 8, 8, 9]
    assert dealt.grid(4, 2, 5, 148) == 5 and dealt.grid(12, 4, 1, 148) == 1
