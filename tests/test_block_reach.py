"""Which elements the groups of eight of dropout and of the norm touch, by the arithmetic that their kernels use
(csrc/soma_eights.hpp), compiled for the host: every element of every row once, and nothing read at once that is not
aligned or lies outside the array."""
import os
import shutil
import subprocess

import pytest

from conftest import ROOT

PROGRAM = r"""
#include <cstdio>
#include <vector>

#include "soma_eights.hpp"

using namespace soma;

static long wrong = 0;

static void fail(const char* what, int64_t size, int64_t rows, int64_t width, int64_t stride, int64_t row) {
  if (wrong++ < 20) std::printf("%s: element of %ld bytes, [%ld][%ld], rows %ld apart, row %ld\n", what, size, rows, width, stride, row);
}

template <class Of>
static void array(int64_t size, int64_t rows, int64_t width, int64_t stride, int64_t groups, Of of) {
  const bool vec = in_eights(true, stride, width, size);
  const int64_t end = (rows - 1) * stride + width;
  std::vector<int> seen(end);
  for (int64_t row = 0; row < rows; ++row)
    for (int64_t i = 0; i < groups; ++i) {
      const auto g = of(row, i);
      if (g.hi <= g.lo) continue;
      const int64_t at = row * stride + g.col;
      for (int k = g.lo; k < g.hi; ++k) {
        if (g.col + k < 0 || g.col + k >= width) fail("not of its row", size, rows, width, stride, row);
        else ++seen[at + k];
      }
      if (!reads_whole(vec, row + 1 == rows, g.lo, g.hi)) continue;
      if (at < 0 || at + 8 > end) fail("outside", size, rows, width, stride, row);
      if (at * size % 16) fail("not aligned", size, rows, width, stride, row);
    }
  for (int64_t row = 0; row < rows; ++row)
    for (int64_t c = 0; c < width; ++c)
      if (seen[row * stride + c] != 1) fail("not once", size, rows, width, stride, row);
}

template <int kLanes>
static void norm(int64_t size, int64_t rows, int64_t width, int64_t stride, int groups) {
  const auto walk = [&](auto ragged) {
    array(size, rows, width, stride, kLanes * groups, [&](int64_t row, int64_t i) {
      return Group<kLanes, ragged()>(static_cast<int>(row), static_cast<int>(width), static_cast<int>(i % kLanes), static_cast<int>(i / kLanes));
    });
  };
  struct Yes { constexpr bool operator()() const { return true; } };
  struct No { constexpr bool operator()() const { return false; } };
  if (width % 8) walk(Yes{});
  else walk(No{});
}

int main() {
  for (int64_t size : {2, 4})
    for (int64_t width = 1; width <= 40; ++width)
      for (int64_t rows = 1; rows <= 20; ++rows)
        for (int64_t stride = width; stride <= width + 17; ++stride) {
          array(size, rows, width, stride, groups_of(width), [&](int64_t row, int64_t i) { return Eight(row, width, i); });
          norm<64>(size, rows, width, stride, 1);
        }
  for (int64_t size : {2, 4})
    for (int64_t width : {505, 511, 513, 1015, 1017, 4097})
      for (int64_t rows = 1; rows <= 9; ++rows)
        for (int64_t stride : {width, width + 4, width + 8}) norm<64>(size, rows, width, stride, static_cast<int>(groups_of(width) + 63) / 64);
  std::printf("%ld wrong\n", wrong);
  return wrong != 0;
}
"""


def test_groups_of_eight_stay_inside_their_arrays(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ is not installed")
    source, program = tmp_path / "reach.cpp", tmp_path / "reach"
    source.write_text(PROGRAM)
    subprocess.check_call([cxx, "-std=c++20", "-O1", "-Wall", "-I", os.path.join(ROOT, "paper_2609_37899_amd", "csrc"), "-o",
                           str(program), str(source)])
    out = subprocess.run([str(program)], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, out.stdout
