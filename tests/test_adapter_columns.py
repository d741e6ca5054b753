"""The columns of the adapters' outer products, walked on the host over the kernel's own index rule; needs no GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def walk(tmp_path, program):
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(program)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2207_01260_amd", "csrc"), str(src), "-o", str(exe)])
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout


# Sides up to three work-groups wide; V numbers at once where the row holds as many, otherwise those that it holds.
READS = r"""
#include "adapter_columns.hpp"
#include <cstdio>
#include <initializer_list>
using namespace cprune;
int main() {
  long outside = 0;
  for (int v : {4, 8}) for (int c = 1; c <= 3 * 16 * v; ++c)
    for (int group = 0; group <= (c - 1) / (16 * v); ++group) for (int lane = 0; lane < 16; ++lane) {
      const OuterLane at = outer_lane(c, v, group, lane);
      const int count = at.there >= v ? v : at.there > 0 ? at.there : 0;
      if (count && (at.column < 0 || at.column + count > c)) ++outside;
      if (c >= v && count != v) ++outside;
    }
  std::printf("%ld lanes read outside of their row\n", outside);
  return outside != 0;
}
"""


def test_every_lane_reads_within_its_row(tmp_path):
    walk(tmp_path, READS)
    # the kernel's count is the rule's
    text = open(os.path.join(ROOT, "paper_2207_01260_amd", "csrc", "adapter_kernel.hpp")).read()
    assert "load_some(from, mine.there)" in text and "outer_lane(side.c, V, group, t & 15)" in text


# Column `column + i` of a lane's sums is the row's number there: every column is stored, and a column that two lanes store is the same number for both, which is so
# where both have V numbers from their column on, or one of them has it in a place that is there.
COLUMNS = r"""
#include "adapter_columns.hpp"
#include <cstdio>
#include <initializer_list>
#include <vector>
using namespace cprune;
int main() {
  long wrong = 0;
  for (int v : {4, 8}) for (int c = 1; c <= 3 * 16 * v; ++c) {
    std::vector<int> stored(c, 0);
    for (int group = 0; group <= (c - 1) / (16 * v); ++group) for (int lane = 0; lane < 16; ++lane) {
      const OuterLane at = outer_lane(c, v, group, lane);
      std::vector<int> held(v, -1);                             // what the products multiply: the row's columns, zeros past them
      for (int i = 0; i < v && i < at.there; ++i) held[i] = at.column + i;
      for (int i = 0; i < v; ++i) {
        if ((group * 16 + lane) * v >= c || at.column + i >= c) continue;
        ++stored[at.column + i];
        if (held[i] != at.column + i) ++wrong;
      }
    }
    for (int n : stored) if (!n) ++wrong;
  }
  std::printf("%ld columns not stored, or with another's sums\n", wrong);
  return wrong != 0;
}
"""


def test_every_column_is_stored_with_its_own_sums(tmp_path):
    walk(tmp_path, COLUMNS)
    csrc = os.path.join(ROOT, "paper_2207_01260_amd", "csrc")
    # the products and the join have one rule
    assert "outer_lane(side.c, V, group, t & 15)" in open(os.path.join(csrc, "adapter_kernel.hpp")).read()
    assert "outer_lane(c, p.v, (int)group, of).column" in open(os.path.join(csrc, "adapter.hip")).read()
