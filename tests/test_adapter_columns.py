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


# Sides up to three work-groups wide, beside one that is thin and beside one that is not; V numbers at once where the row holds as many, otherwise those that it holds.
READS = r"""
#include "adapter_columns.hpp"
#include <cstdio>
#include <initializer_list>
using namespace cprune;
int main() {
  long outside = 0;
  for (int v : {4, 8}) for (int c = 1; c <= 3 * 16 * v; ++c) for (int thin = c < v; thin <= 1; ++thin)
    for (int group = 0; group <= (c - 1) / (16 * v); ++group) for (int lane = 0; lane < 16; ++lane) {
      const OuterLane at = outer_lane(c, v, group, lane, thin != 0);
      const int count = at.there >= v ? v : at.there > 0 ? at.there : 0;
      if (count && (at.column < 0 || at.column + count > c)) ++outside;
      if (!thin && count != v) ++outside;
    }
  std::printf("%ld lanes read outside of their row\n", outside);
  return outside != 0;
}
"""


def test_every_lane_reads_within_its_row(tmp_path):
    walk(tmp_path, READS)
    # the kernel's count is the rule's
    text = open(os.path.join(ROOT, "paper_2207_01260_amd", "csrc", "adapter_kernel.hpp")).read()
    assert "load_some(from, mine.there)" in text and "outer_lane(side.c, V, group, t & 15, THIN)" in text
