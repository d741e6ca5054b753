"""Arrays in LDS that are read or written 16 bytes at a time begin at multiples of 16; needs no GPU."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2207_01260_amd", "csrc")

OFFSETS = r"""
#include <cstddef>
#include "distill_kernel.hpp"
using namespace cprune::distill;
template <int NT> constexpr bool fits() {
  return alignof(Shared<NT>) % 16 == 0 && (offsetof(Shared<NT>, shares) + offsetof(Shares, id)) % 16 == 0 && (offsetof(Shared<NT>, shares) + offsetof(Shares, p)) % 16 == 0;
}
static_assert(fits<64>() && fits<256>() && fits<512>(), "lists are read four numbers at a time");
"""


def test_lists_of_the_distillation(tmp_path):
    src = tmp_path / "offsets.hip"
    src.write_text(OFFSETS)
    include = os.path.join(os.path.dirname(os.path.dirname(CSRC)), "include")
    out = subprocess.run(["hipcc", "--offload-arch=gfx950", "--cuda-host-only", "-fsyntax-only", "-std=c++17", "-I" + CSRC, "-I" + include, str(src)], capture_output=True, text=True)
    assert out.returncode == 0, out.stderr


def test_rows_of_the_adapters():
    text = open(os.path.join(CSRC, "adapter_kernel.hpp")).read()
    for name in ("results", "turned"):
        assert re.search(r"__shared__ alignas\(16\) float %s\[" % name, text), name
