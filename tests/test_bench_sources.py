"""The stamp on the benchmark's traffic figures: of the sources that its network runs."""
import os
import re
import shutil

import pytest

import bench

CSRC = os.path.join(bench.ROOT, "paper_2207_01260_amd", "csrc")


@pytest.fixture()
def copy(tmp_path):
    return shutil.copytree(CSRC, tmp_path / "csrc")


def test_a_kernel_of_the_network_changes_it(copy):
    before = bench.kernel_source_hash(copy)
    assert before == bench.kernel_source_hash()
    for name in ("conv_split_f32.hip", "common.hpp", "conv_launch.hip"):
        with open(copy / name, "a") as f:
            f.write("\n")
        after = bench.kernel_source_hash(copy)
        assert after != before
        before = after


def test_sources_of_other_calls_do_not(copy):
    before = bench.kernel_source_hash(copy)
    for name in ("group_norm.hip", "group_norm_kernel.hpp", "mx4.hip", "mx4_kernel.hpp"):
        with open(copy / name, "a") as f:
            f.write("\n")
    assert bench.kernel_source_hash(copy) == before


def test_no_other_source_includes_them():
    for name in os.listdir(CSRC):
        if name.endswith((".hip", ".hpp")) and not name.startswith(bench.APART):
            included = re.findall(r'#include "([^"]+)"', open(os.path.join(CSRC, name)).read())
            assert not [i for i in included if os.path.basename(i).startswith(bench.APART)], name
