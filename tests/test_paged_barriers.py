"""The cluster barriers of the decode over pages are `.aligned`: all threads of a warp must run them together, which the code sees to right
before each (after a branch of some of a warp's threads, or a loop that they leave apart, a warp need not have joined again)."""
import glob
import os
import re

import pytest

from paper_2603_14303_b200 import build

FILES = sorted(glob.glob(os.path.join(build.CSRC, "paged*.cu*")))


def _barriers(path):
    lines = [re.sub(r"//.*", "", line).strip() for line in open(path)]
    lines = [line for line in lines if line]
    return [(i, lines) for i, line in enumerate(lines) if "barrier.cluster" in line and ".aligned" in line]


@pytest.mark.parametrize("path", FILES, ids=os.path.basename)
def test_warps_join_before_an_aligned_barrier(path):
    for i, lines in _barriers(path):
        assert lines[i - 1] == "__syncwarp();", lines[i - 1:i + 1]


def test_the_barriers_are_found():
    assert sum(len(_barriers(path)) for path in FILES) >= 3
