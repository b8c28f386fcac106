"""The kernels on a cache kept in pages start before the kernel ahead of them ends: what that one may still write is not read as read-only data."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_15312_b200", "csrc")


@pytest.mark.parametrize("name", ["paged.cuh", "tree_attention.cuh", "tree_plan.h", "verify_sampled.cuh"])
def test_no_read_only_loads_in_kernels_that_start_early(name):
    with open(os.path.join(CSRC, name)) as fh:
        code = re.sub(r"//[^\n]*", "", fh.read())
    assert not re.search(r"\b__ldg\b|\bld\.global\.nc|\bld_nc_|__restrict__", code)
