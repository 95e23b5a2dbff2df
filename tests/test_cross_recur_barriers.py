"""Barriers of the cross attention's and the recurrence's kernels are lds_barrier() (or
cross_barrier()), which wait for the wave's own LDS operations themselves: a plain
__syncthreads() leaves that to the compiler, which has been seen to drop it in loops."""
import glob
import os

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_20744_amd", "csrc")


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "vda_cross*.hip")) + glob.glob(os.path.join(CSRC, "vda_recur*.hip"))),
                         ids=os.path.basename)
def test_no_plain_barrier(path):
    with open(path) as f:
        assert "__syncthreads" not in f.read()
