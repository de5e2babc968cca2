"""Limits of the dense entry points that their cost and their arithmetic set."""
import os

import numpy as np
import pytest

B = pytest.importorskip("paper_2510_23621_amd.binding")
pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libmace_amd.so not built")


@pytest.mark.parametrize("experts", [1, 64, 512])
def test_counts_that_every_block_of_the_sort_reads_are_bounded(experts):
    """Each block reads the counts of all of them, which the workspace holds: it must not
    grow with the slots, or the whole would grow with their square."""
    def need(slots):
        return B.mace_route_workspace_bytes(B.mace_route_desc(slots, 1, experts, 8, 0, 8, 8))
    assert 0 < need(1 << 22) <= need(1 << 30) <= 256 + 512 * (experts + 1) * 4
