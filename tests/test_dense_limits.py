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


@pytest.mark.parametrize("dtype,n_in,n_out", [(0, 512, 2048), (0, 2048, 2048), (0, 1023, 1023), (1, 511, 2049),
                                              (2, 1023, 2047), (1, 512, 2048)])
def test_partial_sums_of_weight_gradients_are_no_more_than_fill_the_chip(dtype, n_in, n_out):
    """Two blocks of 128 x 128 FP32 sums per CU, or one of 256 x 256 where rows are aligned 16-bit ones."""
    d = B.mace_linear_desc(36864, n_in, n_out, 1, dtype, 0, n_in, n_out, n_out, n_out)
    blocks = 512 * 128 * 128 if dtype == 0 or n_in % 8 else 256 * 256 * 256
    assert B.mace_linear_backward_workspace_bytes(d, False, True) <= blocks * 4 + 512
