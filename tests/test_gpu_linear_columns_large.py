"""Launches of more threads than one axis of a grid holds: 1024 groups of 2^20 columns."""
import pytest
import torch

from dense_common import U32

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")


def test_every_group_and_column():
    """One row in every hundredth group and in the last; products of one term, within 9
    FP32 roundings (as product_error has it); a bias gradient of one row is that row."""
    torch.cuda.empty_cache()
    groups, m = 1024, 1 << 20
    used = [*range(0, groups, 100), groups - 1]
    n = len(used)
    counts = torch.zeros(groups, dtype=torch.int64)
    counts[used] = 1
    off = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)]).int().cuda()
    x = torch.randn(n, 1, device="cuda")
    w = torch.randn(groups, 1, m, device="cuda")
    dy = torch.randn(n, m, device="cuda")
    y = L.linear(x, w, offsets=off)
    want = x.double() * w[used, 0].double()
    assert ((y.double() - want).abs() <= 9 * U32 * want.abs()).all()
    dx, dw, db = L.linear_backward(dy, x, w, offsets=off)
    want = x.double() * dy.double()
    assert ((dw[used, 0].double() - want).abs() <= 9 * U32 * want.abs()).all()
    assert torch.equal(db[used], dy)
    terms = dy.double() * w[used, 0].double()
    assert ((dx[:, 0].double() - terms.sum(1)).abs() <= (m + 8) * U32 * terms.abs().sum(1)).all()
    idle = torch.ones(groups, dtype=torch.bool)
    idle[used] = False
    assert not dw[idle.cuda()].any() and not db[idle.cuda()].any()
    del w, dw, db
    torch.cuda.empty_cache()
