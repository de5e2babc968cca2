"""The order of more slots than the sort's blocks take one chunk each."""
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")


@pytest.mark.parametrize("n,k,E", [((1 << 21) + 4099, 1, 3), (700001, 3, 512), (1 << 22, 2, 64), (6000001, 4, 37)])
def test_order(n, k, E):
    """Against torch's stable sort, a tenth of the slots dropped."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    e = torch.randint(0, E, (n, k), generator=gen, device="cuda", dtype=torch.int32)
    e[torch.rand(n, k, generator=gen, device="cuda") < 0.1] = -1
    p = L.route(e, E)
    key = torch.where(e < 0, E, e).reshape(-1)
    order = torch.sort(key, stable=True).indices
    assert torch.equal(p.slot_of_row.long(), order)
    assert torch.equal(order[p.row_of_slot.reshape(-1).long()], torch.arange(n * k, device="cuda"))
    count = torch.bincount(key, minlength=E + 1)
    assert torch.equal(p.offsets.long(), torch.cat([count.new_zeros(1), count[:E].cumsum(0)]))


def test_skewed_order():
    """One expert takes nearly all of nine million slots, in long runs."""
    n, E = 9000001, 100
    e = torch.full((n, 1), 42, dtype=torch.int32, device="cuda")
    e[::4097] = 7
    e[-5:] = 0
    p = L.route(e, E)
    assert torch.equal(p.slot_of_row.long(), torch.sort(e.reshape(-1), stable=True).indices)
