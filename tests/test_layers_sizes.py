"""Sizes that the library's 32-bit fields cannot hold are refused, not wrapped."""
import pytest
import torch

from test_layers_calls import machine  # noqa: F401

L = pytest.importorskip("paper_2510_23621_amd.layers")
WIDE = 2 ** 32 + 8


def empty(*shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype, device="cuda:0")


@pytest.mark.parametrize("call", [
    lambda: L.linear(empty(1, WIDE), empty(WIDE, 8)), lambda: L.linear(empty(1, 8), empty(8, WIDE)),
    lambda: L.linear(empty(1, 1), empty(WIDE, 1, 1), offsets=empty(WIDE + 1, dtype=torch.int32)),
    lambda: L.linear_backward(empty(1, WIDE), empty(1, 8), empty(8, WIDE)),
    lambda: L.route(empty(1, WIDE, dtype=torch.int32), 4), lambda: L.route(empty(4, 2, dtype=torch.int32), WIDE),
    lambda: L.route(empty(4, 2, dtype=torch.int32), -WIDE),
    lambda: L.orthogonalise(empty(8, WIDE)), lambda: L.orthogonalise(empty(WIDE, 8)),
    lambda: L.route_rows(empty(4, WIDE), plan()), lambda: L.combine_rows(empty(8, WIDE), plan()),
    lambda: L.combine_rows_backward(empty(4, WIDE), empty(8, WIDE), plan())])
def test_refused(machine, call):  # noqa: F811
    with pytest.raises(ValueError):
        call()
    assert not machine.calls


def plan():
    return L.Route(empty(4, 2, dtype=torch.int32), empty(8, dtype=torch.int32), empty(3, dtype=torch.int32))
