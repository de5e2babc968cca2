"""No function of layers.py records a graph: a tensor that asks for a gradient is
refused rather than answered with one that has silently lost it."""
import pytest
import torch

L = pytest.importorskip("paper_2510_23621_amd.layers")


def t(*shape, grad=False, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype, requires_grad=grad)


PLAN = L.Route(t(4, 2, dtype=torch.int32), t(8, dtype=torch.int32), t(3, dtype=torch.int32))
CALLS = {"x": lambda g: L.linear(t(4, 8, grad=g), t(8, 8)),
         "w": lambda g: L.linear(t(4, 8), t(8, 8, grad=g)),
         "bias": lambda g: L.linear(t(4, 8), t(8, 8), bias=t(8, grad=g)),
         "residual": lambda g: L.linear(t(4, 8), t(8, 8), None, t(4, 8, grad=g)),
         "dy": lambda g: L.linear_backward(t(4, 8, grad=g), t(4, 8), t(8, 8)),
         "route_rows": lambda g: L.route_rows(t(4, 8, grad=g), PLAN),
         "combine_rows": lambda g: L.combine_rows(t(8, 8, grad=g), PLAN),
         "weights": lambda g: L.combine_rows(t(8, 8), PLAN, weights=t(4, 2, grad=g)),
         "dout": lambda g: L.combine_rows_backward(t(4, 8, grad=g), t(8, 8), PLAN),
         "drows": lambda g: L.route_rows_backward(t(8, 8, grad=g), PLAN),
         "g": lambda g: L.orthogonalise(t(4, 8, grad=g))}


@pytest.mark.parametrize("name", CALLS)
def test_refused_while_gradients_are_recorded(name):
    with pytest.raises(ValueError, match="no_grad"):
        CALLS[name](True)
    with torch.no_grad(), pytest.raises(ValueError, match="GPU"):   # (then the host tensors are what is wrong)
        CALLS[name](True)
    with pytest.raises(ValueError, match="GPU"):
        CALLS[name](False)
