"""Gradients as autograd hands them on: expanded, transposed, of strided rows."""
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")


def layouts(n, c, gen):
    one = torch.randn(1, 1, generator=gen, device="cuda")
    yield "of a sum", one.expand(n, c)
    yield "of a sum over rows", torch.randn(1, c, generator=gen, device="cuda").expand(n, c)
    yield "of a sum over columns", torch.randn(n, 1, generator=gen, device="cuda").expand(n, c)
    yield "of a transpose", torch.randn(c, n, generator=gen, device="cuda").t()


def test_linear_backward():
    gen = torch.Generator(device="cuda").manual_seed(0)
    x, w = torch.randn(50, 24, generator=gen, device="cuda"), torch.randn(24, 40, generator=gen, device="cuda")
    _, z = L.linear(x, w, act="silu", save=True)
    for name, dy in layouts(50, 40, gen):
        want = L.linear_backward(dy.contiguous(), x, w, z, act="silu")
        for a, b in zip(L.linear_backward(dy, x, w, z, act="silu"), want):
            assert torch.equal(a, b), name


def test_routing():
    gen = torch.Generator(device="cuda").manual_seed(0)
    e = torch.randint(-1, 5, (30, 2), generator=gen, device="cuda", dtype=torch.int32)
    p, w = L.route(e, 5), torch.rand(30, 2, generator=gen, device="cuda")
    rows = torch.randn(60, 16, generator=gen, device="cuda")
    for name, dout in layouts(30, 16, gen):
        want = L.combine_rows_backward(dout.contiguous(), rows, p, w)
        for a, b in zip(L.combine_rows_backward(dout, rows, p, w), want):
            assert torch.equal(a, b), name
    for name, drows in layouts(60, 16, gen):
        assert torch.equal(L.route_rows_backward(drows, p), L.route_rows_backward(drows.contiguous(), p)), name
