"""The 8-bit layer at rows and weights whose integer sums times one of the two scales leave FP32's
range where the result does not: y against FP64."""
import numpy as np
import pytest
import torch

from dense_common import DTYPES, U, U32, act64, within

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")


def values(p):
    return p.values.double().cpu(), p.scales.double().cpu()


# the one-launch form, tiles of 64 x 64, 128 x 128 and 256 x 256
@pytest.mark.parametrize("n,k,m", [(1, 2048, 40), (16, 500, 33), (300, 130, 2056), (2048, 96, 2048), (6144, 64, 2048)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("size_x,size_w", [(1e36, 1e-3), (1e36, 1e-30), (3e37, 2e-9), (1e-30, 1e35), (1e-37, 1e30), (1e16, 1e16)])
def test_products_of_far_scales(size_x, size_w, n, k, m, dtype):
    gen = torch.Generator().manual_seed(k)
    x = ((torch.rand(n, k, generator=gen) + 0.5) * size_x).to(DTYPES[dtype])
    if n > 2:
        x[1] = x[1] / x[1].max()   # an ordinary row beside the others
    w = ((torch.rand(k, m, generator=gen) + 0.5) * (size_w / k)).to(DTYPES[dtype])
    bias = torch.full((m,), size_x * size_w).to(DTYPES[dtype])
    w8 = L.pack_weights(w.cuda())
    q, s = values(L.pack_rows(x.cuda()))
    qw, sw = values(w8)
    T = ((q @ qw[0].t()) * s[:, None]) * sw[0]   # (FP64 holds every product of these)
    for act in ("none", "silu"):
        y = L.linear8(x.cuda(), w8, bias.cuda(), act=act)
        assert torch.equal(y, L.linear8(L.pack_rows(x.cuda()), w8, bias.cuda(), act=act, dtype=DTYPES[dtype]))
        Z = T + bias.double()
        Y = act64(Z, act)
        u = U[dtype]
        # the sum as FP32, two scales, the bias; silu's slope is at most 1.1 and its own error 16 roundings
        e = 1.1 * (4 * U32 * T.abs() + 2 * U32 * Z.abs()) + 16 * U32 * (Y.abs() + Z.abs()) + 2.0 ** -126
        within(y, Y, e + u * Y.abs() * (1 + 2 * u), f"{act} y")


@pytest.mark.parametrize("n,k,m", [(2, 64, 24), (300, 130, 2056)])
def test_results_beyond_the_range(n, k, m):
    """Infinite where the exact result is, and zero where the sum is zero, whatever the scales."""
    x = torch.full((n, k), 1e30, device="cuda")
    w = torch.full((k, m), 1e30, device="cuda")
    w[::2, 1] = -1e30
    y = L.linear8(x, L.pack_weights(w))
    assert (y[:, 0] == float("inf")).all()
    assert (y[:, 1] == 0).all()
    x[0, 0] = float("nan")
    y = L.linear8(x, L.pack_weights(w))
    assert torch.isnan(y[0]).all() and not torch.isnan(y[1:]).any()


@pytest.mark.parametrize("n,k,m", [(12, 64, 24), (300, 130, 2056), (2048, 96, 2048), (6144, 64, 2048)])
def test_rows_do_not_meet(n, k, m):
    """A large and a non-finite row leave the others' bits."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(n, k, generator=gen, device="cuda")
    w = L.pack_weights(torch.randn(k, m, generator=gen, device="cuda") * 1e-6)
    want = L.linear8(x, w, act="gelu")
    x[3] *= 1e36
    x[5, 0] = float("nan")
    y = L.linear8(x, w, act="gelu")
    assert torch.isfinite(y[3]).all() and torch.isnan(y[5]).all()
    keep = [i for i in range(n) if i not in (3, 5)]
    assert torch.equal(y[keep], want[keep])
