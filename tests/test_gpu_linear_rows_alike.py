"""A row's result does not depend on its place in a tile, nor on the tile: the same bits."""
import pytest
import torch

from dense_common import DTYPES

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("n,k,m", [(6144, 64, 2048), (4096, 64, 1024), (4100, 65, 1026), (1024, 72, 1000), (300, 64, 130)])
def test_rows_alike(n, k, m, act, dtype):
    gen = torch.Generator().manual_seed(m)
    x, r = (torch.randn(1, c, generator=gen).to(DTYPES[dtype]).cuda().expand(n, c).contiguous() for c in (k, m))
    w, b = (torch.randn(*s, generator=gen).to(DTYPES[dtype]).cuda() for s in ((k, m), (m,)))
    y = L.linear(x, w, b, r, act=act)
    assert torch.equal(y, y[:1].expand(n, m))
    y8 = L.linear8(x, L.pack_weights(w), b, r, act=act)
    assert torch.equal(y8, y8[:1].expand(n, m))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("n,m", [(6144, 2048), (8192, 512), (6145, 1026)])
def test_tiles_alike(n, m, act, dtype):
    """The first rows of a launch in wide tiles (256 and 128 rows) and alone, in tiles of 64: the same
    sums in the same order, and one rounding of act(z) + r (its last product and the residual's
    addition are one operation) in each."""
    k = 192
    gen = torch.Generator().manual_seed(m)
    x, r = (torch.randn(n, c, generator=gen).to(DTYPES[dtype]).cuda() for c in (k, m))
    w, b = (torch.randn(*s, generator=gen).to(DTYPES[dtype]).cuda() for s in ((k, m), (m,)))
    y = L.linear(x, w, b, r, act=act)
    few = L.linear(x[:64], w, b, r[:64], act=act)
    assert torch.equal(y[:64], few)
