"""Weights' gradients from 8-bit rows with an activation: the input's operand is exact, so that the
terms of the products are rounded once (dz), not twice; and what a row that is not finite reaches."""
import pytest
import torch

from dense_common import DTYPES, SLOPE2, TINY, U, U32, randn, slope64, within

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")


def stands_for(p):
    return p.values[:, :p.columns].double().cpu() * p.scales.double().cpu()[:, None]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,n_in,n_out", [(1, 512, 512), (24, 97, 211), (40, 64, 72)])
def test_one_rounding_of_the_terms(rows, n_in, n_out, act, dtype):
    """Groups of a row each: dW = x dz^T has one term, off by dz's rounding and its own. With x rounded
    too a part of the elements (1 to 3 of 1000) is off by more than two roundings."""
    gen = torch.Generator().manual_seed(rows)
    x = randn(rows, n_in, gen=gen, dtype=dtype) * torch.exp2(torch.linspace(-6, 6, rows)).to(DTYPES[dtype])[:, None]
    z, dy = randn(rows, n_out, gen=gen, dtype=dtype), randn(rows, n_out, gen=gen, dtype=dtype, scale=4.0)
    w = randn(rows, n_in, n_out, gen=gen, dtype=dtype)
    off = torch.arange(rows + 1, dtype=torch.int32)
    x8, z8 = L.pack_rows(x.cuda()), L.pack_rows(z.cuda())
    dw = L.linear_backward8(dy.cuda(), x8, w.cuda(), z8, offsets=off.cuda(), act=act)[1]
    X, Z, DY = stands_for(x8), stands_for(z8), dy.double()
    u, tiny = U[dtype], TINY[dtype]
    DZ = DY * slope64(Z, act)
    edz = DY.abs() * (SLOPE2 * U32 * Z.abs() + 32 * U32 * (1 + Z.abs()))
    edz = edz + (u + 2 * U32) * (DZ.abs() + edz) + tiny   # the scale's rest in FP32, the rounding
    DW = X[:, :, None] * DZ[:, None, :]
    e = X.abs()[:, :, None] * edz[:, None, :] * (1 + 4 * U32)
    within(dw, DW, e + u * (DW.abs() + e) + tiny, "dw")
    # the same bound does not hold of the definition with x rounded to the type
    twice = X.to(DTYPES[dtype]).double()[:, :, None] * DZ.to(DTYPES[dtype]).double()[:, None, :]
    twice = twice.to(DTYPES[dtype]).double()
    assert ((twice - DW).abs() > e + u * (DW.abs() + e) + tiny).any()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n_in,n_out", [(40, 24), (97, 33), (256, 264)])
def test_row_that_is_not_finite(n_in, n_out, dtype):
    """Its group's weights' gradients are NaN, other groups' and dx and db the same bits as without it."""
    gen = torch.Generator().manual_seed(7)
    x, z, dy = (randn(90, c, gen=gen, dtype=dtype).cuda() for c in (n_in, n_out, n_out))
    w = randn(3, n_in, n_out, gen=gen, dtype=dtype).cuda()
    off = torch.tensor([0, 30, 71, 90], dtype=torch.int32, device="cuda")
    z8 = L.pack_rows(z)
    want = L.linear_backward8(dy, L.pack_rows(x), w, z8, offsets=off, act="silu")
    for bad in (float("inf"), float("nan")):
        x[40, 5] = bad
        dx, dw, db = L.linear_backward8(dy, L.pack_rows(x), w, z8, offsets=off, act="silu")
        assert torch.isnan(dw[1]).all() and torch.equal(dw[0], want[1][0]) and torch.equal(dw[2], want[1][2])
        keep = [i for i in range(90) if i != 40]
        assert torch.equal(db, want[2]) and torch.equal(dx[keep], want[0][keep])
        u = U[dtype]
        DX = (dy[40].double() * slope64(stands_for(z8)[40].cuda(), "silu")) @ w[1].double().t()
        mag = dy[40].double().abs() @ w[1].double().abs().t() * 1.13
        within(dx[40], DX.cpu(), ((2 * u + u * u + (n_out + 100) * U32) * mag).cpu() + TINY[dtype] * n_out, "dx")


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_the_same_bits_again(dtype):
    gen = torch.Generator().manual_seed(8)
    x, z, dy = (randn(9000, c, gen=gen, dtype=dtype).cuda() for c in (97, 211, 211))
    w = randn(4, 97, 211, gen=gen, dtype=dtype).cuda()
    off = torch.tensor([0, 3000, 3001, 8000, 8990], dtype=torch.int32, device="cuda")
    x8, z8 = L.pack_rows(x), L.pack_rows(z)
    want = L.linear_backward8(dy, x8, w, z8, offsets=off, act="gelu")
    for _ in range(5):
        got = L.linear_backward8(dy, x8, w, z8, offsets=off, act="gelu")
        assert all(torch.equal(a, b) for a, b in zip(got, want))
