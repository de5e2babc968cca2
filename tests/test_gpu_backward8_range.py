"""Gradients of linear layers from 8-bit rows at the ends of the 16-bit types' ranges, against FP64
at the values that the rows stand for.

With an activation the products' operands are the input's integers times a power of two and
dz times the rest f of the row's scale, in (1/2, 1]. Where no power keeps the integers within the
type, x is rounded to the type and f is 1: dz, and with it dx and db, never depend on the
size of x."""
import pytest
import torch

from dense_common import DTYPES, TINY, U, U32, within

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")
LARGEST = {"fp16": 65504.0, "bf16": 3.3895313892515355e38}
END = {"fp16": 65520.0, "bf16": 511 * 2.0 ** 119}   # half a step more: from there on results are infinite


def stands_for(p):
    return p.values[:, :p.columns].double().cpu() * p.scales.double().cpu()[:, None]


def near(got, want, bound, dtype, what):
    """`within`, and infinity where the exact value is past END by more than its bound; what may come
    out either way is not compared."""
    got, end = got.detach().cpu().double(), END[dtype]
    past, inside = want.abs() - bound > end, want.abs() + bound < end
    assert (got[past] == torch.sign(want[past]) * float("inf")).all(), f"{what}: past the type's range"
    within(got[inside], want[inside], bound[inside], what)


def slopes_of_one(n, m):
    """Pre-activations of 90 as 8-bit rows: SiLU's slope there is 1 to FP32, so that dz = dy."""
    return L.pack_rows(torch.full((n, m), 90.0, device="cuda"))


def check(x8, dy, w, dtype, ex):
    """dx, dw and db of a layer whose slopes are 1, with ex [n, n_in] a bound of the error of x's operand."""
    n, m = dy.shape
    dx, dw, db = L.linear_backward8(dy.cuda(), x8, w.cuda(), slopes_of_one(n, m), act="silu")
    u, tiny = U[dtype], TINY[dtype]
    X, DY, W = stands_for(x8), dy.double(), w.double()
    # the slope and f dz: FP32 roundings, and one of the type (tiny: near zero, over f)
    edz = (u + 8 * U32) * DY.abs() + tiny
    DX, mx = DY @ W.t(), (DY.abs() + edz) @ W.abs().t()
    edx = edz @ W.abs().t() + (m + 10) * U32 * mx
    near(dx, DX, edx + u * (DX.abs() + edx) + tiny, dtype, "dx")
    edb = 8 * U32 * DY.abs().sum(0) + (n + 8) * U32 * DY.abs().sum(0)
    near(db, DY.sum(0), edb + u * (DY.sum(0).abs() + edb) + tiny, dtype, "db")
    if ex is None:
        return dw
    DW = X.t() @ DY
    edw = (X.abs() + ex).t() @ edz + ex.t() @ DY.abs()
    edw = edw + (n + 10) * U32 * ((X.abs() + ex).t() @ (DY.abs() + edz))
    near(dw, DW, edw + u * (DW.abs() + edw) + tiny, dtype, "dw")


@pytest.mark.parametrize("n,n_in,n_out", [(3, 24, 16), (70, 97, 33), (300, 256, 264)])
def test_rows_that_binary16_cannot_hold(n, n_in, n_out):
    """Rows of 1e6 in 8 bits, packed from float32: their gradients' dz of 5000 stays as it is."""
    gen = torch.Generator().manual_seed(0)
    x = torch.randn(n, n_in, generator=gen)
    x[1] *= 1e6
    x[2] *= 1e30
    dy = (5000 * torch.randn(n, n_out, generator=gen)).half()
    w = (torch.randn(n_in, n_out, generator=gen) * 0.01).half()
    dw = check(L.pack_rows(x.cuda()), dy, w, "fp16", None)
    assert not torch.isfinite(dw).all()   # x itself is infinite in binary16


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("n,n_in,n_out", [(3, 24, 16), (70, 97, 33)])
def test_largest_dz_of_largest_rows(n, n_in, n_out, dtype):
    """Rows up to the type's largest number, whose scale over the largest power of two is a little above one."""
    gen = torch.Generator().manual_seed(1)
    big = LARGEST[dtype]
    x = (torch.rand(n, n_in, generator=gen) - 0.5).to(DTYPES[dtype])
    x[:, 0] = big
    dy = torch.full((n, n_out), big).to(DTYPES[dtype])
    w = (torch.rand(n_in, n_out, generator=gen) / (4 * n_out)).to(DTYPES[dtype])
    x8 = L.pack_rows(x.cuda())
    n_, m = dy.shape
    dx, _, _ = L.linear_backward8(dy.cuda(), x8, w.cuda(), slopes_of_one(n_, m), act="silu", bias=False)
    DX = dy.double() @ w.double().t()
    u = U[dtype]
    within(dx, DX, (2 * u + u * u + (m + 20) * U32) * DX.abs() + TINY[dtype], "dx")


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_weights_gradient_of_largest_rows(dtype):
    """x = q s rounded to the type: one rounding of it."""
    gen = torch.Generator().manual_seed(2)
    big = LARGEST[dtype]
    x = ((torch.rand(20, 40, generator=gen) - 0.5) * big).to(DTYPES[dtype])
    x[:, 3] = big
    dy = (torch.randn(20, 16, generator=gen) * 2.0 ** -8).to(DTYPES[dtype])
    w = torch.randn(40, 16, generator=gen).to(DTYPES[dtype])
    x8 = L.pack_rows(x.cuda())
    assert (x8.scales.cpu() > big / 128).all()   # above the largest power of two whose 127-fold the type holds
    check(x8, dy, w, dtype, U[dtype] * stands_for(x8).abs())


@pytest.mark.parametrize("n", [1, 4, 16])
@pytest.mark.parametrize("size", [1e-7, 3e-7, 1e-6, 3e-6, 4e-6, 1e-5])
def test_weights_gradient_of_smallest_binary16_rows(size, n):
    """Rows down to binary16's smallest numbers. From scales of 2^-25 up the integers times a power
    of two are exact; below, x is rounded to binary16: the numbers that the rows were packed from lie
    within half a scale of q s, and the nearest number does at the most."""
    gen = torch.Generator().manual_seed(3)
    x = ((torch.rand(n, 60, generator=gen) - 0.5) * 2 * size).half()
    x[:, 5] = size
    dy = (2000 * torch.randn(n, 48, generator=gen)).half()
    w = (torch.randn(60, 48, generator=gen) * 0.01).half()
    x8 = L.pack_rows(x.cuda())
    X, s = stands_for(x8), x8.scales.double().cpu()[:, None].expand(n, 60)
    ex = torch.where(s > 2.0 ** -25, 0 * s, (s / 2 * (1 + 2.0 ** -20)).clamp_max(2.0 ** -25) + 2 * U32 * X.abs())
    check(x8, dy, w, "fp16", ex)


def test_rows_below_binary16():
    """Rows of 1e-9 to 1e-12 packed from float32: x is zero in binary16, and dx and db what they are."""
    gen = torch.Generator().manual_seed(4)
    x = torch.randn(30, 40, generator=gen) * 10.0 ** -torch.linspace(9, 12, 30)[:, None]
    dy = (2000 * torch.randn(30, 24, generator=gen)).half()
    w = (torch.randn(40, 24, generator=gen) * 0.01).half()
    x8 = L.pack_rows(x.cuda())
    check(x8, dy, w, "fp16", torch.full((30, 40), 2.0 ** -25, dtype=torch.float64))
