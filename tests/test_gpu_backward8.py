"""Gradients of linear layers from an input and a pre-activation kept as 8-bit rows,
against FP64 at the values that the rows stand for.

Bounds as for linear_backward, where z stands exactly here (an FP32 product, one
rounding), and one rounding more: x = q s is rounded to the operands' type."""
import numpy as np
import pytest
import torch

from dense_common import DTYPES, SLOPE2, TINY, U, U32, randn, slope64, within

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")


def stands_for(p):
    """FP64 values of 8-bit rows."""
    return p.values[:, :p.columns].double().cpu() * p.scales.double().cpu()[:, None]


def strided(t, pad, shift):
    buf = torch.full((t.shape[0], t.shape[1] + pad + shift), float("nan"), dtype=t.dtype, device="cuda")
    return buf[:, shift:shift + t.shape[1]].copy_(t)


def case(n, n_in, n_out, dtype, act, sizes=None, tail=0, bias=True, pad=0, shift=0):
    gen = torch.Generator().manual_seed(n_in + n_out)
    off, groups = None, 1
    if sizes is not None:
        off = [0, *np.cumsum(sizes).tolist()]
        n, groups = off[-1] + tail, len(sizes)
    kept = off[-1] if off else n
    x, z = randn(n, n_in, gen=gen, dtype=dtype), randn(n, n_out, gen=gen, dtype=dtype)
    w = randn(groups, n_in, n_out, gen=gen, dtype=dtype, scale=n_in ** -0.5)
    dy = randn(n, n_out, gen=gen, dtype=dtype, scale=0.3)
    dyd = strided(dy, pad, shift)
    x8, z8 = L.pack_rows(x.cuda()), L.pack_rows(z.cuda()) if act != "none" else None
    offd = torch.tensor(off, dtype=torch.int32, device="cuda") if off else None
    X, Z = stands_for(x8), stands_for(z8) if z8 else None
    if tail:   # rows of no group are not read, whatever they hold
        dyd[kept:] = float("inf")
        x8.scales[kept:] = float("nan")
        if z8:
            z8.scales[kept:] = float("nan")
    wd = w.cuda()
    kw = dict(offsets=offd, act=act)
    dx, dw, db = L.linear_backward8(dyd, x8, wd, z8, bias=bias, **kw)
    u, tiny = U[dtype], TINY[dtype]
    ux = u if dtype != "fp32" else 0   # (q s in FP32 is one FP32 rounding, counted with the sums)
    for g, (a, e) in enumerate(zip(off[:-1], off[1:]) if off else [(0, n)]):
        tag = f"group {g} rows {a}:{e}"
        DY, W, Xg = dy[a:e].double(), w[g].double(), X[a:e]
        slope = slope64(Z[a:e], act) if act != "none" else torch.ones_like(DY)
        DZ = DY * slope
        edz = torch.zeros_like(DZ)
        if act != "none":
            edz = DY.abs() * (SLOPE2 * U32 * Z[a:e].abs() + 32 * U32 * (1 + Z[a:e].abs())) + tiny
        edz_r = edz + (u * (DZ.abs() + edz) if act != "none" else 0)
        DX = DZ @ W.t()
        edx = edz_r @ W.abs().t() + (n_out + 8) * U32 * ((DZ.abs() + edz_r) @ W.abs().t())
        within(dx[a:e], DX, edx + u * (DX.abs() + edx) + tiny, tag + " dx")
        DW = Xg.t() @ DZ
        mag = Xg.abs().t() @ (DZ.abs() + edz_r)
        edw = Xg.abs().t() @ edz_r + (ux + tiny) * mag + tiny * (DZ.abs() + edz_r).sum(0) + (e - a + 10) * U32 * mag
        within(dw[g], DW, edw + u * (DW.abs() + edw) + tiny, tag + " dw")
        if bias:
            DB = DZ.sum(0)
            edb = edz.sum(0) + (e - a + 8) * U32 * (DZ.abs() + edz).sum(0)
            within(db[g], DB, edb + u * (DB.abs() + edb) + tiny, tag + " db")
    assert (dx[kept:] == 0).all()
    only_x = L.linear_backward8(dyd, x8, wd, z8, bias=False, need_dw=False, **kw)
    only_w = L.linear_backward8(dyd, x8, wd, z8, bias=False, need_dx=False, **kw)
    assert only_x[1] is None and only_x[2] is None and only_w[0] is None
    assert torch.equal(only_x[0], dx) and torch.equal(only_w[1], dw)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n,n_in,n_out", [(1, 1, 1), (1, 128, 128), (2, 7, 5), (3, 64, 1), (16, 16, 17), (65, 8, 72),
                                          (130, 97, 211), (257, 130, 129), (300, 200, 8)])
def test_one_group(n, n_in, n_out, dtype):
    for act in ("none", "silu", "gelu"):
        case(n, n_in, n_out, dtype, act, bias=act != "gelu")


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("sizes,tail", [([5], 0), ([0, 3, 0, 0, 70, 1], 0), ([0, 0], 9), ([1] * 70 + [40], 11), ([129, 0, 257], 65)])
def test_groups(sizes, tail, dtype):
    case(None, 48, 40, dtype, "silu", sizes, tail)
    case(None, 31, 21, dtype, "gelu", sizes, tail)
    case(None, 31, 24, dtype, "none", sizes, tail)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (1, 0), (0, 1), (16, 8)])
def test_strided_rows(pad, shift, dtype):
    case(75, 64, 80, dtype, "silu", pad=pad, shift=shift)
    case(75, 64, 80, dtype, "none", pad=pad, shift=shift)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n,n_in,n_out,sizes", [(5001, 70, 66, None), (4100, 256, 520, None), (None, 512, 264, [2000, 1, 3000]),
                                                (33000, 32, 16, None)])
def test_many_rows(n, n_in, n_out, sizes, dtype):
    case(n, n_in, n_out, dtype, "silu", sizes)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n,n_in,n_out,sizes", [(12288, 1024, 64, None), (12300, 1032, 72, None), (None, 1024, 64, [6000, 0, 6300]),
                                                (1500, 1024, 1048, None)])
def test_wide_tiles(n, n_in, n_out, sizes, dtype):
    """dx, or dW, in 256 x 256 tiles."""
    case(n, n_in, n_out, dtype, "gelu", sizes)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_short_sums_over_many_rows(dtype):
    """dx as the form with weights in registers gives it (1026 runs of 512 rows, 64 columns)."""
    case(525000, 64, 24, dtype, "silu")


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_same_as_the_layer_at_the_unpacked_input(dtype):
    """Without an activation it is linear_backward at the unpacked rows, bit for bit."""
    gen = torch.Generator().manual_seed(0)
    x, w, dy = (randn(*s, gen=gen, dtype=dtype).cuda() for s in [(900, 72), (72, 40), (900, 40)])
    x8 = L.pack_rows(x)
    got = L.linear_backward8(dy, x8, w)
    want = L.linear_backward(dy, L.unpack_rows(x8, DTYPES[dtype]), w)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_gradient_of_expanded_dy():
    x8 = L.pack_rows(torch.randn(100, 24, device="cuda"))
    w = torch.randn(24, 16, device="cuda")
    one = torch.ones(1, 1, device="cuda").expand(100, 16)
    got, want = L.linear_backward8(one, x8, w), L.linear_backward8(one.contiguous(), x8, w)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_no_rows():
    x8 = L.pack_rows(torch.empty(0, 24, device="cuda"))
    dx, dw, db = L.linear_backward8(torch.empty(0, 16, device="cuda"), x8, torch.randn(24, 16, device="cuda"))
    assert dx.shape == (0, 24) and (dw == 0).all() and (db == 0).all()


def test_gradient_against_differences():
    """Central differences of sum(c act(x W + b)) in W and b at the x and z that the rows
    stand for: z is what the rows give for x W + b, so W is taken as zero and the bias as z's
    column (rows that are alike). h = 2^-6: truncation h^2 / 6 |act'''| below 1e-4."""
    gen = torch.Generator().manual_seed(5)
    b = torch.randn(16, generator=gen)
    x8, z8 = L.pack_rows(torch.randn(50, 24, generator=gen).cuda()), L.pack_rows(b.expand(50, 16).contiguous().cuda())
    X, Z = stands_for(x8), stands_for(z8)
    c = torch.randn(50, 16, generator=gen)
    dx, dw, db = L.linear_backward8(c.cuda(), x8, torch.zeros(24, 16, device="cuda"), z8, act="silu")
    v, vb, h = torch.randn(24, 16, generator=gen).double(), torch.randn(16, generator=gen).double(), 2.0 ** -6
    v /= 5

    def loss(t):
        z = Z + t * (X @ v + vb)
        return (c.double() * z / (1 + torch.exp(-z))).sum().item()
    want = (loss(h) - loss(-h)) / (2 * h)
    got = (dw.cpu().double() * v).sum().item() + (db.cpu().double() * vb).sum().item()
    size = (c.double().abs() * (X @ v + vb).abs()).sum().item()
    assert abs(got - want) <= 2e-3 * size
    assert (dx == 0).all()


def test_offsets_beyond_32_bits():
    """More than 2^31 elements of x8, of its 16-bit operand and of dx."""
    n, k, m = (1 << 20) + 77, 2064, 24
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, z, dy = (torch.zeros(n, c, dtype=torch.bfloat16, device="cuda") for c in (k, m, m))
    for t in (x, z, dy):
        t[-50:] = torch.randn(50, t.shape[1], generator=gen, device="cuda").bfloat16()
    w = (torch.randn(k, m, generator=gen, device="cuda") * k ** -0.5).bfloat16()
    x8, z8 = L.pack_rows(x), L.pack_rows(z)
    assert x8.values.numel() > 1 << 31
    dx, dw, db = L.linear_backward8(dy, x8, w, z8, act="silu")
    tail = [L.pack_rows(t[-50:].contiguous()) for t in (x, z)]
    want = L.linear_backward8(dy[-50:].contiguous(), tail[0], w, tail[1], act="silu")
    assert torch.equal(dx[-50:], want[0]) and not dx[:-50].any()
    X, dz = stands_for(tail[0]), dy[-50:].cpu().double() * slope64(stands_for(tail[1]), "silu")
    DW, mag = X.t() @ dz, X.abs().t() @ dz.abs()
    u = U["bf16"]   # dz's rounding and the result's, and FP32 sums of 50 terms that are not zero
    within(dw, DW, (u * (1 + 2 * u) + 64 * U32) * mag + u * DW.abs() + TINY["bf16"], "dw")
    within(db, dz.sum(0), 100 * U32 * dz.abs().sum(0) + u * dz.sum(0).abs() * (1 + u), "db")


def test_captured_beside_an_eager_graph():
    x, z, w, dy = (torch.randn(*s, device="cuda").bfloat16() for s in [(2000, 96), (2000, 64), (2, 96, 64), (2000, 64)])
    off = torch.tensor([0, 700, 1990], dtype=torch.int32, device="cuda")

    def step(stream=None):
        x8, z8 = L.pack_rows(x, stream=stream), L.pack_rows(z, stream=stream)
        return L.linear_backward8(dy, x8, w, z8, offsets=off, act="silu", stream=stream)
    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = step(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    leaf = w.clone().requires_grad_()
    alive = (leaf * 2).sum()   # an eager graph that lives through the capture
    g = torch.cuda.CUDAGraph()
    with torch.no_grad(), torch.cuda.graph(g):
        out = step()
    for _ in range(3):
        for t in out:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    alive.backward()
    assert (leaf.grad == 2).all()
