"""8-bit rows and weights bit for bit against the definition in exact arithmetic
(FP64 quotients of FP32 numbers decide the nearest integer), and the linear layer
on them against FP64: integer sums are exact, so its error is that of a few FP32
roundings and of the result's own."""
import numpy as np
import pytest
import torch

from dense_common import DTYPES, SLOPE1, TINY, U, U32, act64, randn, within

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")
SMALLEST = np.float32(2.0 ** -126)


def oracle(x):
    """q (int64) and scales (float32) of the rows of a float64 array of finite values."""
    big = abs(x).max(1)
    scale = np.maximum((big / 127).astype(np.float32), SMALLEST)
    q = np.rint(x / scale.astype(np.float64)[:, None])   # (a half of FP32 numbers' quotient is exact in FP64)
    return q.astype(np.int64), scale


def strided(t, pad, shift=0):
    buf = torch.full((t.shape[0], t.shape[1] + pad + shift), float("nan"), dtype=t.dtype, device="cuda")
    return buf[:, shift:shift + t.shape[1]].copy_(t)


def check_pack(x, pad=0, shift=0):
    p = L.pack_rows(strided(x, pad, shift))
    q, scale = oracle(x.double().numpy())
    n, c = x.shape
    assert p.columns == c and p.values.shape == (n, -(-c // 16) * 16)
    assert np.array_equal(p.scales.cpu().numpy(), scale)
    assert np.array_equal(p.values.cpu().numpy()[:, :c], q) and not p.values[:, c:].any()
    for dtype in DTYPES.values():
        got = L.unpack_rows(p, dtype)
        want = torch.from_numpy(q.astype(np.float32) * scale[:, None]).to(dtype)
        assert torch.equal(got.cpu(), want)
    return p, q, scale


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n,c,pad,shift", [(1, 1, 0, 0), (1, 2048, 0, 0), (3, 15, 0, 0), (5, 16, 16, 0), (70, 17, 1, 0),
                                           (64, 128, 0, 0), (33, 97, 3, 5), (9, 515, 0, 1), (257, 1024, 8, 8),
                                           (4, 4097, 0, 0), (3, 20000, 0, 0), (2, 131072, 0, 0), (1000, 8, 0, 0)])
def test_pack(n, c, pad, shift, dtype):
    gen = torch.Generator().manual_seed(n + c)
    x = randn(n, c, gen=gen, dtype=dtype) * torch.exp(3 * torch.randn(n, 1, generator=gen)).to(DTYPES[dtype])
    check_pack(x, pad, shift)


def test_halves_go_to_even():
    """Rows whose quotients are halves exactly (scale 1 and 3), and their neighbours in FP32."""
    h = torch.arange(-126.5, 127, 1.0)
    x = torch.stack([torch.cat([h, torch.tensor([127.0])]), 3 * torch.cat([h, torch.tensor([127.0])])])
    near = torch.cat([torch.nextafter(x, torch.full_like(x, 1e9)), torch.nextafter(x, torch.full_like(x, -1e9))])
    near[:, -1] = torch.tensor([127.0, 381.0, 127.0, 381.0])
    check_pack(torch.cat([x, near]))


def test_quotients_next_to_halves():
    """Scales of all significands, values at the FP32 numbers around (k + 1/2) scale."""
    rng = np.random.default_rng(0)
    rows = []
    for _ in range(300):
        big = np.float32(rng.uniform(1, 2) * 2.0 ** rng.integers(-100, 100))
        s = np.float32(np.float64(big) / 127)
        at = ((np.arange(-126, 126) + 0.5) * np.float64(s)).astype(np.float32)
        rows.append(np.concatenate([[big], at, np.nextafter(at, np.float32(np.inf)), np.nextafter(at, np.float32(-np.inf))]))
    check_pack(torch.from_numpy(np.stack(rows).astype(np.float32)))


def test_ends_of_the_range():
    tiny = 2.0 ** -149
    x = torch.tensor([[0.0, -0.0, 0.0], [tiny, -tiny, 0.0], [2.0 ** -126, 2.0 ** -127, -tiny], [127 * 2.0 ** -126, 2.0 ** -127, 3 * 2.0 ** -127],
                      [2.0 ** -119, 3 * 2.0 ** -127, 1e-38], [3.0e38, 1e38, -2.9e38], [1e-30, 1e-33, 4e-31]])
    check_pack(x)
    x[0, 1], x[2, 0], x[4, 2] = float("inf"), float("nan"), -float("inf")
    p = L.pack_rows(x.cuda())
    bad = torch.tensor([0, 2, 4])
    assert torch.isnan(p.scales.cpu()[bad]).all() and not p.values.cpu()[bad].any()
    keep = torch.tensor([1, 3, 5, 6])
    assert np.array_equal(p.scales.cpu()[keep].numpy(), oracle(x[keep].double().numpy())[1])
    assert torch.isnan(L.unpack_rows(p)[bad.cuda()]).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("g,k,m", [(1, 1, 1), (1, 128, 64), (3, 97, 211), (2, 17, 65), (1, 2048, 130), (5, 16, 8)])
def test_pack_weights(g, k, m, dtype):
    w = randn(g, k, m, gen=torch.Generator().manual_seed(k), dtype=dtype)
    p = L.pack_weights((w[0] if g == 1 else w).cuda())
    for i in range(g):
        q, scale = oracle(w[i].double().numpy().T)
        assert np.array_equal(p.scales[i].cpu().numpy(), scale) and np.array_equal(p.values[i, :, :k].cpu().numpy(), q)
    assert p.n_in == k and not p.values[:, :, k:].any()


def test_pack_weights_over_more_than_one_row_of_blocks():
    """1024 groups of 2049 tiles of columns: more than 2^21 blocks."""
    g, m = 1024, 131130
    w = torch.zeros(g, 1, m, dtype=torch.float16, device="cuda")
    w[-1] = torch.randn(1, m, device="cuda").half()
    w[0, 0, 5] = 2
    p = L.pack_weights(w)
    x = w[-1, 0].double()
    assert torch.equal(p.scales[-1].double(), (x.abs() / 127).float().clamp_min(2.0 ** -126).double())
    assert torch.equal(p.values[-1, :, 0].double(), 127 * x.sign()) and not p.values[:, :, 1:].any()
    assert p.values[0, 5, 0] == 127 and not p.values[1:-1].any()


def offsets_of(sizes, tail=0):
    off = torch.tensor([0] + list(sizes)).cumsum(0)
    return off.tolist(), int(off[-1]) + tail


def check_linear(n, k, m, dtype, act="none", sizes=None, tail=0, bias=True, residual=True, pad=0, shift=0, seed=0):
    gen = torch.Generator().manual_seed(seed + k)
    off, groups = None, 1
    if sizes is not None:
        off, n = offsets_of(sizes, tail)
        groups = len(sizes)
    x = randn(n, k, gen=gen, dtype=dtype)
    w = randn(groups, k, m, gen=gen, dtype=dtype, scale=k ** -0.5)
    b = randn(groups, m, gen=gen, dtype=dtype, scale=0.3) if bias else None
    r = randn(n, m, gen=gen, dtype=dtype) if residual else None
    kept = off[-1] if off else n
    xd = strided(x, pad, shift)
    rd = strided(r, pad, shift) if residual else None
    if tail:
        xd[kept:] = float("nan")
    offd = torch.tensor(off, dtype=torch.int32, device="cuda") if off else None
    w8 = L.pack_weights(w.cuda())
    bd = b.cuda() if bias else None
    y = L.linear8(xd, w8, bd, rd, offsets=offd, act=act)
    assert torch.equal(y, L.linear8(L.pack_rows(xd), w8, bd, rd, offsets=offd, act=act, dtype=DTYPES[dtype]))
    u = U[dtype]
    for g in range(groups):
        a, e = (off[g], off[g + 1]) if off else (0, n)
        if a == e:
            continue
        q, s = oracle(x[a:e].double().numpy())
        qw, sw = oracle(w[g].double().numpy().T)
        T = torch.from_numpy((q @ qw.T) * (s.astype(np.float64)[:, None] * sw.astype(np.float64)[None]))
        Z = T + (b[g].double() if bias else 0)
        ez = 4 * U32 * T.abs() + 2 * U32 * Z.abs()   # the sum as FP32, two scales; the bias
        Y = act64(Z, act) + (r[a:e].double() if residual else 0)
        ey = (SLOPE1 * ez if act != "none" else ez) + 16 * U32 * (act64(Z, act).abs() + Z.abs() + Y.abs()) + TINY[dtype]
        within(y[a:e], Y, ey + u * Y.abs() * (1 + 2 * u), f"group {g} rows {a}:{e}")
    assert (y[kept:] == 0).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n,k,m", [(1, 1, 1), (1, 128, 128), (1, 2048, 2048), (2, 7, 5), (3, 64, 1), (15, 17, 33), (16, 16, 17), (17, 130, 64),
                                   (33, 97, 211), (64, 128, 64), (65, 8, 72), (130, 1000, 130), (257, 129, 300), (40, 2047, 96)])
def test_linear(n, k, m, dtype):
    check_linear(n, k, m, dtype, "silu")
    check_linear(n, k, m, dtype, bias=False, residual=False)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,k,m", [(1, 50000, 40), (1, 8192, 1100), (2, 20001, 33), (3, 9000, 50), (7, 6100, 40), (9, 3000, 70),
                                   (16, 3500, 30), (5, 60000, 20)])
def test_linear_few_rows_of_long_sums(n, k, m, dtype):
    check_linear(n, k, m, dtype, "silu")


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("sizes,tail", [([5], 0), ([0, 3, 0, 0, 70, 1], 0), ([0, 0], 9), ([64, 64, 128], 0), ([1] * 70 + [40], 11),
                                        ([129, 0, 257], 65), ([700, 3], 0)])
def test_linear_groups(sizes, tail, dtype):
    check_linear(None, 48, 40, dtype, "silu", sizes, tail)
    check_linear(None, 31, 21, dtype, "gelu", sizes, tail)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,k,m,sizes", [(9000, 64, 64, None), (4100, 300, 520, None), (None, 257, 1032, [1500, 2, 2700]),
                                         (33000, 33, 24, None), (6144, 256, 2048, None)])
def test_linear_many_rows(n, k, m, sizes, dtype):
    check_linear(n, k, m, dtype, "gelu", sizes)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (1, 0), (0, 1), (16, 8)])
def test_linear_strided(pad, shift, dtype):
    check_linear(75, 64, 80, dtype, "silu", pad=pad, shift=shift)
    check_linear(300, 128, 130, dtype, pad=pad, shift=shift)


def test_largest_sums_are_exact():
    """All products 127 * 127 over the longest sum: 2114060288, next to 2^31."""
    k = 131072
    x, w = torch.ones(2, k, device="cuda"), torch.ones(k, 3, device="cuda")
    x[1] = -1
    y = L.linear8(x, L.pack_weights(w)).cpu()
    s = float(np.float32(1 / 127))
    want = torch.tensor([[1.0], [-1.0]]).double() * (127.0 * 127 * k * s * s)
    within(y, want.expand(2, 3), 4 * U32 * want.abs().expand(2, 3), "y")


def test_non_finite_rows_alone():
    x, w = torch.randn(70, 40, device="cuda"), L.pack_weights(torch.randn(40, 24, device="cuda"))
    want = L.linear8(x, w)
    x[5, 3], x[66, 0] = float("nan"), float("inf")
    y = L.linear8(x, w)
    assert torch.isnan(y[[5, 66]]).all()
    keep = [i for i in range(70) if i not in (5, 66)]
    assert torch.equal(y[keep], want[keep])


def test_no_rows():
    w = L.pack_weights(torch.randn(24, 8, device="cuda"))
    assert L.linear8(torch.empty(0, 24, device="cuda"), w).shape == (0, 8)
    p = L.pack_rows(torch.empty(0, 24, device="cuda"))
    assert p.values.shape == (0, 32) and L.unpack_rows(p).shape == (0, 24) and L.linear8(p, w).shape == (0, 8)


def test_other_stream_and_graph():
    x, w = torch.randn(3000, 200, device="cuda").bfloat16(), torch.randn(3, 200, 96, device="cuda").bfloat16()
    off = torch.tensor([0, 1000, 1001, 2900], dtype=torch.int32, device="cuda")

    def step(stream=None):
        w8 = L.pack_weights(w, stream=stream)
        p = L.pack_rows(x, stream=stream)
        return (w8.values, w8.scales, p.values, p.scales, L.unpack_rows(p, torch.bfloat16, stream=stream),
                L.linear8(x, w8, offsets=off, act="silu", stream=stream), L.linear8(p, w8, offsets=off, stream=stream),
                L.linear8(x[:1], w8._replace(values=w8.values[:1], scales=w8.scales[:1]), stream=stream))
    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = step(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for _ in range(3):
        for t in out:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_offsets_beyond_32_bits():
    """More than 2^31 elements of x, of its integers and of y."""
    n, k = (1 << 20) + 77, 2064
    x = torch.zeros(n, k, dtype=torch.bfloat16, device="cuda")
    x[-50:] = torch.randn(50, k, device="cuda").bfloat16()
    p = L.pack_rows(x)
    assert p.values.numel() > 1 << 31
    q = L.pack_rows(x[-50:].contiguous())
    assert torch.equal(p.values[-50:], q.values) and torch.equal(p.scales[-50:], q.scales) and not p.values[:-50].any()
    back = L.unpack_rows(p, torch.bfloat16)
    assert torch.equal(back[-50:], L.unpack_rows(q, torch.bfloat16)) and not back[:-50].any()
    w = L.pack_weights(torch.randn(k, 2056, device="cuda").bfloat16())
    y = L.linear8(p, w, dtype=torch.bfloat16)
    assert y.numel() > 1 << 31
    assert torch.equal(y[-50:], L.linear8(q, w, dtype=torch.bfloat16)) and not y[:-50].any()
