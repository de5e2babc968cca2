"""Newton-Schulz orthogonalisation of rank-deficient matrices over many steps.

In exact arithmetic a zero singular value stays zero; rounding puts something of
the order of the arithmetic's unit there, which every step multiplies by a
until it, too, reaches the plateau.  So the part of the result in the matrix's
own r left directions is compared with the iteration of those r rows alone, in
FP64, and the rest only has to stay on the plateau.

Bounds.  (1.5, -0.5, 0) converges to singular values of 1 and contracts errors
there, so an error is at most a start's 8 2^-23 times the growth 1.2 / s_min of
the smallest non-zero singular value (as in test_gpu_orthogonalise.py).  The
default steps neither converge nor contract on their plateau (slope up to 1.7
of 0.68 .. 1.13), so there, after the five to eight steps that reach it, only
the plateau itself is asked for: 0.6 to 1.25, and no more than 1.25 anywhere."""
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")
CLASSIC = (1.5, -0.5, 0.0)
DEFAULT = L.NEWTON_SCHULZ[0]


def deficient(kind, m, n, seed):
    """[2, m, n] FP32 matrices of rank below min(m, n), exactly representable rows."""
    gen = torch.Generator().manual_seed(seed)
    short = min(m, n)
    if kind == "two equal rows":
        r = short - 1
        g = torch.randn(2, r, max(m, n), generator=gen)
        g = torch.cat([g, g[:, :1]], 1)
    elif kind == "repeated rows":
        r = max(1, short // 3)
        g = torch.randn(2, r, max(m, n), generator=gen)[:, torch.arange(short) % r]
    else:   # a few rows, the others zero
        r = max(1, short // 3)
        g = torch.zeros(2, short, max(m, n))
        g[:, :r] = torch.randn(2, r, max(m, n), generator=gen)
    return (g if m <= n else g.transpose(1, 2).contiguous()), r


def iterate(x, coef):
    for a, b, c in coef:
        A = x @ x.t()
        x = a * x + (b * A + c * A @ A) @ x
    return x


SHAPES = [(24, 40), (40, 24), (5, 7), (16, 200), (32, 32), (12, 700), (700, 12), (48, 300), (300, 60), (64, 1280),
          (48, 48), (100, 70), (140, 200)]
KINDS = ["two equal rows", "repeated rows", "zero rows"]


@pytest.mark.parametrize("steps", [8, 16, 24, 40, 64])
@pytest.mark.parametrize("m,n", SHAPES)
@pytest.mark.parametrize("kind", KINDS)
def test_converging_steps(kind, m, n, steps):
    g, r = deficient(kind, m, n, m + n)
    out = L.orthogonalise(g.cuda(), (CLASSIC,) * steps, eps=0.0).cpu().double()
    assert torch.isfinite(out).all()
    for i in range(2):
        x, o = g[i].double(), out[i]
        if m > n:
            x, o = x.t(), o.t()
        u, s, _ = torch.linalg.svd(x, full_matrices=False)
        u, s = u[:, :r], s[:r] / torch.linalg.norm(s)
        want = iterate(u.t() @ x / torch.linalg.norm(x), (CLASSIC,) * steps)
        err = (torch.linalg.norm(u.t() @ o - want) / torch.linalg.norm(want)).item()
        assert err <= 8 * 2.0 ** -23 * 1.2 / s[-1].item(), (kind, i, err, s[-1].item())
        assert torch.linalg.svdvals(o)[0].item() <= 1.001


@pytest.mark.parametrize("steps", [8, 12, 16, 24, 64])
@pytest.mark.parametrize("m,n", SHAPES)
@pytest.mark.parametrize("kind", KINDS)
def test_default_steps_stay_on_their_plateau(kind, m, n, steps):
    g, r = deficient(kind, m, n, m + n)
    out = L.orthogonalise(g.cuda(), (DEFAULT,) * steps, eps=0.0).cpu().double()
    assert torch.isfinite(out).all()
    for i in range(2):
        x, o = g[i].double(), out[i]
        if m > n:
            x, o = x.t(), o.t()
        u = torch.linalg.svd(x, full_matrices=False)[0][:, :r]
        s = torch.linalg.svdvals(u.t() @ o)
        assert 0.6 <= s[-1].item() and torch.linalg.svdvals(o)[0].item() <= 1.25, (kind, i, s)
