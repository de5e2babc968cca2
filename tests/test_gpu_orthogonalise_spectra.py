"""Newton-Schulz orthogonalisation to the accuracy of the result's type, whatever
the matrix's spectrum and the schedule.

Bound, on |out - ref|_F: the error of rounding the FP64 reference to the type
(of which the kernel's own rounding differs only where its value crosses to the
next number: 10 % of it), and an error of FP32 arithmetic, 8 2^-23 |ref|_F times
the growth min(prod a, 1.2 / s_min) of an error in the weakest direction (as in
test_gpu_orthogonalise.py)."""
import math

import pytest
import torch

from dense_common import DTYPES

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")


def matrix(kind, m, n, seed=0):
    gen = torch.Generator().manual_seed(seed)
    g = torch.randn(m, n, generator=gen)
    if kind == "repeated rows":
        g = g[torch.arange(m) % (m // 4)]
    elif kind == "block":   # only 8 x 8 non-zero
        g[8:] = 0
        g[:, 8:] = 0
    elif kind == "strong rows":   # above weak noise
        g[8:] *= 1e-4
    elif kind == "scaled":   # rows and columns of different scales
        g = g * torch.exp(torch.randn(m, 1, generator=gen)) * torch.exp(torch.randn(1, n, generator=gen))
    return g


def check(g, dtype, coef):
    g = g.to(DTYPES[dtype])
    out = L.orthogonalise(g.cuda(), coef).double()
    x = g.cuda().double()
    x = x / (torch.linalg.norm(x) + 1e-7)
    s = torch.linalg.svdvals(x.cpu())
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    for a, b, c in coef:
        A = x @ x.t().contiguous()
        x = a * x + (b * A + c * A @ A) @ x
    ref = x.t() if tall else x
    rounding = torch.linalg.norm(ref.to(DTYPES[dtype]).double() - ref).item()
    growth = min(math.prod(c[0] for c in coef), 1.2 / max(s[-1].item(), 1e-12))
    bound = 1.1 * rounding + 8 * 2.0 ** -23 * max(growth, 1.0) * torch.linalg.norm(ref).item()
    err = torch.linalg.norm(out - ref).item()
    assert err <= bound, (err, rounding, bound)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("kind,m,n", [("repeated rows", 512, 512), ("block", 129, 129), ("strong rows", 200, 256),
                                      ("scaled", 128, 256), ("scaled", 515, 300), ("gaussian", 128, 2048),
                                      ("gaussian", 300, 140)])
def test_spectra(kind, m, n, dtype):
    check(matrix(kind, m, n), dtype, L.NEWTON_SCHULZ)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("coef", [L.NEWTON_SCHULZ * 2, L.NEWTON_SCHULZ[:3], ((1.5, -0.5, 0.0),) * 12,
                                  ((2.0, -1.5, 0.5),) * 6, ((0.5, 0.0, 0.0),) * 3], ids=str)
def test_schedules(coef, dtype):
    check(matrix("gaussian", 128, 256, 1), dtype, coef)
