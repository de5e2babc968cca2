"""The wide tiles of the linear layers and of the iteration, at sizes that no
tile divides: more than 256 blocks of 128 x 128, or 192 of 256 x 256."""
import pytest
import torch

from dense_common import DTYPES
from test_gpu_linear_layers import case

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")


# forward and dx as 256 x 256 tiles (25 x 9 of them) or 128 x 128 (40 x 9), operands
# at any alignment, dW in 256 x 256 over ten splits
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n,n_in,n_out", [(6200, 136, 2056), (6200, 2056, 136), (6203, 137, 2051), (5000, 136, 1100),
                                          (5000, 1104, 136), (5001, 1101, 135), (5400, 520, 2056)])
def test_linear(n, n_in, n_out, dtype):
    case(n, n_in, n_out, dtype, "silu", seed=n_in)


GROUPS = [513, 700, 1027, 600, 0, 1300, 899, 1161]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n_in,n_out", [(136, 2056), (2056, 136), (129, 2050)])
def test_groups(n_in, n_out, dtype):
    case(None, n_in, n_out, dtype, "gelu", GROUPS, 65, seed=n_in)


def test_strided_rows():
    for dtype in ("bf16", "fp16"):
        case(6200, 136, 2056, dtype, "silu", pad=16, shift=8, seed=3)
        case(6200, 2056, 136, dtype, "none", pad=8, seed=4)


# half-wide and 128 x 128 blocks of the symmetric products, the last ones short
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("b,m,n", [(65, 211, 300), (65, 300, 211), (30, 300, 515), (130, 200, 260), (130, 260, 200),
                                   (7, 520, 1100), (1, 2900, 2905)])
def test_orthogonalise(b, m, n, dtype):
    """Every matrix against the iteration in FP64. Bound on |out - ref|_F / |ref|_F:
    8 2^-23 a^5 for FP32's arithmetic (errors grow as the weakest direction does, at most
    a^5 = 484), and one rounding to the type, 2^-8 and 2^-11 at most."""
    gen = torch.Generator(device="cuda").manual_seed(b + m)
    r = min(m, n) // 4
    g = torch.randn(b, m, r, generator=gen, device="cuda") @ torch.randn(b, r, n, generator=gen, device="cuda") * r ** -0.5
    g = ((g + 0.3 * torch.randn(b, m, n, generator=gen, device="cuda")) * 0.01).to(DTYPES[dtype])
    out = L.orthogonalise(g)
    tol = 8 * 2.0 ** -23 * 3.4445 ** 5 + {"fp32": 0.0, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[dtype]
    for i in range(b):
        x = g[i].double()
        x = x / (torch.linalg.norm(x) + 1e-7)
        x = x.t().contiguous() if m > n else x
        for ca, cb, cc in L.NEWTON_SCHULZ:
            A = x @ x.t().contiguous()
            x = ca * x + (cb * A + cc * (A @ A)) @ x
        x = x.t() if m > n else x
        err = (torch.linalg.norm(out[i].double() - x) / torch.linalg.norm(x)).item()
        assert err <= tol, (i, err, tol)
