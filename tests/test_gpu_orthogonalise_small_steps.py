"""Steps that shrink every singular value, and steps that grow them again."""
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")


@pytest.mark.parametrize("m,n", [(24, 40), (48, 300), (100, 100), (140, 300)])
@pytest.mark.parametrize("steps", [((2.0 ** -12, 0.0, 0.0), (2.0 ** 12, 0.0, 0.0)), ((0.05, 0.0, 0.0), (1.5, -0.5, 0.0)),
                                   ((2.0 ** -10, 0.0, 0.0), (300.0, -1e6, 0.0)), ((1.5, -0.5, 0.0), (2.0 ** -14, 0.0, 0.0)),
                                   ((0.0, 0.0, 0.0), (3.0, 0.0, 0.0)), ((0.0, 0.01, 0.0),),
                                   ((0.0, 1e-8, 0.0),), ((2.0 ** -20, 0.0, 0.0), (2.0 ** 20, 0.0, 0.0)),
                                   ((2.0 ** -10, 0.0, 0.0), (0.0, 1e8, 0.0))], ids=str)
def test_against_fp64(steps, m, n):
    """Bound: 8 2^-22 (a pair's digits and FP32 sums, per element) of the norm that the steps'
    largest singular value could have, |g|_F = 1 times the largest |P(s^2)| of each step."""
    gen = torch.Generator().manual_seed(m)
    g = torch.randn(2, m, n, generator=gen)
    out = L.orthogonalise(g.cuda(), steps).cpu().double()
    for i in range(2):
        x = g[i].double() / torch.linalg.norm(g[i].double())
        scale, top = 1.0, 1.0
        for a, b, c in steps:
            grid = torch.linspace(0, top * top, 10001, dtype=torch.float64)
            p = (a + b * grid + c * grid * grid).abs()
            scale, top = scale * p.max().item(), (p * grid.sqrt()).max().item()
            A = x @ x.t()
            x = a * x + (b * A + c * A @ A) @ x
        assert torch.linalg.norm(out[i] - x) <= 8 * 2.0 ** -22 * scale, (torch.linalg.norm(out[i] - x), scale)


def test_few_rows_take_any():
    g = torch.randn(2, 20, 50).cuda()
    out = L.orthogonalise(g, ((2.0 ** -20, 0.0, 0.0), (2.0 ** 20, 0.0, 0.0)))
    want = g / torch.linalg.norm(g, dim=(1, 2), keepdim=True)
    assert torch.allclose(out, want, rtol=1e-6, atol=0)
