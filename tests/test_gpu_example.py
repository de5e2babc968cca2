"""The distillation example trains: its routed student explains most of the
variance of the teacher's energies within a few steps, on finite gradients that
agree with differences of the loss."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_student_learns():
    import distil_head
    first, last = distil_head.train(60, log=lambda *a, **k: None)
    assert last < 0.25 * first and last < 0.25, (first, last)


def test_gradients_of_the_whole_step():
    """Central differences along a random direction of every parameter. The choice
    of experts must not change between the three evaluations; h = 1e-3 leaves FP32
    rounding (1e-7 / h) and truncation (h^2) below 2 % of the slope."""
    import distil_head as D
    gen = torch.Generator().manual_seed(3)
    x, y = torch.randn(200, 20, generator=gen).cuda(), torch.randn(200, 1, generator=gen).cuda()
    p = D.init(20)
    p["router.w"] *= 20   # well separated choices
    _, g = D.step(p, x, y)
    for k in p:
        v = torch.randn(p[k].shape, generator=gen).cuda()
        h = 1e-3
        plus, _ = D.step({**p, k: p[k] + h * v}, x, y)
        minus, _ = D.step({**p, k: p[k] - h * v}, x, y)
        slope = (plus.double() - minus.double()).item() / (2 * h)
        got = (g[k].double() * v.double()).sum().item()
        scale = (g[k].double().norm() * v.double().norm() / v.numel() ** 0.5).item()
        assert abs(got - slope) <= 0.02 * abs(slope) + 0.02 * scale, (k, got, slope, scale)
