"""Activations over the whole range of the types, infinities among them, in each
kernel that applies one: the value of the definition (NaN where that is
inf / inf or -inf 0), to 2^-20 relative and 2^-120 absolute (below z = -88 SiLU
is under 2^-120; 2^-20 is above the activations' 2e-7 and FP32's own rounding),
and one rounding to the type."""
import math

import pytest
import torch

from dense_common import DTYPES, TINY, U, act64

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")
INF = math.inf
VALUES = [INF, 3.2e38, 2.4e38, 2.3e38, 1e38, 1e20, 6e4, 300.0, 100.0, 89.0, 88.0, 87.0, 30.0, 10.0, 1.0, 0.0, -1.0, -10.0,
          -30.0, -80.0, -87.0, -88.0, -89.0, -100.0, -300.0, -6e4, -1e20, -1e37, -1e38, -3.2e38]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n,m", [(30, 3), (30, 128), (3000, 520), (300000, 128)])   # thin or small tiles, tiles, streamed rows
def test_values(n, m, dtype, act):
    t = DTYPES[dtype]
    x = torch.tensor(VALUES).to(t)
    if dtype == "fp32" and n > 30:   # (infinite FP32 operands are split to NaN there)
        x[0] = 3.3e38
    x = x.repeat(n // len(VALUES))[:, None].cuda()
    y, z = L.linear(x, torch.ones(1, m, dtype=t, device="cuda"), act=act, save=True)
    want_z = x.cpu().double()
    assert torch.equal(z.cpu().double(), want_z.expand(-1, m))
    want = act64(want_z, act)
    got = y.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want).expand(-1, m))
    inf = torch.isinf(want)[:, 0]
    assert torch.equal(got[inf], want[inf].expand(-1, m))
    ok = torch.isfinite(want)[:, 0]
    bound = (2.0 ** -20 + U[dtype]) * want.abs() + max(2.0 ** -120, TINY[dtype])
    over = ((got - want).abs() - bound)[ok]
    assert over.max().item() <= 0, x[ok][int(over.argmax()) // m]


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_minus_infinity_is_as_the_definition_has_it(act):
    x = torch.tensor([[-INF]], device="cuda")
    assert torch.isnan(act64(x.cpu().double(), act)).all()
    for t in (torch.float32, torch.bfloat16, torch.float16):
        assert torch.isnan(L.linear(x.to(t), torch.ones(1, 16, dtype=t, device="cuda"), act=act)).all()
