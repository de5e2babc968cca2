"""8-bit rows at FP32's largest numbers: what is finite comes back finite."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")
LARGEST = 3.4028234663852886e38


@pytest.mark.parametrize("columns", [1, 40, 5000, 9000])
def test_largest_numbers(columns):
    """127 times the scale is a number: the quotient by 127 rounded to nearest would give infinity."""
    x = torch.zeros(4, columns)
    x[0, 0], x[1, -1] = LARGEST, -LARGEST
    x[2, 0] = float(np.nextafter(np.float32(LARGEST), np.float32(0)))
    x[3, 0] = 3.4e38
    p = L.pack_rows(x.cuda())
    got = L.unpack_rows(p).cpu()
    assert torch.isfinite(got).all()
    # within half a step of 1 / 254 and the scale's rounding
    assert ((got.double() - x.double()).abs() <= x.double().abs().max(1, keepdim=True).values * (1 / 254 + 2.0 ** -22)).all()
    assert torch.equal(got[:, 1:-1], x[:, 1:-1])
    w = L.pack_weights(x.t().contiguous().cuda())
    assert torch.equal(w.values[0], p.values) and torch.equal(w.scales[0], p.scales)
    # the layer at these rows (an FP32 product's operands end at 2^128 (1 - 2^-9): no gradients here)
    one = L.pack_weights(torch.full((columns, 2), 2.0 ** -20, device="cuda"))
    want = (p.values[:, :columns].double() * p.scales.double()[:, None]).sum(1, keepdim=True) * 2.0 ** -20
    y = L.linear8(x.cuda(), one)
    assert ((y.double() - want).abs() <= 2.0 ** -21 * want.abs()).all()
