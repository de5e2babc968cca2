"""The combine's gradient of rows that are a few columns of a wide tensor."""
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")


def test_gradient_of_strided_rows_is_no_wider_than_the_rows():
    """Rows that are a few columns of a wide tensor: their gradient takes the columns only."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    e = torch.randint(-1, 5, (300, 2), generator=gen, device="cuda", dtype=torch.int32)
    p, w = L.route(e, 5), torch.rand(300, 2, generator=gen, device="cuda")
    dout = torch.randn(300, 16, generator=gen, device="cuda")
    wide = torch.randn(600, 5000, generator=gen, device="cuda")
    for rows in (wide[:, 8:24], wide[:, 3:19]):
        for weights in (w, None):
            drows, dw = L.combine_rows_backward(dout, rows, p, weights)
            assert drows.is_contiguous() and drows.untyped_storage().nbytes() == 600 * 16 * 4
            want = L.combine_rows_backward(dout, rows.contiguous(), p, weights)
            assert torch.equal(drows, want[0]) and (dw is None if weights is None else torch.equal(dw, want[1]))
