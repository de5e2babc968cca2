"""Rows past the threads that one axis of a grid holds."""
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2510_23621_amd.layers")


def test_rows_past_the_threads_of_one_axis():
    """2^32 vectors of 16 bytes and more, 69 GB of rows: one expert and one choice, so that
    every direction copies."""
    torch.cuda.empty_cache()
    n, width, part = (1 << 26) + 5, 512, 1 << 20
    p = L.route(torch.zeros(n, 1, dtype=torch.int32, device="cuda"), 1)
    base = torch.randn(part, width, device="cuda").bfloat16()

    def piece(i):
        return base[:min(part, n - i)] * (1 + i // part % 3)

    def check(t):
        for i in range(0, n, part):
            assert torch.equal(t[i:i + part], piece(i)), i
    x = torch.empty(n, width, dtype=torch.bfloat16, device="cuda")
    for i in range(0, n, part):
        x[i:i + part] = piece(i)
    rows = L.route_rows(x, p)
    del x
    check(rows)
    out = L.combine_rows(rows, p)
    del rows
    check(out)
    drows, _ = L.combine_rows_backward(out, out, p)
    del out
    check(drows)
    del drows
    torch.cuda.empty_cache()
