"""Shared pieces of the dense operators' tests: unit roundoffs, FP64 forms of
the activations, and the elementwise bound of a product's error."""
import math

import torch

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
U = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}   # relative error of one rounding
U32 = 2.0 ** -24
TINY = {"fp32": 2.0 ** -126, "bf16": 2.0 ** -126, "fp16": 2.0 ** -24}   # absolute error of one rounding near zero
SLOPE2 = 0.8   # bound of |silu''| (0.5) and |gelu''| (0.798)
SLOPE1 = 1.13   # bound of |silu'| (1.0999) and |gelu'| (1.129)


def randn(*shape, gen, dtype, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(DTYPES[dtype])


def act64(z, act):
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2))
    return z


def slope64(z, act):
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s + z * s * (1 - s)
    if act == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def product_error(a, b, length):
    """Bound of |fl(a @ b) - a @ b|: `length` FP32 additions and products in any
    order, and the split products' dropped terms (below two FP32 roundings)."""
    return (length + 8) * U32 * (a.abs() @ b.abs())


def within(got, want, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.isfinite(got).all(), f"{what}: non-finite"
    over = (got - want).abs() - bound
    worst = over.max().item() if over.numel() else -1.0
    assert worst <= 0, f"{what}: error exceeds its bound by {worst:.3e} at {int(over.argmax())} of {tuple(want.shape)}"
