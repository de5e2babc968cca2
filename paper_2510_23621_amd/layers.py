"""Dense operators on torch tensors: grouped linear layers, rows sorted by
expert and back, Newton-Schulz orthogonalisation, and the gradients of the
first two.  torch allocates results and workspaces, the library's kernels do
the work on ``stream`` (default: the current one).

Tensors are float32, bfloat16 or float16 on one GPU; rows may be strided
(any row stride, columns adjacent).  Tensors of another stream are the
caller's to order, as with any torch operation.
"""
from __future__ import annotations

from contextlib import nullcontext
from typing import NamedTuple

import numpy as np
import torch

from . import binding as B

DTYPES = {torch.float32: B.MACE_TYPE_FP32, torch.bfloat16: B.MACE_TYPE_BF16, torch.float16: B.MACE_TYPE_FP16}
ACTIVATIONS = {"none": B.MACE_ACT_NONE, "silu": B.MACE_ACT_SILU, "gelu": B.MACE_ACT_GELU}
# a, b, c of five steps that bring singular values from about 0.01..1 to about 0.7..1.2
NEWTON_SCHULZ = ((3.4445, -4.7750, 2.0315),) * 5


def _on(stream):
    """Allocations belong to the stream that uses them."""
    return nullcontext() if stream is None else torch.cuda.stream(stream)


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _rows(t, name: str, shape, like) -> int:
    """Leading dimension of a [rows, columns] tensor, after checking it."""
    _need(tuple(t.shape) == tuple(shape), f"{name} must be {tuple(shape)}, not {tuple(t.shape)}")
    _need(t.dtype == like.dtype and t.device == like.device, f"{name} must have x's dtype and device")
    n, c = shape
    if n == 0:
        return c
    s = t.stride()
    if n == 1:
        _need(c == 1 or s[1] == 1, f"{name}'s columns must be adjacent")
        return c
    _need((c == 1 or s[1] == 1) and s[0] >= c, f"{name}'s columns must be adjacent and its rows apart")
    return s[0]


def _whole(t, name: str, shape, dtype, device):
    _need(tuple(t.shape) == tuple(shape) and t.dtype == dtype and t.device == device and t.is_contiguous(),
          f"{name} must be contiguous {tuple(shape)} {dtype} on {device}")


def _linear_desc(x, w, bias, offsets, act):
    _need(x.dim() == 2 and x.is_cuda and x.dtype in DTYPES, "x must be a [rows, n_in] GPU tensor of a supported dtype")
    _need(act in ACTIVATIONS, f"act must be one of {sorted(ACTIVATIONS)}")
    _need(w.dim() in (2, 3), "w must be [n_in, n_out] or [groups, n_in, n_out]")
    n, n_in = x.shape
    groups, n_out = (1 if w.dim() == 2 else w.shape[0]), w.shape[-1]
    _whole(w, "w", (*w.shape[:-2], n_in, n_out), x.dtype, x.device)
    if bias is not None:
        _whole(bias, "bias", (*w.shape[:-2], n_out), x.dtype, x.device)
    if offsets is not None:
        _whole(offsets, "offsets", (groups + 1,), torch.int32, x.device)
    else:
        _need(groups == 1, "more than one group needs offsets")
    d = B.mace_linear_desc(n, n_in, n_out, groups, DTYPES[x.dtype], ACTIVATIONS[act], _rows(x, "x", x.shape, x), n_out,
                           n_out, n_out)
    return d


def linear(x, w, bias=None, residual=None, *, offsets=None, act: str = "none", save: bool = False, stream=None):
    """y = act(x W_g + b_g) + residual for the rows offsets[g]:offsets[g+1] of
    each group g (int32 offsets on the device; None: one group).  Rows behind
    the last group give zeros.  With save, returns (y, z): z is what
    linear_backward needs, the value before the activation (None without one)."""
    d = _linear_desc(x, w, bias, offsets, act)
    shape = (d.n_rows, d.n_out)
    if residual is not None:
        d.ld_residual = _rows(residual, "residual", shape, x)
    with _on(stream):
        y = torch.empty(shape, dtype=x.dtype, device=x.device)
        z = torch.empty(shape, dtype=x.dtype, device=x.device) if save and act != "none" else None
        B.mace_linear_forward(d, x, w, bias, residual, offsets, y, z, stream)
    return (y, z) if save else y


def linear_backward(dy, x, w, z=None, *, offsets=None, act: str = "none", bias: bool = True, need_dx: bool = True,
                    need_dw: bool = True, stream=None):
    """(dx, dw, db) of `linear` from dy; z as `linear` saved it.  The residual's
    gradient is dy itself.  bias, need_dx, need_dw: which ones are wanted (None
    in the others' places)."""
    d = _linear_desc(x, w, None, offsets, act)
    shape = (d.n_rows, d.n_out)
    ld_dy = _rows(dy, "dy", shape, x)
    if act != "none":
        _need(z is not None, "an activation's gradient needs z")
        d.ld_preact = _rows(z, "z", shape, x)
    with _on(stream):
        dx = torch.empty((d.n_rows, d.n_in), dtype=x.dtype, device=x.device) if need_dx else None
        dw = torch.empty_like(w) if need_dw else None
        db = torch.empty((*w.shape[:-2], d.n_out), dtype=x.dtype, device=x.device) if bias else None
        nbytes = B.mace_linear_backward_workspace_bytes(d, bias, need_dw)
        if nbytes == 0:   # sizes the library does not take: the call itself says which way
            nbytes = 1
        ws = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
        B.mace_linear_backward(d, dy, ld_dy, x, w, z, offsets, dx, d.n_in, dw, db, ws, nbytes, stream)
    return dx, dw, db


class Route(NamedTuple):
    """Order of the (token, choice) slots sorted by expert (`route`)."""
    row_of_slot: torch.Tensor   # int32 [tokens, top_k]
    slot_of_row: torch.Tensor   # int32 [tokens * top_k], slot = token * top_k + choice
    offsets: torch.Tensor       # int32 [n_experts + 1]


def route(expert, n_experts: int, *, stream=None) -> Route:
    """The stable sort of the slots of expert (int32 [tokens, top_k]) by expert;
    slots with an index outside 0..n_experts-1 are dropped, behind the others."""
    _need(expert.dim() == 2 and expert.is_cuda, "expert must be a [tokens, top_k] GPU tensor")
    _whole(expert, "expert", expert.shape, torch.int32, expert.device)
    n, k = expert.shape
    d = B.mace_route_desc(n, k, n_experts, 1, B.MACE_TYPE_FP32, 1, 1)
    with _on(stream):
        # one allocation: the orders, the offsets
        buf = torch.empty(2 * n * k + n_experts + 1, dtype=torch.int32, device=expert.device)
        r = Route(buf[:n * k].view(n, k), buf[n * k:2 * n * k], buf[2 * n * k:])
        nbytes = B.mace_route_workspace_bytes(d) if n * k > 4096 else 0
        ws = torch.empty(nbytes, dtype=torch.uint8, device=expert.device) if nbytes else None
        B.mace_route_build(d, expert, r.row_of_slot, r.slot_of_row, r.offsets, ws, nbytes, stream)
    return r


def _route_desc(plan: Route, t, name: str, rows: bool):
    _need(t.dim() == 2 and t.is_cuda and t.dtype in DTYPES, f"{name} must be a 2-d GPU tensor of a supported dtype")
    n, k = plan.row_of_slot.shape
    ld = _rows(t, name, (n * k if rows else n, t.shape[1]), t)
    width = t.shape[1]
    return B.mace_route_desc(n, k, plan.offsets.shape[0] - 1, width, DTYPES[t.dtype], width if rows else ld,
                             ld if rows else width)


def _weights(weights, plan: Route):
    if weights is not None:
        _whole(weights, "weights", plan.row_of_slot.shape, torch.float32, plan.row_of_slot.device)


def route_rows(x, plan: Route, *, stream=None):
    """[tokens * top_k, width] rows in expert order; zeros for dropped slots."""
    d = _route_desc(plan, x, "x", False)
    with _on(stream):
        rows = torch.empty((plan.slot_of_row.shape[0], d.width), dtype=x.dtype, device=x.device)
        B.mace_route_gather(d, x, plan.row_of_slot, plan.offsets, rows, stream)
    return rows


def combine_rows(rows, plan: Route, weights=None, *, stream=None):
    """[tokens, width]: each token's kept rows times their weights (float32
    [tokens, top_k], None: ones), summed."""
    d = _route_desc(plan, rows, "rows", True)
    _weights(weights, plan)
    with _on(stream):
        out = torch.empty((d.n_tokens, d.width), dtype=rows.dtype, device=rows.device)
        B.mace_route_combine(d, rows, weights, plan.row_of_slot, plan.offsets, out, stream)
    return out


def combine_rows_backward(dout, rows, plan: Route, weights=None, *, stream=None):
    """(drows, dweights) of `combine_rows`; dweights is None without weights."""
    d = _route_desc(plan, dout, "dout", False)
    _weights(weights, plan)
    d.ld_rows = _rows(rows, "rows", (d.n_tokens * d.top_k, d.width), dout)
    with _on(stream):
        # rows and their gradient share a leading dimension
        buf = torch.empty((d.n_tokens * d.top_k, d.ld_rows), dtype=dout.dtype, device=dout.device)
        drows = buf if d.ld_rows == d.width else buf[:, :d.width]
        dw = None if weights is None else torch.empty_like(weights)
        B.mace_route_combine_backward(d, dout, rows, weights, plan.row_of_slot, plan.offsets, drows, dw, stream)
    return drows, dw


def route_rows_backward(drows, plan: Route, *, stream=None):
    """Gradient of `route_rows` with respect to x."""
    return combine_rows(drows, plan, None, stream=stream)


def orthogonalise(g, coefficients=NEWTON_SCHULZ, *, eps: float = 1e-7, stream=None):
    """Newton-Schulz steps (a, b, c) on g / (|g|_F + eps), x <- a x + (b A + c A A) x
    with A = x x^T: [rows, cols] or a batch [batch, rows, cols], columns adjacent."""
    _need(g.dim() in (2, 3) and g.is_cuda and g.dtype in DTYPES,
          "g must be a [(batch,) rows, cols] GPU tensor of a supported dtype")
    coef = np.ascontiguousarray(coefficients, dtype=np.float64).reshape(-1, 3)
    m = g if g.dim() == 3 else g[None]
    b, rows, cols = m.shape
    if m.numel() and not ((cols == 1 or m.stride(2) == 1) and (rows == 1 or m.stride(1) >= cols) and m.stride(0) >= 0):
        raise ValueError("g's columns must be adjacent and its rows apart")
    d = B.mace_orthogonalise_desc(b, rows, cols, DTYPES[g.dtype], len(coef), m.stride(1) if rows > 1 else cols,
                                  m.stride(0), cols, rows * cols, eps)
    with _on(stream):
        out = torch.empty(g.shape, dtype=g.dtype, device=g.device)
        nbytes = B.mace_orthogonalise_workspace_bytes(d) or 1
        ws = torch.empty(nbytes, dtype=torch.uint8, device=g.device)
        B.mace_orthogonalise(d, m, coef, out, ws, nbytes, stream)
    return out
