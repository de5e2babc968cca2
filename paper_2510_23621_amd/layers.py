"""Dense operators on torch tensors: grouped linear layers, rows sorted by
expert and back, Newton-Schulz orthogonalisation, and the gradients of the
first two.  torch allocates results and workspaces, the library's kernels do
the work on ``stream`` (a torch.cuda.Stream; default: the current one).

Tensors are float32, bfloat16 or float16 on one GPU, whichever is current, and
``stream`` is one of that GPU's; rows may be strided (any row stride, columns
adjacent), and gradients handed to a backward function (dy, dout, drows) in any
order, at the price of a copy.  Tensors of another stream are the caller's to
order, as with any torch operation.  Nothing here records a graph for autograd:
the backward functions are called by the program, under torch.no_grad() or on
detached tensors, and tensors that ask for a gradient are refused otherwise.

The checks are written out in each function: a small layer's call is bound by
the host, and one costs about as much as its kernel.
"""
from __future__ import annotations

from functools import wraps
from typing import NamedTuple

import numpy as np
import torch

from . import binding as B

DTYPES = {torch.float32: B.MACE_TYPE_FP32, torch.bfloat16: B.MACE_TYPE_BF16, torch.float16: B.MACE_TYPE_FP16}
ACTIVATIONS = {"none": B.MACE_ACT_NONE, "silu": B.MACE_ACT_SILU, "gelu": B.MACE_ACT_GELU}
# a, b, c of five steps that bring singular values from about 0.01..1 to about 0.7..1.2: the
# ones published with the Muon optimiser (K. Jordan and others, 2024)
NEWTON_SCHULZ = ((3.4445, -4.7750, 2.0315),) * 5


def _streamed(f):
    """Runs f on the device of its first tensor, as the library launches on the
    current device, and with `stream` as the current stream, so that what it
    allocates belongs to the stream that uses it.  Refuses tensors that ask for
    a gradient: the result would have lost it without a word."""
    first = f.__code__.co_varnames[0]

    @wraps(f)
    def on(*args, stream=None, **kw):
        if torch.is_grad_enabled():
            for t in (*args, *kw.values()):
                if getattr(t, "requires_grad", False):
                    raise ValueError(f"{f.__name__} records no gradients: call it under torch.no_grad() or on "
                                     "detached tensors")
        device = (args[0] if args else kw[first]).get_device()   # (-1: a host tensor, which f refuses)
        if stream is not None:
            if stream.device.index != device:
                raise ValueError(f"stream is of device {stream.device}, {first} of {device}")
            with torch.cuda.stream(stream):   # (makes its device current, too)
                return f(*args, **kw)
        if device < 0 or device == torch._C._cuda_getDevice():
            return f(*args, **kw)
        with torch.cuda.device(device):
            return f(*args, **kw)
    return on


def _current_stream(t) -> int:
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _leading(t, name: str) -> int:
    """Leading dimension of a matrix, whose columns have to be adjacent."""
    n, c = t.shape
    if t.is_contiguous():
        return c
    s0, s1 = t.stride()
    if (s1 != 1 and c > 1 and n > 0) or (s0 < c and n > 1):
        raise ValueError(f"{name}'s columns must be adjacent and its rows apart")
    return s0 if n > 1 else c


def _gradient(t):
    """t as the kernels can read it: autograd hands on expanded and transposed gradients."""
    if t.is_contiguous() or t.dim() == 2 and t.stride(1) == 1 and t.stride(0) >= t.shape[1]:
        return t
    return t.contiguous()


def _rows(t, n: int, c: int, like, name: str) -> int:
    """Leading dimension of t, which has to be [n, c] and of like's dtype and device."""
    if t.shape != (n, c):
        raise ValueError(f"{name} must be {(n, c)}, not {tuple(t.shape)}")
    if t.dtype is not like.dtype or t.get_device() != like.get_device():
        raise ValueError(f"{name} must have the first tensor's dtype and device")
    return _leading(t, name)


def _whole(t, shape, dtype, like, name: str):
    if t.shape != shape or t.dtype is not dtype or t.get_device() != like.get_device() or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous {tuple(shape)} {dtype} on {like.device}")


def _too_large(name: str):
    # (the descriptors' fields have 32 bits and would wrap; what fits, the library itself takes or refuses)
    raise ValueError(f"{name} has more than 2^31 - 1 columns, groups or choices")


def _gpu_matrix(t, name: str) -> int:
    """The library's number of t's dtype; t has to be a matrix on a GPU."""
    dtype = DTYPES.get(t.dtype)
    if dtype is None or t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{name} must be a 2-d GPU tensor of float32, bfloat16 or float16")
    if t.shape[1] >> 31:
        _too_large(name)
    return dtype


def _linear_desc(x, w, offsets, act):
    dtype, a = _gpu_matrix(x, "x"), ACTIVATIONS.get(act)
    if a is None:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}")
    n, n_in = x.shape
    shape = w.shape
    if len(shape) == 3:
        groups, k, n_out = shape
    elif len(shape) == 2:
        groups, (k, n_out) = 1, shape
    else:
        raise ValueError("w must be [n_in, n_out] or [groups, n_in, n_out]")
    if k != n_in or w.dtype is not x.dtype or w.get_device() != x.get_device() or not w.is_contiguous():
        raise ValueError(f"w must be contiguous with {n_in} input rows, of x's dtype and device")
    if (groups | n_out) >> 31:
        _too_large("w")
    if offsets is not None:
        _whole(offsets, (groups + 1,), torch.int32, x, "offsets")
    elif groups != 1:
        raise ValueError("more than one group needs offsets")
    return B.mace_linear_desc(n, n_in, n_out, groups, dtype, a, _leading(x, "x"), n_out, n_out, n_out)


@_streamed
def linear(x, w, bias=None, residual=None, *, offsets=None, act: str = "none", save: bool = False):
    """y = act(x W_g + b_g) + residual for the rows offsets[g]:offsets[g+1] of
    each group g (int32 offsets on the device; None: one group).  Rows behind
    the last group give zeros.  With save, returns (y, z): z is what
    linear_backward needs, the value before the activation (None without one)."""
    d = _linear_desc(x, w, offsets, act)
    n, m = d.n_rows, d.n_out
    if bias is not None:
        _whole(bias, (*w.shape[:-2], m), x.dtype, x, "bias")
    if residual is not None:
        d.ld_residual = _rows(residual, n, m, x, "residual")
    y = x.new_empty((n, m))
    z = x.new_empty((n, m)) if save and d.act else None
    B._check(B.lib().mace_linear_forward(d, x.data_ptr(), w.data_ptr(), None if bias is None else bias.data_ptr(),
                                         None if residual is None else residual.data_ptr(),
                                         None if offsets is None else offsets.data_ptr(), y.data_ptr(),
                                         None if z is None else z.data_ptr(), _current_stream(x)),
             "mace_linear_forward")
    return (y, z) if save else y


@_streamed
def linear_backward(dy, x, w, z=None, *, offsets=None, act: str = "none", bias: bool = True, need_dx: bool = True,
                    need_dw: bool = True):
    """(dx, dw, db) of `linear` from dy; z as `linear` saved it.  The residual's
    gradient is dy itself.  bias, need_dx, need_dw: which ones are wanted (None
    in the others' places)."""
    d = _linear_desc(x, w, offsets, act)
    n, m = d.n_rows, d.n_out
    dy = _gradient(dy)
    ld_dy = _rows(dy, n, m, x, "dy")
    if d.act:
        if z is None:
            raise ValueError("an activation's gradient needs z")
        d.ld_preact = _rows(z, n, m, x, "z")
    else:
        z = None
    dx = x.new_empty((n, d.n_in)) if need_dx else None
    dw = torch.empty_like(w) if need_dw else None
    db = x.new_empty((*w.shape[:-2], m)) if bias else None
    lib = B.lib()
    # (0 for sizes the library does not take: the call itself says which error)
    nbytes = lib.mace_linear_backward_workspace_bytes(d, bias, need_dw) or 1
    ws = x.new_empty(nbytes, dtype=torch.uint8)
    B._check(lib.mace_linear_backward(d, dy.data_ptr(), ld_dy, x.data_ptr(), w.data_ptr(),
                                      None if z is None else z.data_ptr(),
                                      None if offsets is None else offsets.data_ptr(),
                                      None if dx is None else dx.data_ptr(), d.n_in,
                                      None if dw is None else dw.data_ptr(), None if db is None else db.data_ptr(),
                                      ws.data_ptr(), nbytes, _current_stream(x)), "mace_linear_backward")
    return dx, dw, db


class Route(NamedTuple):
    """Order of the (token, choice) slots sorted by expert (`route`)."""
    row_of_slot: torch.Tensor   # int32 [tokens, top_k]
    slot_of_row: torch.Tensor   # int32 [tokens * top_k], slot = token * top_k + choice
    offsets: torch.Tensor       # int32 [n_experts + 1]


@_streamed
def route(expert, n_experts: int) -> Route:
    """The stable sort of the slots of expert (int32 [tokens, top_k]) by expert;
    slots with an index outside 0..n_experts-1 are dropped, behind the others."""
    if expert.dim() != 2 or not expert.is_cuda or expert.dtype is not torch.int32 or not expert.is_contiguous():
        raise ValueError("expert must be a contiguous int32 [tokens, top_k] GPU tensor")
    n, k = expert.shape
    if k >> 31 or not -1 << 31 <= n_experts < 1 << 31:
        _too_large("expert")
    d = B.mace_route_desc(n, k, n_experts, 1, B.MACE_TYPE_FP32, 1, 1)
    lib = B.lib()
    s = n * k
    rows, slots = torch.empty_like(expert), expert.new_empty(s)
    offsets = expert.new_empty(max(n_experts, 0) + 1)
    nbytes = lib.mace_route_workspace_bytes(d) if s > 4096 else 0
    ws = expert.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    B._check(lib.mace_route_build(d, expert.data_ptr(), rows.data_ptr(), slots.data_ptr(), offsets.data_ptr(),
                                  None if ws is None else ws.data_ptr(), nbytes, _current_stream(expert)),
             "mace_route_build")
    return Route(rows, slots, offsets)


def _check_plan(plan: Route, like, weights=None):
    device, slots = like.get_device(), plan.row_of_slot.numel()
    for t in plan:
        if t.get_device() != device or t.dtype is not torch.int32 or not t.is_contiguous():
            raise ValueError(f"the plan's tensors must be contiguous int32 on {like.device}")
    if plan.slot_of_row.numel() != slots:
        raise ValueError(f"the plan's slot_of_row must have {slots} elements")
    if weights is not None:
        _whole(weights, plan.row_of_slot.shape, torch.float32, like, "weights")


@_streamed
def route_rows(x, plan: Route):
    """[tokens * top_k, width] rows in expert order; zeros for dropped slots."""
    dtype = _gpu_matrix(x, "x")
    n, k = plan.row_of_slot.shape
    tokens, width = x.shape
    if tokens != n:
        raise ValueError(f"x must have {n} rows, not {tokens}")
    _check_plan(plan, x)
    ld = _leading(x, "x")
    d = B.mace_route_desc(n, k, plan.offsets.shape[0] - 1, width, dtype, ld, width)
    rows = x.new_empty((n * k, width))
    B._check(B.lib().mace_route_gather(d, x.data_ptr(), plan.slot_of_row.data_ptr(), plan.offsets.data_ptr(),
                                       rows.data_ptr(), _current_stream(x)), "mace_route_gather")
    return rows


@_streamed
def combine_rows(rows, plan: Route, weights=None):
    """[tokens, width]: each token's kept rows times their weights (float32
    [tokens, top_k], None: ones), summed."""
    return _combine(rows, plan, weights)


def _combine(rows, plan: Route, weights=None):
    dtype = _gpu_matrix(rows, "rows")
    n, k = plan.row_of_slot.shape
    slots, width = rows.shape
    if slots != n * k:
        raise ValueError(f"rows must have {n * k} rows, not {slots}")
    ld = _leading(rows, "rows")
    _check_plan(plan, rows, weights)
    d = B.mace_route_desc(n, k, plan.offsets.shape[0] - 1, width, dtype, width, ld)
    out = rows.new_empty((n, width))
    B._check(B.lib().mace_route_combine(d, rows.data_ptr(), None if weights is None else weights.data_ptr(),
                                        plan.row_of_slot.data_ptr(), plan.offsets.data_ptr(), out.data_ptr(),
                                        _current_stream(rows)), "mace_route_combine")
    return out


@_streamed
def combine_rows_backward(dout, rows, plan: Route, weights=None):
    """(drows, dweights) of `combine_rows`; dweights is None without weights."""
    dout = _gradient(dout)
    dtype = _gpu_matrix(dout, "dout")
    n, k = plan.row_of_slot.shape
    tokens, width = dout.shape
    if tokens != n:
        raise ValueError(f"dout must have {n} rows, not {tokens}")
    ld = _leading(dout, "dout")
    ld_rows = _rows(rows, n * k, width, dout, "rows")
    _check_plan(plan, dout, weights)
    drows = dout.new_empty((n * k, width))
    dw = None if weights is None else torch.empty_like(weights)
    lib, stream = B.lib(), _current_stream(dout)

    def call(ld_rows, drows, dw):   # (the library takes one leading dimension for rows and their gradient)
        d = B.mace_route_desc(n, k, plan.offsets.shape[0] - 1, width, dtype, ld, ld_rows)
        B._check(lib.mace_route_combine_backward(d, dout.data_ptr(), rows.data_ptr(),
                                                 None if weights is None else weights.data_ptr(),
                                                 plan.row_of_slot.data_ptr(), plan.offsets.data_ptr(),
                                                 None if drows is None else drows.data_ptr(),
                                                 None if dw is None else dw.data_ptr(), stream),
                 "mace_route_combine_backward")
    if ld_rows == width or dw is None:   # (without weights' gradients the rows are not read)
        call(width, drows, dw)
    else:
        call(ld_rows, None, dw)
        call(width, drows, None)
    return drows, dw


@_streamed
def route_rows_backward(drows, plan: Route):
    """Gradient of `route_rows` with respect to x."""
    return _combine(_gradient(drows), plan)


def _coefficients(steps) -> np.ndarray:
    """float64 [n, 3] on the host."""
    if not hasattr(steps, "__len__"):
        steps = list(steps)
    if len(steps) == 0:
        return np.empty((0, 3))
    try:
        coef = np.array(steps, dtype=np.float64, order="C")
    except ValueError:   # (of different lengths)
        coef = None
    if coef is None or coef.ndim != 2 or coef.shape[1] != 3:
        raise ValueError("coefficients must be triples (a, b, c), one per step")
    return coef


@_streamed
def orthogonalise(g, coefficients=NEWTON_SCHULZ, *, eps: float = 1e-7):
    """Newton-Schulz steps (a, b, c) on g / (|g|_F + eps), x <- a x + (b A + c A A) x
    with A = x x^T: [rows, cols] or a batch [batch, rows, cols], columns adjacent."""
    dtype = DTYPES.get(g.dtype)
    if dtype is None or g.dim() not in (2, 3) or not g.is_cuda:
        raise ValueError("g must be a [(batch,) rows, cols] GPU tensor of float32, bfloat16 or float16")
    coef = _coefficients(coefficients)
    if g.dim() == 3:
        (b, rows, cols), (sb, s0, s1) = g.shape, g.stride()
    else:
        (rows, cols), (s0, s1), b, sb = g.shape, g.stride(), 1, 0
    if (s1 != 1 and cols > 1 or s0 < cols and rows > 1 or sb < 0) and g.numel():
        raise ValueError("g's columns must be adjacent and its rows apart")
    if (rows | cols) >> 31:
        _too_large("g")
    d = B.mace_orthogonalise_desc(b, rows, cols, dtype, len(coef), s0 if rows > 1 else cols, sb, cols, rows * cols, eps)
    out = g.new_empty(g.shape)
    lib = B.lib()
    nbytes = lib.mace_orthogonalise_workspace_bytes(d) or 1
    ws = g.new_empty(nbytes, dtype=torch.uint8)
    B._check(lib.mace_orthogonalise(d, g.data_ptr(), coef.ctypes.data, out.data_ptr(), ws.data_ptr(), nbytes,
                                    _current_stream(g)), "mace_orthogonalise")
    return out
