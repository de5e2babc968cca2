"""Dense operators on torch tensors: grouped linear layers, embeddings, the
choice of experts, rows sorted by expert and back, Newton-Schulz
orthogonalisation, and the gradients of all but the last; linear layers served
in 8 bits, and their gradients from activations kept in 8 bits.  torch allocates
results and workspaces, the library's kernels do the work on ``stream`` (a
torch.cuda.Stream; default: the current one).

Tensors are float32, bfloat16 or float16 on one GPU, whichever is current, and
``stream`` is one of that GPU's; rows may be strided (any row stride, columns
adjacent), and gradients handed to a backward function (dy, dout, drows, dweights) in any
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
SCORES = {"softmax": B.MACE_SCORES_SOFTMAX, "sigmoid": B.MACE_SCORES_SIGMOID}
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
    packed = any("Rows8" in a or "Weights8" in a for a in f.__annotations__.values())   # (tuples of tensors)

    @wraps(f)
    def on(*args, stream=None, **kw):
        if torch.is_grad_enabled():
            for t in (*args, *kw.values()):
                if getattr(t, "requires_grad", False) or packed and isinstance(t, tuple) and any(
                        getattr(u, "requires_grad", False) for u in t):
                    raise ValueError(f"{f.__name__} records no gradients: call it under torch.no_grad() or on "
                                     "detached tensors")
        t = args[0] if args else kw[first]
        device = (t[0] if packed and isinstance(t, tuple) else t).get_device()   # (-1: a host tensor, which f refuses)
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


class Choice(NamedTuple):
    """The experts of each token, best first, and their weights (`choose_experts`)."""
    expert: torch.Tensor    # int32 [tokens, top_k], -1 where fewer are left
    weights: torch.Tensor   # float32 [tokens, top_k]


def _choose_desc(logits, top_k, groups, top_groups, scores, normalise, scale):
    dtype, kind = _gpu_matrix(logits, "logits"), SCORES.get(scores)
    if kind is None:
        raise ValueError(f"scores must be one of {sorted(SCORES)}")
    n, e = logits.shape
    for v in (top_k, groups, top_groups):
        if not 0 < v < 1 << 31:
            raise ValueError("top_k, groups and top_groups must be positive 32-bit integers")
    return B.mace_choose_desc(n, e, top_k, groups, top_groups, dtype, kind, bool(normalise), _leading(logits, "logits"), scale)


@_streamed
def choose_experts(logits, top_k: int, *, bias=None, scores: str = "softmax", groups: int = 1, top_groups: int | None = None,
                   normalise: bool = True, scale: float = 1.0) -> Choice:
    """The top_k experts of each token by score + bias and their weights, scale
    times the scores (softmax or sigmoid of logits [tokens, experts]), divided by
    the chosen ones' sum if `normalise`.  bias (float32 [experts]) sways the
    choice only.  groups: runs of experts of which the top_groups (default: all)
    with the largest sums of their two best take part.  Equal ones go by the
    lower index.  A logit of -infinity or the type's lowest value masks its
    expert; where fewer than top_k are left the expert is -1, which `route`
    drops, and the weight 0.  A token with a NaN gets NaN weights."""
    d = _choose_desc(logits, top_k, groups, groups if top_groups is None else top_groups, scores, normalise, scale)
    if bias is not None:
        _whole(bias, (d.n_experts,), torch.float32, logits, "bias")
    expert = logits.new_empty((d.n_tokens, top_k), dtype=torch.int32)
    weights = logits.new_empty((d.n_tokens, top_k), dtype=torch.float32)
    B._check(B.lib().mace_choose_forward(d, logits.data_ptr(), None if bias is None else bias.data_ptr(),
                                         expert.data_ptr(), weights.data_ptr(), _current_stream(logits)),
             "mace_choose_forward")
    return Choice(expert, weights)


@_streamed
def choose_experts_backward(dweights, logits, expert, *, scores: str = "softmax", normalise: bool = True,
                            scale: float = 1.0):
    """Gradient of the logits from dweights (float32 [tokens, top_k]) and the
    experts that `choose_experts` chose, which themselves have no gradient."""
    if expert.dim() != 2:
        raise ValueError("expert must be [tokens, top_k]")
    n, k = expert.shape
    if dweights.dim() != 2 or not dweights.is_cuda:
        raise ValueError(f"dweights must be a float32 {(n, k)} GPU tensor")
    d = _choose_desc(logits, k, 1, 1, scores, normalise, scale)
    if not dweights.is_contiguous():
        dweights = dweights.contiguous()
    _whole(expert, (d.n_tokens, k), torch.int32, logits, "expert")
    _whole(dweights, (d.n_tokens, k), torch.float32, logits, "dweights")
    dlogits = logits.new_empty(logits.shape)
    B._check(B.lib().mace_choose_backward(d, dweights.data_ptr(), logits.data_ptr(), expert.data_ptr(),
                                          dlogits.data_ptr(), d.n_experts, _current_stream(logits)),
             "mace_choose_backward")
    return dlogits


def _ids(ids):
    if ids.dtype is not torch.int32 or not ids.is_cuda or not ids.is_contiguous():
        raise ValueError("ids must be a contiguous int32 GPU tensor")


@_streamed
def embed(ids, table, *, scale: float = 1.0):
    """scale table[ids] for int32 ids of any shape: [*ids.shape, width], zeros
    for ids outside the table (-1, say, in a padded batch)."""
    _ids(ids)
    dtype = _gpu_matrix(table, "table")
    v, width = table.shape
    if table.get_device() != ids.get_device():
        raise ValueError("table must be on ids' device")
    d = B.mace_embed_desc(ids.numel(), v, width, dtype, _leading(table, "table"), width, scale)
    out = table.new_empty((*ids.shape, width))
    B._check(B.lib().mace_embed_forward(d, table.data_ptr(), ids.data_ptr(), out.data_ptr(), _current_stream(ids)),
             "mace_embed_forward")
    return out


@_streamed
def embed_backward(dout, ids, n_rows: int, *, scale: float = 1.0):
    """Gradient [n_rows, width] of the table of `embed`, in dout's dtype."""
    _ids(ids)
    if dout.dim() < 1 or dout.shape[:-1] != ids.shape or dout.get_device() != ids.get_device():
        raise ValueError(f"dout must be {(*ids.shape, 'width')} on ids' device")
    if not 0 < n_rows < 1 << 31:
        raise ValueError("n_rows must be a positive 32-bit integer")
    width = dout.shape[-1]
    dout = _gradient(dout if dout.dim() == 2 else dout.reshape(ids.numel(), width))
    d = B.mace_embed_desc(ids.numel(), n_rows, width, _gpu_matrix(dout, "dout"), width, _leading(dout, "dout"), scale)
    dtable = dout.new_empty((n_rows, width))
    lib = B.lib()
    # (0 for sizes the library does not take: the call itself says which error)
    nbytes = lib.mace_embed_backward_workspace_bytes(d) or 1
    ws = dout.new_empty(nbytes, dtype=torch.uint8)
    B._check(lib.mace_embed_backward(d, dout.data_ptr(), ids.data_ptr(), dtable.data_ptr(), ws.data_ptr(), nbytes,
                                     _current_stream(dout)), "mace_embed_backward")
    return dtable


class Rows8(NamedTuple):
    """Rows of 8-bit integers with a scale each (`pack_rows`): values[i, :columns] * scales[i]."""
    values: torch.Tensor   # int8 [n, columns rounded up to a multiple of 16]
    scales: torch.Tensor   # float32 [n]
    columns: int


class Weights8(NamedTuple):
    """Weights of 8-bit integers with a scale for each output column (`pack_weights`)."""
    values: torch.Tensor   # int8 [groups, n_out, n_in rounded up to a multiple of 16]
    scales: torch.Tensor   # float32 [groups, n_out]
    n_in: int


def _check_rows8(r: Rows8, name: str):
    v, s, c = r
    if v.dim() != 2 or v.dtype is not torch.int8 or not v.is_cuda or not v.is_contiguous() or not 0 < c <= v.shape[1]:
        raise ValueError(f"{name}'s values must be contiguous int8 [n, columns, padded] on a GPU")
    if s.dtype is not torch.float32 or s.shape != v.shape[:1] or s.get_device() != v.get_device() or not s.is_contiguous():
        raise ValueError(f"{name}'s scales must be contiguous float32 [n] on {v.device}")


@_streamed
def pack_rows(x) -> Rows8:
    """x's rows as the nearest 8-bit integers in -127..127 and a float32 scale,
    the row's largest magnitude / 127, each: half the size of a 16-bit activation
    kept for the backward (`linear_backward8`), and an operand of `linear8`.  A
    row with a non-finite element gets the scale NaN."""
    dtype = _gpu_matrix(x, "x")
    n, c = x.shape
    ld = (c + 15) // 16 * 16
    d = B.mace_rows8_desc(n, c, dtype, _leading(x, "x"), ld)
    values, scales = x.new_empty((n, ld), dtype=torch.int8), x.new_empty(n, dtype=torch.float32)
    B._check(B.lib().mace_pack_rows(d, x.data_ptr(), values.data_ptr(), scales.data_ptr(), _current_stream(x)),
             "mace_pack_rows")
    return Rows8(values, scales, c)


@_streamed
def unpack_rows(rows: Rows8, dtype: torch.dtype = torch.float32):
    """[n, columns] values that rows stand for, rounded once to dtype."""
    _check_rows8(rows, "rows")
    if dtype not in DTYPES:
        raise ValueError("dtype must be float32, bfloat16 or float16")
    values, scales, c = rows
    d = B.mace_rows8_desc(values.shape[0], c, DTYPES[dtype], c, values.shape[1])
    x = values.new_empty((values.shape[0], c), dtype=dtype)
    B._check(B.lib().mace_unpack_rows(d, values.data_ptr(), scales.data_ptr(), x.data_ptr(), _current_stream(values)),
             "mace_unpack_rows")
    return x


@_streamed
def pack_weights(w) -> Weights8:
    """w [n_in, n_out] or [groups, n_in, n_out] for `linear8`: 8-bit integers and
    a float32 scale for each output column of each group."""
    dtype = DTYPES.get(w.dtype)
    if dtype is None or w.dim() not in (2, 3) or not w.is_cuda or not w.is_contiguous():
        raise ValueError("w must be a contiguous [(groups,) n_in, n_out] GPU tensor of float32, bfloat16 or float16")
    g, k, m = w.shape if w.dim() == 3 else (1, *w.shape)
    if (g | k | m) >> 31:
        _too_large("w")
    ld = (k + 15) // 16 * 16
    values, scales = w.new_empty((g, m, ld), dtype=torch.int8), w.new_empty((g, m), dtype=torch.float32)
    B._check(B.lib().mace_pack_weights(g, k, m, dtype, w.data_ptr(), values.data_ptr(), ld, scales.data_ptr(),
                                       _current_stream(w)), "mace_pack_weights")
    return Weights8(values, scales, k)


@_streamed
def linear8(x, w: Weights8, bias=None, residual=None, *, offsets=None, act: str = "none", dtype: torch.dtype | None = None):
    """`linear` in 8 bits: y = act(x W_g + b_g) + residual with x's rows rounded as
    `pack_rows` does and weights of `pack_weights`; the products' sums are exact.
    x: [n, n_in] of float32, bfloat16 or float16, or Rows8; dtype (for Rows8 only;
    default float32) is that of bias, residual and y."""
    values, w_scales, n_in = w
    if values.dim() != 3 or values.dtype is not torch.int8 or not values.is_contiguous() or not 0 < n_in <= values.shape[2]:
        raise ValueError("w must be Weights8 as pack_weights gives them")
    groups, m, ld_w = values.shape
    a = ACTIVATIONS.get(act)
    if a is None:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}")
    if isinstance(x, tuple):
        _check_rows8(x, "x")
        x, x_scales, c = x
        dtype = torch.float32 if dtype is None else dtype
        if dtype not in DTYPES:
            raise ValueError("dtype must be float32, bfloat16 or float16")
        like, ld_x = x.new_empty(0, dtype=dtype), x.shape[1]
    else:
        _gpu_matrix(x, "x")
        if dtype is not None and dtype is not x.dtype:
            raise ValueError("dtype is x's, but for Rows8")
        x_scales, c, like, ld_x = None, x.shape[1], x, _leading(x, "x")
    n = x.shape[0]
    if c != n_in or values.get_device() != x.get_device():
        raise ValueError(f"w must have {c} input rows and be on x's device")
    _whole(w_scales, (groups, m), torch.float32, x, "w's scales")
    if offsets is not None:
        _whole(offsets, (groups + 1,), torch.int32, x, "offsets")
    elif groups != 1:
        raise ValueError("more than one group needs offsets")
    d = B.mace_linear_desc(n, n_in, m, groups, DTYPES[like.dtype], a, ld_x, m, m, m)
    if bias is not None:
        if bias.shape != (groups, m) and (groups != 1 or bias.shape != (m,)):
            raise ValueError(f"bias must be {(groups, m)}")
        _whole(bias, bias.shape, like.dtype, x, "bias")
    if residual is not None:
        d.ld_residual = _rows(residual, n, m, like, "residual")
    y = like.new_empty((n, m))
    lib = B.lib()
    # (0 for sizes the library does not take: the call itself says which error; 256: nothing is kept in it)
    nbytes = 0 if x_scales is not None else lib.mace_linear8_workspace_bytes(d)
    ws = x.new_empty(nbytes, dtype=torch.uint8) if nbytes > 256 else None
    B._check(lib.mace_linear8_forward(d, x.data_ptr(), None if x_scales is None else x_scales.data_ptr(),
                                      values.data_ptr(), ld_w, w_scales.data_ptr(),
                                      None if bias is None else bias.data_ptr(),
                                      None if residual is None else residual.data_ptr(),
                                      None if offsets is None else offsets.data_ptr(), y.data_ptr(),
                                      None if ws is None else ws.data_ptr(), nbytes, _current_stream(x)),
             "mace_linear8_forward")
    return y


@_streamed
def linear_backward8(dy, x: Rows8, w, z: Rows8 | None = None, *, offsets=None, act: str = "none", bias: bool = True,
                     need_dx: bool = True, need_dw: bool = True):
    """(dx, dw, db) of `linear` from dy, with x and z (what `linear` saved) kept as
    8-bit rows of `pack_rows` since the forward: the gradients at the values that
    they stand for.  Of 16-bit types with an activation dz is rounded to the type
    before both products, as in `linear_backward`, with a factor of 1/2 to 1 of x's
    scales (relative error 2.3e-3 in bfloat16 and 2.9e-4 in float16, where the
    result's rounding alone is 1.7e-3 and 2.1e-4); x is exact, but rounded to the
    type too, infinite where that is, in rows above its range (127 * 2**9, bfloat16
    127 * 2**121) or with a scale of 2**-25 or less in float16.  Without an
    activation x is rounded to the type, and dy is taken as it is."""
    dy = _gradient(dy)
    dtype, a = _gpu_matrix(dy, "dy"), ACTIVATIONS.get(act)
    if a is None:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}")
    _check_rows8(x, "x")
    n, m = dy.shape
    groups, k, n_out = w.shape if w.dim() == 3 else (1, *w.shape) if w.dim() == 2 else (0, 0, 0)
    if groups == 0 or n_out != m or w.dtype is not dy.dtype or w.get_device() != dy.get_device() or not w.is_contiguous():
        raise ValueError(f"w must be contiguous [(groups,) n_in, {m}], of dy's dtype and device")
    if (groups | k) >> 31:
        _too_large("w")
    if x.values.shape[0] != n or x.columns != k or x.values.get_device() != dy.get_device():
        raise ValueError(f"x must stand for {(n, k)} on dy's device")
    if offsets is not None:
        _whole(offsets, (groups + 1,), torch.int32, dy, "offsets")
    elif groups != 1:
        raise ValueError("more than one group needs offsets")
    ld_z = m
    if a:
        if z is None:
            raise ValueError("an activation's gradient needs z")
        _check_rows8(z, "z")
        if z.values.shape[0] != n or z.columns != m or z.values.get_device() != dy.get_device():
            raise ValueError(f"z must stand for {(n, m)} on dy's device")
        ld_z = z.values.shape[1]
    d = B.mace_linear_desc(n, k, m, groups, dtype, a, x.values.shape[1], m, m, ld_z)
    dx = dy.new_empty((n, k)) if need_dx else None
    dw = torch.empty_like(w) if need_dw else None
    db = dy.new_empty((*w.shape[:-2], m)) if bias else None
    lib = B.lib()
    nbytes = lib.mace_linear_backward8_workspace_bytes(d, bias, need_dw) or 1
    ws = dy.new_empty(nbytes, dtype=torch.uint8)
    B._check(lib.mace_linear_backward8(d, dy.data_ptr(), _leading(dy, "dy"), x.values.data_ptr(), x.scales.data_ptr(),
                                       w.data_ptr(), z.values.data_ptr() if a else None,
                                       z.scales.data_ptr() if a else None,
                                       None if offsets is None else offsets.data_ptr(),
                                       None if dx is None else dx.data_ptr(), k,
                                       None if dw is None else dw.data_ptr(), None if db is None else db.data_ptr(),
                                       ws.data_ptr(), nbytes, _current_stream(dy)), "mace_linear_backward8")
    return dx, dw, db


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
