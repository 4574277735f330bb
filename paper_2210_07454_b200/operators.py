"""Operators of language models beside the optimiser step: layer norm, the loss of a linear head over a large vocabulary,
orthogonalised updates of matrix parameters, the products of a layer of experts, dropout, and the clipped policy loss.

Argument marshalling only, like ``binding``: every operator runs in the CUDA library (``sk_layer_norm`` and so on in
``include/sketched_amsgrad.h``, which states the formulas).  Tensors are CUDA tensors of one device whose rows are
contiguous; rows may be any distance apart.  Calls are asynchronous on torch's current stream of that device, or on
``stream`` (a ``torch.cuda.Stream``), behind what that stream has been given before: if the inputs are still being written elsewhere, let it wait
first.  Workspaces come from torch's allocator.  Outputs are allocated unless given; wait for ``stream`` before reading them elsewhere.

The calls are not part of torch's autograd: results carry no history, whether or not the inputs require gradients.  A backward pass is a call of its own, with
the tensors that it needs; inside a torch graph, wrap the pair in a ``torch.autograd.Function``.

A small call costs the host a few microseconds more than its kernels, so the checks below ask cheap questions first.
"""
from __future__ import annotations

import ctypes as C
import functools

import torch

from .binding import SkError, _check, lib

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_HALF = {torch.bfloat16: 1, torch.float16: 2}
_F32 = {torch.float32: 0}
_INT64 = {torch.int64: 0}
_INDEX = {torch.int64: 64, torch.int32: 32}

# Newton-Schulz step X <- a X + (b A + c A^2) X, A = X X^T: the coefficients published with the Muon optimiser (K. Jordan and others, 2024)
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _shortcut(owner, name, public):
    """torch's inner function if this torch has it (a microsecond of the host's time each), else what its public interface offers."""
    for part in name.split("."):
        owner = getattr(owner, part, None)
    return owner or public


_raw_stream = _shortcut(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)
_current_device = _shortcut(torch._C, "_cuda_getDevice", lambda: torch.cuda.current_device())
_empty_here = _shortcut(torch._C, "_dynamo.guards._empty_strided_cuda",                     # 0.7 us; torch.empty_like 1.3, new_empty 1.8
                        lambda shape, stride, dtype: torch.empty_strided(shape, stride, dtype=dtype, device="cuda"))


# ---- checks ---------------------------------------------------------------------------------------------------------------
def _tensor(t, name, types, device=None):
    """The type's code; the tensor is on `device` (an index) if given, else on any CUDA device."""
    try:
        code, where = types[t.dtype], t.get_device()
    except (AttributeError, KeyError):
        if not isinstance(t, torch.Tensor):
            raise SkError(f"{name} must be a CUDA tensor") from None
        raise SkError(f"{name}: type {t.dtype} is not supported here") from None
    if where < 0:
        raise SkError(f"{name} must be a CUDA tensor")
    if device is not None and where != device:
        raise SkError(f"{name} is on device {where}, not on {device}")
    return code


def _ld(t, name):
    """Distance between the rows of a tensor of two or more dimensions, in elements."""
    if t.is_contiguous():
        return t.shape[-1] or 1
    rows, cols = t.shape[-2], t.shape[-1]
    if cols > 1 and t.stride(-1) != 1:
        raise SkError(f"{name}: the entries of a row must be contiguous")
    if rows <= 1:                                # the stride of a single row means nothing
        return max(cols, 1)
    if t.stride(-2) < cols:
        raise SkError(f"{name}: rows that overlap (a broadcast tensor) are not supported: make it contiguous")
    return max(t.stride(-2), 1)


def _rows(t, name):
    """(rows, ld) of a tensor of any dimension seen as rows of its last axis, without a copy."""
    cols = t.shape[-1]
    if cols and t.is_contiguous():
        return t.numel() // cols, cols
    if not cols:
        return 0, 1
    try:
        flat = t.view(-1, cols)
    except RuntimeError:
        raise SkError(f"{name}: the leading axes must be one evenly spaced run of rows (make it contiguous)") from None
    return flat.shape[0], _ld(flat, name)


def _matrix(t, name, types, device=None):
    code = _tensor(t, name, types, device)
    if t.dim() != 2:
        raise SkError(f"{name} must have 2 dimensions, got {t.dim()}")
    return code, _ld(t, name)


def _vector(t, name, n, types, device):
    """Address of a contiguous vector of n."""
    _tensor(t, name, types, device)
    if t.numel() != n or not t.is_contiguous():
        raise SkError(f"{name} must be contiguous and hold {n} values, got shape {tuple(t.shape)}")
    return t.data_ptr()


def _same_shape(t, like, name):
    if t.shape != like.shape:
        raise SkError(f"{name} must have the shape {tuple(like.shape)}, got {tuple(t.shape)}")


# ---- streams, devices, memory ---------------------------------------------------------------------------------------------
def _on(stream, call, *given):
    """call() with `stream` current: what it allocates then belongs to that stream.  (torch hands freed memory out again in the order of
    the stream it was allocated for; taken from the caller's stream, it might still be in use by kernels that `stream` does not wait for.)
    The tensors that are handed back are used on the caller's stream too, and those that were given on `stream`: neither's memory must be
    handed out again before that stream is done with it, whenever the caller drops them."""
    for t in given:
        if isinstance(t, torch.Tensor) and t.is_cuda and t.get_device() != stream.device_index:
            raise SkError(f"the stream is of device {stream.device_index}, a tensor is on device {t.get_device()}")
    caller = torch.cuda.current_stream(stream.device)
    with torch.cuda.stream(stream):
        out = call()
    for t in given:
        if isinstance(t, torch.Tensor):
            t.record_stream(stream)
    for t in out if isinstance(out, tuple) else (out,):
        if t is not None and not any(t is g for g in given):
            t.record_stream(caller)
    return out


def _run(device, fn, *args):
    """Calls into the library with the tensors' device current."""
    if _current_device() == device:
        rc = fn(*args)
        if rc < 0:
            _check(rc)
    else:
        with torch.cuda.device(device):
            _check(fn(*args))


def _elsewhere(device, fn, *args):
    """What a function of the library (a workspace's size) gives for a device that is not current."""
    with torch.cuda.device(device):
        return fn(*args)


def _need(device, size, *args):
    """Bytes of workspace, asked with the tensors' device current."""
    return size(*args) if _current_device() == device else _elsewhere(device, size, *args)


@functools.lru_cache(maxsize=256)
def _size(name, device, *sizes):
    """What a workspace function of the library gives that depends on sizes and the device only."""
    return _need(device, getattr(lib(), name), *sizes)


def _new_on(device):
    """What allocates uninitialised memory on the device of that index: f(shape, stride, dtype)"""
    if _current_device() == device:
        return _empty_here
    return lambda shape, stride, dtype: torch.empty_strided(shape, stride, dtype=dtype, device=f"cuda:{device}")


def _new(shape, stride, dtype, device):
    """Uninitialised memory on the device of that index."""
    if _current_device() == device:
        return _empty_here(shape, stride, dtype)
    return torch.empty_strided(shape, stride, dtype=dtype, device=f"cuda:{device}")


def _new_like(t, dtype, device):
    """A contiguous tensor of t's shape."""
    if t.is_contiguous():
        return _new(tuple(t.shape), t.stride(), dtype, device)   # a plain tuple is asked for
    return torch.empty_like(t, dtype=dtype, memory_format=torch.contiguous_format)


def _workspace(nbytes, device):
    return _new((nbytes,), (1,), torch.uint8, device) if nbytes else None


def _wrote(*given):
    """Tensors of the caller's that a call writes: autograd's check for tensors changed in place learns of it."""
    for t in given:
        if isinstance(t, torch.Tensor):
            torch.autograd.graph.increment_version(t)


def _p(t):
    return t.data_ptr() if t is not None else None


# ---- layer norm -----------------------------------------------------------------------------------------------------------
def _norm_weights(weight, bias, cols, device):
    """The weights' common type and their addresses."""
    if cols < 1:
        raise SkError("the last axis must not be empty")
    pw = pb = None
    if weight is not None:
        pw = _vector(weight, "weight", cols, _TYPES, device)
    if bias is not None:
        if weight is not None and bias.dtype != weight.dtype:
            raise SkError(f"bias has type {bias.dtype}, weight {weight.dtype}")
        pb = _vector(bias, "bias", cols, _TYPES, device)
    first = weight if weight is not None else bias
    return (0 if first is None else _TYPES[first.dtype]), pw, pb


def layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, stream=None):
    """y = (x - mean) rstd weight + bias over the last axis.  x: (..., cols) fp32, bf16 or fp16; weight, bias: (cols,) or None.
    Returns (y, mean, rstd): y like x, mean and rstd fp32 of x's leading shape."""
    if stream is not None:
        return _on(stream, lambda: layer_norm(x, weight, bias, eps, out), x, weight, bias, out)
    code = _tensor(x, "x", _TYPES)
    shape = x.shape
    if not shape:
        raise SkError("x must have at least 1 dimension")
    device, cols = x.get_device(), shape[-1]
    wcode, pw, pb = _norm_weights(weight, bias, cols, device)
    rows, ld = _rows(x, "x")
    if out is None:
        y, ld_y = _new_like(x, x.dtype, device), cols
    else:
        if _tensor(out, "out", _TYPES, device) != code:
            raise SkError(f"out has type {out.dtype}, x {x.dtype}")
        _same_shape(out, x, "out")
        y, ld_y = out, _rows(out, "out")[1]
    if len(shape) == 2:
        mean, rstd = _new((rows,), (1,), torch.float32, device), _new((rows,), (1,), torch.float32, device)
    else:
        mean = x.new_empty(shape[:-1], dtype=torch.float32)
        rstd = torch.empty_like(mean)
    _run(device, lib().sk_layer_norm, x.data_ptr(), ld, y.data_ptr(), ld_y, code, rows, cols, pw, pb, wcode, eps, mean.data_ptr(), rstd.data_ptr(),
         _raw_stream(device))
    if out is not None:
        _wrote(out)
    return y, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd, dx=None, dweight=None, dbias=None, stream=None):
    """Gradients of ``layer_norm`` from dy and what it returned.  Returns (dx, dweight, dbias): dx like x; dweight, dbias (cols,) of
    weight's type (fp32 without a weight).  ``dx``, ``dweight``, ``dbias``: tensors to write into, False to leave one out."""
    if stream is not None:
        return _on(stream, lambda: layer_norm_backward(dy, x, weight, mean, rstd, dx, dweight, dbias), dy, x, weight, mean, rstd, dx, dweight, dbias)
    given_outputs = None if dx is None and dweight is None and dbias is None else (dx, dweight, dbias)
    code = _tensor(x, "x", _TYPES)
    device, cols = x.get_device(), x.shape[-1] if x.dim() else 0
    if _tensor(dy, "dy", _TYPES, device) != code:
        raise SkError(f"dy has type {dy.dtype}, x {x.dtype}")
    _same_shape(dy, x, "dy")
    wcode, pw, _ = _norm_weights(weight, None, cols, device)
    (rows, ld), (_, ld_dy) = _rows(x, "x"), _rows(dy, "dy")
    pm, pr = _vector(mean, "mean", rows, _F32, device), _vector(rstd, "rstd", rows, _F32, device)
    ld_dx, pdx = cols, None
    if dx is None:
        dx = _new_like(x, x.dtype, device)
        pdx = dx.data_ptr()
    elif dx is False:
        dx = None
    else:
        if _tensor(dx, "dx", _TYPES, device) != code:
            raise SkError(f"dx has type {dx.dtype}, x {x.dtype}")
        _same_shape(dx, x, "dx")
        ld_dx, pdx = _rows(dx, "dx")[1], dx.data_ptr()
    given = dweight if isinstance(dweight, torch.Tensor) else dbias if isinstance(dbias, torch.Tensor) else weight
    dtype = torch.float32 if given is None else given.dtype
    pdw = pdb = None
    if dweight is None:
        dweight = _new((cols,), (1,), dtype, device)
        pdw = dweight.data_ptr()
    elif dweight is False:
        dweight = None
    else:
        pdw = _vector(dweight, "dweight", cols, _TYPES, device)
    if dbias is None:
        dbias = _new((cols,), (1,), dtype, device)
        pdb = dbias.data_ptr()
    elif dbias is False:
        dbias = None
    else:
        pdb = _vector(dbias, "dbias", cols, _TYPES, device)
        if dbias.dtype != dtype:
            raise SkError(f"dbias has type {dbias.dtype}, dweight {dtype}")
    need = 0
    if rows and (pdw or pdb):
        size = lib().sk_layer_norm_backward_workspace
        need = size(rows, cols) if _current_device() == device else _elsewhere(device, size, rows, cols)
    ws = _workspace(need, device)
    _run(device, lib().sk_layer_norm_backward, dy.data_ptr(), ld_dy, x.data_ptr(), ld, pdx, ld_dx, code, rows, cols, pw, wcode, pm, pr, pdw, pdb,
         _TYPES[dtype], _p(ws), need, _raw_stream(device))
    if given_outputs:
        _wrote(*given_outputs)
    return dx, dweight, dbias


# ---- linear cross entropy ---------------------------------------------------------------------------------------------------
def _head(hidden, weight, targets):
    code, ld_h = _matrix(hidden, "hidden", _HALF)
    device = hidden.get_device()
    wcode, ld_w = _matrix(weight, "weight", _HALF, device)
    if wcode != code:
        raise SkError(f"hidden has type {hidden.dtype}, weight {weight.dtype}")
    (tokens, width), (vocab, other) = hidden.shape, weight.shape
    if width != other:
        raise SkError(f"hidden has width {width}, weight {other}")
    if vocab < 1 or width < 1:
        raise SkError("the vocabulary and the width must not be empty")
    return device, code, tokens, vocab, width, ld_h, ld_w, _vector(targets, "targets", tokens, _INT64, device)


def linear_cross_entropy(hidden, weight, targets, stream=None):
    """Softmax cross entropy of the logits hidden weight^T, which are never stored.  hidden: (tokens, width), weight: (vocab, width),
    both bf16 or both fp16; targets: (tokens,) int64, negative = the token takes no part.  Returns (loss, lse), fp32 (tokens,)."""
    if stream is not None:
        return _on(stream, lambda: linear_cross_entropy(hidden, weight, targets), hidden, weight, targets)
    device, code, tokens, vocab, width, ld_h, ld_w, pt = _head(hidden, weight, targets)
    loss, lse = _new((tokens,), (1,), torch.float32, device), _new((tokens,), (1,), torch.float32, device)
    ph, pw = hidden.data_ptr(), weight.data_ptr()
    size, sizes = lib().sk_linear_cross_entropy_workspace, (ph, ld_h, pw, ld_w, tokens, vocab, width)
    need = size(*sizes) if _current_device() == device else _elsewhere(device, size, *sizes)
    ws = _workspace(need, device)
    _run(device, lib().sk_linear_cross_entropy, ph, ld_h, pw, ld_w, code, tokens, vocab, width, pt, loss.data_ptr(), lse.data_ptr(), _p(ws), need,
         _raw_stream(device))
    return loss, lse


def linear_cross_entropy_backward(dloss, hidden, weight, targets, lse, dhidden=None, dweight=None, stream=None):
    """Gradients of ``linear_cross_entropy`` from dloss (fp32, the gradient with respect to every token's loss) and the lse it
    returned.  Returns (dhidden, dweight) of the inputs' type.  ``dhidden``, ``dweight``: tensors to write into (of the inputs' type or
    fp32; views of the gradient array of a step are fine), False to leave one out.  Beyond 64 tokens the gradient of the logits is rounded to the inputs'
    type before the two products that take it, whatever the type of the outputs; up to 64 it is a pair of such values.  Sums are fp32."""
    if stream is not None:
        return _on(stream, lambda: linear_cross_entropy_backward(dloss, hidden, weight, targets, lse, dhidden, dweight), dloss, hidden, weight, targets, lse, dhidden, dweight)
    device, code, tokens, vocab, width, ld_h, ld_w, pt = _head(hidden, weight, targets)
    pd, pl = _vector(dloss, "dloss", tokens, _F32, device), _vector(lse, "lse", tokens, _F32, device)
    types = {hidden.dtype: code, torch.float32: 0}
    outs = []
    for t, name, like in ((dhidden, "dhidden", hidden), (dweight, "dweight", weight)):
        if t is None:
            outs.append((_new_like(like, like.dtype, device), width, code))
        elif t is False:
            outs.append((None, width, code))
        else:
            tcode, ld = _matrix(t, name, types, device)
            _same_shape(t, like, name)
            outs.append((t, ld, tcode))
    (dh, ld_dh, type_dh), (dw, ld_dw, type_dw) = outs
    ph, pw = hidden.data_ptr(), weight.data_ptr()
    size, sizes = lib().sk_linear_cross_entropy_backward_workspace, (ph, ld_h, pw, ld_w, tokens, vocab, width)
    need = size(*sizes) if _current_device() == device else _elsewhere(device, size, *sizes)
    ws = _workspace(need, device)
    _run(device, lib().sk_linear_cross_entropy_backward, pd, ph, ld_h, pw, ld_w, code, tokens, vocab, width, pt, pl, _p(dh), ld_dh, type_dh, _p(dw),
         ld_dw, type_dw, _p(ws), need, _raw_stream(device))
    if dhidden is not None or dweight is not None:
        _wrote(dhidden, dweight)
    return dh, dw


# ---- orthogonalised updates -------------------------------------------------------------------------------------------------
def _batch_of(t, name, like, types, device):
    """(address, ld, stride of the batch, type) of (rows, cols) or (batch, rows, cols)"""
    if t is None:
        return None, 0, 0, 0
    code = _tensor(t, name, types, device)
    if t is not like:
        _same_shape(t, like, name)
    return t.data_ptr(), _ld(t, name), t.stride(0) if t.dim() == 3 else 0, code


def orthogonalize(update, momentum=None, beta=0.95, nesterov=True, steps=5, coefficients=COEFFICIENTS, eps=1e-7, out=None,
                  stream=None):
    """The orthogonalised update of matrix parameters: ``steps`` Newton-Schulz products on U / (|U| + eps), U = update, or with a
    momentum (fp32, updated in place) momentum = beta momentum + update and U = update + beta momentum (nesterov) or momentum.
    update: (rows, cols) or (batch, rows, cols).  Returns out: the same shape, bf16 (fp16 for an fp16 update) unless given.
    Inside, matrices are fp16 with a common scale and sums fp32.  For a bf16 output X is a pair of them in the product P X of all but the last two
    steps: within some 1.1e-3 (2-norm, relative) of the formulas' before the output's own rounding (1.7e-3).  For an fp16 output X, A and P are
    pairs throughout: the error is the output's own rounding (2.1e-4), at 1.4 to 2.2 times the time."""
    if stream is not None:
        return _on(stream, lambda: orthogonalize(update, momentum, beta, nesterov, steps, coefficients, eps, out), update, momentum, out)
    if not isinstance(update, torch.Tensor) or update.dim() not in (2, 3):
        raise SkError("update must be a CUDA tensor of 2 or 3 dimensions")
    device = update.get_device() if update.is_cuda else None
    pu, ld_u, s_u, code = _batch_of(update, "update", update, _TYPES, device)
    pm, ld_m, s_m, _ = _batch_of(momentum, "momentum", update, _F32, device)
    if len(coefficients) != 3:
        raise SkError("coefficients are three numbers (a, b, c)")
    given_out = out
    if out is None:
        out = _new_like(update, torch.float16 if update.dtype == torch.float16 else torch.bfloat16, device)
    po, ld_o, s_o, out_code = _batch_of(out, "out", update, _HALF, device)
    batch, (rows, cols) = (update.shape[0] if update.dim() == 3 else 1), update.shape[-2:]
    size = lib().sk_orthogonalize_workspace
    need = size(batch, rows, cols) if _current_device() == device else _elsewhere(device, size, batch, rows, cols)
    ws = _workspace(need, device)
    _run(device, lib().sk_orthogonalize, pu, ld_u, s_u, code, pm, ld_m, s_m, beta, int(nesterov), po, ld_o, s_o, out_code, batch, rows, cols, steps,
         (C.c_float * 3)(*coefficients), eps, _p(ws), need, _raw_stream(device))
    if momentum is not None or given_out is not None:
        _wrote(momentum, given_out)
    return out


# ---- products grouped by expert ---------------------------------------------------------------------------------------------
def sort_by_expert(experts, groups, stream=None):
    """Brings assignments of rows to experts into the order that ``grouped_linear`` takes.  experts: a contiguous tensor of n values, int64 or
    int32; what lies outside 0..groups-1 belongs to no expert and comes last.  Returns (order, places, offsets), int64: order (n,), the assignments sorted
    by expert, equal ones in the order they have; places, like experts, where each one went (order[places[i]] = i); offsets (groups + 1,),
    the places at which the experts' assignments begin and end.

    With k experts for each token (experts: (tokens, k)) the rows are x[order // k], and a token's results are y[places]: (tokens, k, out)."""
    if stream is not None:
        return _on(stream, lambda: sort_by_expert(experts, groups), experts)
    wide = _tensor(experts, "experts", _INDEX)
    if not experts.is_contiguous():
        raise SkError("experts must be contiguous")
    if groups < 1 or groups > 2048:
        raise SkError("groups must be in 1..2048")
    device, shape = experts.get_device(), experts.shape
    n = shape[0] if len(shape) == 1 else experts.numel()
    new = _new_on(device)
    order, offsets = new((n,), (1,), torch.int64), new((groups + 1,), (1,), torch.int64)
    places = new((n,), (1,), torch.int64) if len(shape) == 1 else _new_like(experts, torch.int64, device)
    need = _size("sk_sort_by_expert_workspace", device, n, groups)
    ws = new((need,), (1,), torch.uint8) if need else None
    _run(device, lib().sk_sort_by_expert, experts.data_ptr(), wide, n, groups, order.data_ptr(), places.data_ptr(), offsets.data_ptr(), _p(ws), need,
         _raw_stream(device))
    return order, places, offsets


def _grouped(x, weight, offsets):
    """What both directions take: (device, code, rows, groups, width, out, ld_x, ld_w, stride_w, address of the offsets)"""
    code = _tensor(x, "x", _HALF)
    device = x.get_device()
    if _tensor(weight, "weight", _HALF, device) != code:
        raise SkError(f"x has type {x.dtype}, weight {weight.dtype}")
    if x.dim() != 2 or weight.dim() != 3:
        raise SkError(f"x must have 2 dimensions and weight 3, got {x.dim()} and {weight.dim()}")
    (rows, width), (groups, out, other) = x.shape, weight.shape
    if width != other:
        raise SkError(f"x has width {width}, weight {other}")
    if groups < 1 or width < 1 or out < 1:
        raise SkError("the groups, the width and the outputs must not be empty")
    if weight.is_contiguous():
        ld_w, s_w = width, out * width
    else:
        ld_w, s_w = _ld(weight, "weight"), weight.stride(0)
    return device, code, rows, groups, width, out, width if x.is_contiguous() else _ld(x, "x"), ld_w, s_w, _vector(offsets, "offsets", groups + 1, _INT64, device)


def grouped_linear(x, weight, offsets, out=None, stream=None):
    """y[i] = weight[g] x[i] for the rows i of every group g: offsets[g] <= i < offsets[g + 1].  x: (rows, width), weight: (groups, out, width), both
    bf16 or both fp16; offsets: (groups + 1,) int64 on the same device (see ``sort_by_expert``), not decreasing, which the host never reads.  Returns
    (rows, out) of x's type.  Rows of no group are zero, or left as they were in an ``out`` that is given."""
    if stream is not None:
        return _on(stream, lambda: grouped_linear(x, weight, offsets, out), x, weight, offsets, out)
    device, code, rows, groups, width, n, ld_x, ld_w, s_w, po = _grouped(x, weight, offsets)
    new = _new_on(device)
    if out is None:
        y, ld_y = new((rows, n), (n, 1), x.dtype), n
    else:
        ycode, ld_y = _matrix(out, "out", _HALF, device)
        if ycode != code:
            raise SkError(f"out has type {out.dtype}, x {x.dtype}")
        if out.shape != (rows, n):
            raise SkError(f"out must have the shape {(rows, n)}, got {tuple(out.shape)}")
        y = out
    px, pw = x.data_ptr(), weight.data_ptr()
    L = lib()
    py = y.data_ptr()
    need = _need(device, L.sk_grouped_linear_workspace, px, ld_x, pw, ld_w, s_w, rows, groups, width, n, py, ld_y)
    ws = new((need,), (1,), torch.uint8) if need else None
    _run(device, L.sk_grouped_linear, px, ld_x, pw, ld_w, s_w, code, rows, groups, width, n, po, py, ld_y, out is None, _p(ws), need, _raw_stream(device))
    if out is not None:
        _wrote(out)
    return y


def grouped_linear_backward(dy, x, weight, offsets, dx=None, dweight=None, stream=None):
    """Gradients of ``grouped_linear``.  Returns (dx, dweight) of the inputs' type: dx like x (rows of no group are zero, or left as they were in a given one),
    dweight like weight (zero for a group without rows).  ``dx``, ``dweight``: tensors to write into (dweight of the inputs' type or fp32; a view of
    the gradient array of a step is fine), False to leave one out.  Sums are fp32."""
    if stream is not None:
        return _on(stream, lambda: grouped_linear_backward(dy, x, weight, offsets, dx, dweight), dy, x, weight, offsets, dx, dweight)
    device, code, rows, groups, width, n, ld_x, ld_w, s_w, po = _grouped(x, weight, offsets)
    if _tensor(dy, "dy", _HALF, device) != code:
        raise SkError(f"dy has type {dy.dtype}, x {x.dtype}")
    if dy.shape != (rows, n):
        raise SkError(f"dy must have the shape {(rows, n)}, got {tuple(dy.shape)}")
    ld_dy, given_outputs, fill, ld_dx, new = n if dy.is_contiguous() else _ld(dy, "dy"), (dx, dweight), dx is None, width, _new_on(device)
    if dx is None:
        dx = new((rows, width), (width, 1), x.dtype)
    elif dx is False:
        dx = None
    else:
        xcode, ld_dx = _matrix(dx, "dx", _HALF, device)
        if xcode != code:
            raise SkError(f"dx has type {dx.dtype}, x {x.dtype}")
        _same_shape(dx, x, "dx")
    wcode, ld_dw, s_dw = code, width, n * width
    if dweight is None:
        dweight = new((groups, n, width), (n * width, width, 1), x.dtype)
    elif dweight is False:
        dweight = None
    else:
        wcode = _tensor(dweight, "dweight", {weight.dtype: code, torch.float32: 0}, device)
        _same_shape(dweight, weight, "dweight")
        ld_dw, s_dw = _ld(dweight, "dweight"), dweight.stride(0)
    pd, px, pw, pdx, pdw = dy.data_ptr(), x.data_ptr(), weight.data_ptr(), _p(dx), _p(dweight)
    L = lib()
    need = _need(device, L.sk_grouped_linear_backward_workspace, pd, ld_dy, px, ld_x, pw, ld_w, s_w, rows, groups, width, n, pdx, ld_dx, pdw, ld_dw, s_dw, wcode)
    ws = new((need,), (1,), torch.uint8) if need else None
    _run(device, L.sk_grouped_linear_backward, pd, ld_dy, px, ld_x, pw, ld_w, s_w, code, rows, groups, width, n, po, pdx, ld_dx, fill, pdw,
         ld_dw, s_dw, wcode, _p(ws), need, _raw_stream(device))
    if given_outputs[0] is not None or given_outputs[1] is not None:
        _wrote(*given_outputs)
    return dx, dweight


# ---- dropout ------------------------------------------------------------------------------------------------------------------
def _seed(seed, device):
    """(value, address) of a seed: a whole number, or one on the device"""
    if isinstance(seed, torch.Tensor):
        _vector(seed, "seed", 1, _INT64, device)
        return 0, seed.data_ptr()
    try:
        value = int(seed)
        if value == seed:                            # nothing that had to be rounded
            return value & 0xFFFFFFFFFFFFFFFF, None
    except (TypeError, ValueError, OverflowError):
        pass
    raise SkError("seed must be a whole number or a CUDA tensor of one int64")


def dropout(x, p, seed, residual=None, out=None, stream=None):
    """residual + x / (1 - p) where a value stays, residual where it is dropped, with probability p.  Which ones stay is a function of the seed and the
    value's number in x (in row order, whatever its strides): there is no mask to keep.  x: fp32, bf16 or fp16 of any shape; residual: like x, or None
    (zero).  p is rounded to a multiple of 2^-16.  seed: a whole number (modulo 2^64), another one for every use, or a CUDA tensor of one int64 that is read when
    the kernel runs (a captured call can then be replayed with another).  Returns a tensor like x; ``out`` may be x or residual."""
    if stream is not None:
        return _on(stream, lambda: dropout(x, p, seed, residual, out), x, seed, residual, out)
    code = _tensor(x, "x", _TYPES)
    shape = x.shape
    if not shape:
        raise SkError("x must have at least 1 dimension")
    device, cols, whole = x.get_device(), shape[-1], x.is_contiguous()
    rows, ld = (x.numel() // cols if cols else 0, cols) if whole else _rows(x, "x")
    pr, ld_r = None, cols
    if residual is not None:
        if _tensor(residual, "residual", _TYPES, device) != code:
            raise SkError(f"residual has type {residual.dtype}, x {x.dtype}")
        if residual.shape != shape:
            _same_shape(residual, x, "residual")
        pr = residual.data_ptr()
        if not residual.is_contiguous():
            ld_r = _rows(residual, "residual")[1]
    if out is None:
        y, ld_y = (_new_on(device)(tuple(shape), x.stride(), x.dtype) if whole else _new_like(x, x.dtype, device)), cols
    else:
        if _tensor(out, "out", _TYPES, device) != code:
            raise SkError(f"out has type {out.dtype}, x {x.dtype}")
        _same_shape(out, x, "out")
        y, ld_y = out, _rows(out, "out")[1]
    value, at = _seed(seed, device)
    _run(device, lib().sk_dropout, x.data_ptr(), ld, pr, ld_r, y.data_ptr(), ld_y, code, rows, cols, p, value, at, _raw_stream(device))
    if out is not None:
        _wrote(out)
    return y


def dropout_backward(dy, p, seed, dx=None, stream=None):
    """Gradient of ``dropout`` with respect to x, from dy with the p and the seed of the forward pass (that of the residual is dy).  Returns dx, which may
    be given and may be dy."""
    return dropout(dy, p, seed, None, dx, stream)


# ---- policy loss ----------------------------------------------------------------------------------------------------------------
_OF = {"tokens": 0, "sequences": 1}


def _policy(nll, old_nll, advantages, targets, offsets, reference_nll, clip, kl, advantage_of):
    """The arguments that both directions share, from nll to kl, and (device, tokens, sequences)"""
    _tensor(nll, "nll", _F32)
    if not nll.is_contiguous():
        raise SkError("nll must be contiguous")
    device, tokens = nll.get_device(), nll.numel()
    pn, pold = nll.data_ptr(), _vector(old_nll, "old_nll", tokens, _F32, device)
    pt = _vector(targets, "targets", tokens, _INT64, device) if targets is not None else None
    sequences, po = 1, None
    if offsets is not None:
        _tensor(offsets, "offsets", _INT64, device)
        sequences = offsets.numel() - 1
        if sequences < 1 or not offsets.is_contiguous():
            raise SkError("offsets must be contiguous and hold at least 2 values")
        po = offsets.data_ptr()
    of = _OF.get(advantage_of)
    if of is None:
        raise SkError(f"advantage_of must be 'tokens' or 'sequences', got {advantage_of!r}")
    pa = _vector(advantages, "advantages", sequences if of else tokens, _F32, device)
    pr = _vector(reference_nll, "reference_nll", tokens, _F32, device) if reference_nll is not None else None
    try:
        low, high = clip
    except (TypeError, ValueError):
        raise SkError("clip is two numbers (low, high)") from None
    return (pn, pold, pa, of, pt, po, sequences, pr, tokens, low, high, kl), device, tokens, sequences


def policy_loss(nll, old_nll, advantages, targets=None, offsets=None, reference_nll=None, clip=(0.2, 0.2), kl=0.0, average="tokens",
                advantage_of="tokens", stream=None):
    """The clipped policy loss with a KL term, over losses as ``linear_cross_entropy`` returns them (negative log probabilities of the tokens drawn).
    With r = exp(old_nll - nll), A the advantage, e = nll - reference_nll, a token's loss is
    -min(r A, min(max(r, 1 - clip[0]), 1 + clip[1]) A) + kl (exp(e) - e - 1).

    nll, old_nll, reference_nll: fp32, (tokens,); advantages: fp32, one for each token or (advantage_of="sequences") each sequence; targets: (tokens,) int64, tokens
    with a negative one take no part (the vector that the head takes); offsets: (sequences + 1,) int64, where the sequences begin and end (None: all
    tokens are one).  average: "tokens" (every token counts the same) or "sequences" (every sequence, and its tokens among one another).
    Returns (result, norm): result (3,) fp32 is the loss, the mean of exp(e) - e - 1, the share of clipped tokens, all in the same average; norm (sequences,) fp32
    is what a token counts, for the backward pass."""
    if stream is not None:
        return _on(stream, lambda: policy_loss(nll, old_nll, advantages, targets, offsets, reference_nll, clip, kl, average, advantage_of), nll, old_nll,
                   advantages, targets, offsets, reference_nll)
    args, device, tokens, sequences = _policy(nll, old_nll, advantages, targets, offsets, reference_nll, clip, kl, advantage_of)
    if average not in _OF:
        raise SkError(f"average must be 'tokens' or 'sequences', got {average!r}")
    new = _new_on(device)
    result, norm = new((3,), (1,), torch.float32), new((sequences,), (1,), torch.float32)
    need = _size("sk_policy_loss_workspace", device, tokens, sequences)
    ws = new((need,), (1,), torch.uint8) if need else None
    _run(device, lib().sk_policy_loss, *args, _OF[average], result.data_ptr(), norm.data_ptr(), _p(ws), need, _raw_stream(device))
    return result, norm


def policy_loss_backward(dloss, nll, old_nll, advantages, norm, targets=None, offsets=None, reference_nll=None, clip=(0.2, 0.2), kl=0.0,
                         advantage_of="tokens", dnll=None, stream=None):
    """Gradient of ``policy_loss``'s loss with respect to nll, from the norm it returned and its other arguments: what
    ``linear_cross_entropy_backward`` takes as dloss.  dloss: fp32 of one value, or None (1).  Returns dnll (tokens,) fp32, zero for tokens that take no
    part; ``dnll``, if given, may be nll."""
    if stream is not None:
        return _on(stream, lambda: policy_loss_backward(dloss, nll, old_nll, advantages, norm, targets, offsets, reference_nll, clip, kl, advantage_of, dnll),
                   dloss, nll, old_nll, advantages, norm, targets, offsets, reference_nll, dnll)
    args, device, tokens, sequences = _policy(nll, old_nll, advantages, targets, offsets, reference_nll, clip, kl, advantage_of)
    pl = _vector(dloss, "dloss", 1, _F32, device) if dloss is not None else None
    pm = _vector(norm, "norm", sequences, _F32, device)
    if dnll is None:
        out = _new((tokens,), (1,), torch.float32, device)
    else:
        _vector(dnll, "dnll", tokens, _F32, device)
        out = dnll
    _run(device, lib().sk_policy_loss_backward, pl, *args, pm, out.data_ptr(), _raw_stream(device))
    if dnll is not None:
        _wrote(dnll)
    return out


def sync(stream=None, device=None) -> None:
    """Waits for the stream (default: torch's current one) and raises if an operator's kernel reported an inconsistency."""
    with torch.cuda.device(device if device is not None else torch.cuda.current_device()):
        _check(lib().sk_operators_sync((stream or torch.cuda.current_stream()).cuda_stream))
