"""Operators of language models beside the optimiser step: layer norm, the loss of a linear head over a large vocabulary,
and orthogonalised updates of matrix parameters.

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

import torch

from .binding import SkError, _check, lib

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_HALF = {torch.bfloat16: 1, torch.float16: 2}
_F32 = {torch.float32: 0}
_INT64 = {torch.int64: 0}

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
        _check(fn(*args))
    else:
        with torch.cuda.device(device):
            _check(fn(*args))


def _elsewhere(device, fn, *args):
    """What a function of the library (a workspace's size) gives for a device that is not current."""
    with torch.cuda.device(device):
        return fn(*args)


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


def sync(stream=None, device=None) -> None:
    """Waits for the stream (default: torch's current one) and raises if an operator's kernel reported an inconsistency."""
    with torch.cuda.device(device if device is not None else torch.cuda.current_device()):
        _check(lib().sk_operators_sync((stream or torch.cuda.current_stream()).cuda_stream))
