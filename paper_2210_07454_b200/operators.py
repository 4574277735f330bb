"""Operators of language models beside the optimiser step: layer norm, the loss of a linear head over a large vocabulary,
and orthogonalised updates of matrix parameters.

Argument marshalling only, like ``binding``: every operator runs in the CUDA library (``sk_layer_norm`` and so on in
``include/sketched_amsgrad.h``, which states the formulas).  Tensors are CUDA tensors of one device whose rows are
contiguous; rows may be any distance apart.  Calls are asynchronous on torch's current stream of that device, or on
``stream`` (a ``torch.cuda.Stream``); workspaces come from torch's allocator.  Outputs are allocated unless given.
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import SkError, _check, lib

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_HALF = (torch.bfloat16, torch.float16)

COEFFICIENTS = (3.4445, -4.7750, 2.0315)         # Newton-Schulz step X <- a X + (b A + c A^2) X, A = X X^T


def _matrix(t, name, dtypes=tuple(_TYPES)):
    """A 2-d CUDA tensor with contiguous rows; returns its leading dimension."""
    _tensor(t, name, dtypes)
    if t.dim() != 2:
        raise SkError(f"{name} must have 2 dimensions, got {t.dim()}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise SkError(f"{name}: the entries of a row must be contiguous")
    return _ld(t)


def _ld(t):
    if t.shape[-2] <= 1:                         # the stride of a single row means nothing
        return max(t.shape[-1], 1)
    if t.stride(-2) < t.shape[-1]:
        raise SkError("rows that overlap (a broadcast tensor) are not supported: make it contiguous")
    return max(t.stride(-2), 1)


def _tensor(t, name, dtypes):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise SkError(f"{name} must be a CUDA tensor")
    if t.dtype not in dtypes:
        raise SkError(f"{name}: type {t.dtype} is not supported here")


def _vector(t, name, n, dtypes):
    _tensor(t, name, dtypes)
    if t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise SkError(f"{name} must be a contiguous vector of {n}, got shape {tuple(t.shape)}")
    return t.data_ptr()


class _Call:
    """The device, the stream and the workspace of one call."""

    def __init__(self, first, others, stream):
        for t in others:
            if t is not None and t.device != first.device:
                raise SkError(f"tensors on different devices: {first.device} and {t.device}")
        self.device = first.device
        self.stream = stream
        self.ptr = (stream or torch.cuda.current_stream(self.device)).cuda_stream
        self.guard = None

    def __enter__(self):
        if torch.cuda.current_device() != self.device.index:
            self.guard = torch.cuda.device(self.device)
            self.guard.__enter__()
        return self

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)

    def new(self, shape, dtype):
        t = torch.empty(shape, dtype=dtype, device=self.device)
        if self.stream is not None:              # allocated on the current stream, used on another
            t.record_stream(self.stream)
        return t

    def workspace(self, nbytes):
        return self.new(nbytes, torch.uint8) if nbytes else None


def _p(t):
    return t.data_ptr() if t is not None else None


def layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, stream=None):
    """y = (x - mean) rstd weight + bias over the last axis.  x: (..., cols) fp32, bf16 or fp16; weight, bias: (cols,) or None.
    Returns (y, mean, rstd): y like x, mean and rstd fp32 of x's leading shape."""
    _tensor(x, "x", tuple(_TYPES))
    if x.dim() < 1:
        raise SkError("x must have at least 1 dimension")
    flat = _rows(x, "x")
    rows, cols = flat.shape
    wtype = _norm_weights(weight, bias, cols)
    with _Call(x, (weight, bias, out), stream) as call:
        y = call.new(x.shape, x.dtype) if out is None else out
        flat_y = _rows(_like(y, x, "out"), "out")
        mean, rstd = call.new(x.shape[:-1], torch.float32), call.new(x.shape[:-1], torch.float32)
        _check(lib().sk_layer_norm(flat.data_ptr(), _ld(flat), flat_y.data_ptr(), _ld(flat_y), _TYPES[x.dtype], rows, cols, _p(weight),
                                   _p(bias), wtype, eps, mean.data_ptr(), rstd.data_ptr(), call.ptr))
    return y, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd, dx=None, dweight=None, dbias=None, stream=None):
    """Gradients of ``layer_norm`` from dy and what it returned.  Returns (dx, dweight, dbias): dx like x; dweight, dbias (cols,) of
    weight's type (fp32 without a weight).  ``dx``, ``dweight``, ``dbias``: tensors to write into, False to leave one out."""
    _tensor(x, "x", tuple(_TYPES))
    _like(dy, x, "dy")
    fx, fdy = _rows(x, "x"), _rows(dy, "dy")
    rows, cols = fx.shape
    wtype = _norm_weights(weight, None, cols)
    pm, pr = (_vector(t.reshape(-1) if isinstance(t, torch.Tensor) else t, name, rows, (torch.float32,)) for t, name in ((mean, "mean"), (rstd, "rstd")))
    sums = [t for t in (dweight, dbias) if t is not None and t is not False]
    dtype = sums[0].dtype if sums else weight.dtype if weight is not None else torch.float32
    with _Call(x, (dy, weight, mean, rstd, dx or None if not isinstance(dx, torch.Tensor) else dx, *sums), stream) as call:
        dx = None if dx is False else call.new(x.shape, x.dtype) if dx is None else _like(dx, x, "dx")
        fdx = _rows(dx, "dx") if dx is not None else None
        dweight, dbias = (None if t is False else call.new((cols,), dtype) if t is None else t for t in (dweight, dbias))
        for t, name in ((dweight, "dweight"), (dbias, "dbias")):
            if t is not None:
                _vector(t, name, cols, (dtype,))
        need = lib().sk_layer_norm_backward_workspace(rows, cols) if rows and (dweight is not None or dbias is not None) else 0
        ws = call.workspace(need)
        _check(lib().sk_layer_norm_backward(fdy.data_ptr(), _ld(fdy), fx.data_ptr(), _ld(fx), _p(fdx), _ld(fdx) if fdx is not None else 0,
                                            _TYPES[x.dtype], rows, cols, _p(weight), wtype, pm, pr, _p(dweight), _p(dbias),
                                            _TYPES[dtype], _p(ws), need, call.ptr))
    return dx, dweight, dbias


def _like(t, x, name):
    _tensor(t, name, (x.dtype,))
    if t.shape != x.shape:
        raise SkError(f"{name} must have the shape {tuple(x.shape)}, got {tuple(t.shape)}")
    return t


def _rows(t, name):
    """(..., cols) as (rows, cols) without a copy."""
    try:
        flat = t.view(-1, t.shape[-1]) if t.numel() else t.reshape(t.shape[:-1].numel(), t.shape[-1])
    except RuntimeError:
        raise SkError(f"{name}: the leading axes must be one evenly spaced run of rows (make it contiguous)") from None
    _matrix(flat, name)
    return flat


def _norm_weights(weight, bias, cols):
    if cols < 1:
        raise SkError("the last axis must not be empty")
    dtype = next((t.dtype for t in (weight, bias) if isinstance(t, torch.Tensor)), torch.float32)
    for t, name in ((weight, "weight"), (bias, "bias")):
        if t is not None:
            _vector(t, name, cols, (dtype,) if dtype in _TYPES else tuple(_TYPES))
    return _TYPES[dtype]


def _head(hidden, weight, targets):
    ld_h, ld_w = _matrix(hidden, "hidden", _HALF), _matrix(weight, "weight", (hidden.dtype,) if hidden.dtype in _HALF else _HALF)
    if hidden.shape[1] != weight.shape[1]:
        raise SkError(f"hidden has width {hidden.shape[1]}, weight {weight.shape[1]}")
    if weight.shape[0] < 1 or weight.shape[1] < 1:
        raise SkError("the vocabulary and the width must not be empty")
    _vector(targets, "targets", hidden.shape[0], (torch.int64,))
    return hidden.shape[0], weight.shape[0], weight.shape[1], ld_h, ld_w


def linear_cross_entropy(hidden, weight, targets, stream=None):
    """Softmax cross entropy of the logits hidden weight^T, which are never stored.  hidden: (tokens, width), weight: (vocab, width),
    both bf16 or both fp16; targets: (tokens,) int64, negative = the token takes no part.  Returns (loss, lse), fp32 (tokens,)."""
    tokens, vocab, width, ld_h, ld_w = _head(hidden, weight, targets)
    with _Call(hidden, (weight, targets), stream) as call:
        loss, lse = call.new((tokens,), torch.float32), call.new((tokens,), torch.float32)
        need = lib().sk_linear_cross_entropy_workspace(hidden.data_ptr(), ld_h, weight.data_ptr(), ld_w, tokens, vocab, width)
        ws = call.workspace(need)
        _check(lib().sk_linear_cross_entropy(hidden.data_ptr(), ld_h, weight.data_ptr(), ld_w, _TYPES[hidden.dtype], tokens, vocab, width,
                                             targets.data_ptr(), loss.data_ptr(), lse.data_ptr(), _p(ws), need, call.ptr))
    return loss, lse


def linear_cross_entropy_backward(dloss, hidden, weight, targets, lse, dhidden=None, dweight=None, stream=None):
    """Gradients of ``linear_cross_entropy`` from dloss (fp32, the gradient with respect to every token's loss) and the lse it
    returned.  Returns (dhidden, dweight) of the inputs' type.  ``dhidden``, ``dweight``: tensors to write into (of the inputs' type or
    fp32; views of the gradient array of a step are fine), False to leave one out."""
    tokens, vocab, width, ld_h, ld_w = _head(hidden, weight, targets)
    for t, name in ((dloss, "dloss"), (lse, "lse")):
        _vector(t, name, tokens, (torch.float32,))
    given = [t for t in (dhidden, dweight) if isinstance(t, torch.Tensor)]
    with _Call(hidden, (weight, targets, dloss, lse, *given), stream) as call:
        outs = []
        for t, name, like in ((dhidden, "dhidden", hidden), (dweight, "dweight", weight)):
            t = None if t is False else call.new(like.shape, like.dtype) if t is None else t
            if t is not None:
                ld = _matrix(t, name, (like.dtype, torch.float32))
                if t.shape != like.shape:
                    raise SkError(f"{name} must have the shape {tuple(like.shape)}, got {tuple(t.shape)}")
            outs.append((t, ld if t is not None else 0, _TYPES[t.dtype] if t is not None else 0))
        (dh, ld_dh, type_dh), (dw, ld_dw, type_dw) = outs
        need = lib().sk_linear_cross_entropy_backward_workspace(hidden.data_ptr(), ld_h, weight.data_ptr(), ld_w, tokens, vocab, width)
        ws = call.workspace(need)
        _check(lib().sk_linear_cross_entropy_backward(dloss.data_ptr(), hidden.data_ptr(), ld_h, weight.data_ptr(), ld_w, _TYPES[hidden.dtype], tokens,
                                                      vocab, width, targets.data_ptr(), lse.data_ptr(), _p(dh), ld_dh, type_dh, _p(dw), ld_dw,
                                                      type_dw, _p(ws), need, call.ptr))
    return dh, dw


def orthogonalize(update, momentum=None, beta=0.95, nesterov=True, steps=5, coefficients=COEFFICIENTS, eps=1e-7, out=None,
                  stream=None):
    """The orthogonalised update of matrix parameters: ``steps`` Newton-Schulz products on U / (|U| + eps), U = update, or with a
    momentum (fp32, updated in place) momentum = beta momentum + update and U = update + beta momentum (nesterov) or momentum.
    update: (rows, cols) or (batch, rows, cols).  Returns out: the same shape, bf16 (fp16 for an fp16 update) unless given."""
    _tensor(update, "update", tuple(_TYPES))
    if update.dim() not in (2, 3):
        raise SkError(f"update must have 2 or 3 dimensions, got {update.dim()}")
    if momentum is not None:
        _tensor(momentum, "momentum", (torch.float32,))
    if len(coefficients) != 3:
        raise SkError("coefficients are three numbers (a, b, c)")
    with _Call(update, (momentum, out), stream) as call:
        if out is None:
            out = call.new(update.shape, torch.float16 if update.dtype == torch.float16 else torch.bfloat16)
        _tensor(out, "out", _HALF)
        views = []
        for t, name in ((update, "update"), (momentum, "momentum"), (out, "out")):
            if t is None:
                views.append((None, 0, 0))
                continue
            if t.shape != update.shape:
                raise SkError(f"{name} must have the shape {tuple(update.shape)}, got {tuple(t.shape)}")
            t3 = t if t.dim() == 3 else t.unsqueeze(0)
            if t3.shape[2] > 1 and t3.stride(2) != 1:
                raise SkError(f"{name}: the entries of a row must be contiguous")
            views.append((t.data_ptr(), _ld(t3), t3.stride(0)))
        batch, rows, cols = update.shape if update.dim() == 3 else (1, *update.shape)
        need = lib().sk_orthogonalize_workspace(batch, rows, cols)
        ws = call.workspace(need)
        (pu, ld_u, s_u), (pm, ld_m, s_m), (po, ld_o, s_o) = views
        _check(lib().sk_orthogonalize(pu, ld_u, s_u, _TYPES[update.dtype], pm, ld_m, s_m, beta, int(nesterov), po, ld_o, s_o, _TYPES[out.dtype],
                                      batch, rows, cols, steps, (C.c_float * 3)(*coefficients), eps, _p(ws), need, call.ptr))
    return out


def sync(stream=None, device=None) -> None:
    """Waits for the stream (default: torch's current one) and raises if an operator's kernel reported an inconsistency."""
    with torch.cuda.device(device if device is not None else torch.cuda.current_device()):
        _check(lib().sk_operators_sync((stream or torch.cuda.current_stream()).cuda_stream))
