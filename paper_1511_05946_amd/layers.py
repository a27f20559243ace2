"""Rows for a cascade and their normalisation, on libacdc.so.

What a language model of cascades needs besides them: ``acdc.forward`` takes
rows of N values, and

* ``embedding``    makes such rows of tokens (``embedding_backward``: the
                   weight's gradient);
* ``layer_norm``   brings rows back to mean 0 and variance 1 between cascades
                   and in front of ``losses.vocab_loss`` (``layer_norm_backward``:
                   the gradients of rows, weight and bias).

Argument marshalling only; the work is enqueued on the current torch stream.
Values are float32 or bfloat16, sums and statistics are held in float32.  Rows
are [rows, width], each contiguous and the rows any distance apart; the rows
that go in and those that come out may differ in type (``dtype``), so that a
bfloat16 weight gives a cascade its float32 rows and a cascade's rows reach a
bfloat16 loss without a pass of their own.  The ``*_autograd`` functions are the
differentiable forms (first derivatives; a second one raises).
"""

from __future__ import annotations

import functools
import math
from typing import NamedTuple, Optional

import torch

from ._lib import lib
from .acdc import _call, _check, _once, _ptr, _wrote
from .losses import _DTYPES, _aligned_workspace, _apart, _capturable, _index, _matrix, _native, _sizes, _values, _workspace


class LayerNorm(NamedTuple):
    y: torch.Tensor
    saved: Optional[torch.Tensor]      # [rows, 2]: mean and 1 / deviation, for layer_norm_backward


def _code(dtype):
    """The type as the binding's native part takes it; None where it cannot."""
    return -1 if dtype is None else _DTYPES.get(dtype)


def _type(name, dtype, default):
    if dtype is None:
        return default
    if dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32 or bfloat16, not {dtype}")
    return dtype


def _rows_of(name, t, rows, width, device, dtype=None):
    """The stride of [rows, width] values on `device`."""
    n, w, stride = _matrix(name, t, device)
    if (n, w) != (rows, width) or (dtype is not None and t.dtype is not dtype):
        raise ValueError(f"{name} must be [{rows}, {width}]{'' if dtype is None else f' {dtype}'}, got {tuple(t.shape)} {t.dtype}")
    return stride


def _width_vector(name, t, width, device):
    if t is None:
        return
    if t.shape != (width,) or t.device != device or t.dtype not in _DTYPES or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 or bfloat16 vector of {width} values on {device}, got "
                         f"{tuple(t.shape)} {t.dtype} on {t.device}")
    _values(name, t)


def _one_type(name, a, b):
    if a is not None and b is not None and a.dtype is not b.dtype:
        raise ValueError(f"{name} must have one type, got {a.dtype} and {b.dtype}")
    t = a if a is not None else b
    return 0 if t is None else _DTYPES[t.dtype]


# ------------------------------------------------------------------- layer norm


@functools.lru_cache(maxsize=512)
def _norm_bytes(rows, width):
    _sizes(rows=rows, columns=width)
    return lib().acdc_norm_workspace_size(rows, width)


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, dtype=None, save: bool = False, out=None) -> LayerNorm:
    """y = (x - mean) / sqrt(variance + eps) * weight + bias for each row, mean
    and variance over the row (``weight`` None: 1, ``bias`` None: 0).  y is of
    ``dtype`` (default: x's); ``save`` returns what ``layer_norm_backward`` needs."""
    r = _native(x, "norm", weight, bias, eps, _code(dtype), save, out)
    if r is not None:
        return LayerNorm(*r)
    rows, width, x_stride = _matrix("x", x)
    device = x.device
    _width_vector("weight", weight, width, device)
    _width_vector("bias", bias, width, device)
    vector_type = _one_type("weight and bias", weight, bias)
    if not 0.0 <= eps < float("inf"):
        raise ValueError(f"eps must be >= 0 and finite, got {eps}")
    if out is None:
        y = torch.empty(rows, width, dtype=_type("dtype", dtype, x.dtype), device=device)
        y_stride = width
    else:
        y, y_stride = out, _rows_of("out", out, rows, width, device, _type("dtype", dtype, out.dtype))
        _apart("out", out, ("x", x), ("weight", weight), ("bias", bias))
    saved = torch.empty(rows, 2, device=device) if save else None
    rc = _call(lib().acdc_norm_forward, device, x.data_ptr(), _DTYPES[x.dtype], x_stride, _ptr(weight), _ptr(bias), vector_type,
               eps, y.data_ptr(), _DTYPES[y.dtype], y_stride, _ptr(saved), rows, width)
    _check(rc, "acdc_norm_forward")
    _wrote(out)
    return LayerNorm(y, saved)


def layer_norm_backward(x, grad_y, weight, saved, out=None, grads=None, accumulate: bool = False, grad=(True, True, True),
                        dtype=None, workspace=None):
    """(grad_x, grad_weight, grad_bias) of ``layer_norm(x, weight, ...)`` from
    dL/dy, the last two summed over the rows.  ``out``: a tensor to write grad_x
    into (grad_y itself, if it has x's type).  ``grads`` = (grad_weight, grad_bias)
    tensors to write into, or with ``accumulate`` to add to (either may be None:
    not wanted); otherwise they are made, of ``dtype`` (default: the weight's, or
    float32).  ``grad`` tells which of the three are wanted."""
    want_x, want_w, want_b = grad
    gw, gb = grads if grads is not None else (None, None)
    r = _native(x, "norm_backward", grad_y, weight, saved, out, gw, gb, grads is not None, accumulate, want_x, want_w, want_b,
                _code(dtype), workspace)
    if r is not None:
        return r
    rows, width, x_stride = _matrix("x", x)
    device = x.device
    gy_stride = _rows_of("grad_y", grad_y, rows, width, device)
    _width_vector("weight", weight, width, device)
    if saved.shape != (rows, 2) or saved.dtype is not torch.float32 or saved.device != device or not saved.is_contiguous():
        raise ValueError(f"saved must be the contiguous float32 [{rows}, 2] tensor of the forward call")
    _values("saved", saved)
    gx = None
    gx_stride = width
    if want_x:
        gx = torch.empty(rows, width, dtype=x.dtype, device=device) if out is None else out
        if out is not None:
            gx_stride = _rows_of("out", out, rows, width, device, x.dtype)
            same = out.data_ptr() == grad_y.data_ptr() and gx_stride == gy_stride and out.dtype is grad_y.dtype
            _apart("out", out, ("x", x), ("weight", weight), ("saved", saved), *(() if same else (("grad_y", grad_y),)))
    if grads is not None:
        gw, gb = gw if want_w else None, gb if want_b else None
        for name, t in (("grad_weight", gw), ("grad_bias", gb)):
            if t is not None:
                _width_vector(name, t, width, device)
                _apart(name, t, ("x", x), ("grad_y", grad_y), ("weight", weight), ("saved", saved), ("out", gx),
                       ("grad_bias", gb if t is gw else None))
    else:
        if accumulate:
            raise ValueError("accumulate needs the gradient tensors to add into (grads=...)")
        made = _type("dtype", dtype, torch.float32 if weight is None else weight.dtype)
        gw = torch.empty(width, dtype=made, device=device) if want_w else None
        gb = torch.empty(width, dtype=made, device=device) if want_b else None
    grads_type = _one_type("grad_weight and grad_bias", gw, gb)
    need = _norm_bytes(rows, width)
    ws = _workspace(workspace, need, device)
    rc = _call(lib().acdc_norm_backward, device, x.data_ptr(), _DTYPES[x.dtype], x_stride, grad_y.data_ptr(), _DTYPES[grad_y.dtype],
               gy_stride, _ptr(weight), 0 if weight is None else _DTYPES[weight.dtype], saved.data_ptr(), _ptr(gx), gx_stride,
               _ptr(gw), _ptr(gb), grads_type, 1 if accumulate else 0, rows, width, ws.data_ptr(), need)
    _check(rc, "acdc_norm_backward")
    _wrote(out if want_x else None, *(() if grads is None else (gw, gb)))
    return gx, gw, gb


# -------------------------------------------------------------------- embedding


@functools.lru_cache(maxsize=512)
def _embedding_bytes(rows, width, classes):
    _sizes(rows=rows, columns=width, classes=classes)
    return lib().acdc_embedding_workspace_size(rows, width, classes)


def _finite(scale):
    if not math.isfinite(scale):
        raise ValueError(f"scale must be finite, got {scale}")


def embedding(tokens, weight, scale: float = 1.0, dtype=None, out=None):
    """scale * weight[tokens]: [rows, width] of ``dtype`` (default: the weight's).
    A negative token gives a row of zeros, one past the weight's rows a row of NaN."""
    r = _native(weight, "embedding", scale, _code(dtype), out, first=tokens)
    if r is not None:
        return r
    classes, width, stride = _matrix("weight", weight)
    device = weight.device
    rows = tokens.shape[0] if tokens.dim() == 1 else -1
    bits = _index("tokens", tokens, rows, device)
    if classes < 1:
        raise ValueError("weight must have a class at least")
    _finite(scale)
    if out is None:
        y = torch.empty(rows, width, dtype=_type("dtype", dtype, weight.dtype), device=device)
        y_stride = width
    else:
        y, y_stride = out, _rows_of("out", out, rows, width, device, _type("dtype", dtype, out.dtype))
        _apart("out", out, ("weight", weight), ("tokens", tokens))
    rc = _call(lib().acdc_embedding_forward, device, tokens.data_ptr(), bits, weight.data_ptr(), _DTYPES[weight.dtype], stride,
               scale, y.data_ptr(), _DTYPES[y.dtype], y_stride, rows, width, classes)
    _check(rc, "acdc_embedding_forward")
    _wrote(out)
    return y


def embedding_backward(tokens, grad_rows, classes: int, scale: float = 1.0, dtype=None, grad_weight=None,
                       accumulate: bool = False, workspace=None):
    """The gradient [classes, width] of ``embedding``'s weight from dL/drows, summed
    in the order of the rows.  ``grad_weight``: a tensor to write it into, or with
    ``accumulate`` to add it to (a weight that the loss shares: its gradient); only
    the tokens' rows of it are read and written then.  Otherwise it is made, of
    ``dtype`` (default: that of ``grad_rows``)."""
    r = _native(grad_rows, "embedding_backward", classes, scale, _code(dtype), grad_weight, accumulate, workspace, first=tokens)
    if r is not None:
        return r
    rows, width, stride = _matrix("grad_rows", grad_rows)
    device = grad_rows.device
    bits = _index("tokens", tokens, rows, device)
    if classes < 1:
        raise ValueError(f"classes must be positive, got {classes}")
    _sizes(classes=classes)
    _finite(scale)
    if grad_weight is None:
        if accumulate:
            raise ValueError("accumulate needs the grad_weight to add to")
        gw = torch.empty(classes, width, dtype=_type("dtype", dtype, grad_rows.dtype), device=device)
        gw_stride = width
    else:
        gw, gw_stride = grad_weight, _rows_of("grad_weight", grad_weight, classes, width, device,
                                              _type("dtype", dtype, grad_weight.dtype))
        _apart("grad_weight", gw, ("grad_rows", grad_rows), ("tokens", tokens))
    need = _embedding_bytes(rows, width, classes)
    ws = _aligned_workspace(workspace, need, device)
    rc = _call(lib().acdc_embedding_backward, device, tokens.data_ptr(), bits, grad_rows.data_ptr(), _DTYPES[grad_rows.dtype], stride,
               scale, gw.data_ptr(), _DTYPES[gw.dtype], gw_stride, 1 if accumulate else 0, rows, width, classes, ws.data_ptr(), need)
    _check(rc, "acdc_embedding_backward")
    _wrote(grad_weight)
    return gw


def workspace_bytes(rows: int, width: int, classes: int = 1) -> int:
    """Bytes of workspace that either backward call takes for these sizes."""
    return max(_norm_bytes(rows, width), _embedding_bytes(rows, width, classes))


# ------------------------------------------------------------------- autograd


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, dtype):
        r = layer_norm(x, weight, bias, eps, dtype, save=True)
        ctx.save_for_backward(x, weight, r.saved)
        ctx.bias_type = None if bias is None else bias.dtype
        return r.y

    @staticmethod
    def backward(ctx, grad_y):
        x, weight, saved = ctx.saved_tensors
        dtype = weight.dtype if weight is not None else ctx.bias_type
        got = layer_norm_backward(x, grad_y.contiguous(), weight, saved, grad=ctx.needs_input_grad[:3], dtype=dtype)
        return *(_once("layer_norm_autograd", g, x, grad_y, weight) for g in got), None, None


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, weight, scale, dtype):
        ctx.save_for_backward(tokens)
        ctx.classes, ctx.scale, ctx.dtype = weight.shape[0], scale, weight.dtype
        return embedding(tokens, weight, scale, dtype)

    @staticmethod
    def backward(ctx, grad_rows):
        tokens, = ctx.saved_tensors
        g = embedding_backward(tokens, grad_rows.contiguous(), ctx.classes, ctx.scale, dtype=ctx.dtype)
        return None, _once("embedding_autograd", g, grad_rows), None, None


def layer_norm_autograd(x, weight=None, bias=None, eps: float = 1e-5, dtype=None):
    """``layer_norm(...).y``, differentiable in x, weight and bias."""
    _capturable("layer_norm_autograd", x, weight, bias)
    return _LayerNorm.apply(x, weight, bias, eps, dtype)


def embedding_autograd(tokens, weight, scale: float = 1.0, dtype=None):
    """``embedding(...)``, differentiable in the weight."""
    _capturable("embedding_autograd", weight)
    return _Embedding.apply(tokens, weight, scale, dtype)
