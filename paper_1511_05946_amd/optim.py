"""AdamW over a list of tensors and the global norm of their gradients, on
libacdc.so: the step that turns a cascade's ``grad_A``, ``grad_D`` and
``grad_bias`` into new diagonals, all tensors in one or a few launches.

Argument marshalling only; the work is enqueued on the current torch stream.
Parameters are float32, bfloat16 or complex64 (stepped as pairs of reals, as
the cascade's gradients of complex layers are dL/dRe + i dL/dIm), contiguous;
gradients float32 or bfloat16 (complex64 for complex parameters), conjugate
views among them.

The moments of a tensor are made by ``moments(param, bits)``:

* 32 bits: ``(m, v)``, float32;
* 8 bits: ``(m, v, m_scale, v_scale)``, m and v float8 (e4m3) codes with a
  float32 scale per 256 elements, m = code * scale and sqrt(v) = code * scale:
  2.03 bytes an element instead of 8.
"""

from __future__ import annotations

import ctypes
import struct

import torch

from ._lib import binding, lib
from .acdc import _call, _check, _has_memory, _wrote

SCALE_BLOCK = 256
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.complex64: 0}
_RECORD = struct.Struct("=7Qqffii")   # struct acdc_adamw_tensor


def _real_numel(t) -> int:
    return 2 * t.numel() if t.dtype is torch.complex64 else t.numel()


def _lazy(t) -> bool:
    """A view that torch marks as conjugated or negated without touching the
    memory that it shares with its base."""
    return t.is_conj() or t.is_neg()


def _listed(items):
    return items if isinstance(items, (list, tuple)) else list(items)


def _native_stream(tensors):
    """The current stream, if the native part of the binding can take tensors
    of the first one's device; None leaves them to the code that checks one by
    one and says what is wrong."""
    if not tensors or not isinstance(tensors[0], torch.Tensor):
        return None
    device = tensors[0].get_device()
    if device < 0 or device != torch._C._cuda_getDevice():
        return None
    return torch._C._cuda_getCurrentRawStream(device)


def moments(param, bits: int = 32):
    """Moments of zero for one parameter, in 32 or 8 bits."""
    n = _real_numel(param)
    device = param.device
    if bits == 32:
        return torch.zeros(n, device=device), torch.zeros(n, device=device)
    if bits != 8:
        raise ValueError(f"moments are kept in 32 or 8 bits, not {bits}")
    blocks = -(-n // SCALE_BLOCK)
    codes = [torch.zeros(n, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn) for _ in range(2)]
    return (*codes, torch.zeros(blocks, device=device), torch.zeros(blocks, device=device))


def _refuse_moments(i, state, n, device):
    if len(state) not in (2, 4):
        raise ValueError(f"moments[{i}] must be (m, v) or (m, v, m_scale, v_scale)")
    dtype = torch.float32 if len(state) == 2 else torch.float8_e4m3fn
    for k, t in enumerate(state):
        want, size = (dtype, n) if k < 2 else (torch.float32, -(-n // SCALE_BLOCK))
        if t.dtype is not want or t.numel() != size or not t.is_contiguous() or t.device != device:
            raise ValueError(f"moments[{i}][{k}] must be {size} contiguous {want} values on {device}, got "
                             f"{tuple(t.shape)} {t.dtype} on {t.device}")
        if _lazy(t):
            raise ValueError(f"moments[{i}][{k}] is a conjugate or negative view")
        if not _has_memory(t):
            raise ValueError(f"moments[{i}][{k}] is without memory")


def _refuse(i, p, g, master, n, device):
    if p.dtype not in _TYPES or not p.is_contiguous() or p.device != device:
        raise ValueError(f"params[{i}] must be a contiguous float32, bfloat16 or complex64 tensor, all on one device; got "
                         f"{p.dtype} on {p.device}")
    wanted = "complex64" if p.dtype is torch.complex64 else "float32 or bfloat16"
    if g is None or g.shape != p.shape or g.device != device or not g.is_contiguous() or \
            g.dtype not in _TYPES or (g.dtype is torch.complex64) != (p.dtype is torch.complex64):
        got = "None" if g is None else f"{tuple(g.shape)} {g.dtype} on {g.device}"
        raise ValueError(f"grads[{i}] must be a contiguous {wanted} tensor of shape {tuple(p.shape)} on {device}, got {got}")
    if master is not None and (p.dtype is not torch.bfloat16 or master.dtype is not torch.float32 or
                               master.numel() != n or not master.is_contiguous() or master.device != device):
        raise ValueError(f"masters[{i}] must be the contiguous float32 copy of a bfloat16 parameter of {n} elements")
    if _lazy(p) or (master is not None and _lazy(master)):
        raise ValueError(f"params[{i}] and its master must not be conjugate or negative views: they are written in place")
    for name, t in (("params", p), ("grads", g), ("masters", master)):
        if t is not None and not _has_memory(t):
            raise ValueError(f"{name}[{i}] is without memory")


def adamw_step(params, grads, moments, step: int, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.01,
               masters=None, grad_scale=None):
    """One AdamW step of every tensor, in place (lists or other iterables of as many each):

        m = beta1 m + (1 - beta1) g        v = beta2 v + (1 - beta2) g^2
        w = w (1 - lr weight_decay) - lr m / (1 - beta1^step) / (sqrt(v / (1 - beta2^step)) + eps)

    ``step`` counts from 1 (captured into a graph, every replay is the captured
    step, with its ``lr`` and bias correction).  ``lr`` and ``weight_decay`` are
    numbers or one number per tensor (diagonals near 1 are usually not decayed).
    ``masters``: per tensor the float32 copy of a bfloat16 parameter that is
    updated and rounded into it, or None.  ``grad_scale``: a float32 tensor of one
    value that multiplies every gradient, such as ``grad_norm(...)[1:]``; where it
    is not finite, or -0, the step leaves everything as it is: what ``grad_norm``
    with a ``max_norm`` gives for gradients that hold a NaN or an infinity."""
    params, grads, moments = _listed(params), _listed(grads), _listed(moments)
    if masters is not None:
        masters = _listed(masters)
    stream = _native_stream(params)
    if stream is not None:
        rc = binding().adamw(params, grads, moments, masters, lr, weight_decay, betas[0], betas[1], eps, step, grad_scale,
                             stream)
        if rc is not None:
            return _check(rc, "acdc_adamw_step")
    count = len(params)
    if len(grads) != count or len(moments) != count or (masters is not None and len(masters) != count):
        raise ValueError("params, grads, moments and masters must be lists of one length")
    lrs = [lr] * count if isinstance(lr, (int, float)) else list(lr)
    decays = [weight_decay] * count if isinstance(weight_decay, (int, float)) else list(weight_decay)
    if len(lrs) != count or len(decays) != count:
        raise ValueError("lr and weight_decay must be numbers or one number per tensor")
    if count == 0:
        return
    device = params[0].device
    size = _RECORD.size
    records = bytearray(size * count)
    resolved = []   # (kept until the step is enqueued)
    for i in range(count):
        p, g, state = params[i], grads[i], moments[i]
        master = masters[i] if masters is not None else None
        n = _real_numel(p)
        _refuse(i, p, g, master, n, device)
        _refuse_moments(i, state, n, device)
        if _lazy(g):   # as autograd hands out the gradient of a parameter that was used conjugated
            g = g.resolve_conj().resolve_neg()
            resolved.append(g)
        scales = (state[2].data_ptr(), state[3].data_ptr()) if len(state) == 4 else (0, 0)
        _RECORD.pack_into(records, size * i, p.data_ptr(), 0 if master is None else master.data_ptr(), g.data_ptr(),
                          state[0].data_ptr(), state[1].data_ptr(), *scales, n, lrs[i], decays[i],
                          _TYPES[p.dtype], _TYPES[g.dtype])
    if grad_scale is not None and (grad_scale.numel() != 1 or grad_scale.dtype is not torch.float32 or
                                   grad_scale.device != device or not _has_memory(grad_scale)):
        raise ValueError(f"grad_scale must be one float32 value on {device}")
    if grad_scale is not None:
        grad_scale = grad_scale.resolve_neg()
    buf = (ctypes.c_char * len(records)).from_buffer(records)
    rc = _call(lib().acdc_adamw_step, device, ctypes.addressof(buf), count, float(betas[0]), float(betas[1]),
               float(eps), int(step), None if grad_scale is None else grad_scale.data_ptr())
    _check(rc, "acdc_adamw_step")
    _wrote(*params, *(masters or ()), *(t for state in moments for t in state))


def grad_norm(grads, max_norm=None, out=None):
    """[norm, scale] on the device: the 2-norm of all gradients together and the
    factor min(1, max_norm / (norm + 1e-6)) that clips them (1 without
    ``max_norm``), which ``adamw_step`` takes as ``grad_scale=result[1:]``. The 0 of
    an infinite norm is -0, with which the step is left out as with NaN."""
    grads = _listed(grads)
    stream = _native_stream(grads)
    if stream is not None and (max_norm is None or max_norm > 0):
        r = binding().grad_norm(grads, max_norm or 0.0, out, stream)
        if r.__class__ is int:
            _check(r, "acdc_grad_norm")
        elif r is not None:
            return r
    count = len(grads)
    if count == 0:
        raise ValueError("grad_norm needs a tensor at least")
    if max_norm is not None and not max_norm > 0:
        raise ValueError(f"max_norm must be positive, got {max_norm}")
    device = grads[0].device
    ptrs, sizes, types = [], [], []
    for i, g in enumerate(grads):
        if g.dtype not in _TYPES or not g.is_contiguous() or g.device != device:
            raise ValueError(f"grads[{i}] must be a contiguous float32, bfloat16 or complex64 tensor, all on one device; "
                             f"got {g.dtype} on {g.device}")
        if not _has_memory(g):
            raise ValueError(f"grads[{i}] is without memory")
        ptrs.append(g.data_ptr())
        sizes.append(_real_numel(g))
        types.append(_TYPES[g.dtype])
    given = out
    if out is None:
        out = torch.empty(2, device=device)
    elif out.shape != (2,) or out.dtype is not torch.float32 or out.device != device or not out.is_contiguous() or \
            _lazy(out) or not _has_memory(out):
        raise ValueError(f"out must be a contiguous float32 vector of 2 values on {device}")
    ptrs, sizes, types = struct.pack(f"{count}Q", *ptrs), struct.pack(f"{count}q", *sizes), struct.pack(f"{count}i", *types)
    need = lib().acdc_grad_norm_workspace_size(sizes, count)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device=device)
    rc = _call(lib().acdc_grad_norm, device, ptrs, sizes, types, count, float(max_norm or 0.0), out.data_ptr(),
               ws.data_ptr(), need)
    _check(rc, "acdc_grad_norm")
    _wrote(given)
    return out
