"""Losses over rows of logits and their gradients, on libacdc.so.

They stand between a cascade's forward and backward pass: ``y`` is read as
logits over its ``N`` classes (or, as ``y[:, :V]``, over the first V), and the
gradient that a loss returns is the ``grad_y`` that ``acdc.backward`` takes.

* ``token_logprobs``    log-probability of one class per row (and the entropy),
                        with ``token_logprobs_backward`` for its gradient;
* ``policy_loss``       clipped policy loss with a KL term and an entropy bonus;
* ``preference_loss``   preference loss over pairs of sequences of rows.

Argument marshalling only, like the cascade's binding: every step of the
computation runs in HIP kernels on the current torch stream.  Logits are
float32 or bfloat16, [rows, classes], each row contiguous and the rows any
distance apart; gradients have the logits' dtype.  ``out`` may be the logits
themselves, or other columns of the same rows.  Targets are int32 or int64, one
class per row; a row with a negative target takes no part (its logits do not
matter, its gradient is 0), and a target past the classes gives NaN.  The
``*_autograd`` functions are the differentiable forms (first derivatives; a
second one raises).
"""

from __future__ import annotations

import functools
import struct
from typing import NamedTuple, Optional

import torch

from ._lib import binding, lib
from .acdc import _call, _check, _has_memory, _once, _ptr, _wrote

_DTYPES = {torch.float32: 0, torch.bfloat16: 1}
_BITS = {torch.int32: 32, torch.int64: 64}


class TokenLogprobs(NamedTuple):
    logp: torch.Tensor                 # [rows]
    entropy: Optional[torch.Tensor]    # [rows]
    saved: Optional[torch.Tensor]      # [rows, 4], for token_logprobs_backward


class PolicyLoss(NamedTuple):
    stats: torch.Tensor                # [6]: loss, policy, kl, entropy, clipped share, ratio
    logp: torch.Tensor                 # [rows]
    grad_logits: Optional[torch.Tensor]
    saved: Optional[torch.Tensor]      # [rows, 4]
    row_grads: Optional[torch.Tensor]  # [2, rows]: dL/dlogp, dL/dentropy


class PreferenceLoss(NamedTuple):
    stats: torch.Tensor                # [5]: loss, accuracy, margin, preferred reward, other reward
    logp: torch.Tensor                 # [rows]
    grad_logits: Optional[torch.Tensor]
    saved: Optional[torch.Tensor]      # [rows, 4]
    row_grads: Optional[torch.Tensor]  # [2, rows]


def _native(logits, name, *args):
    """The call by the binding's native part, or None where the logits are not
    on the current device or an argument is not plainly what it should be (the
    code below then says what is wrong)."""
    device = logits.get_device()
    if device < 0 or device != torch._C._cuda_getDevice():
        return None
    r = getattr(binding(), name)(logits, *args, torch._C._cuda_getCurrentRawStream(device))
    if type(r) is int:
        _check(r, f"acdc_{name}")
    return r


def _values(name, t):
    if t.is_neg():
        raise ValueError(f"{name} is a view that stands for the negative of its memory: give its resolve_neg()")
    if not _has_memory(t):
        raise ValueError(f"{name} is without memory: its storage was freed")


def _logits(x, name="logits"):
    if x.dim() != 2:
        raise ValueError(f"{name} must be [rows, classes], got {tuple(x.shape)}")
    rows, classes = x.shape
    if classes < 1:
        raise ValueError(f"{name} must have a class at least")
    if x.dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32 or bfloat16, not {x.dtype}")
    stride, inner = x.stride()
    if classes > 1 and inner != 1:
        raise ValueError(f"{name} must have contiguous rows (stride 1 along the classes, got {inner})")
    if rows <= 1:
        stride = max(stride, classes)
    if stride < classes:
        raise ValueError(f"{name} has overlapping rows (stride {stride}, {classes} classes)")
    _values(name, x)
    return rows, classes, stride


def _vector(name, t, n, device, dtype=torch.float32):
    if t is None:
        return
    if t.shape != (n,) or t.device != device or t.dtype is not dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} vector of {n} values on {device}, got "
                         f"{tuple(t.shape)} {t.dtype} on {t.device}")
    _values(name, t)


def _index(name, t, n, device):
    if t.dtype not in _BITS:
        raise ValueError(f"{name} must be int32 or int64, not {t.dtype}")
    _vector(name, t, n, device, t.dtype)
    return _BITS[t.dtype]


def _gradient(logits, out, rows, classes):
    """The tensor the gradient is written into, and its row stride."""
    if out is None:
        return torch.empty(rows, classes, dtype=logits.dtype, device=logits.device), classes
    if out.shape != logits.shape or out.dtype is not logits.dtype or out.device != logits.device:
        raise ValueError(f"out must be like logits, {tuple(logits.shape)} {logits.dtype} on {logits.device}")
    return out, _logits(out, "out")[2]


def _saved(saved, rows, device):
    if saved.shape != (rows, 4) or saved.dtype is not torch.float32 or saved.device != device or \
            not saved.is_contiguous():
        raise ValueError(f"saved must be the contiguous float32 [{rows}, 4] tensor of the forward call")
    _values("saved", saved)


@functools.lru_cache(maxsize=512)
def _logprob_bytes(rows, classes, dtype):
    return lib().acdc_logprob_workspace_size(rows, classes, dtype)


@functools.lru_cache(maxsize=512)
def _policy_bytes(rows, classes, dtype):
    return lib().acdc_policy_workspace_size(rows, classes, dtype)


@functools.lru_cache(maxsize=512)
def _preference_bytes(rows, classes, dtype, pairs):
    return lib().acdc_preference_workspace_size(rows, classes, dtype, pairs)


def workspace_bytes(logits, pairs: int = 0) -> int:
    """Bytes of workspace that any of the calls takes for these logits
    (``pairs`` of sequences for the preference loss)."""
    rows, classes, _ = _logits(logits)
    dtype = _DTYPES[logits.dtype]
    return max(_logprob_bytes(rows, classes, dtype), _policy_bytes(rows, classes, dtype),
               _preference_bytes(rows, classes, dtype, pairs))


def _workspace(ws, need, device):
    if ws is None:
        return torch.empty(max(need, 1), dtype=torch.uint8, device=device)
    if ws.dtype is not torch.uint8 or ws.dim() != 1 or ws.numel() < need or ws.device != device or not ws.is_contiguous():
        raise ValueError(f"workspace must be a contiguous uint8 vector of at least {need} bytes on {device}")
    _values("workspace", ws)
    return ws


def token_logprobs(logits, targets, entropy: bool = False, save: bool = False, workspace=None) -> TokenLogprobs:
    """Log-probability of each row's target under softmax(logits), with
    ``entropy`` the entropy of each row, with ``save`` what
    ``token_logprobs_backward`` needs."""
    r = _native(logits, "logprobs", targets, entropy, save, workspace)
    if r is not None:
        return TokenLogprobs(*r)
    rows, classes, stride = _logits(logits)
    device = logits.device
    bits = _index("targets", targets, rows, device)
    dtype = _DTYPES[logits.dtype]
    logp = torch.empty(rows, device=device)
    ent = torch.empty(rows, device=device) if entropy else None
    saved = torch.empty(rows, 4, device=device) if save else None
    need = _logprob_bytes(rows, classes, dtype)
    ws = _workspace(workspace, need, device)
    rc = _call(lib().acdc_logprob_forward, device, logits.data_ptr(), dtype, stride, targets.data_ptr(), bits, rows,
               classes, logp.data_ptr(), _ptr(ent), _ptr(saved), ws.data_ptr(), need)
    _check(rc, "acdc_logprob_forward")
    return TokenLogprobs(logp, ent, saved)


def token_logprobs_backward(logits, targets, saved, grad_logp, grad_entropy=None, scale=None, out=None):
    """dL/dlogits from dL/dlogp and dL/dentropy of each row, times ``scale`` (a
    tensor of one value on the device) if given."""
    r = _native(logits, "logprobs_backward", targets, saved, grad_logp, grad_entropy, scale, out)
    if r is not None:
        return r
    rows, classes, stride = _logits(logits)
    device = logits.device
    bits = _index("targets", targets, rows, device)
    _saved(saved, rows, device)
    _vector("grad_logp", grad_logp, rows, device)
    _vector("grad_entropy", grad_entropy, rows, device)
    if scale is not None:
        _vector("scale", scale.reshape(-1), 1, device)
    grad, grad_stride = _gradient(logits, out, rows, classes)
    rc = _call(lib().acdc_logprob_backward, device, logits.data_ptr(), _DTYPES[logits.dtype], stride,
               targets.data_ptr(), bits, saved.data_ptr(), grad_logp.data_ptr(), _ptr(grad_entropy), _ptr(scale),
               grad.data_ptr(), grad_stride, rows, classes)
    _check(rc, "acdc_logprob_backward")
    _wrote(out)
    return grad


def _results(logits, rows, stats, grad, save, out):
    device = logits.device
    classes = logits.shape[1]
    g, grad_stride = _gradient(logits, out, rows, classes) if grad else (None, classes)
    saved = torch.empty(rows, 4, device=device) if save else None
    row_grads = torch.empty(2, rows, device=device) if save else None
    return torch.empty(stats, device=device), torch.empty(rows, device=device), g, grad_stride, saved, row_grads


def policy_loss(logits, actions, logp_old, advantages, logp_ref=None, weights=None, clip=(0.2, 0.2),
                kl_coef: float = 0.0, entropy_coef: float = 0.0, mean: bool = True, grad_scale: float = 1.0,
                grad: bool = True, save: bool = False, out=None, workspace=None) -> PolicyLoss:
    """Clipped policy loss of one action per row.  With ratio = exp(logp -
    logp_old) and k = logp_ref - logp, each row's loss is

        -min(ratio a, clamp(ratio, 1 - clip[0], 1 + clip[1]) a)
        + kl_coef (exp(k) - k - 1) - entropy_coef entropy

    and the total its mean (or, with ``mean`` off, its sum) under ``weights``
    (>= 0; a row of weight 0 takes no part).  With ``kl_coef`` 0 ``logp_ref``
    serves the stats alone.  ``grad_scale`` multiplies the gradient of the logits
    (a loss scale, or 1 / steps of an accumulation).
    ``grad`` off computes the values alone; ``save`` returns what
    ``token_logprobs_backward`` needs to compute the gradient later."""
    low, high = clip
    r = _native(logits, "policy", actions, logp_old, advantages, logp_ref, weights, low, high, kl_coef, entropy_coef,
                grad_scale, mean, grad, save, out, workspace)
    if r is not None:
        return PolicyLoss(*r)
    rows, classes, stride = _logits(logits)
    device = logits.device
    bits = _index("actions", actions, rows, device)
    if kl_coef != 0.0 and logp_ref is None:
        raise ValueError("kl_coef needs logp_ref")
    if not (low >= 0 and high >= 0):
        raise ValueError(f"clip must be two distances >= 0, got {clip}")
    for name, t in (("logp_old", logp_old), ("logp_ref", logp_ref), ("advantages", advantages), ("weights", weights)):
        _vector(name, t, rows, device)
    dtype = _DTYPES[logits.dtype]
    stats, logp, g, grad_stride, saved, row_grads = _results(logits, rows, 6, grad, save, out)
    need = _policy_bytes(rows, classes, dtype)
    ws = _workspace(workspace, need, device)
    params = struct.pack("5fi", low, high, kl_coef, entropy_coef, grad_scale, 1 if mean else 0)
    rc = _call(lib().acdc_policy_loss, device, logits.data_ptr(), dtype, stride, actions.data_ptr(), bits,
               logp_old.data_ptr(), _ptr(logp_ref), advantages.data_ptr(), _ptr(weights), rows, classes, params,
               stats.data_ptr(), logp.data_ptr(), _ptr(g), grad_stride, _ptr(saved), _ptr(row_grads), ws.data_ptr(),
               need)
    _check(rc, "acdc_policy_loss")
    _wrote(out if grad else None)
    return PolicyLoss(stats, logp, g, saved, row_grads)


def preference_loss(logits, targets, offsets, logp_ref, beta: float = 0.1, label_smoothing: float = 0.0,
                    grad_scale: float = 1.0, grad: bool = True, save: bool = False, out=None,
                    workspace=None) -> PreferenceLoss:
    """Preference loss over pairs of sequences.  Sequence s holds the rows
    offsets[s] .. offsets[s + 1] - 1 (``offsets``: int32 or int64, one more than
    the sequences); sequence 2p is the preferred one of pair p, 2p + 1 the
    other.  reward = beta sum(logp - logp_ref) over a sequence's rows with a
    target, margin = the difference of a pair's rewards, and the loss the mean of

        -(1 - label_smoothing) log sigmoid(margin) - label_smoothing log sigmoid(-margin)
    """
    r = _native(logits, "preference", targets, offsets, logp_ref, beta, label_smoothing, grad_scale, grad, save, out,
                workspace)
    if r is not None:
        return PreferenceLoss(*r)
    rows, classes, stride = _logits(logits)
    device = logits.device
    bits = _index("targets", targets, rows, device)
    if offsets.dim() != 1 or offsets.numel() % 2 != 1:
        raise ValueError("offsets must hold 2 * pairs + 1 values: where each sequence begins, and the end")
    offset_bits = _index("offsets", offsets, offsets.numel(), device)
    _vector("logp_ref", logp_ref, rows, device)
    if not 0.0 <= label_smoothing <= 1.0:
        raise ValueError(f"label_smoothing must lie in [0, 1], got {label_smoothing}")
    pairs = offsets.numel() // 2
    dtype = _DTYPES[logits.dtype]
    stats, logp, g, grad_stride, saved, row_grads = _results(logits, rows, 5, grad, save, out)
    need = _preference_bytes(rows, classes, dtype, pairs)
    ws = _workspace(workspace, need, device)
    params = struct.pack("3f", beta, label_smoothing, grad_scale)
    rc = _call(lib().acdc_preference_loss, device, logits.data_ptr(), dtype, stride, targets.data_ptr(), bits,
               offsets.data_ptr(), offset_bits, logp_ref.data_ptr(), rows, classes, pairs, params, stats.data_ptr(),
               logp.data_ptr(), _ptr(g), grad_stride, _ptr(saved), _ptr(row_grads), ws.data_ptr(), need)
    _check(rc, "acdc_preference_loss")
    _wrote(out if grad else None)
    return PreferenceLoss(stats, logp, g, saved, row_grads)


# ------------------------------------------------------------------- autograd


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets):
        r = token_logprobs(logits, targets, entropy=True, save=True)
        ctx.save_for_backward(logits, targets, r.saved)
        return r.logp, r.entropy

    @staticmethod
    def backward(ctx, grad_logp, grad_entropy):
        logits, targets, saved = ctx.saved_tensors
        grad = token_logprobs_backward(logits, targets, saved, grad_logp.contiguous(), grad_entropy.contiguous())
        return _once("token_logprobs_autograd", grad, logits, grad_logp, grad_entropy), None


class _Loss(torch.autograd.Function):
    """A loss of the row statistics: the forward reads the logits once and
    keeps dL/dlogp and dL/dentropy of each row, the backward reads them again
    and writes the gradient, times the loss's own upstream gradient."""

    @staticmethod
    def forward(ctx, logits, targets, loss, args, options):
        if options.get("out") is not None:
            raise ValueError("out is not for the differentiable form: autograd makes the gradient's tensor")
        r = loss(logits, targets, *args, grad=False, save=True, **options)
        ctx.grad_scale, ctx.call = options.get("grad_scale", 1.0), loss.__name__ + "_autograd"
        ctx.save_for_backward(logits, targets, r.saved, r.row_grads)
        ctx.mark_non_differentiable(r.stats, r.logp)
        return r.stats[0].clone(), r.stats, r.logp

    @staticmethod
    def backward(ctx, grad_loss, _stats, _logp):
        logits, targets, saved, row_grads = ctx.saved_tensors
        scale = grad_loss.reshape(1).float()
        if ctx.grad_scale != 1.0:
            scale = scale * ctx.grad_scale
        grad = token_logprobs_backward(logits, targets, saved, row_grads[0], row_grads[1], scale=scale)
        return _once(ctx.call, grad, logits, grad_loss), None, None, None, None


def token_logprobs_autograd(logits, targets):
    """(logp, entropy), differentiable in the logits."""
    return _TokenLogprobs.apply(logits, targets)


def policy_loss_autograd(logits, actions, logp_old, advantages, **options):
    """(loss, stats, logp) of ``policy_loss``; the loss is differentiable in the
    logits, and ``grad_scale`` multiplies their gradient as it does there."""
    return _Loss.apply(logits, actions, policy_loss, (logp_old, advantages), options)


def preference_loss_autograd(logits, targets, offsets, logp_ref, **options):
    """(loss, stats, logp) of ``preference_loss``; the loss is differentiable in the
    logits, and ``grad_scale`` multiplies their gradient as it does there."""
    return _Loss.apply(logits, targets, preference_loss, (offsets, logp_ref), options)
