"""Losses over rows of logits and their gradients, on libacdc.so.

They stand between a cascade's forward and backward pass: ``y`` is read as
logits over its ``N`` classes (or, as ``y[:, :V]``, over the first V), and the
gradient that a loss returns is the ``grad_y`` that ``acdc.backward`` takes.

* ``token_logprobs``    log-probability of one class per row (and the entropy),
                        with ``token_logprobs_backward`` for its gradient;
* ``policy_loss``       clipped policy loss with a KL term and an entropy bonus;
* ``preference_loss``   preference loss over pairs of sequences of rows.

Where a vocabulary is wider than a row, the logits are ``hidden @ weight.T`` of a
cascade's rows and a weight [classes, width], and they are not kept:

* ``vocab_loss``        cross entropy over the vocabulary, with the gradients of
                        rows and weight;
* ``vocab_logprobs``    log-probability of one class per row, with
                        ``vocab_logprobs_backward`` for the gradients.

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
import math
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


class VocabLogprobs(NamedTuple):
    logp: torch.Tensor                 # [rows]
    saved: Optional[torch.Tensor]      # [rows, 2], for vocab_logprobs_backward


class VocabLoss(NamedTuple):
    stats: torch.Tensor                # [2]: loss, sum of the weights
    logp: torch.Tensor                 # [rows]
    grad_hidden: Optional[torch.Tensor]
    grad_weight: Optional[torch.Tensor]
    saved: Optional[torch.Tensor]      # [rows, 2]
    row_grads: Optional[torch.Tensor]  # [rows]: dL/dlogp


def _native(logits, name, *args, first=None):
    """The call by the binding's native part (``first``: an argument before the
    logits), or None where the logits are not on the current device or an
    argument is not plainly what it should be (the code below then says what is
    wrong)."""
    device = logits.get_device()
    if device < 0 or device != torch._C._cuda_getDevice():
        return None
    if first is not None:
        args = (logits, *args)
        logits = first
    r = getattr(binding(), name)(logits, *args, torch._C._cuda_getCurrentRawStream(device))
    if type(r) is int:
        _check(r, f"acdc_{name}")
    return r


def _values(name, t):
    if t.is_neg():
        raise ValueError(f"{name} is a view that stands for the negative of its memory: give its resolve_neg()")
    if not _has_memory(t):
        raise ValueError(f"{name} is without memory: its storage was freed")


def _sizes(**sizes):
    """Sizes that the C entry points take in 32 bits: a longer one would come there as another."""
    for name, n in sizes.items():
        if n > 0x7fffffff:
            raise ValueError(f"{n} {name}: at most 2^31 - 1 are supported")


def _logits(x, name="logits"):
    if x.dim() != 2:
        raise ValueError(f"{name} must be [rows, classes], got {tuple(x.shape)}")
    rows, classes = x.shape
    if classes < 1:
        raise ValueError(f"{name} must have a class at least")
    _sizes(rows=rows, classes=classes)
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


# ----------------------------------------------------- losses over a vocabulary


def _matrix(name, t, device=None):
    """(rows, width, stride) of float32 or bfloat16 rows."""
    if t.dim() != 2:
        raise ValueError(f"{name} must be [rows, width], got {tuple(t.shape)}")
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    rows, width = t.shape
    if width < 1:
        raise ValueError(f"{name} must have a column at least")
    _sizes(rows=rows, columns=width)
    stride, inner = t.stride()
    if width > 1 and inner != 1:
        raise ValueError(f"{name} must have contiguous rows (stride 1 along the width, got {inner})")
    if rows <= 1:
        stride = max(stride, width)
    if stride < width:
        raise ValueError(f"{name} has overlapping rows (stride {stride}, width {width})")
    _values(name, t)
    return rows, width, stride


@functools.lru_cache(maxsize=512)
def _vocab_bytes(rows, width, classes, dtype, gradient):
    _sizes(rows=rows, columns=width, classes=classes)
    need = lib().acdc_vocab_workspace_size(rows, width, classes, dtype, gradient)
    if need == 0:
        raise ValueError(f"{rows} rows of {width} over {classes} classes: at most 2^24 rows, a width of 2^17 and 2^27 classes "
                         "are supported")
    return need


def vocab_workspace_bytes(hidden, weight, grad: bool = True) -> int:
    """Bytes of workspace of the calls below for this hidden and weight."""
    return _vocab_bytes(*hidden.shape, weight.shape[0], _DTYPES[hidden.dtype], 1 if grad else 0)


def _vocab_head(hidden, weight, targets, grad, workspace):
    """The packed description of the inputs, and the workspace."""
    rows, width, stride = _matrix("hidden", hidden)
    device = hidden.device
    classes, weight_width, weight_stride = _matrix("weight", weight, device)
    if weight.dtype is not hidden.dtype:
        raise ValueError(f"hidden and weight must have one type, got {hidden.dtype} and {weight.dtype}")
    if weight_width != width:
        raise ValueError(f"weight is {tuple(weight.shape)}: its rows must have hidden's width {width}")
    if classes < 1:
        raise ValueError("weight must have a class at least")
    bits = _index("targets", targets, rows, device)
    dtype = _DTYPES[hidden.dtype]
    need = _vocab_bytes(rows, width, classes, dtype, 1 if grad else 0)
    head = struct.pack("3Q3q4i", hidden.data_ptr(), weight.data_ptr(), targets.data_ptr(), stride, weight_stride, rows,
                       width, classes, dtype, bits)
    return head, _aligned_workspace(workspace, need, device), need


def _aligned_workspace(ws, need, device):
    if ws is not None and ws.data_ptr() % 256 != 0:
        raise ValueError("workspace must begin at a multiple of 256 bytes")
    return _workspace(ws, need, device)


def _apart(name, out, *others):
    """Whether `out` shares memory with an input: refused, as it is written while they are read."""
    if out.numel() == 0:
        return
    def span(t):
        last = sum((n - 1) * s for n, s in zip(t.shape, t.stride()))
        return t.data_ptr(), t.data_ptr() + (last + 1) * t.element_size()
    a, b = span(out)
    for other, t in others:
        if t is not None and t.numel() > 0:
            c, d = span(t)
            if a < d and c < b:
                raise ValueError(f"{name} overlaps {other}")


def _vocab_grads(hidden, weight, out, grad_weight, accumulate, wanted, *read):
    """(packed description, grad_hidden, grad_weight) for the gradients in `wanted`; `read`: what
    else the call reads, (name, tensor) each."""
    gh = gw = None
    gh_stride = gw_stride = 0
    if wanted[0]:
        gh = torch.empty(hidden.shape, dtype=hidden.dtype, device=hidden.device) if out is None else out
        _, _, gh_stride = _matrix("out", gh, hidden.device)
        if gh.shape != hidden.shape or gh.dtype is not hidden.dtype:
            raise ValueError(f"out must be like hidden, {tuple(hidden.shape)} {hidden.dtype}")
    if wanted[1]:
        if grad_weight is None:
            if accumulate:
                raise ValueError("accumulate needs the grad_weight to add to")
            gw = torch.empty(weight.shape, dtype=weight.dtype, device=weight.device)
        else:
            gw = grad_weight
        _, _, gw_stride = _matrix("grad_weight", gw, hidden.device)
        if gw.shape != weight.shape or (gw.dtype is not weight.dtype and gw.dtype is not torch.float32):
            raise ValueError(f"grad_weight must be {tuple(weight.shape)} {weight.dtype} or float32, got {tuple(gw.shape)} {gw.dtype}")
    if out is not None and gh is not None:
        _apart("out", gh, ("hidden", hidden), ("weight", weight), ("grad_weight", gw), *read)
    if grad_weight is not None and gw is not None:
        _apart("grad_weight", gw, ("hidden", hidden), ("weight", weight), *read)
    record = struct.pack("2Q2q2i", 0 if gh is None else gh.data_ptr(), 0 if gw is None else gw.data_ptr(), gh_stride, gw_stride,
                         0 if gw is None else _DTYPES[gw.dtype], 1 if accumulate else 0)
    return record, gh, gw


def _wants(grad):
    """Which of (grad_hidden, grad_weight) a call computes."""
    if grad in (True, False):
        return bool(grad), bool(grad)
    if grad not in ("hidden", "weight"):
        raise ValueError(f"grad must be True, False, 'hidden' or 'weight', not {grad!r}")
    return grad == "hidden", grad == "weight"


def vocab_logprobs(hidden, weight, targets, save: bool = False, workspace=None) -> VocabLogprobs:
    """Log-probability of each row's target under softmax(hidden @ weight.T),
    with ``save`` what ``vocab_logprobs_backward`` needs."""
    r = _native(hidden, "vocab_logprobs", weight, targets, save, workspace)
    if r is not None:
        return VocabLogprobs(*r)
    head, ws, need = _vocab_head(hidden, weight, targets, False, workspace)
    rows, device = hidden.shape[0], hidden.device
    logp = torch.empty(rows, device=device)
    saved = torch.empty(rows, 2, device=device) if save else None
    rc = _call(lib().acdc_vocab_logprob, device, head, logp.data_ptr(), _ptr(saved), ws.data_ptr(), need)
    _check(rc, "acdc_vocab_logprob")
    return VocabLogprobs(logp, saved)


def vocab_logprobs_backward(hidden, weight, targets, saved, grad_logp, scale=None, grad=True, out=None, grad_weight=None,
                            accumulate: bool = False, workspace=None):
    """(grad_hidden, grad_weight) from dL/dlogp of each row, times ``scale`` (a
    tensor of one value on the device) if given.  ``grad`` may be "hidden" or
    "weight" for one of them (the other is None).  ``out``: a tensor to write
    grad_hidden into; ``grad_weight``: one to write, or with ``accumulate`` to
    add, the weight's gradient into, float32 or of the weight's type."""
    wanted = _wants(grad)
    r = _native(hidden, "vocab_backward", weight, targets, saved, grad_logp, scale, *wanted, out, grad_weight, accumulate,
                workspace)
    if r is not None:
        return r
    head, ws, need = _vocab_head(hidden, weight, targets, True, workspace)
    rows, device = hidden.shape[0], hidden.device
    if saved.shape != (rows, 2) or saved.dtype is not torch.float32 or saved.device != device or not saved.is_contiguous():
        raise ValueError(f"saved must be the contiguous float32 [{rows}, 2] tensor of the forward call")
    _values("saved", saved)
    _vector("grad_logp", grad_logp, rows, device)
    if scale is not None:
        _vector("scale", scale.reshape(-1), 1, device)
    record, gh, gw = _vocab_grads(hidden, weight, out, grad_weight, accumulate, wanted, ("targets", targets), ("saved", saved),
                                  ("grad_logp", grad_logp), ("scale", scale))
    rc = _call(lib().acdc_vocab_backward, device, head, saved.data_ptr(), grad_logp.data_ptr(), _ptr(scale), record,
               ws.data_ptr(), need)
    _check(rc, "acdc_vocab_backward")
    _wrote(out if wanted[0] else None, grad_weight if wanted[1] else None)
    return gh, gw


def vocab_loss(hidden, weight, targets, weights=None, mean: bool = True, grad_scale: float = 1.0, grad=True,
               save: bool = False, out=None, grad_weight=None, accumulate: bool = False, workspace=None) -> VocabLoss:
    """Cross entropy of softmax(hidden @ weight.T) at one target per row: the
    mean (or, with ``mean`` off, the sum) of -logp under ``weights`` (>= 0; a row
    of weight 0, or with a negative target, takes no part).  The logits are
    computed in pieces of the vocabulary and not kept.  ``grad``, ``out``,
    ``grad_weight`` and ``accumulate`` as in ``vocab_logprobs_backward``;
    ``grad_scale`` multiplies the gradients.  ``save`` returns what
    ``vocab_logprobs_backward`` needs to compute them later."""
    wanted = _wants(grad)
    r = _native(hidden, "vocab_loss", weight, targets, weights, mean, grad_scale, *wanted, save, out, grad_weight,
                accumulate, workspace)
    if r is not None:
        return VocabLoss(*r)
    any_grad = wanted[0] or wanted[1]
    head, ws, need = _vocab_head(hidden, weight, targets, any_grad, workspace)
    rows, device = hidden.shape[0], hidden.device
    _vector("weights", weights, rows, device)
    if not math.isfinite(grad_scale):
        raise ValueError(f"grad_scale must be finite, got {grad_scale}")
    record, gh, gw = _vocab_grads(hidden, weight, out, grad_weight, accumulate, wanted, ("targets", targets),
                                  ("weights", weights)) if any_grad else (None, None, None)
    stats, logp = torch.empty(2, device=device), torch.empty(rows, device=device)
    saved = torch.empty(rows, 2, device=device) if save else None
    row_grads = torch.empty(rows, device=device) if save else None
    params = struct.pack("fi", grad_scale, 1 if mean else 0)
    rc = _call(lib().acdc_vocab_loss, device, head, _ptr(weights), params, stats.data_ptr(), logp.data_ptr(), _ptr(saved),
               _ptr(row_grads), record, ws.data_ptr(), need)
    _check(rc, "acdc_vocab_loss")
    _wrote(out if wanted[0] else None, grad_weight if wanted[1] else None)
    return VocabLoss(stats, logp, gh, gw, saved, row_grads)


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


def _capturable(call, *inputs):
    """Refuses to take into a captured graph what was made outside of it on the default
    stream: its backward pass would make that stream wait for the captured one, which
    ends the process.  A leaf is made there with the first operation on it, and stays
    while any result of one lives.  Without gradients there is no backward pass."""
    if torch.is_grad_enabled() and inputs[0].is_cuda and torch.cuda.is_current_stream_capturing() and \
            binding().made_on_default_stream(*inputs):
        raise RuntimeError(f"{call} is captured while results of its inputs that were computed on the default stream are "
                           "alive: drop them (and their losses) before the capture, or compute them on another stream")


class _VocabLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, targets):
        r = vocab_logprobs(hidden, weight, targets, save=True)
        ctx.save_for_backward(hidden, weight, targets, r.saved)
        return r.logp

    @staticmethod
    def backward(ctx, grad_logp):
        return *_vocab_gradients(ctx, "vocab_logprobs_autograd", grad_logp.contiguous(), None, grad_logp), None


def _vocab_gradients(ctx, call, grad_logp, scale, upstream):
    hidden, weight, targets, saved = ctx.saved_tensors[:4]
    wanted = ctx.needs_input_grad[:2]
    if not any(wanted):
        return None, None
    grad = True if all(wanted) else "hidden" if wanted[0] else "weight"
    got = vocab_logprobs_backward(hidden, weight, targets, saved, grad_logp, scale=scale, grad=grad)
    return tuple(_once(call, g, hidden, weight, upstream) for g in got)


class _VocabLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, targets, weights, mean, grad_scale):
        r = vocab_loss(hidden, weight, targets, weights, mean, grad=False, save=True)
        ctx.grad_scale = grad_scale
        ctx.save_for_backward(hidden, weight, targets, r.saved, r.row_grads)
        ctx.mark_non_differentiable(r.stats, r.logp)
        return r.stats[0].clone(), r.stats, r.logp

    @staticmethod
    def backward(ctx, grad_loss, _stats, _logp):
        scale = grad_loss.reshape(1).float()
        if ctx.grad_scale != 1.0:
            scale = scale * ctx.grad_scale
        return *_vocab_gradients(ctx, "vocab_loss_autograd", ctx.saved_tensors[4], scale, grad_loss), None, None, None, None


def vocab_logprobs_autograd(hidden, weight, targets):
    """``vocab_logprobs(...).logp``, differentiable in hidden and weight."""
    _capturable("vocab_logprobs_autograd", hidden, weight)
    return _VocabLogprobs.apply(hidden, weight, targets)


def vocab_loss_autograd(hidden, weight, targets, weights=None, mean: bool = True, grad_scale: float = 1.0):
    """(loss, stats, logp) of ``vocab_loss``; the loss is differentiable in hidden
    and weight, and ``grad_scale`` multiplies their gradients as it does there."""
    _capturable("vocab_loss_autograd", hidden, weight)
    return _VocabLoss.apply(hidden, weight, targets, weights, mean, grad_scale)


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
