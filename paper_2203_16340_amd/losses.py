"""Losses on the logits of a vocabulary, with their gradients: token log-probabilities, distillation from a teacher's top
logits, the clipped policy loss and the preference loss.  The tensors are checked and the results made in csrc/losses_binding.cpp
(_losses.so); formulas and conventions are in include/lbfgsb.h, whose structs are mirrored here for callers without torch.

Logits are 2-d float32, bfloat16 or float16 CUDA tensors with unit column stride (rows may be spaced apart and start on any
element).  Everything is enqueued on torch's current stream of the logits' device; nothing synchronises.  Every call
returns plain tensors without history, whether the logits require a gradient (or carry a tangent) or not: the gradient is a result, and
`logits.backward(r.grad)` hands it on to whatever made the logits.  A gradient written over the logits counts as an
operation in place: if what made them kept them (a tanh does), backward refuses.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import NamedTuple, Optional

from . import OK, _check, lib

BF16, F16 = 2, 3
I32, I64 = 0, 1
KL_KINDS = {"k1": 1, "k2": 2, "k3": 3}
PAIR_KINDS = {"sigmoid": 0, "hinge": 1, "ipo": 2}


class Logits(C.Structure):
    _fields_ = [("dtype", C.c_int), ("rows", C.c_int64), ("vocab", C.c_int64), ("ld", C.c_int64), ("z", C.c_void_p),
                ("temperature", C.c_double), ("grad", C.c_void_p), ("ld_grad", C.c_int64)]


class Teacher(C.Structure):
    _fields_ = [("index_type", C.c_int), ("logit_type", C.c_int), ("top", C.c_int64), ("ld", C.c_int64), ("index", C.c_void_p),
                ("logit", C.c_void_p), ("lse", C.c_void_p)]


class Rollout(C.Structure):
    _fields_ = [("labels", C.c_void_p), ("old_logp", C.c_void_p), ("advantage", C.c_void_p), ("ref_logp", C.c_void_p),
                ("weight", C.c_void_p)]


class PolicyOptions(C.Structure):
    _fields_ = [("clip_low", C.c_double), ("clip_high", C.c_double), ("kl_coef", C.c_double), ("entropy_coef", C.c_double),
                ("kl_kind", C.c_int)]


class PreferenceOptions(C.Structure):
    _fields_ = [("kind", C.c_int), ("length_normalised", C.c_int), ("beta", C.c_double), ("label_smoothing", C.c_double),
                ("margin", C.c_double)]


def declare(L) -> None:
    """Argument types of the entry points, on the loaded library."""
    vp, i64, dbl, size = C.c_void_p, C.c_int64, C.c_double, C.c_size_t
    lg = C.POINTER(Logits)
    L.lbfgsb_logits_workspace_bytes.restype = size
    L.lbfgsb_logits_workspace_bytes.argtypes = [lg]
    for name, args in (("token_logprob", [lg, vp, vp, vp, vp, vp, vp, size, vp]),
                       ("token_logprob_grad", [lg, vp, vp, vp, vp, vp, vp, vp]),
                       ("token_logprob_stats", [lg, vp, vp, vp, vp, vp, vp, vp, vp, size, vp]),
                       ("token_logprob_stats_grad", [lg, vp, vp, vp, vp, vp, vp, vp]),
                       ("distill_loss", [lg, C.POINTER(Teacher), vp, dbl, vp, vp, vp, size, vp]),
                       ("policy_loss", [lg, C.POINTER(Rollout), C.POINTER(PolicyOptions), dbl, vp, vp, vp, vp, vp, size, vp]),
                       ("preference_loss", [i64, i64, vp, vp, vp, vp, vp, C.POINTER(PreferenceOptions), dbl, vp, vp, vp, vp, vp])):
        f = getattr(L, "lbfgsb_" + name)
        f.restype, f.argtypes = C.c_int, args


class _TokenLogprob(NamedTuple):
    logp: "torch.Tensor"
    lse: "torch.Tensor"
    lse_rest: "torch.Tensor"
    entropy: Optional["torch.Tensor"]


class TokenLogprob(_TokenLogprob):
    """What token_logprob returns.  Beside the tuple's entries, for the way back: stats, whose first two rows are
    every row's largest logit and its sum of exponentials; a tuple that was taken apart and put together again has none (None)."""
    stats = None


class DistillLoss(NamedTuple):
    loss: "torch.Tensor"
    row_loss: "torch.Tensor"
    grad: Optional["torch.Tensor"]


class PolicyLoss(NamedTuple):
    loss: "torch.Tensor"
    row_loss: "torch.Tensor"
    logp: "torch.Tensor"
    entropy: Optional["torch.Tensor"]
    grad: Optional["torch.Tensor"]


class PreferenceLoss(NamedTuple):
    loss: "torch.Tensor"
    pair_loss: "torch.Tensor"
    rewards: "torch.Tensor"
    grad: Optional["torch.Tensor"]


_torch = None
_native = None


def _load():
    """torch and the binding, when the first of these functions is called (the package itself loads neither)."""
    global _torch, _native
    import torch
    lib()
    try:
        from . import _losses
    except ImportError as e:
        raise RuntimeError(f"{os.path.join(os.path.dirname(__file__), '_losses.so')} does not load ({e}): build it with "
                           "`python -m paper_2203_16340_amd.build`; there is no fallback path") from e
    _torch, _native = torch, _losses
    return _losses


def _call(f, t, *args):
    """f on torch's current stream of the device of t; raises what the C entry refuses, and returns the rest."""
    if not isinstance(t, _torch.Tensor) or not t.is_cuda:
        raise TypeError("the tensors must be on a GPU")
    index = t.get_device()
    if _torch.cuda.current_device() != index:
        with _torch.cuda.device(index):
            rc, *out = f(*args, _torch.cuda.current_stream().cuda_stream)
    else:
        # (the current stream's handle without an object around it: 0.1 us for 1.9)
        rc, *out = f(*args, _torch._C._cuda_getCurrentRawStream(index))
    if rc != OK:
        _check(rc)
    return out


def _kind(kinds: dict, kind: str, name: str) -> int:
    if kind not in kinds:
        raise ValueError(f"{name} must be one of {', '.join(kinds)} (got {kind!r})")
    return kinds[kind]


def _gradient(grad):
    """(a new one is wanted, the one to write to) of a `grad` argument"""
    return (grad, None) if grad is True or grad is False else (False, grad)


def token_logprob(logits, labels, *, temperature: float = 1.0, entropy: bool = False) -> TokenLogprob:
    """lbfgsb_token_logprob: log-probability of each row's label (int64; negative: ignored), the row's log-sum-exp (lse + lse_rest
    is more exact) and, if asked for, its entropy."""
    native = _native or _load()
    *out, stats = _call(native.token_logprob, logits, logits, labels, temperature, entropy)
    r = TokenLogprob(*out)
    r.stats = stats
    return r


def token_logprob_grad(logits, labels, forward: TokenLogprob, d_logp, *, temperature: float = 1.0, d_entropy=None, grad=True):
    """lbfgsb_token_logprob_grad: the gradient with respect to the logits of something whose gradient with respect to logp
    (and entropy) is d_logp (and d_entropy).  forward: what token_logprob returned for these logits at this temperature (with
    the entropy, for d_entropy); of one without stats, lse and lse_rest are used, and rows whose shares they do not tell, such as one
    held whole at float32's lowest value at temperature 1.5, get NaN.  grad: a tensor to write to (the logits themselves: in place), or True for a new one."""
    native = _native or _load()
    if grad is False or grad is None:
        raise TypeError("grad must be True or a tensor")
    return _call(native.token_logprob_grad, logits, logits, labels, forward.lse, forward.lse_rest, forward.entropy,
                 getattr(forward, "stats", None), d_logp, d_entropy,
                 temperature, _gradient(grad)[1])[0]


def distill_loss(logits, teacher_index, teacher_logit, *, teacher_lse=None, temperature: float = 1.0, weight=None, scale: float = 1.0,
                 grad=True) -> DistillLoss:
    """lbfgsb_distill_loss: divergence of the student's rows from a teacher known by its top logits.  teacher_index: (rows, top)
    int32 or int64, negative = padding; teacher_logit: (rows, top) of a logits type; teacher_lse: rows entries, the
    teacher's log-sum-exp at this temperature, or None (the top logits are then all there is).  grad: True (a new tensor), a
    tensor to write to (the logits themselves: in place), or False."""
    native = _native or _load()
    return DistillLoss(*_call(native.distill_loss, logits, logits, teacher_index, teacher_logit, teacher_lse, weight, temperature, scale,
                              *_gradient(grad)))


def policy_loss(logits, labels, old_logp, advantage, *, ref_logp=None, weight=None, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_coef: float = 0.0, kl_kind: str = "k3", entropy_coef: float = 0.0, entropy: bool = False, temperature: float = 1.0,
                scale: float = 1.0, grad=True) -> PolicyLoss:
    """lbfgsb_policy_loss: the clipped policy loss of every token with its KL term and entropy bonus, from the logits to their
    gradient in one call.  labels: int64, the tokens taken (negative: not counted); weight: the mask and the mean (for
    instance 1 / tokens, or 1 / (answers * tokens of the answer)).  entropy: return it too.  grad: as for distill_loss."""
    native = _native or _load()
    return PolicyLoss(*_call(native.policy_loss, logits, logits, labels, old_logp, advantage, ref_logp, weight, clip_low, clip_high, kl_coef,
                             _kind(KL_KINDS, kl_kind, "kl_kind"), entropy_coef, entropy, temperature, scale, *_gradient(grad)))


def preference_loss(logp, ref_logp, offsets, *, mask=None, weight=None, beta: float = 0.1, kind: str = "sigmoid",
                    label_smoothing: float = 0.0, margin: float = 0.0, length_normalised: bool = False, scale: float = 1.0,
                    grad: bool = True) -> PreferenceLoss:
    """lbfgsb_preference_loss: the loss on pairs of answers from their tokens' log-probabilities, and its gradient with respect to
    them (which token_logprob_grad takes to the logits).  offsets: int64, 2 pairs + 1 entries, the chosen answers and then
    the rejected ones; ref_logp: None for a loss without a reference; mask: bool or uint8, a token each."""
    native = _native or _load()
    return PreferenceLoss(*_call(native.preference_loss, logp, logp, ref_logp, offsets, mask, weight, beta, _kind(PAIR_KINDS, kind, "kind"),
                                 label_smoothing, margin, length_normalised, scale, grad))
