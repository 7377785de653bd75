"""Losses on the logits of a vocabulary, with their gradients: token log-probabilities, distillation from a teacher's top
logits, the clipped policy loss and the preference loss.  Argument marshalling only; formulas and conventions are in
include/lbfgsb.h.

Logits are 2-d float32, bfloat16 or float16 CUDA tensors with unit column stride (rows may be spaced apart and start on any
element).  Everything is enqueued on torch's current stream of the logits' device; nothing synchronises.  Every call
returns plain tensors: the gradient is a result, and `logits.backward(r.grad)` hands it on to whatever made the logits.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional

from . import _check, lib

BF16, F16 = 2, 3
I32, I64 = 0, 1
KL_KINDS = {"k1": 1, "k2": 2, "k3": 3}
PAIR_KINDS = {"sigmoid": 0, "hinge": 1, "ipo": 2}
MAX_TOP = 1024


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
                       ("distill_loss", [lg, C.POINTER(Teacher), vp, dbl, vp, vp, vp, size, vp]),
                       ("policy_loss", [lg, C.POINTER(Rollout), C.POINTER(PolicyOptions), dbl, vp, vp, vp, vp, vp, size, vp]),
                       ("preference_loss", [i64, i64, vp, vp, vp, vp, vp, C.POINTER(PreferenceOptions), dbl, vp, vp, vp, vp, vp])):
        f = getattr(L, "lbfgsb_" + name)
        f.restype, f.argtypes = C.c_int, args


class TokenLogprob(NamedTuple):
    logp: "torch.Tensor"
    lse: "torch.Tensor"
    lse_rest: "torch.Tensor"
    entropy: Optional["torch.Tensor"]


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


# What torch calls the types, filled when torch is first needed (the package itself does not load it).
_torch = None
_LOGIT_TYPES: dict = {}
_INDEX_TYPES: dict = {}


def _load_torch():
    global _torch
    import torch
    _torch = torch
    _LOGIT_TYPES.update({torch.float32: 1, torch.bfloat16: BF16, torch.float16: F16})
    _INDEX_TYPES.update({torch.int32: I32, torch.int64: I64})
    return torch


def _call(name: str, device, *args) -> None:
    """The entry point, on torch's current stream of `device`."""
    f, index = getattr(lib(), name), device.index
    if _torch.cuda.current_device() != index:
        with _torch.cuda.device(device):
            _check(f(*args, _torch.cuda.current_stream().cuda_stream))
    else:
        # (the current stream's handle without an object around it: 0.1 us for 1.9)
        _check(f(*args, _torch._C._cuda_getCurrentRawStream(index)))


def _logit_type(t, name: str) -> int:
    torch = _torch or _load_torch()
    dtype = _LOGIT_TYPES.get(t.dtype) if isinstance(t, torch.Tensor) else None
    if dtype is None or not t.is_cuda or t.dim() != 2 or (t.stride(1) != 1 and t.shape[1] != 1):
        raise TypeError(f"{name} must be a 2-d float32/bfloat16/float16 CUDA tensor with unit column stride")
    return dtype


def _stride(t) -> int:
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _vector(t, name: str, numel: int, device, dtype=None) -> int:
    """The address of a contiguous 1-d tensor of `numel` entries (float32 if not said otherwise)."""
    torch = _torch or _load_torch()
    if dtype is None:
        dtype = torch.float32
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.device != device or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {str(dtype)[6:]} tensor on {device}")
    if t.shape != (numel,):
        raise ValueError(f"{name} must have {numel} entries, got shape {tuple(t.shape)}")
    return t.data_ptr()


def _maybe(t, name: str, numel: int, device):
    return None if t is None else _vector(t, name, numel, device)


def _logits(z, temperature: float, grad):
    """The logits struct and the gradient's tensor.  grad: True = a new one, False/None = none, or a tensor to write to."""
    dtype = _logit_type(z, "logits")
    rows, vocab = z.shape
    ld = z.stride(0) if rows > 1 else vocab
    if grad is False or grad is None:
        return Logits(dtype, rows, vocab, ld, z.data_ptr(), temperature, None, 0), None
    if grad is True:
        grad = _torch.empty_like(z) if z.is_contiguous() else z.new_empty(z.shape)   # (the first is the cheaper call)
    elif _logit_type(grad, "grad") != dtype or grad.shape != z.shape or grad.device != z.device:
        raise TypeError("grad must have the type, shape and device of the logits")
    return Logits(dtype, rows, vocab, ld, z.data_ptr(), temperature, grad.data_ptr(), _stride(grad)), grad


def _rows(z, count: int):
    """New float32 tensors on the device of z, `count` of them of one entry a row and then one of no dimension."""
    empty, dev, f32, n = _torch.empty, z.device, _torch.float32, z.shape[0]
    return [empty(n, dtype=f32, device=dev) for _ in range(count)] + [empty((), dtype=f32, device=dev)]


def _workspace(lg: Logits, device):
    """A workspace for one call (torch keeps it until the stream is done with it) and its size."""
    n = lib().lbfgsb_logits_workspace_bytes(C.byref(lg))
    return (None, 0) if n == 0 else (_torch.empty(n, dtype=_torch.uint8, device=device), n)


def _address(t):
    return None if t is None else t.data_ptr()


def _kind(kinds: dict, kind: str, name: str) -> int:
    if kind not in kinds:
        raise ValueError(f"{name} must be one of {', '.join(kinds)} (got {kind!r})")
    return kinds[kind]


def token_logprob(logits, labels, *, temperature: float = 1.0, entropy: bool = False) -> TokenLogprob:
    """lbfgsb_token_logprob: log-probability of each row's label (int64; negative: ignored), the row's log-sum-exp (lse + lse_rest
    is more exact) and, if asked for, its entropy."""
    lg, _ = _logits(logits, temperature, None)
    n, dev = logits.shape[0], logits.device
    y = _vector(labels, "labels", n, dev, _torch.int64)
    out = _torch.empty((4 if entropy else 3, n), dtype=_torch.float32, device=dev).unbind(0)
    ws, nbytes = _workspace(lg, dev)
    _call("lbfgsb_token_logprob", dev, C.byref(lg), y, out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(),
          out[3].data_ptr() if entropy else None, _address(ws), nbytes)
    return TokenLogprob(out[0], out[1], out[2], out[3] if entropy else None)


def token_logprob_grad(logits, labels, forward: TokenLogprob, d_logp, *, temperature: float = 1.0, d_entropy=None, grad=True):
    """lbfgsb_token_logprob_grad: the gradient with respect to the logits of something whose gradient with respect to logp
    (and entropy) is d_logp (and d_entropy).  forward: what token_logprob returned for these logits (with the entropy, for
    d_entropy).  grad: a tensor to write to (the logits themselves: in place), or True for a new one."""
    if grad is False or grad is None:
        raise TypeError("grad must be True or a tensor")
    lg, out = _logits(logits, temperature, grad)
    n, dev = logits.shape[0], logits.device
    y = _vector(labels, "labels", n, dev, _torch.int64)
    _call("lbfgsb_token_logprob_grad", dev, C.byref(lg), y, _vector(forward.lse, "lse", n, dev),
          _maybe(forward.lse_rest, "lse_rest", n, dev), _maybe(forward.entropy, "entropy", n, dev),
          _vector(d_logp, "d_logp", n, dev), _maybe(d_entropy, "d_entropy", n, dev))
    return out


def distill_loss(logits, teacher_index, teacher_logit, *, teacher_lse=None, temperature: float = 1.0, weight=None, scale: float = 1.0,
                 grad=True) -> DistillLoss:
    """lbfgsb_distill_loss: divergence of the student's rows from a teacher known by its top logits.  teacher_index: (rows, top)
    int32 or int64, negative = padding; teacher_logit: (rows, top) of a logits type; teacher_lse: rows entries, the
    teacher's log-sum-exp at this temperature, or None (the top logits are then all there is).  grad: True (a new tensor), a
    tensor to write to (the logits themselves: in place), or False."""
    lg, out = _logits(logits, temperature, grad)
    n, dev = logits.shape[0], logits.device
    ttype = _logit_type(teacher_logit, "teacher_logit")
    itype = _INDEX_TYPES.get(teacher_index.dtype) if isinstance(teacher_index, _torch.Tensor) else None
    if itype is None or teacher_index.dim() != 2 or (teacher_index.stride(1) != 1 and teacher_index.shape[1] != 1):
        raise TypeError("teacher_index must be a 2-d int32/int64 tensor with unit column stride")
    if teacher_index.shape != teacher_logit.shape or teacher_index.shape[0] != n:
        raise ValueError(f"teacher_index and teacher_logit must both be ({n}, top), got {tuple(teacher_index.shape)}, {tuple(teacher_logit.shape)}")
    if teacher_index.device != dev or teacher_logit.device != dev:
        raise TypeError(f"the teacher's tensors must be on {dev}")
    if _stride(teacher_index) != _stride(teacher_logit):
        raise ValueError("teacher_index and teacher_logit must have the same row stride")
    t = Teacher(itype, ttype, teacher_index.shape[1], _stride(teacher_index), teacher_index.data_ptr(),
                teacher_logit.data_ptr(), _maybe(teacher_lse, "teacher_lse", n, dev))
    row, loss = _rows(logits, 1)
    ws, nbytes = _workspace(lg, dev)
    _call("lbfgsb_distill_loss", dev, C.byref(lg), C.byref(t), _maybe(weight, "weight", n, dev), float(scale), loss.data_ptr(),
          row.data_ptr(), _address(ws), nbytes)
    return DistillLoss(loss, row, out)


def policy_loss(logits, labels, old_logp, advantage, *, ref_logp=None, weight=None, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_coef: float = 0.0, kl_kind: str = "k3", entropy_coef: float = 0.0, entropy: bool = False, temperature: float = 1.0,
                scale: float = 1.0, grad=True) -> PolicyLoss:
    """lbfgsb_policy_loss: the clipped policy loss of every token with its KL term and entropy bonus, from the logits to their
    gradient in one call.  labels: int64, the tokens taken (negative: not counted); weight: the mask and the mean (for
    instance 1 / tokens, or 1 / (answers * tokens of the answer)).  entropy: return it too.  grad: as for distill_loss."""
    lg, out = _logits(logits, temperature, grad)
    n, dev = logits.shape[0], logits.device
    p = Rollout(_vector(labels, "labels", n, dev, _torch.int64), _vector(old_logp, "old_logp", n, dev),
                _vector(advantage, "advantage", n, dev), _maybe(ref_logp, "ref_logp", n, dev), _maybe(weight, "weight", n, dev))
    o = PolicyOptions(float(clip_low), float(clip_high), float(kl_coef), float(entropy_coef), _kind(KL_KINDS, kl_kind, "kl_kind"))
    *rows, loss = _rows(logits, 3 if entropy else 2)
    ws, nbytes = _workspace(lg, dev)
    _call("lbfgsb_policy_loss", dev, C.byref(lg), C.byref(p), C.byref(o), float(scale), loss.data_ptr(), rows[0].data_ptr(),
          rows[1].data_ptr(), rows[2].data_ptr() if entropy else None, _address(ws), nbytes)
    return PolicyLoss(loss, rows[0], rows[1], rows[2] if entropy else None, out)


def preference_loss(logp, ref_logp, offsets, *, mask=None, weight=None, beta: float = 0.1, kind: str = "sigmoid",
                    label_smoothing: float = 0.0, margin: float = 0.0, length_normalised: bool = False, scale: float = 1.0,
                    grad: bool = True) -> PreferenceLoss:
    """lbfgsb_preference_loss: the loss on pairs of answers from their tokens' log-probabilities, and its gradient with respect to
    them (which token_logprob_grad takes to the logits).  offsets: int64, 2 pairs + 1 entries, the chosen answers and then
    the rejected ones; ref_logp: None for a loss without a reference; mask: bool or uint8, a token each."""
    torch = _torch or _load_torch()
    if not (isinstance(logp, torch.Tensor) and logp.is_cuda):
        raise TypeError("logp must be a CUDA tensor")
    if not (isinstance(offsets, torch.Tensor) and offsets.dim() == 1 and offsets.shape[0] % 2 == 1):
        raise ValueError("offsets must have 2 * pairs + 1 entries")
    dev, n, pairs = logp.device, logp.numel(), offsets.shape[0] // 2
    o = PreferenceOptions(_kind(PAIR_KINDS, kind, "kind"), int(bool(length_normalised)), float(beta), float(label_smoothing), float(margin))
    args = (_vector(logp, "logp", n, dev), _maybe(ref_logp, "ref_logp", n, dev), _vector(offsets, "offsets", 2 * pairs + 1, dev, _torch.int64),
            None if mask is None else _vector(mask.view(torch.uint8) if mask.dtype == torch.bool else mask, "mask", n, dev, torch.uint8),
            _maybe(weight, "weight", pairs, dev))
    out = torch.empty(n, dtype=torch.float32, device=dev) if grad else None
    pair, rewards = torch.empty(pairs, dtype=torch.float32, device=dev), torch.empty(2 * pairs, dtype=torch.float32, device=dev)
    loss = torch.empty((), dtype=torch.float32, device=dev)
    _call("lbfgsb_preference_loss", dev, n, pairs, *args, C.byref(o), float(scale), loss.data_ptr(), pair.data_ptr(), rewards.data_ptr(),
          _address(out))
    return PreferenceLoss(loss, pair, rewards, out)
