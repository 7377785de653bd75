"""What makes rollouts for the losses on logits: products with 4-bit weights, tokens drawn from logits by given numbers, and
verification of drafted tokens against a target's logits.  The tensors are checked and the results made in
csrc/rollouts_binding.cpp (in _losses.so); formulas and conventions are in include/lbfgsb.h, whose structs are mirrored here.

Logits are as for the losses: float32, bfloat16 or float16 CUDA tensors whose last dimension has unit stride.  Everything is enqueued on
torch's current stream of their device; nothing synchronises, and results carry no history.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional

from . import losses
from .losses import Logits, _call, _load


class Weights4Struct(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("group", C.c_int64), ("scale_type", C.c_int), ("codes", C.c_void_p),
                ("scale", C.c_void_p), ("zero", C.c_void_p)]


class Drafts(C.Structure):
    _fields_ = [("dtype", C.c_int), ("requests", C.c_int64), ("drafts", C.c_int64), ("vocab", C.c_int64), ("z", C.c_void_p), ("ld", C.c_int64),
                ("ld_request", C.c_int64), ("temperature", C.c_double), ("draft_z", C.c_void_p), ("draft_ld", C.c_int64),
                ("draft_ld_request", C.c_int64), ("draft_temperature", C.c_double), ("draft_logp", C.c_void_p), ("drafted", C.c_void_p),
                ("lengths", C.c_void_p), ("uniform", C.c_void_p), ("last_uniform", C.c_void_p)]


def declare(L) -> None:
    """Argument types of the entry points, on the loaded library."""
    vp, i64, size, num = C.c_void_p, C.c_int64, C.c_size_t, C.c_int
    w, lg, d = C.POINTER(Weights4Struct), C.POINTER(Logits), C.POINTER(Drafts)
    for name, arg in (("packed4_bytes", w), ("draw_workspace_bytes", lg), ("verify_workspace_bytes", d)):
        f = getattr(L, "lbfgsb_" + name)
        f.restype, f.argtypes = size, [arg]
    L.lbfgsb_matvec4_workspace_bytes.restype, L.lbfgsb_matvec4_workspace_bytes.argtypes = size, [w, i64, num]
    for name, args in (("quantize4", [num, i64, vp, w, vp]), ("pack4", [w, vp, size, vp]),
                       ("matvec4", [w, vp, i64, num, i64, vp, num, i64, vp, vp, size, vp]),
                       ("draw_tokens", [lg, vp, vp, vp, vp, size, vp]), ("verify_draft", [d, vp, vp, vp, vp, size, vp])):
        f = getattr(L, "lbfgsb_" + name)
        f.restype, f.argtypes = num, args


class Codes4(NamedTuple):
    codes: "torch.Tensor"
    scale: "torch.Tensor"
    zero: Optional["torch.Tensor"]


class Weights4:
    """Weights of 4 bits as matvec4 reads them (pack4 makes them): `rows` outputs, `cols` inputs, a scale (and zero) for every `group`
    columns of a row.  A `packed` that was stored is given back with the same numbers; matvec4 refuses one that is too short for them."""

    def __init__(self, packed, rows: int, cols: int, group: int, scale_type: int, has_zero: bool):
        self.packed, self.rows, self.cols, self.group = packed, rows, cols, group
        self._rest = (rows, cols, group, scale_type, has_zero)

    def __repr__(self) -> str:
        return f"Weights4({self.rows} x {self.cols}, groups of {self.group}, {self.packed.numel()} bytes on {self.packed.device})"


class DrawTokens(NamedTuple):
    tokens: "torch.Tensor"
    logp: "torch.Tensor"


class VerifyDraft(NamedTuple):
    tokens: "torch.Tensor"
    count: "torch.Tensor"
    logp: "torch.Tensor"


def quantize4(weight, *, group: int = 128, symmetric: bool = False, scale_dtype=None) -> Codes4:
    """lbfgsb_quantize4: the nearest 4-bit codes of a (rows, cols) matrix, two a byte, the even column in the low four bits, with a scale and
    (symmetric: without) a zero for each `group` columns.  scale_dtype: that of the weight unless given."""
    native = losses._native or _load()
    return Codes4(*_call(native.quantize4, weight, weight, group, symmetric, scale_dtype))


def pack4(codes, scale, zero=None, *, cols: Optional[int] = None, group: int = 128) -> Weights4:
    """lbfgsb_pack4: codes (rows, ceil(cols / 2)) uint8, scale and zero (rows, ceil(cols / group)) of one logits type; w = scale (code - zero),
    and 8 in the place of zeros that are None.  cols: 2 * codes.shape[1] unless given.  The tensors are not kept."""
    native = losses._native or _load()
    if cols is None:
        cols = 2 * codes.shape[-1]
    packed, scale_type = _call(native.pack4, codes, codes, scale, zero, cols, group)
    return Weights4(packed, codes.shape[0], cols, group, scale_type, zero is not None)


def matvec4(x, weights: Weights4, *, dtype=None, out=None):
    """lbfgsb_matvec4: x W^T for a few rows x (tokens, cols), in x's dtype or float32 (dtype=torch.float32).  out: a (tokens, rows) tensor of
    either to write to, which counts as an operation in place."""
    native = losses._native or _load()
    return _call(native.matvec4, x, x, weights.packed, *weights._rest, dtype, out)[0]


def draw_tokens(logits, uniform, *, temperature: float = 1.0) -> DrawTokens:
    """lbfgsb_draw_tokens: a token for each row of (rows, vocab) logits from a float32 number in [0, 1) for each, the first at which the
    running sum of probabilities passes it, and its log-probability."""
    native = losses._native or _load()
    return DrawTokens(*_call(native.draw_tokens, logits, logits, uniform, temperature))


def verify_draft(logits, drafted, uniform, last_uniform, *, draft_logits=None, draft_logp=None, lengths=None, temperature: float = 1.0,
                 draft_temperature: Optional[float] = None) -> VerifyDraft:
    """lbfgsb_verify_draft: how many of each request's drafted tokens stand against the target's logits (requests, drafts + 1, vocab), and the
    token after them.  drafted: (requests, drafts) int64; uniform: as many float32 numbers in [0, 1), last_uniform: one for each request;
    draft_logits: (requests, drafts, vocab) of the logits' dtype, or None for a drafter that is certain of its tokens; draft_logp: what
    draw_tokens gave with the drafted tokens (None: worked out from draft_logits); lengths: int64, drafts of each request where they are fewer,
    negative for one that has ended.  draft_temperature: that of the target unless given.
    Returns tokens and logp (requests, drafts + 1), -1 and 0 behind what is emitted, and count."""
    native = losses._native or _load()
    return VerifyDraft(*_call(native.verify_draft, logits, logits, drafted, uniform, last_uniform, draft_logits, draft_logp, lengths, temperature,
                              temperature if draft_temperature is None else draft_temperature))
