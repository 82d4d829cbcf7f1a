"""ctypes binding of what stands around the experts of a transformer block
(include/moe_block.h): argument marshalling only, like ``experts``.

    logits [T, E] --choose--> ids, gates --the layer--> y [T, H] --join--> the stream, the next block's input

Tensors are contiguous and on the GPU.  Every function takes ``stream`` (a torch
stream; default: the current one) and only enqueues work on it; outputs that are not
given with ``out`` are allocated for that stream, and ones that are count as changed
in place, as in ``experts``.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from . import binding as _b
from .binding import MoeError, Workspace
from .experts import (MX4, _FLOAT, _F32, _I32, _MOST, _TYPES, _U8, _BF16, _check, _empty, _mx4_check,
                      _status_word, _stream, _too_large, _two, _written)

EXPORTED = (
    "moe_choose", "moe_choose_grad", "moe_join", "moe_join_grad_scratch_size", "moe_join_grad",
    "moe_few_scratch_size", "moe_few_forward", "moe_few_forward_mx4", "moe_block_abi_version",
)

FEW_TOKENS = 16                              # tokens of layer_few
_SCORES = {"softmax": 0, "sigmoid": 1}       # moe_score_t
_NONE, _TOKEN, _CHANNEL = 0, 1, 2            # moe_gate_t
_lib = None


def lib() -> ctypes.CDLL:
    """The HIP library with this module's functions declared."""
    global _lib
    if _lib is None:
        L = _b.lib()
        vp, sz, i32, f32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_float
        L.moe_choose.argtypes = [vp] * 4 + [i32] * 6 + [f32, vp]
        L.moe_choose_grad.argtypes = [vp] * 4 + [i32] * 6 + [f32, vp, vp]
        L.moe_join.argtypes = [vp] * 8 + [i32] * 7 + [f32, ctypes.c_double, f32, vp]
        L.moe_join_grad_scratch_size.argtypes = [i32] * 2
        L.moe_join_grad.argtypes = [vp] * 13 + [i32] * 7 + [f32, ctypes.c_double, f32, vp, sz, vp]
        L.moe_few_scratch_size.argtypes = [i32] * 5
        L.moe_few_forward.argtypes = [vp] * 6 + [i32] * 7 + [vp, sz, vp]
        L.moe_few_forward_mx4.argtypes = [vp] * 8 + [i32] * 7 + [vp, sz, vp]
        for name in EXPORTED:
            getattr(L, name).restype = sz if name.endswith("_size") else ctypes.c_int
        _lib = L
    return _lib


def _ptr(t):
    return None if t is None else t.data_ptr()


def _place(stream, *tensors):
    """The handle of the stream to launch on; all of a call is on the current device."""
    device = torch.cuda.current_device() if _b._raw_device is None else _b._raw_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise TypeError(f"expected tensors on the current device ({device}), got one on {t.device}")
    if stream is not None and stream.device_index != device:
        raise TypeError(f"expected a stream of the current device ({device}), got one of {stream.device_index}")
    return _stream(stream)


# ---- the router's choice ---------------------------------------------------------------

class Choice(NamedTuple):
    """expert_ids int32 and gates fp32 [T, topk], as sort_by_expert and layer_few take
    them; slots without an expert: -1 and 0."""
    expert_ids: torch.Tensor
    gates: torch.Tensor


def _score(score):
    if score not in _SCORES:
        raise ValueError(f"score: expected one of {', '.join(_SCORES)}, got {score!r}")
    return _SCORES[score]


def choose(logits, topk: int, bias=None, score: str = "softmax", renormalize: bool = True, scale: float = 1.0,
           out: Optional[Choice] = None, stream=None) -> Choice:
    """moe_choose: logits [T, E] (bf16 or fp32) to the experts of the topk largest
    logits + bias (fp32 [E]; it acts on the choice alone), ties to the lower index,
    and their gates: scale times the score (softmax over all experts, or sigmoid),
    renormalised over the chosen or not.  Logits of -inf are never chosen."""
    T, E = _two(logits, "logits", _FLOAT)
    if (T | E | topk) > _MOST:
        _too_large("moe_choose")
    if bias is not None:
        _check(bias, "bias", (E,), _F32)
    given, shape = out, (T, topk)
    L = lib()
    if out is None:
        out = Choice(_empty(shape, torch.int32, logits.device, stream), _empty(shape, torch.float32, logits.device, stream))
    else:
        _check(out[0], "expert_ids", shape, _I32)
        _check(out[1], "gates", shape, _F32)
    r = L.moe_choose(logits.data_ptr(), _ptr(bias), out[0].data_ptr(), out[1].data_ptr(), T, E, topk,
                     _TYPES[logits.dtype], _score(score), renormalize, scale, _place(stream, logits, bias, *out))
    if r < 0:
        raise MoeError(r, "moe_choose")
    if given is not None:
        _written(given)
    return out


def choose_grad(d_gates, logits, expert_ids, score: str = "softmax", renormalize: bool = True, scale: float = 1.0,
                out=None, workspace: Optional[Workspace] = None, stream=None):
    """moe_choose_grad: the gates' gradient fp32 [T, topk], the logits and the chosen
    ids to the logits' gradient [T, E], of their type."""
    T, E = shape = _two(logits, "logits", _FLOAT)
    topk = _two(expert_ids, "expert_ids", _I32)[1]
    if (T | E | topk) > _MOST:
        _too_large("moe_choose_grad")
    _check(expert_ids, "expert_ids", (T, topk), _I32)
    _check(d_gates, "d_gates", (T, topk), _F32)
    given = out
    if out is None:
        out = _empty(shape, logits.dtype, logits.device, stream)
    else:
        _check(out, "out", shape, (logits.dtype,))
    r = lib().moe_choose_grad(d_gates.data_ptr(), logits.data_ptr(), expert_ids.data_ptr(), out.data_ptr(), T, E, topk,
                              _TYPES[logits.dtype], _score(score), renormalize, scale, _status_word(workspace),
                              _place(stream, d_gates, logits, expert_ids, out))
    if r < 0:
        raise MoeError(r, "moe_choose_grad")
    if given is not None:
        _written((given,))
    return out


# ---- the residual join -------------------------------------------------------------------

class Joined(NamedTuple):
    """The residual stream after a block [T, H], and its norm, the next block's input
    (None without one)."""
    h: torch.Tensor
    z: Optional[torch.Tensor]


class JoinGrads(NamedTuple):
    """Gradients of join's h, y, after, gate and before (fp32 for the last three), None
    for what the join did not have."""
    h: Optional[torch.Tensor]
    y: Optional[torch.Tensor]
    after: Optional[torch.Tensor]
    gate: Optional[torch.Tensor]
    before: Optional[torch.Tensor]


def _weights(T, H, after, gate, before):
    """The kind of gate and the type that norms' weights and the gate share."""
    dtype = None
    for what, t in (("after", after), ("before", before)):
        if t is not None:
            dtype = dtype or t.dtype
            _check(t, what, (H,), _FLOAT if dtype in _FLOAT and dtype == t.dtype else (dtype,))
    kind = _NONE
    if gate is not None:
        dtype = dtype or gate.dtype
        kind = _CHANNEL if gate.shape == (1, H) else _TOKEN
        _check(gate, "gate", (1, H) if kind == _CHANNEL else (T, 1), (dtype,) if dtype in _FLOAT else _FLOAT)
    return kind, _TYPES[dtype] if dtype is not None else 1


def _rng(rng, drop):
    if not 0.0 <= drop < 1.0:
        raise ValueError(f"drop: expected a probability below 1, got {drop}")
    if drop > 0.0:
        if rng is None:
            raise TypeError("rng: dropout needs one, int64 [2] (seed, offset)")
        _check(rng, "rng", (2,), (torch.int64,))
        return rng.data_ptr()
    return None


def join(h, y=None, after=None, gate=None, scale: float = 1.0, drop: float = 0.0, rng=None, before=None,
         eps: float = 1e-6, out: Optional[Joined] = None, dtype=torch.bfloat16, stream=None) -> Joined:
    """moe_join: y [T, H], a block's output, onto the residual stream h [T, H] (each
    bf16 or fp32): h + scale drop(gate norm(y) after), and that normalised times
    `before` (of `dtype`), the next block's input.
      after, before  weights [H] of the norms after and before a block, or None
      gate           [T, 1] (of tokens) or [1, H] (of channels), or None; of the
                     weights' type (all bf16 or all fp32)
      drop           dropout's probability; rng: int64 [2] on the GPU, seed and offset,
                     read as the call runs (a program gives every call numbers of its own)
    h None: nothing to add to (the result is of y's type).  y None: h's norm alone.
    out: where both go (out.h may be h itself; out.z None without `before`)."""
    if h is None and y is None:
        raise TypeError("expected h, y or both")
    some = h if h is not None else y
    T, H = shape = _two(some, "h" if h is not None else "y", _FLOAT)
    if (T | H) > _MOST:
        _too_large("moe_join")
    if y is not None and h is not None:
        _check(y, "y", shape, _FLOAT)
    kind, w_type = _weights(T, H, after, gate, before)
    seeds, given, L = _rng(rng, drop), out, lib()
    if out is None:
        x = h if y is None else _empty(shape, some.dtype, some.device, stream)
        z = None if before is None else _empty(shape, dtype, some.device, stream)
        out = Joined(x, z)
    x, z = out
    if y is not None:
        _check(x, "out.h", shape, (some.dtype,))
    if before is not None:
        _check(z, "out.z", shape, _FLOAT)
    r = L.moe_join(_ptr(h), _ptr(y), _ptr(after), _ptr(gate), _ptr(before), seeds,
                   None if y is None else x.data_ptr(), None if before is None else z.data_ptr(), T, H,
                   _TYPES[some.dtype], 0 if y is None else _TYPES[y.dtype], 0 if before is None else _TYPES[z.dtype],
                   w_type, kind, scale, drop, eps,
                   _place(stream, h, y, after, gate, before, rng if seeds else None, x, z if before is not None else None))
    if r < 0:
        raise MoeError(r, "moe_join")
    if given is not None:
        if y is not None:
            _written((x,) if before is None else (x, z))
        elif before is not None:
            _written((z,))
    return out


def join_grad_scratch_size(T: int, H: int) -> int:
    return 0 if max(T, H) > _MOST else int(lib().moe_join_grad_scratch_size(T, H))


def join_grad(d_h, d_z, h, y=None, after=None, gate=None, scale: float = 1.0, drop: float = 0.0, rng=None, before=None,
              eps: float = 1e-6, out: Optional[JoinGrads] = None, residual: bool = True, scratch=None,
              stream=None) -> JoinGrads:
    """moe_join_grad: from the gradients of join's results, d_h [T, H] (of the stream's
    type) and d_z [T, H] (either may be None), its other arguments as they were, and h,
    the stream as join returned it (read with d_z only).  residual False: join had no h
    (no gradient of it).  out: where the gradients go, None for ones that are not wanted
    (out.h may be d_h).  scratch: uint8, at least join_grad_scratch_size bytes."""
    some = d_h if d_h is not None else h
    if some is None:
        raise TypeError("expected d_h, or d_z and h")
    T, H = shape = _two(some, "d_h" if d_h is not None else "h", _FLOAT)
    if (T | H) > _MOST:
        _too_large("moe_join_grad")
    dtype, dev = some.dtype, some.device
    if d_z is not None:
        if before is None or h is None:
            raise TypeError("d_z: expected `before` and h with it")
        _check(h, "h", shape, (dtype,))
        _check(d_z, "d_z", shape, _FLOAT)
    if y is not None:
        _check(y, "y", shape, _FLOAT)
    kind, w_type = _weights(T, H, after, gate, before)
    seeds, L = _rng(rng, drop), lib()
    if out is None:
        f32 = torch.float32
        given = None
        out = JoinGrads(_empty(shape, dtype, dev, stream) if residual else None,
                        _empty(shape, y.dtype, dev, stream) if y is not None else None,
                        _empty((H,), f32, dev, stream) if after is not None else None,
                        _empty(gate.shape, f32, dev, stream) if gate is not None else None,
                        _empty((H,), f32, dev, stream) if before is not None else None)
    else:
        given = out
        for what, t, s, types in (("out.h", out.h, shape, (dtype,)), ("out.y", out.y, shape, (y.dtype,) if y is not None else ()),
                                  ("out.after", out.after, (H,), _F32),
                                  ("out.gate", out.gate, gate.shape if gate is not None else (), _F32),
                                  ("out.before", out.before, (H,), _F32)):
            if t is not None:
                _check(t, what, s, types)
    if scratch is None and (out.after is not None or out.before is not None or (out.gate is not None and kind == _CHANNEL)):
        scratch = _empty((L.moe_join_grad_scratch_size(T, H),), torch.uint8, dev, stream)
    room = 0
    if scratch is not None:
        _check(scratch, "scratch", scratch.shape, _U8)
        room = scratch.numel()
    r = L.moe_join_grad(_ptr(d_h), _ptr(d_z), _ptr(h) if d_z is not None else None, _ptr(y), _ptr(after), _ptr(gate),
                        _ptr(before), seeds, _ptr(out.h), _ptr(out.y), _ptr(out.after), _ptr(out.gate), _ptr(out.before),
                        T, H, _TYPES[dtype], 0 if y is None else _TYPES[y.dtype], 0 if d_z is None else _TYPES[d_z.dtype],
                        w_type, kind, scale, drop, eps, scratch.data_ptr() if room else None, room,
                        _place(stream, d_h, d_z, h if d_z is not None else None, y, after, gate, before,
                               rng if seeds else None, scratch, *out))
    if r < 0:
        raise MoeError(r, "moe_join_grad")
    if given is not None:
        _written(tuple(t for t in given if t is not None))
    return out


# ---- the post-router layer for a few tokens --------------------------------------------------

def layer_few_scratch_size(T: int, H: int, I: int, E: int, topk: int) -> int:
    return 0 if max(T, H, I, E, topk) > _MOST else int(lib().moe_few_scratch_size(T, H, I, E, topk))


def layer_few(hidden, w1, w2, expert_ids, gates, first_expert: int = 0, out=None, dtype=torch.float32, scratch=None,
              stream=None):
    """moe_few_forward or, with weights in MX4, moe_few_forward_mx4: the post-router
    layer for up to FEW_TOKENS tokens, without a sort.  hidden bf16 [T, H]; w1 and w2
    either bf16 as layer_forward takes them (w1 packed [E, H, 2I], w2 [E, I, H]) or both
    MX4 as layer_forward_mx4 takes them (activations stay bf16 here); expert_ids int32 and
    gates fp32 [T, topk] (ids outside [first_expert, first_expert + E): no expert); returns
    out [T, H] (`dtype`: fp32 or bf16).  scratch: uint8, at least
    layer_few_scratch_size bytes (allocated if None)."""
    T, H = _two(hidden, "hidden", _BF16)
    shape = _two(expert_ids, "expert_ids", _I32)
    topk = shape[1]
    if shape[0] != T:
        raise TypeError(f"expert_ids: {shape[0]} tokens, hidden {T}")
    _check(gates, "gates", shape, _F32)
    mx4 = isinstance(w1, MX4)
    if mx4 != isinstance(w2, MX4):
        raise TypeError("w1 and w2: expected both in bf16 or both in MX4")
    if mx4:
        if len(w1.codes.shape) != 3 or w1.codes.shape[1] % 2 or w1.K != H:
            raise TypeError(f"w1: expected [E, 2I, {H}] in MX4, got {tuple(w1.codes.shape)}, K = {w1.K}")
        E, I = w1.codes.shape[0], w1.codes.shape[1] // 2
        _mx4_check(w1, "w1", (E, 2 * I))
        if w2.K != I:
            raise TypeError(f"w2: K is {w2.K}, expected {I}")
        _mx4_check(w2, "w2", (E, H))
    else:
        if w2.dim() != 3:
            raise TypeError(f"w2: expected [E, I, H], got {tuple(w2.shape)}")
        E, I = w2.shape[:2]
        _check(w1, "w1", (E, H, 2 * I), _BF16)
        _check(w2, "w2", (E, I, H), _BF16)
    if (T | H | I | E | topk) > _MOST or not -_MOST <= first_expert + 1 <= _MOST + 1:
        _too_large("layer_few")
    given = out
    if out is None:
        out = _empty((T, H), dtype, hidden.device, stream)
    _check(out, "out", (T, H), _FLOAT)
    L = lib()
    if scratch is None:
        scratch = _empty((L.moe_few_scratch_size(T, H, I, E, topk),), torch.uint8, hidden.device, stream)
    _check(scratch, "scratch", scratch.shape, _U8)
    rest = (expert_ids.data_ptr(), gates.data_ptr(), out.data_ptr(), T, H, I, E, topk, first_expert, _TYPES[out.dtype],
            scratch.data_ptr(), scratch.numel(),
            _place(stream, hidden, *(w1[:2] + w2[:2] if mx4 else (w1, w2)), expert_ids, gates, out, scratch))
    if mx4:
        r = L.moe_few_forward_mx4(hidden.data_ptr(), w1.codes.data_ptr(), w1.scales.data_ptr(), w2.codes.data_ptr(),
                                  w2.scales.data_ptr(), *rest)
    else:
        r = L.moe_few_forward(hidden.data_ptr(), w1.data_ptr(), w2.data_ptr(), *rest)
    if r < 0:
        raise MoeError(r, "layer_few")
    if given is not None:
        _written((given,))
    return out
