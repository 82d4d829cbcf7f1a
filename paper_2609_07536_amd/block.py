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
from .experts import (MX4, _BF16, _F32, _FLOAT, _I32, _MOST, _TYPES, _U8, _check, _empty, _mx4_shapes,
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


_I64 = (torch.int64,)


def _here(stream):
    """The current device (-2 without one: no tensor is on it) and the handle of the stream
    to launch on."""
    if torch.cuda.is_initialized() and _b._raw_device is not None:
        device = _b._raw_device()
        if stream is None:
            return device, _b._raw_stream(device)
    elif torch.cuda.is_available():
        device = torch.cuda.current_device()
    else:
        return -2, None
    if stream is not None and stream.device_index != device:
        raise TypeError(f"expected a stream of the current device ({device}), got one of {stream.device_index}")
    return device, _stream(stream)


def _fits(t, what, shape, dtypes, device):
    """_check, and that the tensor is on the current device."""
    if t.get_device() == device and t.dtype in dtypes and t.shape == shape and t.is_contiguous():
        return
    _check(t, what, shape, dtypes)
    raise TypeError(f"{what}: expected a tensor on the current device ({device}), got one on {t.device}")


def _matrix(t, what, dtypes, device):
    """_two, on the current device."""
    shape = t.shape
    if t.get_device() == device and len(shape) == 2 and t.dtype in dtypes and t.is_contiguous():
        return shape
    _two(t, what, dtypes)
    raise TypeError(f"{what}: expected a tensor on the current device ({device}), got one on {t.device}")


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
    L, (device, handle) = lib(), _here(stream)
    T, E = _matrix(logits, "logits", _FLOAT, device)
    if (T | E | topk) > _MOST:
        _too_large("moe_choose")
    if bias is not None:
        _fits(bias, "bias", (E,), _F32, device)
    given, shape = out, (T, topk)
    if out is None:
        out = Choice(_empty(shape, torch.int32, logits.device, stream), _empty(shape, torch.float32, logits.device, stream))
    else:
        _fits(out[0], "expert_ids", shape, _I32, device)
        _fits(out[1], "gates", shape, _F32, device)
    r = L.moe_choose(logits.data_ptr(), _ptr(bias), out[0].data_ptr(), out[1].data_ptr(), T, E, topk,
                     _TYPES[logits.dtype], _score(score), renormalize, scale, handle)
    if r < 0:
        raise MoeError(r, "moe_choose")
    if given is not None:
        _written(given)
    return out


def choose_grad(d_gates, logits, expert_ids, score: str = "softmax", renormalize: bool = True, scale: float = 1.0,
                out=None, workspace: Optional[Workspace] = None, stream=None):
    """moe_choose_grad: the gates' gradient fp32 [T, topk], the logits and the chosen
    ids to the logits' gradient [T, E], of their type."""
    L, (device, handle) = lib(), _here(stream)
    T, E = shape = _matrix(logits, "logits", _FLOAT, device)
    chosen = _matrix(expert_ids, "expert_ids", _I32, device)
    topk = chosen[1]
    if chosen[0] != T:
        raise TypeError(f"expert_ids: {chosen[0]} tokens, logits {T}")
    if (T | E | topk) > _MOST:
        _too_large("moe_choose_grad")
    _fits(d_gates, "d_gates", chosen, _F32, device)
    given = out
    if out is None:
        out = _empty(shape, logits.dtype, logits.device, stream)
    else:
        _fits(out, "out", shape, (logits.dtype,), device)
    r = L.moe_choose_grad(d_gates.data_ptr(), logits.data_ptr(), expert_ids.data_ptr(), out.data_ptr(), T, E, topk,
                          _TYPES[logits.dtype], _score(score), renormalize, scale, _status_word(workspace), handle)
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


def _weights(T, H, after, gate, before, device):
    """The kind of gate and the type that norms' weights and the gate share."""
    types = _FLOAT
    if after is not None:
        _fits(after, "after", (H,), types, device)
        types = (after.dtype,)
    if before is not None:
        _fits(before, "before", (H,), types, device)
        types = (before.dtype,)
    kind = _NONE
    if gate is not None:
        kind = _CHANNEL if gate.shape == (1, H) else _TOKEN
        _fits(gate, "gate", (1, H) if kind == _CHANNEL else (T, 1), types, device)
        types = (gate.dtype,)
    return kind, _TYPES[types[0]]


def _rng(rng, drop, device):
    if drop == 0.0:
        return None
    if not 0.0 <= drop < 1.0:
        raise ValueError(f"drop: expected a probability below 1, got {drop}")
    if rng is None:
        raise TypeError("rng: dropout needs one, int64 [2] (seed, offset)")
    _fits(rng, "rng", (2,), _I64, device)
    return rng.data_ptr()


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
    out: where both go (out.h may be h itself, and without y is it or None; out.z None
    without `before`)."""
    if h is None and y is None:
        raise TypeError("expected h, y or both")
    L, (device, handle) = lib(), _here(stream)
    some = h if h is not None else y
    T, H = shape = _matrix(some, "h" if h is not None else "y", _FLOAT, device)
    if (T | H) > _MOST:
        _too_large("moe_join")
    if y is not None and h is not None:
        _fits(y, "y", shape, _FLOAT, device)
    kind, w_type = _weights(T, H, after, gate, before, device)
    seeds, given, h_type = _rng(rng, drop, device), out, some.dtype
    if out is None:
        x = h if y is None else _empty(shape, h_type, some.device, stream)
        z = None if before is None else _empty(shape, dtype, some.device, stream)
        out = Joined(x, z)
    x, z = out
    if y is not None:
        _fits(x, "out.h", shape, (h_type,), device)
    elif x is not h:
        if x is not None and x.data_ptr() != h.data_ptr():
            raise TypeError("out.h: without y the stream goes on in h; expected None or h")
        out = Joined(h, z)
    if before is not None:
        _fits(z, "out.z", shape, _FLOAT, device)
    elif z is not None:
        raise TypeError("out.z: there is no norm without `before`; expected None")
    r = L.moe_join(_ptr(h), _ptr(y), _ptr(after), _ptr(gate), _ptr(before), seeds,
                   None if y is None else x.data_ptr(), None if before is None else z.data_ptr(), T, H,
                   _TYPES[h_type], 0 if y is None else _TYPES[y.dtype], 0 if before is None else _TYPES[z.dtype],
                   w_type, kind, scale, drop, eps, handle)
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
    (out.h may be d_h).  y is read with `after` or a gate only: without them out.y alone
    says that there was one, and its type.  scratch: uint8, at least join_grad_scratch_size bytes."""
    some = d_h if d_h is not None else h
    if some is None:
        raise TypeError("expected d_h, or d_z and h")
    L, (device, handle) = lib(), _here(stream)
    T, H = shape = _matrix(some, "d_h" if d_h is not None else "h", _FLOAT, device)
    if (T | H) > _MOST:
        _too_large("moe_join_grad")
    dtype, dev = some.dtype, some.device
    if d_z is not None:
        if before is None or h is None:
            raise TypeError("d_z: expected `before` and h with it")
        if h is not some:
            _fits(h, "h", shape, (dtype,), device)
        _fits(d_z, "d_z", shape, _FLOAT, device)
    elif d_h is None:
        raise TypeError("expected d_h, d_z or both")
    if y is not None:
        _fits(y, "y", shape, _FLOAT, device)
    kind, w_type = _weights(T, H, after, gate, before, device)
    seeds, given = _rng(rng, drop, device), out
    if out is None:
        f32 = torch.float32
        out = JoinGrads(_empty(shape, dtype, dev, stream) if residual else None,
                        _empty(shape, y.dtype, dev, stream) if y is not None else None,
                        _empty((H,), f32, dev, stream) if after is not None else None,
                        _empty(gate.shape, f32, dev, stream) if gate is not None else None,
                        _empty((H,), f32, dev, stream) if before is not None else None)
    g_h, g_y, g_after, g_gate, g_before = out
    if given is not None:
        if g_h is not None:
            _fits(g_h, "out.h", shape, (dtype,), device)
        if g_y is not None:
            _fits(g_y, "out.y", shape, _FLOAT if y is None else (y.dtype,), device)
        if g_after is not None:
            _fits(g_after, "out.after", (H,), _F32, device)
        if g_gate is not None:
            _fits(g_gate, "out.gate", gate.shape if gate is not None else (), _F32, device)
        if g_before is not None:
            _fits(g_before, "out.before", (H,), _F32, device)
    if scratch is None and (g_after is not None or g_before is not None or (g_gate is not None and kind == _CHANNEL)):
        scratch = _empty((L.moe_join_grad_scratch_size(T, H),), torch.uint8, dev, stream)
    room = 0
    if scratch is not None:
        _fits(scratch, "scratch", scratch.shape, _U8, device)
        room = scratch.numel()
    like_y = y if y is not None else g_y
    r = L.moe_join_grad(_ptr(d_h), _ptr(d_z), None if d_z is None else h.data_ptr(), _ptr(y), _ptr(after), _ptr(gate),
                        _ptr(before), seeds, _ptr(g_h), _ptr(g_y), _ptr(g_after), _ptr(g_gate), _ptr(g_before),
                        T, H, _TYPES[dtype], 0 if like_y is None else _TYPES[like_y.dtype], 0 if d_z is None else _TYPES[d_z.dtype],
                        w_type, kind, scale, drop, eps, scratch.data_ptr() if room else None, room, handle)
    if r < 0:
        raise MoeError(r, "moe_join_grad")
    if given is not None:
        _written(tuple([t for t in given if t is not None]))
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
    L, (device, handle) = lib(), _here(stream)
    T, H = _matrix(hidden, "hidden", _BF16, device)
    shape = _matrix(expert_ids, "expert_ids", _I32, device)
    topk = shape[1]
    if shape[0] != T:
        raise TypeError(f"expert_ids: {shape[0]} tokens, hidden {T}")
    _fits(gates, "gates", shape, _F32, device)
    mx4 = isinstance(w1, MX4)
    if mx4 != isinstance(w2, MX4):
        raise TypeError("w1 and w2: expected both in bf16 or both in MX4")
    if mx4:
        (c1, s1, K1), (c2, s2, K2) = w1, w2
        if len(c1.shape) != 3 or c1.shape[1] % 2 or K1 != H:
            raise TypeError(f"w1: expected [E, 2I, {H}] in MX4, got {tuple(c1.shape)}, K = {K1}")
        E, N = c1.shape[:2]
        I = N // 2
        if K2 != I:
            raise TypeError(f"w2: K is {K2}, expected {I}")
        codes, scales = _mx4_shapes((E, N), H)
        _fits(c1, "w1.codes", codes, _U8, device)
        _fits(s1, "w1.scales", scales, _U8, device)
        codes, scales = _mx4_shapes((E, H), I)
        _fits(c2, "w2.codes", codes, _U8, device)
        _fits(s2, "w2.scales", scales, _U8, device)
    else:
        if w2.dim() != 3:
            raise TypeError(f"w2: expected [E, I, H], got {tuple(w2.shape)}")
        E, I = w2.shape[:2]
        _fits(w1, "w1", (E, H, 2 * I), _BF16, device)
        _fits(w2, "w2", (E, I, H), _BF16, device)
    if (T | H | I | E | topk) > _MOST or not -_MOST <= first_expert + 1 <= _MOST + 1:
        _too_large("layer_few")
    given = out
    if out is None:
        out = _empty((T, H), dtype, hidden.device, stream)
    _fits(out, "out", (T, H), _FLOAT, device)
    if scratch is None:
        scratch = _empty((L.moe_few_scratch_size(T, H, I, E, topk),), torch.uint8, hidden.device, stream)
    _fits(scratch, "scratch", scratch.shape, _U8, device)
    if mx4:
        r = L.moe_few_forward_mx4(hidden.data_ptr(), c1.data_ptr(), s1.data_ptr(), c2.data_ptr(), s2.data_ptr(),
                                  expert_ids.data_ptr(), gates.data_ptr(), out.data_ptr(), T, H, I, E, topk, first_expert,
                                  _TYPES[out.dtype], scratch.data_ptr(), scratch.numel(), handle)
    else:
        r = L.moe_few_forward(hidden.data_ptr(), w1.data_ptr(), w2.data_ptr(), expert_ids.data_ptr(), gates.data_ptr(),
                              out.data_ptr(), T, H, I, E, topk, first_expert, _TYPES[out.dtype], scratch.data_ptr(),
                              scratch.numel(), handle)
    if r < 0:
        raise MoeError(r, "layer_few")
    if given is not None:
        _written((given,))
    return out
