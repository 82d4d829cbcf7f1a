"""ctypes binding of the operators around and inside the experts
(include/moe_experts.h): argument marshalling only, like ``binding``.

Tensors are contiguous and on the GPU.  Every function takes ``stream`` (a
torch stream; default: the current one) and only enqueues work on it; outputs
that are not given with ``out`` are allocated for that stream, and ones that are
count as changed in place (autograd refuses a backward pass that had saved what
was there before).  ``workspace``
(a ``binding.Workspace`` of at least 512 bytes) is where the row operators
record bad entries of ``slot_rows`` or ``row_ids`` for ``Workspace.status``.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from . import binding as _b
from .binding import MoeError, Workspace

EXPORTED = (
    "moe_sort_scratch_size", "moe_sort_by_expert", "moe_dispatch_rows", "moe_dispatch_rows_grad",
    "moe_combine_rows", "moe_combine_rows_grad", "moe_mx4_quantize", "moe_mx4_quantize_weights",
    "moe_mx4_dequantize", "moe_mx4_product", "moe_mx4_layer_scratch_size", "moe_mx4_layer_forward",
    "moe_experts_abi_version",
)

_TYPES = {torch.bfloat16: 0, torch.float32: 1}   # moe_type_t
_lib = None


def lib() -> ctypes.CDLL:
    """The HIP library with this module's functions declared."""
    global _lib
    if _lib is None:
        L = _b.lib()
        vp, sz, i32, i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int64
        L.moe_sort_scratch_size.argtypes = [i32, i32, i32]
        L.moe_sort_by_expert.argtypes = [vp] * 6 + [i32] * 4 + [vp, sz, vp]
        L.moe_dispatch_rows.argtypes = [vp] * 3 + [i32, i32, i64, i64, vp, vp]
        L.moe_dispatch_rows_grad.argtypes = [vp] * 3 + [i32, i32, i64, i32, i32, i32, vp, vp]
        L.moe_combine_rows.argtypes = [vp] * 4 + [i32, i32, i64, i32, i32, i32, vp, vp]
        L.moe_combine_rows_grad.argtypes = [vp] * 6 + [i32, i32, i64, i32, i32, i32, vp, vp]
        L.moe_mx4_quantize.argtypes = [vp] * 3 + [i64, i32, i32, vp]
        L.moe_mx4_quantize_weights.argtypes = [vp] * 3 + [i32, i32, i32, i32, vp]
        L.moe_mx4_dequantize.argtypes = [vp] * 3 + [i64, i32, i32, vp]
        L.moe_mx4_product.argtypes = [vp] * 7 + [i64, i64, i32, i32, i32, i32, vp, vp]
        L.moe_mx4_layer_scratch_size.argtypes = [i32] * 4
        L.moe_mx4_layer_forward.argtypes = [vp] * 10 + [i32] * 6 + [vp, sz, vp, vp]
        for name in EXPORTED:
            getattr(L, name).restype = sz if name.endswith("_size") else ctypes.c_int
        _lib = L
    return _lib


_BF16, _F32, _I32, _U8 = (torch.bfloat16,), (torch.float32,), (torch.int32,), (torch.uint8,)
_FLOAT = (torch.bfloat16, torch.float32)


def _check(t, what, shape, dtypes):
    if t.dtype in dtypes and t.shape == shape and t.is_cuda and t.is_contiguous():
        return
    raise TypeError(f"{what}: expected a contiguous CUDA tensor of {' or '.join(map(str, dtypes))} and shape "
                    f"{tuple(shape)}, got {t.dtype} {tuple(t.shape)} on {t.device}, strides {t.stride()}")


def _two(t, what, dtypes):
    """The shape of a matrix."""
    shape = t.shape
    if len(shape) == 2 and t.dtype in dtypes and t.is_cuda and t.is_contiguous():
        return shape
    raise TypeError(f"{what}: expected a contiguous CUDA matrix of {' or '.join(map(str, dtypes))}, got {t.dtype} "
                    f"{tuple(shape)} on {t.device}, strides {t.stride()}")


def _stream(stream):
    """The handle of `stream`, or of the current one (by torch's raw accessors, as
    in ``binding``; an int, which a call converts faster than a c_void_p)."""
    if stream is not None:
        return stream.cuda_stream
    if _b._raw_stream is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _b._raw_stream(_b._raw_device())


def _empty(shape, dtype, device, stream):
    """Memory for a launch on `stream`: the caching allocator hands it out again
    only for later work on that stream."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


# The library's sizes are 32 bits, and ctypes cuts a larger int without a word.
_MOST = 2 ** 31 - 1


def _too_large(what):
    raise MoeError(_b.MOE_ERR_UNSUPPORTED, what)


# The library writes through raw pointers, which torch does not see.  Takes a tuple of
# tensors; torch's raw function, where there is one, takes 0.15 us, the public one 0.3.
_written = getattr(torch._C, "_increment_version", torch.autograd.graph.increment_version)


def _done(r, what):
    if r < 0:
        raise MoeError(r, what)


def _status_word(workspace):
    return workspace.ptr if workspace is not None else None


_SORT_WITHOUT_SCRATCH = 4096   # slots, as the C ABI has it: no call to ask for small sorts


class Routing(NamedTuple):
    """A router's choice as rows grouped by expert, as the stage and the grouped
    products take it: expert_offsets int32 [E + 1]; token_ids int32 and gate_w
    fp32 [T topk], of which the first expert_offsets[E] are rows (then -1 and
    0); slot_rows int32 [T, topk], the row of each of a token's slots or -1."""
    expert_offsets: torch.Tensor
    token_ids: torch.Tensor
    gate_w: torch.Tensor
    slot_rows: torch.Tensor


def sort_by_expert(expert_ids, gates, E: int, first_expert: int = 0, out: Optional[Routing] = None,
                   scratch=None, stream=None) -> Routing:
    """moe_sort_by_expert: expert_ids int32 and gates fp32 [T, topk] to a Routing
    (a stable sort by expert).  Ids outside [first_expert, first_expert + E)
    are slots without a row.  scratch: uint8, at least sort_scratch_size bytes."""
    T, topk = shape = _two(expert_ids, "expert_ids", _I32)
    _check(gates, "gates", shape, _F32)
    if (T | topk | E) > _MOST or not -_MOST <= first_expert + 1 <= _MOST + 1:
        _too_large("moe_sort_by_expert")
    n, given = T * topk, out
    if out is None:
        dev = expert_ids.device
        out = Routing(_empty((E + 1,), torch.int32, dev, stream), _empty((n,), torch.int32, dev, stream),
                      _empty((n,), torch.float32, dev, stream), _empty(shape, torch.int32, dev, stream))
    offsets, token_ids, gate_w, slot_rows = out
    _check(offsets, "expert_offsets", (E + 1,), _I32)
    _check(token_ids, "token_ids", (n,), _I32)
    _check(gate_w, "gate_w", (n,), _F32)
    _check(slot_rows, "slot_rows", shape, _I32)
    L, room = lib(), 0
    if n > _SORT_WITHOUT_SCRATCH:
        room = L.moe_sort_scratch_size(T, topk, E)
        if scratch is None:
            scratch = _empty((room,), torch.uint8, expert_ids.device, stream)
        _check(scratch, "scratch", scratch.shape, _U8)
        room = scratch.numel()
    r = L.moe_sort_by_expert(expert_ids.data_ptr(), gates.data_ptr(), offsets.data_ptr(), token_ids.data_ptr(),
                             gate_w.data_ptr(), slot_rows.data_ptr(), T, topk, E, first_expert,
                             scratch.data_ptr() if room else None, room, _stream(stream))
    if r < 0:
        raise MoeError(r, "moe_sort_by_expert")
    if given is not None:
        _written(given)
    return out


def sort_scratch_size(T: int, topk: int, E: int) -> int:
    return 0 if max(T, topk, E) > _MOST else int(lib().moe_sort_scratch_size(T, topk, E))


def dispatch_rows(x, slot_rows, rows: int, out=None, workspace: Optional[Workspace] = None, stream=None):
    """moe_dispatch_rows: x [T, H] of any type to [rows, H], each token's row
    copied to the rows of its slots.  Rows that no slot has are not written."""
    T, topk = _two(slot_rows, "slot_rows", _I32)
    dtypes = (x.dtype,)
    H = _two(x, "x", dtypes)[1]
    if x.shape[0] != T:
        raise TypeError(f"x: {x.shape[0]} rows, slot_rows {T}")
    if (T | topk) > _MOST:
        _too_large("moe_dispatch_rows")
    given = out
    if out is None:
        out = _empty((rows, H), x.dtype, x.device, stream)
    else:
        _check(out, "out", (rows, H), dtypes)
    r = lib().moe_dispatch_rows(x.data_ptr(), slot_rows.data_ptr(), out.data_ptr(), T, topk, rows,
                                H * x.element_size(), _status_word(workspace), _stream(stream))
    if r < 0:
        raise MoeError(r, "moe_dispatch_rows")
    if given is not None:
        _written((given,))
    return out


def dispatch_rows_grad(d, slot_rows, out=None, workspace: Optional[Workspace] = None, stream=None):
    """moe_dispatch_rows_grad: d [rows, H] (bf16 or fp32) to dx [T, H] (of d's type,
    or `out`'s): the sum of each token's rows, in fp32, rounded once."""
    T, topk = _two(slot_rows, "slot_rows", _I32)
    rows, H = _two(d, "d", _FLOAT)
    if (T | topk | H) > _MOST:
        _too_large("moe_dispatch_rows_grad")
    given = out
    if out is None:
        out = _empty((T, H), d.dtype, d.device, stream)
    else:
        _check(out, "out", (T, H), _FLOAT)
    r = lib().moe_dispatch_rows_grad(d.data_ptr(), slot_rows.data_ptr(), out.data_ptr(), T, topk, rows, H,
                                     _TYPES[d.dtype], _TYPES[out.dtype], _status_word(workspace), _stream(stream))
    if r < 0:
        raise MoeError(r, "moe_dispatch_rows_grad")
    if given is not None:
        _written((given,))
    return out


def combine_rows(y, slot_rows, gates, out=None, dtype=torch.float32, workspace: Optional[Workspace] = None,
                 stream=None):
    """moe_combine_rows: y [rows, H] (bf16 or fp32) to out [T, H] (`dtype`: fp32 or
    bf16): the sum of each token's rows weighted by gates fp32 [T, topk], in
    fp32, rounded once."""
    T, topk = shape = _two(slot_rows, "slot_rows", _I32)
    _check(gates, "gates", shape, _F32)
    rows, H = _two(y, "y", _FLOAT)
    if (T | topk | H) > _MOST:
        _too_large("moe_combine_rows")
    given = out
    if out is None:
        out = _empty((T, H), dtype, y.device, stream)
    _check(out, "out", (T, H), _FLOAT)
    r = lib().moe_combine_rows(y.data_ptr(), slot_rows.data_ptr(), gates.data_ptr(), out.data_ptr(), T, topk, rows,
                               H, _TYPES[y.dtype], _TYPES[out.dtype], _status_word(workspace), _stream(stream))
    if r < 0:
        raise MoeError(r, "moe_combine_rows")
    if given is not None:
        _written((given,))
    return out


def combine_rows_grad(d_out, y, slot_rows, gates, out=None, workspace: Optional[Workspace] = None, stream=None):
    """moe_combine_rows_grad: d_out [T, H] and y [rows, H] (each bf16 or fp32) to
    (dy [rows, H] of y's type, dgates fp32 [T, topk]); `out`: that pair."""
    T, topk = shape = _two(slot_rows, "slot_rows", _I32)
    _check(gates, "gates", shape, _F32)
    rows, H = _two(y, "y", _FLOAT)
    if (T | topk | H) > _MOST:
        _too_large("moe_combine_rows_grad")
    _check(d_out, "d_out", (T, H), _FLOAT)
    if out is None:
        dy = _empty((rows, H), y.dtype, y.device, stream)
        dgates = _empty(shape, torch.float32, y.device, stream)
    else:
        dy, dgates = out
        _check(dy, "dy", (rows, H), (y.dtype,))
        _check(dgates, "dgates", shape, _F32)
    r = lib().moe_combine_rows_grad(d_out.data_ptr(), y.data_ptr(), slot_rows.data_ptr(), gates.data_ptr(),
                                    dy.data_ptr(), dgates.data_ptr(), T, topk, rows, H, _TYPES[d_out.dtype],
                                    _TYPES[y.dtype], _status_word(workspace), _stream(stream))
    if r < 0:
        raise MoeError(r, "moe_combine_rows_grad")
    if out is not None:
        _written((dy, dgates))
    return dy, dgates


# ---- microscaled 4-bit floating point -----------------------------------------------

class MX4(NamedTuple):
    """A tensor [..., K] in microscaled 4-bit floating point: codes uint8
    [..., 16 ceil(K / 32)], scales uint8 [..., 4 ceil(K / 128)], K elements a
    row (the layout: include/moe_experts.h)."""
    codes: torch.Tensor
    scales: torch.Tensor
    K: int


def _mx4_shapes(lead, K):
    blocks = (K + 31) >> 5
    return (*lead, 16 * blocks), (*lead, (blocks + 3) & ~3)


def _mx4_check(m, what, lead):
    codes, scales, K = m
    code_shape, scale_shape = _mx4_shapes(lead, K)
    _check(codes, what + ".codes", code_shape, _U8)
    _check(scales, what + ".scales", scale_shape, _U8)


def _mx4_out(out, lead, K, device, stream):
    if out is None:
        codes, scales = _mx4_shapes(lead, K)
        return MX4(_empty(codes, torch.uint8, device, stream), _empty(scales, torch.uint8, device, stream), K)
    if out.K != K:
        raise TypeError(f"out: K is {out.K}, expected {K}")
    _mx4_check(out, "out", lead)
    return out


def mx4_quantize(x, out: Optional[MX4] = None, stream=None) -> MX4:
    """moe_mx4_quantize: x [..., K], bf16 or fp32."""
    shape = x.shape
    _check(x, "x", shape, _FLOAT)
    if len(shape) < 1:
        raise TypeError("x: expected at least one dimension")
    K, lead = shape[-1], shape[:-1]
    if K > _MOST:
        _too_large("moe_mx4_quantize")
    given = out
    out = _mx4_out(out, lead, K, x.device, stream)
    r = lib().moe_mx4_quantize(x.data_ptr(), out[0].data_ptr(), out[1].data_ptr(), lead.numel(), K,
                               _TYPES[x.dtype], _stream(stream))
    if r < 0:
        raise MoeError(r, "moe_mx4_quantize")
    if given is not None:
        _written(given[:2])
    return out


def mx4_quantize_weights(w, out: Optional[MX4] = None, stream=None) -> MX4:
    """moe_mx4_quantize_weights: w [E, K, N] (bf16 or fp32, the layout of w2 and of
    w_gate_up) to the MX4 [E, N, K] that mx4_product reads."""
    _check(w, "w", w.shape, _FLOAT)
    if w.dim() != 3:
        raise TypeError(f"w: expected [E, K, N], got {tuple(w.shape)}")
    E, K, N = w.shape
    if (E | K | N) > _MOST:
        _too_large("moe_mx4_quantize_weights")
    given = out
    out = _mx4_out(out, (E, N), K, w.device, stream)
    _done(lib().moe_mx4_quantize_weights(w.data_ptr(), out[0].data_ptr(), out[1].data_ptr(), E, K, N,
                                         _TYPES[w.dtype], _stream(stream)), "moe_mx4_quantize_weights")
    if given is not None:
        _written(given[:2])
    return out


def mx4_dequantize(m: MX4, out=None, dtype=torch.bfloat16, stream=None):
    """moe_mx4_dequantize: the values of `m` [..., K] as bf16 or fp32 (exact in both)."""
    codes, scales, K = m
    lead = codes.shape[:-1]
    _mx4_check(m, "m", lead)
    if K > _MOST:
        _too_large("moe_mx4_dequantize")
    given = out
    if out is None:
        out = _empty((*lead, K), dtype, codes.device, stream)
    _check(out, "out", (*lead, K), _FLOAT)
    r = lib().moe_mx4_dequantize(codes.data_ptr(), scales.data_ptr(), out.data_ptr(), lead.numel(), K,
                                 _TYPES[out.dtype], _stream(stream))
    if r < 0:
        raise MoeError(r, "moe_mx4_dequantize")
    if given is not None:
        _written((given,))
    return out


def mx4_product(a: MX4, w: MX4, expert_offsets, rows: int, row_ids=None, swiglu: bool = False, out=None,
                workspace: Optional[Workspace] = None, stream=None):
    """moe_mx4_product: a [a_rows, K] and w [E, N, K] to bf16 [rows, N], or with
    swiglu [rows, N / 2]; row_ids int32 (at least `rows`): the row of `a` that
    each row takes.  Rows from expert_offsets[E] on are not written."""
    a_codes, a_scales, K = a
    w_codes, w_scales, _ = w
    a_shape, w_shape = a_codes.shape, w_codes.shape
    if len(a_shape) != 2 or len(w_shape) != 3 or K != w.K:
        raise TypeError(f"expected a [rows, K] and w [E, N, K], got {tuple(a_shape)}, K = {K}, and "
                        f"{tuple(w_shape)}, K = {w.K}")
    a_rows, E, N = a_shape[0], w_shape[0], w_shape[1]
    if (K | E | N) > _MOST:
        _too_large("moe_mx4_product")
    _mx4_check(a, "a", (a_rows,))
    _mx4_check(w, "w", (E, N))
    _check(expert_offsets, "expert_offsets", (E + 1,), _I32)
    if row_ids is not None:
        _check(row_ids, "row_ids", row_ids.shape, _I32)
    have = a_rows if row_ids is None else row_ids.numel()
    if rows > have:
        raise TypeError(f"{rows} rows, but {have} " + ("of a" if row_ids is None else "row_ids"))
    shape = (rows, N // 2 if swiglu else N)
    given = out
    if out is None:
        out = _empty(shape, torch.bfloat16, a_codes.device, stream)
    else:
        _check(out, "out", shape, _BF16)
    r = lib().moe_mx4_product(a_codes.data_ptr(), a_scales.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(),
                              expert_offsets.data_ptr(), None if row_ids is None else row_ids.data_ptr(),
                              out.data_ptr(), a_rows, rows, K, N, E, swiglu, _status_word(workspace),
                              _stream(stream))
    if r < 0:
        raise MoeError(r, "moe_mx4_product")
    if given is not None:
        _written((given,))
    return out


def mx4_layer_scratch_size(T: int, H: int, I: int, topk: int) -> int:
    return 0 if max(T, H, I, topk) > _MOST else int(lib().moe_mx4_layer_scratch_size(T, H, I, topk))


def layer_forward_mx4(hidden, w1: MX4, w2: MX4, routing: Routing, gates, out=None, dtype=torch.float32,
                      scratch=None, workspace: Optional[Workspace] = None, stream=None):
    """moe_mx4_layer_forward, the post-router layer with its experts in 4 bits:
    hidden bf16 [T, H]; w1 [E, 2I, H] and w2 [E, H, I] in MX4
    (mx4_quantize_weights of w_gate_up [E, H, 2I] and w2 [E, I, H]); routing from
    sort_by_expert of gates [T, topk]; returns out [T, H] (`dtype`: fp32 or bf16).
    scratch: uint8, at least mx4_layer_scratch_size bytes (allocated if None)."""
    T, H = _two(hidden, "hidden", _BF16)
    if len(w1.codes.shape) != 3 or w1.codes.shape[1] % 2 or w1.K != H:
        raise TypeError(f"w1: expected [E, 2I, {H}] in MX4, got {tuple(w1.codes.shape)}, K = {w1.K}")
    E, I = w1.codes.shape[0], w1.codes.shape[1] // 2
    _mx4_check(w1, "w1", (E, 2 * I))
    if w2.K != I:
        raise TypeError(f"w2: K is {w2.K}, expected {I}")
    _mx4_check(w2, "w2", (E, H))
    offsets, token_ids, _, slot_rows = routing
    shape = _two(slot_rows, "slot_rows", _I32)
    topk = shape[1]
    if shape[0] != T:
        raise TypeError(f"slot_rows: {shape[0]} tokens, hidden {T}")
    if (T | H | I | E | topk) > _MOST:
        _too_large("moe_mx4_layer_forward")
    _check(gates, "gates", shape, _F32)
    _check(offsets, "expert_offsets", (E + 1,), _I32)
    _check(token_ids, "token_ids", (T * topk,), _I32)
    given = out
    if out is None:
        out = _empty((T, H), dtype, hidden.device, stream)
    _check(out, "out", (T, H), _FLOAT)
    L = lib()
    if scratch is None:
        scratch = _empty((L.moe_mx4_layer_scratch_size(T, H, I, topk),), torch.uint8, hidden.device, stream)
    _check(scratch, "scratch", scratch.shape, _U8)
    r = L.moe_mx4_layer_forward(hidden.data_ptr(), w1.codes.data_ptr(), w1.scales.data_ptr(), w2.codes.data_ptr(),
                                w2.scales.data_ptr(), offsets.data_ptr(), token_ids.data_ptr(), slot_rows.data_ptr(),
                                gates.data_ptr(), out.data_ptr(), T, H, I, E, topk, _TYPES[out.dtype],
                                scratch.data_ptr(), scratch.numel(), _status_word(workspace), _stream(stream))
    if r < 0:
        raise MoeError(r, "moe_mx4_layer_forward")
    if given is not None:
        _written((given,))
    return out
