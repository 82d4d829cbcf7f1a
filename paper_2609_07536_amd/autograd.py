"""A mixture-of-experts block's way from the residual stream to the residual
stream as differentiable functions: their gradients are the library's own kernels
(``experts`` and ``block``).

    ids, gates = autograd.choose(logits, topk)           # logits [T, E]
    routing = experts.sort_by_expert(ids, gates, E)      # ids, gates [T, topk]
    rows = autograd.dispatch(x, routing)                 # [T topk, H], by expert
    ... the experts on rows offsets[e] .. offsets[e + 1] ...
    out = autograd.combine(y, routing, gates)            # [T, H]
    h, x = autograd.join(h, out, before=weight)          # the next block's stream and input

The choice itself (the ids) has no gradient; the gates do, through combine, and the
logits through choose.  ``workspace``: where both directions record bad entries of
slot_rows, as in ``experts``.
"""
from __future__ import annotations

import torch

from . import block as K
from . import experts as X


class _Dispatch(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, slot_rows, workspace):
        ctx.save_for_backward(slot_rows)
        ctx.workspace = workspace
        # rows that no slot has are zeros, as their gradients are
        out = torch.zeros((slot_rows.numel(), x.shape[1]), dtype=x.dtype, device=x.device)
        return X.dispatch_rows(x.contiguous(), slot_rows, slot_rows.numel(), out=out, workspace=workspace)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d):
        (slot_rows,) = ctx.saved_tensors
        return X.dispatch_rows_grad(d.contiguous(), slot_rows, workspace=ctx.workspace), None, None


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, slot_rows, gates, dtype, workspace):
        y, gates = y.contiguous(), gates.contiguous()
        ctx.save_for_backward(y, slot_rows, gates)
        ctx.workspace = workspace
        return X.combine_rows(y, slot_rows, gates, dtype=dtype, workspace=workspace)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d):
        y, slot_rows, gates = ctx.saved_tensors
        out = (torch.zeros_like(y), torch.empty_like(gates))
        dy, dgates = X.combine_rows_grad(d.contiguous(), y, slot_rows, gates, out=out, workspace=ctx.workspace)
        return dy, None, dgates, None, None


def dispatch(x, routing: X.Routing, workspace=None):
    """x [T, H] (bf16 or fp32) to [T topk, H]: each token's row at the rows of its
    slots, zeros at rows that no slot has.  (Without a gradient x may be of any type.)"""
    if x.dtype not in X._TYPES and x.requires_grad and torch.is_grad_enabled():
        raise TypeError(f"x: rows of {x.dtype} can be moved but have no gradient; expected bf16 or fp32")
    return _Dispatch.apply(x, routing.slot_rows, workspace)


def combine(y, routing: X.Routing, gates, dtype=torch.float32, workspace=None):
    """y [T topk, H] (bf16 or fp32) to [T, H]: the sum of each token's rows weighted
    by gates fp32 [T, topk]."""
    rows = routing.slot_rows.numel()
    if y.shape[0] != rows:   # (slots whose rows a shorter y lacks would be dropped)
        raise TypeError(f"y: {y.shape[0]} rows, the routing has {rows} slots")
    return _Combine.apply(y, routing.slot_rows, gates, dtype, workspace)


class _Choose(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, topk, bias, score, renormalize, scale):
        logits = logits.contiguous()
        ids, gates = K.choose(logits, topk, bias, score, renormalize, scale)
        ctx.save_for_backward(logits, ids)
        ctx.how = (score, renormalize, scale)
        ctx.mark_non_differentiable(ids)
        ctx.set_materialize_grads(False)
        return ids, gates

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, _, d):
        if d is None:
            return (None,) * 6
        logits, ids = ctx.saved_tensors
        return (K.choose_grad(d.contiguous(), logits, ids, *ctx.how),) + (None,) * 5


def choose(logits, topk: int, bias=None, score: str = "softmax", renormalize: bool = True, scale: float = 1.0) -> K.Choice:
    """block.choose with the gates' gradient; bias has none (it acts on the choice alone)."""
    return K.Choice(*_Choose.apply(logits, topk, bias, score, renormalize, scale))


class _Join(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h, y, after, gate, before, scale, drop, rng, eps, dtype):
        h, y, after, gate, before = (t if t is None else t.contiguous() for t in (h, y, after, gate, before))
        # (a copy: the program may write the next call's numbers to its own before the backward pass)
        rng = rng.clone() if drop and rng is not None else None
        x, z = K.join(h, y, after, gate, scale, drop, rng, before, eps, dtype=dtype)
        # y is read again for a norm after the block or a gate, the stream for the norm before
        ctx.save_for_backward(y if after is not None or gate is not None else None, after, gate, before, rng,
                              x if before is not None else None)
        ctx.how = (scale, drop, eps)
        ctx.types = (x.dtype, y.dtype if y is not None else None, h is not None)
        ctx.set_materialize_grads(False)
        return x, z

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_x, d_z):
        y, after, gate, before, rng, x = ctx.saved_tensors
        scale, drop, eps = ctx.how
        x_type, y_type, residual = ctx.types
        if d_x is None and d_z is None:
            return (None,) * 10
        d_x, d_z = (d if d is None else d.contiguous() for d in (d_x, d_z))
        some = d_x if d_x is not None else d_z
        need = ctx.needs_input_grad

        def room(wanted, shape, dtype):
            return some.new_empty(shape, dtype=dtype) if wanted else None
        out = K.JoinGrads(room(residual and need[0], some.shape, x_type), room(y_type is not None and need[1], some.shape, y_type),
                          room(after is not None and need[2], some.shape[1:], torch.float32),
                          room(gate is not None and need[3], gate.shape if gate is not None else (), torch.float32),
                          room(before is not None and need[4], some.shape[1:], torch.float32))
        if y is None and out.y is None:
            drop = 0.0   # (nothing that is asked for goes through it)
        K.join_grad(d_x, d_z, x, y, after, gate, scale, drop, rng, before, eps, out=out)
        grads = [g if g is None or t is None else g.to(t.dtype) for g, t in zip(out[2:], (after, gate, before))]
        return (*out[:2], *grads) + (None,) * 5


def join(h, y=None, after=None, gate=None, scale: float = 1.0, drop: float = 0.0, rng=None, before=None,
         eps: float = 1e-6, dtype=torch.bfloat16) -> K.Joined:
    """block.join with the gradients of h, y, after, gate and before.  h None: nothing to
    add to.  y None: the norm of h alone."""
    if y is None:
        if h is None or before is None or after is not None or gate is not None or drop:
            raise TypeError("without y: expected h and `before`, and neither a norm after the block, a gate nor dropout")
        # (the stream itself goes on as it is: its gradient meets the norm's at h)
        return K.Joined(h, _Norm.apply(h, before, eps, dtype))
    return K.Joined(*_Join.apply(h, y, after, gate, before, scale, drop, rng, eps, dtype))


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h, before, eps, dtype):
        h, before = h.contiguous(), before.contiguous()
        ctx.save_for_backward(h, before)
        ctx.eps = eps
        return K.join(h, before=before, eps=eps, dtype=dtype).z

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d):
        h, before = ctx.saved_tensors
        g = K.join_grad(None, d.contiguous(), h, before=before, eps=ctx.eps)
        return g.h, g.before.to(before.dtype), None, None
