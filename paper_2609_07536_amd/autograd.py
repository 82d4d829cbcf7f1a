"""The rows' way to the experts and back as differentiable functions: their
gradients are the library's own kernels (``experts``).

    routing = experts.sort_by_expert(ids, gates, E)      # ids, gates [T, topk]
    rows = autograd.dispatch(x, routing)                 # [T topk, H], by expert
    ... the experts on rows offsets[e] .. offsets[e + 1] ...
    out = autograd.combine(y, routing, gates)            # [T, H]

The choice itself (the ids) has no gradient; the gates do, through combine.
``workspace``: where both directions record bad entries of slot_rows, as in
``experts``.
"""
from __future__ import annotations

import torch

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
