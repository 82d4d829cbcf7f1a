"""MI355X (gfx950) MoE GEMM2 + combine with a launch-time partition selector.

The compute path is the HIP library libmoe_gemm2.so (C ABI in
include/moe_gemm2.h); ``binding`` marshals torch tensors into it.

``experts`` has the operators around and inside the experts (C ABI in
include/moe_experts.h: the sort by expert, dispatch and combine with their
gradients, experts in microscaled 4-bit floating point), ``block`` what stands around
them (include/moe_block.h: the router's choice and the residual join with its norms,
with their gradients, and the layer for a few tokens), ``autograd`` choose, dispatch,
combine and join as differentiable functions; a program imports them by name.
"""
from . import binding  # noqa: F401
from .binding import (MoeError, Workspace, combine, default_params,  # noqa: F401
                      make_workload, select_evaluate, select_partition)
