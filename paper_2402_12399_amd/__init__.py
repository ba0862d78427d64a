"""Rectify-Router MoE-layer forward (and the router-score gradient of its weights) for AMD MI355X (gfx950), and what a model calls
around it: balance loss, dropout with the residual sum, dense projections, each with its gradient.

The product is the HIP library `librr.so` (C ABI in include/rr.h); `binding` marshals torch
tensors into it and `workloads` draws seeded synthetic inputs.  There is no CPU fallback: every
call raises if the library is missing.
"""
from .binding import (  # noqa: F401
    RRConfig, RRError, RRLinearConfig, Tables, alloc_balance_workspace, alloc_linear_workspace, alloc_tables,
    alloc_workspace, library_path, load_library, rr_balance_loss, rr_balance_loss_backward, rr_balance_workspace_bytes,
    rr_capacity, rr_dropout, rr_dropout_backward, rr_init, rr_linear, rr_linear_backward, rr_linear_workspace_bytes,
    rr_moe_forward, rr_profile_enable, rr_profile_read, rr_rectified_dispatch,
    rr_rectified_dispatch_static,
    rr_router_backward, rr_router_scores, rr_slots_per_expert, rr_strerror, rr_workspace_bytes,
    RR_F32, RR_BF16, RR_ACT_GELU, RR_ACT_SWIGLU, RR_ACT_NONE, RR_INTRA_GPU, RR_FILL_IN, RR_POLICY_ARRIVAL,
    RR_QUOTA_PER_GROUP, RR_GRAD_STRAIGHT_THROUGH, RR_GRAD_ACCUMULATE,
)
