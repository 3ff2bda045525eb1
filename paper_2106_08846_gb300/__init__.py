"""GB300 (sm_103a) block-sparse-row x dense product, Y = X W^T + b, and the
operators that stand between two products of a transformer layer.

The product at the centre of "Algorithm to Compilation Co-design" (Section
2.2): a pruned weight stored in BSR form (data, indices, indptr) multiplied
with dense activations; beside it the residual step with its norms
(bsr_residual_norm) and the gated feed-forward block (bsr_gated), forward and
backward. The compute lives in libbsr_gb300.so (include/bsr.h);
this package is its ctypes binding and its build script.
"""
from .bsrlib import (  # noqa: F401
    BSR_BF16, BSR_F32, BsrError, Handle, Plan, bsr_check_device_status, bsr_check_status, bsr_create, bsr_destroy,
    bsr_from_dense, bsr_get_call_info, bsr_get_schedule, bsr_reserve, bsr_spmm, bsr_spmm_batch, bsr_spmm_noalloc, bsr_status_str, load,
    bsr_gated, bsr_gated_backward, bsr_plan_create, bsr_residual_norm, bsr_residual_norm_backward, parse_schedule,
)
