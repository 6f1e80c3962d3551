"""MI355X-native hot path of the universal one-sided matmul (arXiv 2510.08874):
slicing planner, grouping, grouped GEMM and replica sum, products of matrices in 4-bit
microscaled floating point and in 8-bit integers, the gated block, gradients and
orthogonalised updates live in ``libdmm.so``
(sources under ``csrc/``, C ABI in ``include/dmm.h``).  ``binding`` mirrors the
ABI; ``tiles`` allocates tile buffers with torch.  Nothing here computes."""
from .binding import (DMM_BF16, DMM_C_BF16, DMM_DB_F32, DMM_F32, DMM_GELU, DMM_GELU_TANH, DMM_ITERATION_OFFSET, DMM_MX_COLS, DMM_MX_ROWS, DMM_NO_MERGE, DMM_NO_REDUCE, DMM_SEPARATE_REDUCE, DMM_SILU, DMM_STATIONARY_A, DMM_STATIONARY_B, DMM_TIMING, DmmError, Plan, dmm_execute, dmm_execute_backward,  # noqa: F401
                      dmm_gated_backward, dmm_gated_execute, dmm_int_dequantize, dmm_int_execute, dmm_int_gated_execute, dmm_int_quantize, dmm_mx_dequantize,
                      dmm_mx_execute, dmm_mx_quantize, dmm_orthogonalize, dmm_orthogonalize_workspace, dmm_plan, dmm_plan_destroy, dmm_reduce_replicas, dmm_strerror, dmm_version)
