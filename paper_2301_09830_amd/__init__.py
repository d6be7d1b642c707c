"""liboptcc: MI355X-native low-rank power-iteration compressor with error feedback.

The compute path is the HIP library liboptcc.so (csrc/); `optcc` is its thin
ctypes binding over torch tensors.  Build the library with
`python -m paper_2301_09830_amd.build`.
"""

from . import optcc  # noqa: F401
from .optcc import (OCC_ACT_GELU, OCC_ACT_GELU_TANH, OCC_ACT_NONE, OCC_ACT_RELU,  # noqa: F401
                    OCC_ACT_SILU, OCC_BF16, OCC_DEC_OUT_BF16, OCC_DEC_SPLIT_BF16, OCC_F32,
                    OCC_F_BAD_ROWS, OCC_F_NONFINITE, OCC_F_RANK_DEFICIENT, OCC_MAX_CHOICES,
                    OCC_MAX_EXPERTS, OCC_MAX_TEACHER, OCC_NO_MHAT, OccError, Route,
                    alloc_workspace, make_param, make_params, occ_abi_version, occ_adamw_step,
                    occ_combine, occ_combine_bwd, occ_compress, occ_compress_workspace_bytes,
                    occ_decompress, occ_decompress_ex, occ_dispatch, occ_distill_bwd,
                    occ_distill_fwd, occ_err_update, occ_experts_gated_bwd, occ_experts_gated_fwd,
                    occ_experts_linear_bwd, occ_experts_linear_fwd, occ_gated_bwd, occ_gated_fwd,
                    occ_get_flags, occ_linear_bwd, occ_linear_fwd, occ_pipeline_1f1b,
                    occ_profile_begin, occ_profile_end, occ_route_bwd, occ_route_fwd,
                    occ_sc_select, occ_status_str, occ_step, occ_step_batched,
                    occ_step_batched_noalloc, occ_step_rows, occ_step_rows_workspace_bytes,
                    occ_workspace_bytes, occ_workspace_init)
