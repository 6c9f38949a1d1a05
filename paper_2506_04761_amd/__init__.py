"""libloglinear: log-linear attention (forward, backward and decoding) (Guo et al., "Log-Linear
Attention") on MI355X, and the operators around such a mixer: short causal
convolution, selective state space scan, group norm.

The computation lives in the HIP library libloglinear.so (C ABI: include/libloglinear.h);
this package is its Python binding.
"""

from ._lib import (  # noqa: F401
    LL_BF16, LL_F32, LL_GDN, LL_LAMBDA_DIAG, LL_LAMBDA_FULL, LL_MAMBA2, LL_MAMBA2_BWD, LLError, lib, ll_debug_level_map, ll_decode_state_bytes,
    ll_gdn_decode_init, ll_gdn_decode_step, ll_gdn_fwd, ll_gdn_fwd_staged, ll_mamba2_bwd, ll_mamba2_bwd_after_fwd,
    ll_mamba2_bwd_staged, ll_mamba2_bwd_workspace, ll_mamba2_decode_init, ll_mamba2_decode_step, ll_mamba2_fwd,
    ll_mamba2_fwd_grouped, ll_mamba2_fwd_matrix_lambda, ll_mamba2_fwd_noalloc, LL_NOALLOC_SCRATCH_BYTES, ll_mamba2_fwd_matrix_lambda_staged,
    ll_mamba2_fwd_staged, ll_mamba2_matrix_lambda_workspace, ll_num_levels, ll_status_string, ll_supported, ll_workspace_size,
    log_linear_mamba2,
)
from ._layer import (  # noqa: F401
    LL_ACT_NONE, LL_ACT_SILU, ConvGrads, NormGrads, ScanGrads, ll_causal_conv_bwd, ll_causal_conv_bwd_workspace,
    ll_causal_conv_fwd, ll_causal_conv_step, ll_group_norm_bwd, ll_group_norm_fwd, ll_group_norm_stats,
    ll_group_norm_workspace, ll_selective_scan_bwd, ll_selective_scan_fwd, ll_selective_scan_states,
    ll_selective_scan_step, ll_selective_scan_workspace, causal_conv, group_norm, selective_scan,
)
