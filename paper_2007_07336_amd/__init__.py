"""MI355X-native MGRIT-FAS (layer-parallel multigrid) solver for residual networks.

The product is the C-ABI library `libmgrit.so` (HIP kernels for gfx950, see include/mgrit.h);
this package is its thin Python binding.
"""
from .binding import (  # noqa: F401
    MgritError, mgrit_problem_t, make_problem, problem_from_workload, lib,
    mgrit_level_map, mgrit_workspace_bytes, mgrit_adjoint_workspace_bytes,
    mgrit_fas_forward, mgrit_fas_adjoint, mgrit_residual_norm, mgrit_trace_begin, mgrit_trace_end,
    mgrit_fas_forward_static, MGRIT_STATIC_SCRATCH_BYTES,
    mgrit_fc_layers_t, make_fc_layers, mgrit_workspace_bytes_mixed, mgrit_adjoint_workspace_bytes_mixed,
    mgrit_fas_forward_mixed, mgrit_fas_adjoint_mixed, mgrit_residual_norm_mixed,
    MGRIT_ACT_TANH, MGRIT_ACT_RELU, MGRIT_ACT_IDENTITY, MGRIT_FP32, MGRIT_BF16, MGRIT_LOSS_SUM, MGRIT_LOSS_MEAN,
    mgrit_affine_t, make_affine, mgrit_affine_workspace_bytes, mgrit_affine_backward_workspace_bytes,
    mgrit_affine_forward, mgrit_affine_backward,
    mgrit_loss_t, make_loss, mgrit_cross_entropy_workspace_bytes, mgrit_cross_entropy,
    mgrit_tensor_t, make_tensor_list, mgrit_clip_workspace_bytes, mgrit_clip_gradients,
    MGRIT_MX8, MGRIT_MX4, mgrit_packed_t, make_packed, mgrit_packed_bytes, mgrit_pack, mgrit_unpack,
    mgrit_affine_packed_t, make_affine_packed, mgrit_affine_packed_workspace_bytes, mgrit_affine_packed_forward,
    mgrit_affine_kept_workspace_bytes, mgrit_affine_kept_backward,
    MGRIT_NORM_ROOT, MGRIT_NORM_LAYER, MGRIT_GATE_NONE, MGRIT_GATE_FEATURE, MGRIT_GATE_ENTRY,
    mgrit_block_norm_t, make_block_norm, mgrit_block_norm_workspace_bytes, mgrit_block_norm_forward, mgrit_block_norm_backward,
    mgrit_sample_t, make_sample, mgrit_sample_workspace_bytes, mgrit_sample,
)
