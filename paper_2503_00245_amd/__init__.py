"""MI355X-native sparse MoE feed-forward layer (CoSMoEs, arXiv 2503.00245): HIP kernels for
gfx950 behind the C ABI of include/moe.h, plus a ctypes binding of the same names."""
from .binding import (  # noqa: F401
    EXPORTS, FLAG_RESIDUAL, FLAG_SHARED_BASE, LIB_PATH, MOE_BF16, MOE_F32, MoeError, MoeShape,
    MoeWeights, alloc_workspace, lib, make_shape, make_weights, moe_combine, moe_expert_ffn,
    moe_bles_loss, moe_bles_workspace_bytes, moe_delta_uniform, moe_expert_replacements, moe_forward,
    moe_forward_static, moe_forward_timed, STATIC_WORKSPACE_BYTES, moe_offload_counters, moe_permute, moe_route, moe_stack_forward, moe_workspace_bytes, shape_for,
    status_string,
    QUANTISED_EXPORTS, Mxfp4Weights, RouteConfig, SCORE_SIGMOID, SCORE_SOFTMAX, alloc_mxfp4_workspace, make_mxfp4_weights, make_route_config,
    moe_mxfp4_dequantize, moe_mxfp4_experts, moe_mxfp4_forward, moe_mxfp4_pack, moe_mxfp4_quantize, moe_mxfp4_workspace_bytes,
    moe_route_scored, moe_route_scored_backward,
    TRAINING_EXPORTS, Block, alloc_block_stack_workspace, alloc_block_workspace, alloc_dispatch_workspace, alloc_training_workspace, make_block, moe_block_norm,
    moe_block_norm_backward, moe_block_stack_forward, moe_block_stack_workspace_bytes, moe_block_workspace_bytes, moe_collect, moe_collect_backward,
    moe_dispatch, moe_dispatch_backward, moe_dispatch_workspace_bytes, moe_expert_ffn_backward, moe_training_workspace_bytes,
)
