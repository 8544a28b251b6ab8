"""pcpp: PointCNN++ convolution on native points as MVMR, hand-written HIP for MI355X (gfx950).

The package is a thin ctypes binding over libpcpp.so (see include/pcpp.h).  Every step of the
path -- hashed-grid radius search, reordering by (k, o), MVMR forward and both gradients -- runs
in the library's kernels; PyTorch only provides device memory and the stream.  So do the operators that a
training step needs around it: norms, gate and residual between two blocks (pcpp_block_norm_*), activations in
8 bits and the weight gradient that reads them (pcpp_act_*, pcpp_mvmr_bwd_weight_packed), the log
probabilities of a head's classes (pcpp_log_probs_*), and those of its pointwise layers: group norm with an activation
over the clouds of a batch (pcpp_group_norm_*), dropout (pcpp_dropout_*), linear layers in microscaled 4-bit floating point (pcpp_mx_*).
"""
from . import binding
from .binding import (ACT_GELU, ACT_NONE, ACT_RELU, ACT_SILU, BUILD_TEST_SHORT_LISTS, BUILD_TEST_WIDE_KEYS, BUILD_VOXEL, DROP_CLOUDS,
                      DROP_ELEMENTS, DROP_ROWS, NORM_LAYER, NORM_NONE, NORM_RMS, PLAN_BWD_INPUT, PLAN_FWD, PLAN_SPATIAL, BlockNorm,
                      BlockNormGrads, GroupNorm, GroupNormGrads, LogProbs, Mx, MxRows, Packed, PcppError, Random, Triplets, library,
                      pcpp_act_pack, pcpp_act_unpack, pcpp_block_norm_bwd, pcpp_block_norm_fwd, pcpp_build_triplets, pcpp_count_triplets,
                      pcpp_dropout_bwd, pcpp_dropout_fwd, pcpp_group_norm_bwd, pcpp_group_norm_fwd, pcpp_log_probs_bwd,
                      pcpp_log_probs_fwd, pcpp_mvmr_bwd_input, pcpp_mvmr_bwd_weight, pcpp_mvmr_bwd_weight_packed, pcpp_mvmr_fwd,
                      pcpp_mvmr_fwd_static, pcpp_mx_linear, pcpp_mx_pack, pcpp_mx_product, pcpp_mx_unpack, pcpp_tune_plan_order,
                      pcpp_voxel_subsample)

__all__ = ["ACT_GELU", "ACT_NONE", "ACT_RELU", "ACT_SILU", "BUILD_TEST_SHORT_LISTS", "BUILD_TEST_WIDE_KEYS", "BUILD_VOXEL", "BlockNorm",
           "BlockNormGrads", "DROP_CLOUDS", "DROP_ELEMENTS", "DROP_ROWS", "GroupNorm", "GroupNormGrads", "LogProbs", "Mx", "MxRows",
           "NORM_LAYER", "NORM_NONE", "NORM_RMS", "Packed", "pcpp_voxel_subsample", "PLAN_BWD_INPUT", "PLAN_FWD", "PLAN_SPATIAL",
           "PcppError", "Random", "Triplets", "binding", "library", "pcpp_act_pack", "pcpp_act_unpack", "pcpp_block_norm_bwd",
           "pcpp_block_norm_fwd", "pcpp_build_triplets", "pcpp_count_triplets", "pcpp_dropout_bwd", "pcpp_dropout_fwd",
           "pcpp_group_norm_bwd", "pcpp_group_norm_fwd", "pcpp_log_probs_bwd", "pcpp_log_probs_fwd", "pcpp_mvmr_bwd_input",
           "pcpp_mvmr_bwd_weight", "pcpp_mvmr_bwd_weight_packed", "pcpp_mvmr_fwd", "pcpp_mvmr_fwd_static", "pcpp_mx_linear",
           "pcpp_mx_pack", "pcpp_mx_product", "pcpp_mx_unpack", "pcpp_tune_plan_order"]
