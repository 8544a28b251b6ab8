"""pcpp: PointCNN++ convolution on native points as MVMR, hand-written HIP for MI355X (gfx950).

The package is a thin ctypes binding over libpcpp.so (see include/pcpp.h).  Every step of the
path -- hashed-grid radius search, reordering by (k, o), MVMR forward and both gradients -- runs
in the library's kernels; PyTorch only provides device memory and the stream.  So do the operators that a
training step needs around it: norms, gate and residual between two blocks (pcpp_block_norm_*), activations in
8 bits and the weight gradient that reads them (pcpp_act_*, pcpp_mvmr_bwd_weight_packed), and the log
probabilities of a head's classes (pcpp_log_probs_*).
"""
from . import binding
from .binding import (BUILD_TEST_SHORT_LISTS, BUILD_TEST_WIDE_KEYS, BUILD_VOXEL, NORM_LAYER, NORM_NONE, NORM_RMS, PLAN_BWD_INPUT, PLAN_FWD,
                      PLAN_SPATIAL, BlockNorm, BlockNormGrads, LogProbs, Packed, PcppError, Triplets, library, pcpp_act_pack,
                      pcpp_act_unpack, pcpp_block_norm_bwd, pcpp_block_norm_fwd, pcpp_build_triplets, pcpp_count_triplets,
                      pcpp_log_probs_bwd, pcpp_log_probs_fwd, pcpp_mvmr_bwd_input, pcpp_mvmr_bwd_weight,
                      pcpp_mvmr_bwd_weight_packed, pcpp_mvmr_fwd, pcpp_mvmr_fwd_static, pcpp_tune_plan_order, pcpp_voxel_subsample)

__all__ = ["BUILD_TEST_SHORT_LISTS", "BUILD_TEST_WIDE_KEYS", "BUILD_VOXEL", "BlockNorm", "BlockNormGrads", "LogProbs", "NORM_LAYER",
           "NORM_NONE", "NORM_RMS", "Packed", "pcpp_voxel_subsample", "PLAN_BWD_INPUT", "PLAN_FWD", "PLAN_SPATIAL", "PcppError",
           "Triplets", "binding", "library", "pcpp_act_pack", "pcpp_act_unpack", "pcpp_block_norm_bwd", "pcpp_block_norm_fwd",
           "pcpp_build_triplets", "pcpp_count_triplets", "pcpp_log_probs_bwd", "pcpp_log_probs_fwd", "pcpp_mvmr_bwd_input",
           "pcpp_mvmr_bwd_weight", "pcpp_mvmr_bwd_weight_packed", "pcpp_mvmr_fwd", "pcpp_mvmr_fwd_static", "pcpp_tune_plan_order"]
