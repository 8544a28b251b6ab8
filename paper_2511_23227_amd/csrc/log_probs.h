// Arguments of the log probability kernels (log_probs.hip), checked by the entry points; not part of the C ABI.
#pragma once

#include "pcpp_internal.h"

namespace pcpp {

struct LogProbsFwd {
    const void *logits;
    const int32_t *labels;
    float *log_prob, *entropy, *max_log_sum, *top_log_prob;
    int32_t *top_index;
    int64_t n, v, ld;
    int n_top;
};

struct LogProbsBwd {
    const void *logits;
    const int32_t *labels;
    const float *max_log_sum, *entropy, *d_log_prob, *d_entropy;
    void *d_logits;
    int64_t n, v, ld, ld_d;
};

size_t log_probs_workspace_bytes(int64_t n, int64_t v, int n_top);
int log_probs_fwd(const LogProbsFwd &a, int dtype, void *workspace, hipStream_t stream);
int log_probs_bwd(const LogProbsBwd &a, int dtype, hipStream_t stream);

}  // namespace pcpp
