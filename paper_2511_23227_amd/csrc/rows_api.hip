// C ABI entry points of the operators around the convolution: activations in 8 bits, norms between blocks, log probabilities.
// Argument checks and dispatch.  (pcpp_mvmr_bwd_weight_packed lies with the other MVMR calls in pcpp_api.hip.)
#include <math.h>

#include "block_norm.h"
#include "log_probs.h"
#include "pcpp_internal.h"
#include "row_ops.h"

namespace pcpp {

namespace {

constexpr int MAX_CHANNELS = 1024;
constexpr int64_t MAX_PITCH = 1 << 24;                            // (a wave's sixteen rows within 32-bit offsets)

bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
size_t dtype_bytes(int dtype) { return dtype == PCPP_F32 ? 4 : 2; }

int invalid(const char *fn, const char *what)
{
    set_error("%s: %s", fn, what);
    return PCPP_ERR_INVALID_ARG;
}
int unsupported(const char *fn, const char *what)
{
    set_error("%s: %s", fn, what);
    return PCPP_ERR_UNSUPPORTED;
}

int check_rows(const char *fn, int64_t n, int c)
{
    if (n < 0) return invalid(fn, "negative number of rows");
    if (c < 1 || c > MAX_CHANNELS) return unsupported(fn, "channel count outside 1..1024");
    if (n >= INT32_MAX) return unsupported(fn, "sizes must be below 2^31");
    return PCPP_OK;
}

int check_act(const char *fn, const void *x, int dtype, int64_t n, int c, const void *q, const void *codes)
{
    if (int rc = check_rows(fn, n, c)) return rc;
    if (dtype != PCPP_F32 && dtype != PCPP_BF16) return unsupported(fn, "unsupported dtype");
    if (n > 0 && (!x || !q || !codes)) return invalid(fn, "null tensor pointer");
    if (!aligned(x, 16) || !aligned(q, 16) || !aligned(codes, 4)) return invalid(fn, "x and q must be 16-byte aligned, codes 4-byte");
    return PCPP_OK;
}

// what both directions of the block norm share
int check_block(const char *fn, const void *f, int64_t ld_f, const void *gate, int64_t ld_gate, int gate_cols, const float *w_post,
                const float *w_pre, int post_norm, int pre_norm, float scale, float eps, int64_t n, int c, int stream_dtype, int dtype)
{
    if (int rc = check_rows(fn, n, c)) return rc;
    if ((dtype != PCPP_F32 && dtype != PCPP_BF16) || (stream_dtype != dtype && stream_dtype != PCPP_F32))
        return unsupported(fn, "unsupported dtype combination");
    if (post_norm < PCPP_NORM_NONE || post_norm > PCPP_NORM_LAYER || pre_norm < PCPP_NORM_NONE || pre_norm > PCPP_NORM_LAYER)
        return invalid(fn, "unknown kind of norm");
    if (!(eps >= 0.f) || !isfinite(eps) || !isfinite(scale)) return invalid(fn, "eps must be finite and >= 0, residual_scale finite");
    if (gate_cols != 0 && gate_cols != 1 && gate_cols != c) return invalid(fn, "gate_cols must be 0, 1 or c");
    if (n > 0 && (gate != nullptr) != (gate_cols != 0)) return invalid(fn, "gate and gate_cols do not agree");
    if (f && ld_f < c) return invalid(fn, "ld_f < c");
    if (gate && ld_gate < gate_cols) return invalid(fn, "ld_gate < gate_cols");
    if ((f && ld_f >= MAX_PITCH) || (gate && ld_gate >= MAX_PITCH)) return unsupported(fn, "row pitches must be below 2^24");
    if (!aligned(f, dtype_bytes(dtype)) || !aligned(gate, dtype_bytes(dtype)) || !aligned(w_post, 4) || !aligned(w_pre, 4))
        return invalid(fn, "f, gate and the weights must be aligned to their elements");
    return PCPP_OK;
}

int check_logits(const char *fn, const void *logits, int dtype, int64_t n, int64_t v, int64_t ld, const int32_t *labels)
{
    if (n < 0 || v < 1 || ld < v) return invalid(fn, "negative number of rows, no class, or pitch < v");
    if (dtype != PCPP_F32 && dtype != PCPP_BF16) return unsupported(fn, "unsupported dtype");
    if (n >= INT32_MAX || v >= INT32_MAX) return unsupported(fn, "sizes must be below 2^31");
    if (n > 0 && !logits) return invalid(fn, "logits are NULL");
    if (!aligned(logits, dtype_bytes(dtype)) || !aligned(labels, 4)) return invalid(fn, "logits and labels must be aligned to their elements");
    return PCPP_OK;
}

}  // namespace
}  // namespace pcpp

using namespace pcpp;

extern "C" {

size_t pcpp_act_code_bytes(int c) { return c < 1 || c > MAX_CHANNELS ? 0 : (size_t)act_code_bytes(c); }

int pcpp_act_pack(const void *x, int dtype, int64_t n, int c, int8_t *q, uint8_t *codes, void *stream)
{
    if (int rc = check_act("pcpp_act_pack", x, dtype, n, c, q, codes)) return rc;
    if (n == 0) return PCPP_OK;
    return act_pack(x, dtype, n, c, q, codes, static_cast<hipStream_t>(stream));
}

int pcpp_act_unpack(const int8_t *q, const uint8_t *codes, int64_t n, int c, void *x, int dtype, void *stream)
{
    if (int rc = check_act("pcpp_act_unpack", x, dtype, n, c, q, codes)) return rc;
    if (n == 0) return PCPP_OK;
    return act_unpack(q, codes, n, c, x, dtype, static_cast<hipStream_t>(stream));
}

int pcpp_block_norm_fwd(const void *x, const void *f, int64_t ld_f, const void *gate, int64_t ld_gate, int gate_cols, const float *w_post,
                        const float *w_pre, int post_norm, int pre_norm, float residual_scale, float eps, int64_t n, int c, int stream_dtype,
                        int dtype, void *r, void *h, int8_t *fq, uint8_t *fcodes, int8_t *hq, uint8_t *hcodes, void *stream)
{
    const char *fn = "pcpp_block_norm_fwd";
    if (int rc = check_block(fn, f, ld_f, gate, ld_gate, gate_cols, w_post, w_pre, post_norm, pre_norm, residual_scale, eps, n, c, stream_dtype,
                             dtype))
        return rc;
    if (n == 0) return PCPP_OK;
    if (!x) return invalid(fn, "x is NULL");
    if (f ? !r : r != nullptr) return invalid(fn, "r is written exactly if there is a block (f)");
    if (!f && (gate_cols || fq)) return invalid(fn, "a gate or an 8-bit copy of f without f");
    if ((h != nullptr) != (pre_norm != PCPP_NORM_NONE)) return invalid(fn, "h is written exactly if pre_norm is not PCPP_NORM_NONE");
    if (!h && hq) return invalid(fn, "an 8-bit copy of h without h");
    if (!f && !h) return invalid(fn, "nothing to do: neither a block nor a norm");
    if ((fq != nullptr) != (fcodes != nullptr) || (hq != nullptr) != (hcodes != nullptr)) return invalid(fn, "q and codes belong together");
    if (!aligned(x, 16) || !aligned(r, 16) || !aligned(h, 16) || !aligned(fq, 16) || !aligned(hq, 16) || !aligned(fcodes, 4) || !aligned(hcodes, 4))
        return invalid(fn, "x, r, h and q must be 16-byte aligned, codes 4-byte");
    BlockNormFwd a{};
    a.x = x; a.f = f; a.gate = gate; a.w_post = w_post; a.w_pre = w_pre; a.r = r; a.h = h;
    a.f_codes = ActOut{fq, fcodes}; a.h_codes = ActOut{hq, hcodes};
    a.n = n; a.ld_f = ld_f; a.ld_gate = ld_gate;
    a.c = c; a.gate_cols = gate_cols; a.post = post_norm; a.pre = pre_norm;
    a.scale = residual_scale; a.eps = eps; a.inv_c = 1.f / (float)c;
    return block_norm_fwd(a, stream_dtype, dtype, static_cast<hipStream_t>(stream));
}

size_t pcpp_block_norm_workspace_bytes(int64_t n, int c)
{
    return n < 0 || c < 1 || c > MAX_CHANNELS ? 0 : block_norm_bwd_workspace_bytes(n, c);
}

int pcpp_block_norm_bwd(const void *dr, const void *dh, const void *r, const void *f, int64_t ld_f, const int8_t *fq, const uint8_t *fcodes,
                        const void *gate, int64_t ld_gate, int gate_cols, const float *w_post, const float *w_pre, int post_norm, int pre_norm,
                        float residual_scale, float eps, int64_t n, int c, int stream_dtype, int dtype, void *dx, void *df, void *dgate,
                        float *dw_post, float *dw_pre, void *workspace, size_t workspace_bytes, void *stream_)
{
    const char *fn = "pcpp_block_norm_bwd";
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    if (int rc = check_block(fn, f, ld_f, gate, ld_gate, gate_cols, w_post, w_pre, post_norm, pre_norm, residual_scale, eps, n, c, stream_dtype,
                             dtype))
        return rc;
    if (!aligned(dw_post, 4) || !aligned(dw_pre, 4)) return invalid(fn, "the weights' gradients must be 4-byte aligned");
    if (n == 0) {
        if (dw_post)
            if (int rc = fill_u32(reinterpret_cast<uint32_t *>(dw_post), 0u, c, stream)) return rc;
        return dw_pre ? fill_u32(reinterpret_cast<uint32_t *>(dw_pre), 0u, c, stream) : PCPP_OK;
    }
    if ((dh != nullptr) != (pre_norm != PCPP_NORM_NONE) || (r != nullptr) != (pre_norm != PCPP_NORM_NONE))
        return invalid(fn, "dh and r are given exactly if pre_norm is not PCPP_NORM_NONE");
    if (!dr && !dh) return invalid(fn, "neither dr nor dh");
    if (f && fq) return invalid(fn, "f twice, in full and in 8 bits");
    if ((fq != nullptr) != (fcodes != nullptr)) return invalid(fn, "q and codes belong together");
    if (df && !f && !fq && (post_norm != PCPP_NORM_NONE || gate_cols)) return invalid(fn, "f is NULL");
    if (!df && (f || fq || gate_cols || dw_post)) return invalid(fn, "df is NULL though there is a block");
    if ((dgate != nullptr) != (gate_cols != 0)) return invalid(fn, "dgate and gate_cols do not agree");
    if (dw_post && !f && !fq) return invalid(fn, "dw_post without f");
    if (dw_pre && pre_norm == PCPP_NORM_NONE) return invalid(fn, "dw_pre without a pre norm");
    if (!aligned(dr, 16) || !aligned(dh, 16) || !aligned(r, 16) || !aligned(fq, 16) || !aligned(fcodes, 4) || !aligned(dx, 16) || !aligned(df, 16) ||
        !aligned(dgate, 16))
        return invalid(fn, "dr, dh, r, q, dx, df and dgate must be 16-byte aligned, codes 4-byte");
    const size_t need = block_norm_bwd_workspace_bytes(n, c);
    if (!workspace || workspace_bytes < need || !aligned(workspace, 256)) {
        set_error("%s: workspace missing, misaligned or smaller than %zu bytes", fn, need);
        return PCPP_ERR_WORKSPACE;
    }
    BlockNormBwd a{};
    a.dr = dr; a.dh = dh; a.r = r; a.f = f; a.gate = gate; a.f_codes = ActIn{fq, fcodes};
    a.w_post = w_post; a.w_pre = w_pre; a.dx = dx; a.df = df; a.dgate = dgate;
    a.dw_post = dw_post; a.dw_pre = dw_pre; a.part = static_cast<float *>(workspace);
    a.n = n; a.ld_f = ld_f; a.ld_gate = ld_gate;
    a.c = c; a.gate_cols = gate_cols; a.post = post_norm; a.pre = pre_norm;
    a.scale = residual_scale; a.eps = eps; a.inv_c = 1.f / (float)c;
    return block_norm_bwd(a, stream_dtype, dtype, stream);
}

size_t pcpp_log_probs_workspace_bytes(int64_t n, int64_t v, int n_top)
{
    return n < 0 || v < 1 || n_top < 0 || n_top > PCPP_MAX_ALTERNATIVES ? 0 : log_probs_workspace_bytes(n, v, n_top);
}

int pcpp_log_probs_fwd(const void *logits, int dtype, int64_t n, int64_t v, int64_t ld, const int32_t *labels, int n_top, float *log_prob,
                       float *entropy, float *max_log_sum, float *top_log_prob, int32_t *top_index, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *fn = "pcpp_log_probs_fwd";
    if (int rc = check_logits(fn, logits, dtype, n, v, ld, labels)) return rc;
    if (n_top < 0 || n_top > PCPP_MAX_ALTERNATIVES || n_top > v) return invalid(fn, "n_top outside 0 .. min(v, PCPP_MAX_ALTERNATIVES)");
    if (n == 0) return PCPP_OK;
    if (n_top > 0 && (!top_log_prob || !top_index)) return invalid(fn, "top_log_prob or top_index is NULL");
    if (!aligned(log_prob, 4) || !aligned(entropy, 4) || !aligned(max_log_sum, 8) || !aligned(top_log_prob, 4) || !aligned(top_index, 4))
        return invalid(fn, "outputs must be 4-byte aligned, max_log_sum 8-byte");
    const size_t need = log_probs_workspace_bytes(n, v, n_top);
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) {
        set_error("%s: workspace missing, misaligned or smaller than %zu bytes", fn, need);
        return PCPP_ERR_WORKSPACE;
    }
    LogProbsFwd a{};
    a.logits = logits; a.labels = labels;
    a.log_prob = log_prob; a.entropy = entropy; a.max_log_sum = max_log_sum; a.top_log_prob = top_log_prob; a.top_index = top_index;
    a.n = n; a.v = v; a.ld = ld; a.n_top = n_top;
    return log_probs_fwd(a, dtype, workspace, static_cast<hipStream_t>(stream));
}

int pcpp_log_probs_bwd(const void *logits, int dtype, int64_t n, int64_t v, int64_t ld, const int32_t *labels, const float *max_log_sum,
                       const float *entropy, const float *d_log_prob, const float *d_entropy, void *d_logits, int64_t ld_d, void *stream)
{
    const char *fn = "pcpp_log_probs_bwd";
    if (int rc = check_logits(fn, logits, dtype, n, v, ld, labels)) return rc;
    if (ld_d < v) return invalid(fn, "ld_d < v");
    if (n == 0) return PCPP_OK;
    if (!d_logits || !max_log_sum) return invalid(fn, "d_logits or max_log_sum is NULL");
    if (d_entropy && !entropy) return invalid(fn, "d_entropy without entropy");
    if (d_logits == logits && ld_d != ld) return invalid(fn, "d_logits in place of the logits with another pitch");
    if (!aligned(d_logits, dtype_bytes(dtype)) || !aligned(max_log_sum, 8) || !aligned(entropy, 4) || !aligned(d_log_prob, 4) || !aligned(d_entropy, 4))
        return invalid(fn, "tensors must be aligned to their elements, max_log_sum to 8 bytes");
    LogProbsBwd a{};
    a.logits = logits; a.labels = labels; a.max_log_sum = max_log_sum; a.entropy = entropy; a.d_log_prob = d_log_prob; a.d_entropy = d_entropy;
    a.d_logits = d_logits;
    a.n = n; a.v = v; a.ld = ld; a.ld_d = ld_d;
    return log_probs_bwd(a, dtype, static_cast<hipStream_t>(stream));
}

}  // extern "C"
