// C ABI entry points of the pointwise layers' operators: dropout, group norm, rows in microscaled 4-bit floating point and their products.
// Argument checks and dispatch.
#include <float.h>
#include <math.h>

#include "mx.h"

namespace pcpp {

namespace {

constexpr int MAX_CHANNELS = 1024, MAX_DROP_CHANNELS = 65536, MAX_CLOUDS = 65536;
constexpr int64_t MAX_PITCH = 1 << 24, MAX_NORM_PITCH = 1 << 22;  // (the norms: 208 rows within 32-bit offsets)
constexpr int64_t MAX_MX_PITCH = 1 << 25;                         // (32 rows)
constexpr uint64_t MAX_COUNTERS = ((uint64_t)1 << 32) - 65536;

bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
size_t dtype_bytes(int dtype) { return dtype == PCPP_F32 ? 4 : 2; }
bool is_type(int dtype) { return dtype == PCPP_F32 || dtype == PCPP_BF16; }

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

int check_random(const char *fn, const int64_t *random, int64_t n, int64_t c)
{
    if (!aligned(random, 8)) return invalid(fn, "random must be 8-byte aligned");
    if ((uint64_t)n * (uint64_t)ceil_div(c, 8) >= MAX_COUNTERS) return unsupported(fn, "too many random numbers: n * ceil(c / 8) must be below 2^32 - 65536");
    return PCPP_OK;
}
int check_clouds(const char *fn, const int32_t *offsets, int n_clouds)
{
    if (n_clouds < 1 || n_clouds > MAX_CLOUDS) return invalid(fn, "n_clouds outside 1..65536");
    if (!offsets && n_clouds != 1) return invalid(fn, "several clouds without offsets");
    if (!aligned(offsets, 4)) return invalid(fn, "offsets must be 4-byte aligned");
    return PCPP_OK;
}
int check_workspace(const char *fn, const void *workspace, size_t bytes, size_t need)
{
    if (need && (!workspace || bytes < need || !aligned(workspace, 256))) {
        set_error("%s: workspace missing, misaligned or smaller than %zu bytes", fn, need);
        return PCPP_ERR_WORKSPACE;
    }
    return PCPP_OK;
}

int run_dropout(const char *fn, const void *x, int64_t ld_x, const void *residual, const int64_t *random, uint32_t site, float p, int scope,
                const int32_t *offsets, int n_clouds, int64_t n, int c, int in_dtype, int out_dtype, void *y, void *stream)
{
    if (n < 0) return invalid(fn, "negative number of rows");
    if (c < 1 || c > MAX_DROP_CHANNELS) return unsupported(fn, "channel count outside 1..65536");
    if (n >= INT32_MAX) return unsupported(fn, "sizes must be below 2^31");
    if (!is_type(in_dtype) || !is_type(out_dtype)) return unsupported(fn, "unsupported dtype");
    if (!(p >= 0.f && p <= 1.f)) return invalid(fn, "p outside 0 .. 1");
    if (scope < PCPP_DROP_ELEMENTS || scope > PCPP_DROP_CLOUDS) return invalid(fn, "unknown scope");
    if (int rc = check_clouds(fn, offsets, n_clouds)) return rc;
    if (scope != PCPP_DROP_CLOUDS && (offsets || n_clouds != 1)) return invalid(fn, "clouds belong to PCPP_DROP_CLOUDS");
    if (ld_x < c) return invalid(fn, "pitch < c");
    if (ld_x >= MAX_PITCH) return unsupported(fn, "row pitches must be below 2^24");
    if (int rc = check_random(fn, random, n, c)) return rc;
    if (n == 0) return PCPP_OK;
    if (!x || !y || !random) return invalid(fn, "null tensor pointer");
    if (!aligned(x, dtype_bytes(in_dtype)) || !aligned(residual, dtype_bytes(out_dtype)) || !aligned(y, dtype_bytes(out_dtype)))
        return invalid(fn, "tensors must be aligned to their elements");
    if (y == x || y == residual) return invalid(fn, "the output may not be an input");
    DropoutArgs a{};
    a.x = x; a.residual = residual; a.offsets = offsets; a.y = y;
    a.n = n; a.ld_x = ld_x;
    a.c = c; a.scope = scope; a.n_clouds = n_clouds;
    a.drop = make_drop(p, random, site);
    return dropout(a, in_dtype, out_dtype, static_cast<hipStream_t>(stream));
}

// what both directions of the group norm share
int check_norm(const char *fn, int64_t ld_x, const float *w, const float *b, const int32_t *offsets, int n_clouds, int groups, int act, const int64_t *random,
               float p, int64_t n, int c, int dtype)
{
    if (n < 0) return invalid(fn, "negative number of rows");
    if (c < 1 || c > MAX_CHANNELS) return unsupported(fn, "channel count outside 1..1024");
    if (n >= INT32_MAX) return unsupported(fn, "sizes must be below 2^31");
    if (!is_type(dtype)) return unsupported(fn, "unsupported dtype");
    if (groups < 1 || c % groups) return invalid(fn, "groups must divide the channels");
    if (act < PCPP_ACT_NONE || act > PCPP_ACT_GELU) return invalid(fn, "unknown activation");
    if (!(p >= 0.f && p <= 1.f)) return invalid(fn, "p outside 0 .. 1");
    if (p > 0.f && !random) return invalid(fn, "dropout without random");
    if (p > 0.f)
        if (int rc = check_random(fn, random, n, c)) return rc;
    if (int rc = check_clouds(fn, offsets, n_clouds)) return rc;
    if (ld_x < c) return invalid(fn, "pitch < c");
    if (ld_x >= MAX_NORM_PITCH) return unsupported(fn, "row pitches must be below 2^22");
    if (!aligned(w, 4) || !aligned(b, 4)) return invalid(fn, "w and b must be 4-byte aligned");
    return PCPP_OK;
}

int check_mx(const char *fn, int64_t n, int64_t c, int dtype)
{
    if (n < 0 || c < 1) return invalid(fn, "negative number of rows, or no channel");
    if (c >= MX_MAX_CHANNELS) return unsupported(fn, "channel counts must be below 2^24");
    if (n >= INT32_MAX) return unsupported(fn, "sizes must be below 2^31");
    if (!is_type(dtype)) return unsupported(fn, "unsupported dtype");
    return PCPP_OK;
}
int check_product(const char *fn, const uint8_t *b, const uint8_t *b_scales, const float *bias, int act, int64_t n, int64_t m, int64_t k, const void *out,
                  int out_dtype)
{
    if (m < 1) return invalid(fn, "no columns");
    if (m >= MX_MAX_CHANNELS) return unsupported(fn, "m must be below 2^24");
    if (int rc = check_mx(fn, n, k, out_dtype)) return rc;
    if (act < PCPP_ACT_NONE || act > PCPP_ACT_GELU) return invalid(fn, "unknown activation");
    if (n > 0 && (!b || !b_scales || !out)) return invalid(fn, "null tensor pointer");
    if (!aligned(b, 16) || !aligned(b_scales, 4) || !aligned(bias, 4) || !aligned(out, dtype_bytes(out_dtype)))
        return invalid(fn, "codes must be 16-byte aligned, scales and bias 4-byte, out to its elements");
    return PCPP_OK;
}
bool sizes(int64_t n, int64_t m, int64_t k) { return n >= 0 && n < INT32_MAX && m >= 1 && m < MX_MAX_CHANNELS && k >= 1 && k < MX_MAX_CHANNELS; }
size_t linear_codes(int64_t n, int64_t k) { return align_up((size_t)(n * mx_row_bytes(k))); }
size_t linear_scales(int64_t n, int64_t k) { return align_up((size_t)(n * mx_scale_bytes(k))); }

}  // namespace
}  // namespace pcpp

using namespace pcpp;

extern "C" {

int pcpp_dropout_fwd(const void *x, int64_t ld_x, const void *residual, const int64_t *random, uint32_t site, float p, int scope, const int32_t *offsets,
                     int n_clouds, int64_t n, int c, int dtype, int stream_dtype, void *y, void *stream)
{
    const char *fn = "pcpp_dropout_fwd";
    if (stream_dtype != dtype && stream_dtype != PCPP_F32) return unsupported(fn, "unsupported dtype combination");
    return run_dropout(fn, x, ld_x, residual, random, site, p, scope, offsets, n_clouds, n, c, dtype, stream_dtype, y, stream);
}

int pcpp_dropout_bwd(const void *dy, const int64_t *random, uint32_t site, float p, int scope, const int32_t *offsets, int n_clouds, int64_t n, int c, int dtype,
                     int stream_dtype, void *dx, void *stream)
{
    const char *fn = "pcpp_dropout_bwd";
    if (stream_dtype != dtype && stream_dtype != PCPP_F32) return unsupported(fn, "unsupported dtype combination");
    return run_dropout(fn, dy, c, nullptr, random, site, p, scope, offsets, n_clouds, n, c, stream_dtype, dtype, dx, stream);
}

size_t pcpp_group_norm_workspace_bytes(int64_t n, int c, int n_clouds, int groups, int backward)
{
    if (n < 0 || n >= INT32_MAX || c < 1 || c > MAX_CHANNELS || n_clouds < 1 || n_clouds > MAX_CLOUDS || groups < 1 || c % groups) return 0;
    return group_norm_sizes(n, c, n_clouds, groups, backward != 0).bytes;
}

int pcpp_group_norm_fwd(const void *x, int64_t ld_x, const float *w, const float *b, const int32_t *offsets, int n_clouds, int groups, int act, float eps,
                        const int64_t *random, uint32_t site, float p, int64_t n, int c, int dtype, void *y, float *mean_rstd, void *workspace,
                        size_t workspace_bytes, void *stream_)
{
    const char *fn = "pcpp_group_norm_fwd";
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    if (int rc = check_norm(fn, ld_x, w, b, offsets, n_clouds, groups, act, random, p, n, c, dtype)) return rc;
    if (!(eps >= FLT_MIN) || !isfinite(eps)) return invalid(fn, "eps must be finite and at least 2^-126");
    if (!aligned(mean_rstd, 8)) return invalid(fn, "mean_rstd must be 8-byte aligned");
    if (n == 0) return mean_rstd ? fill_u32(reinterpret_cast<uint32_t *>(mean_rstd), 0u, (int64_t)n_clouds * groups * 2, stream) : PCPP_OK;
    if (!x || !y) return invalid(fn, "null tensor pointer");
    if (!aligned(x, dtype_bytes(dtype)) || !aligned(y, 16)) return invalid(fn, "x must be aligned to its elements, y to 16 bytes");
    if (x == y) return invalid(fn, "the output may not be an input");
    const GroupNormSizes s = group_norm_sizes(n, c, n_clouds, groups, false);
    if (int rc = check_workspace(fn, workspace, workspace_bytes, s.bytes)) return rc;
    GroupNormArgs a{};
    a.x = x; a.w = w; a.b = b; a.offsets = offsets; a.y = y;
    a.part = static_cast<float *>(workspace);
    a.stats = mean_rstd || !s.extra ? mean_rstd : reinterpret_cast<float *>(static_cast<char *>(workspace) + s.part);
    a.n = n; a.ld_x = ld_x; a.c = c; a.groups = groups; a.n_clouds = n_clouds; a.act = act; a.eps = eps;
    a.drop = make_drop(p, random, site);
    return group_norm_fwd(a, dtype, stream);
}

int pcpp_group_norm_bwd(const void *dy, const void *x, int64_t ld_x, const float *mean_rstd, const float *w, const float *b, const int32_t *offsets, int n_clouds,
                        int groups, int act, const int64_t *random, uint32_t site, float p, int64_t n, int c, int dtype, void *dx, float *dw, float *db,
                        void *workspace, size_t workspace_bytes, void *stream_)
{
    const char *fn = "pcpp_group_norm_bwd";
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    if (int rc = check_norm(fn, ld_x, w, b, offsets, n_clouds, groups, act, random, p, n, c, dtype)) return rc;
    if (!aligned(dw, 4) || !aligned(db, 4)) return invalid(fn, "the weights' gradients must be 4-byte aligned");
    if (n == 0) {
        if (dw)
            if (int rc = fill_u32(reinterpret_cast<uint32_t *>(dw), 0u, c, stream)) return rc;
        return db ? fill_u32(reinterpret_cast<uint32_t *>(db), 0u, c, stream) : PCPP_OK;
    }
    if (!dy || !x || !mean_rstd) return invalid(fn, "null tensor pointer");
    if (!dx && !dw && !db) return invalid(fn, "nothing to do: no gradient is wanted");
    if (!aligned(x, dtype_bytes(dtype)) || !aligned(dy, 16) || !aligned(dx, 16) || !aligned(mean_rstd, 8))
        return invalid(fn, "x must be aligned to its elements, dy and dx to 16 bytes, mean_rstd to 8");
    if (dx && (dx == dy || dx == x)) return invalid(fn, "the output may not be an input");
    const GroupNormSizes s = group_norm_sizes(n, c, n_clouds, groups, true);
    if (int rc = check_workspace(fn, workspace, workspace_bytes, s.bytes)) return rc;
    GroupNormArgs a{};
    a.x = x; a.dy = dy; a.w = w; a.b = b; a.offsets = offsets; a.dx = dx; a.dw = dw; a.db = db;
    a.stats = const_cast<float *>(mean_rstd);
    a.part = static_cast<float *>(workspace);
    a.coef = s.extra ? reinterpret_cast<float *>(static_cast<char *>(workspace) + s.part) : nullptr;
    a.n = n; a.ld_x = ld_x; a.c = c; a.groups = groups; a.n_clouds = n_clouds; a.act = act;
    a.drop = make_drop(p, random, site);
    return group_norm_bwd(a, dtype, stream);
}

size_t pcpp_mx_row_bytes(int64_t c) { return c < 1 || c >= MX_MAX_CHANNELS ? 0 : (size_t)mx_row_bytes(c); }
size_t pcpp_mx_scale_bytes(int64_t c) { return c < 1 || c >= MX_MAX_CHANNELS ? 0 : (size_t)mx_scale_bytes(c); }

int pcpp_mx_pack(const void *x, int64_t ld_x, int dtype, int64_t n, int64_t c, const int64_t *random, uint32_t site, uint8_t *q, uint8_t *scales, uint8_t *qt,
                 uint8_t *scales_t, void *stream)
{
    const char *fn = "pcpp_mx_pack";
    if (int rc = check_mx(fn, n, c, dtype)) return rc;
    if (ld_x < c) return invalid(fn, "pitch < c");
    if (ld_x >= MAX_MX_PITCH) return unsupported(fn, "row pitches must be below 2^25");
    if (random)
        if (int rc = check_random(fn, random, n, c)) return rc;
    if ((q != nullptr) != (scales != nullptr) || (qt != nullptr) != (scales_t != nullptr)) return invalid(fn, "codes and scales belong together");
    if (qt && n >= MX_MAX_CHANNELS) return unsupported(fn, "columns have fewer than 2^24 rows");
    if (n == 0) return PCPP_OK;
    if (!x || (!q && !qt)) return invalid(fn, "null tensor pointer");
    if (!aligned(x, dtype_bytes(dtype)) || !aligned(q, 16) || !aligned(qt, 16) || !aligned(scales, 4) || !aligned(scales_t, 4))
        return invalid(fn, "x must be aligned to its elements, codes to 16 bytes, scales to 4");
    if (x == q || x == qt || x == scales || x == scales_t) return invalid(fn, "the output may not be an input");
    MxPackArgs a{};
    a.x = x; a.q = q; a.scales = scales; a.qt = qt; a.scales_t = scales_t;
    a.n = n; a.c = c; a.ld_x = ld_x;
    a.random = Random{random, site};
    return mx_pack(a, dtype, static_cast<hipStream_t>(stream));
}

int pcpp_mx_unpack(const uint8_t *q, const uint8_t *scales, int64_t n, int64_t c, void *x, int dtype, void *stream)
{
    const char *fn = "pcpp_mx_unpack";
    if (int rc = check_mx(fn, n, c, dtype)) return rc;
    if (n == 0) return PCPP_OK;
    if (!x || !q || !scales) return invalid(fn, "null tensor pointer");
    if (!aligned(x, dtype_bytes(dtype)) || !aligned(q, 16) || !aligned(scales, 4)) return invalid(fn, "x must be aligned to its elements, codes to 16 bytes, scales to 4");
    if (x == q || x == scales) return invalid(fn, "the output may not be an input");
    return mx_unpack(q, scales, n, c, x, dtype, static_cast<hipStream_t>(stream));
}

size_t pcpp_mx_product_workspace_bytes(int64_t n, int64_t m, int64_t k) { return sizes(n, m, k) ? mx_product_workspace_bytes(n, m, k) : 0; }

int pcpp_mx_product(const uint8_t *a, const uint8_t *a_scales, const uint8_t *b, const uint8_t *b_scales, const float *bias, int act, int64_t n, int64_t m, int64_t k,
                    void *out, int out_dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *fn = "pcpp_mx_product";
    if (int rc = check_product(fn, b, b_scales, bias, act, n, m, k, out, out_dtype)) return rc;
    if (n > 0 && (!a || !a_scales)) return invalid(fn, "null tensor pointer");
    if (!aligned(a, 16) || !aligned(a_scales, 4)) return invalid(fn, "codes must be 16-byte aligned, scales 4-byte");
    if (n == 0) return PCPP_OK;
    if (out == a || out == b || out == a_scales || out == b_scales || out == bias) return invalid(fn, "the output may not be an input");
    if (int rc = check_workspace(fn, workspace, workspace_bytes, mx_product_workspace_bytes(n, m, k))) return rc;
    MxProductArgs p{};
    p.a = a; p.a_scales = a_scales; p.b = b; p.b_scales = b_scales; p.bias = bias; p.out = out; p.part = static_cast<float *>(workspace);
    p.n = n; p.m = m; p.k = k; p.act = act;
    return mx_product(p, out_dtype, static_cast<hipStream_t>(stream));
}

size_t pcpp_mx_linear_workspace_bytes(int64_t n, int64_t m, int64_t k)
{
    if (!sizes(n, m, k) || mx_linear_alone(n, m, k)) return 0;
    return linear_codes(n, k) + linear_scales(n, k) + mx_product_workspace_bytes(n, m, k);
}

int pcpp_mx_linear(const void *x, int64_t ld_x, int x_dtype, const uint8_t *w, const uint8_t *w_scales, const float *bias, int act, int64_t n, int64_t m, int64_t k,
                   void *out, int out_dtype, void *workspace, size_t workspace_bytes, void *stream_)
{
    const char *fn = "pcpp_mx_linear";
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    if (int rc = check_product(fn, w, w_scales, bias, act, n, m, k, out, out_dtype)) return rc;
    if (!is_type(x_dtype)) return unsupported(fn, "unsupported dtype");
    if (ld_x < k) return invalid(fn, "pitch < k");
    if (ld_x >= MAX_MX_PITCH) return unsupported(fn, "row pitches must be below 2^25");
    if (n > 0 && !x) return invalid(fn, "null tensor pointer");
    if (!aligned(x, dtype_bytes(x_dtype))) return invalid(fn, "x must be aligned to its elements");
    if (n == 0) return PCPP_OK;
    if (out == x || out == w || out == w_scales || out == bias) return invalid(fn, "the output may not be an input");
    if (int rc = check_workspace(fn, workspace, workspace_bytes, pcpp_mx_linear_workspace_bytes(n, m, k))) return rc;
    MxProductArgs p{};
    p.b = w; p.b_scales = w_scales; p.bias = bias; p.out = out;
    p.n = n; p.m = m; p.k = k; p.act = act;
    if (mx_linear_alone(n, m, k)) return mx_linear_alone(p, x, x_dtype, ld_x, out_dtype, stream);
    char *at = static_cast<char *>(workspace);
    MxPackArgs a{};
    a.x = x; a.q = reinterpret_cast<uint8_t *>(at); a.scales = a.q + linear_codes(n, k);
    a.n = n; a.c = k; a.ld_x = ld_x;
    if (int rc = mx_pack(a, x_dtype, stream)) return rc;
    p.a = a.q; p.a_scales = a.scales;
    p.part = reinterpret_cast<float *>(at + linear_codes(n, k) + linear_scales(n, k));
    return mx_product(p, out_dtype, stream);
}

}  // extern "C"
