// What the operators of the pointwise layers share: clouds of a batch, activations behind a norm or a product, division by a
// number that the host knows; and their launches.  Not part of the C ABI.
#pragma once

#include "philox.h"
#include "row_ops.h"

namespace pcpp {

// ---- clouds -------------------------------------------------------------------------------------------------------------------
// Rows [offsets[b], offsets[b + 1]) belong to cloud b; without offsets all n rows are one cloud's.  Whatever the array holds, the ranges that
// come out lie inside the tensor.
struct Clouds {
    const int32_t *offsets;
    int count;
    int64_t n;
    __device__ inline int64_t bound(int b) const
    {
        if (!offsets) return b <= 0 ? 0 : n;
        const int64_t v = offsets[b];
        return v < 0 ? 0 : (v < n ? v : n);
    }
    __device__ inline int64_t first(int b) const { return bound(b); }
    __device__ inline int64_t end(int b) const
    {
        const int64_t a = bound(b), e = bound(b + 1);
        return e > a ? e : a;
    }
    // the first cloud that ends behind `row`, `count` if none does
    __device__ inline int at(int64_t row) const
    {
        int lo = 0, hi = count;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (bound(mid + 1) > row) hi = mid;
            else lo = mid + 1;
        }
        return lo;
    }
};

// ---- activations --------------------------------------------------------------------------------------------------------------
__device__ inline float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * z)); }
// The normal distribution below z, (1 + erf(z / sqrt 2)) / 2, and its density without 1 / sqrt(2 pi).  erfc(x) = exp(-x^2) t P(t) with t = 1 / (1 + 0.49 x): P
// of degree 8 by least squares for the relative error over 0 <= x <= 14, reweighted until its largest, 5.5e-8, was level.  In fp32 off by 1.8e-7 at most, and by
// 3e-6 of itself where it is small.  The library's erff took twice the time of the whole epilogue.
__device__ inline float normal(float z, float &density)
{
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.34648232f, __builtin_fabsf(z), 1.f));
    density = __builtin_amdgcn_exp2f(-0.72134752f * z * z);
    float p = -0.0269294106f;
    p = __builtin_fmaf(p, t, 0.137322286f);
    p = __builtin_fmaf(p, t, -0.252138865f);
    p = __builtin_fmaf(p, t, 0.16366231f);
    p = __builtin_fmaf(p, t, -0.0237202372f);
    p = __builtin_fmaf(p, t, 0.106285078f);
    p = __builtin_fmaf(p, t, 0.118834596f);
    p = __builtin_fmaf(p, t, 0.13846641f);
    p = __builtin_fmaf(p, t, 0.138217861f);
    const float below = p * t * density;
    return z < 0.f ? below : 1.f - below;
}
template <int ACT> __device__ inline float activate(float z)
{
    if constexpr (ACT == PCPP_ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
    else if constexpr (ACT == PCPP_ACT_SILU) return z * logistic(z);
    else if constexpr (ACT == PCPP_ACT_GELU) {
        float density;
        return z * normal(z, density);
    } else return z;
}
template <int ACT> __device__ inline float slope(float z)         // the derivative
{
    if constexpr (ACT == PCPP_ACT_RELU) return z > 0.f ? 1.f : (z != z ? z : 0.f);
    else if constexpr (ACT == PCPP_ACT_SILU) {
        const float s = logistic(z);
        return s * (1.f + z * (1.f - s));
    } else if constexpr (ACT == PCPP_ACT_GELU) {
        float density;
        const float below = normal(z, density);
        return __builtin_fmaf(0.39894228f * z, density, below);
    } else return 1.f;
}
template <typename F> void with_act(int act, F f)
{
    switch (act) {
    case PCPP_ACT_RELU: return f(Int<PCPP_ACT_RELU>{});
    case PCPP_ACT_SILU: return f(Int<PCPP_ACT_SILU>{});
    case PCPP_ACT_GELU: return f(Int<PCPP_ACT_GELU>{});
    default: return f(Int<PCPP_ACT_NONE>{});
    }
}

// ---- x / d by a multiplication (Granlund and Montgomery, "Division by invariant integers using multiplication", 1994) ---------------
struct Divisor {
    uint32_t by, mul, s1, s2;
    __device__ inline uint32_t quotient(uint32_t x) const
    {
        const uint32_t t = __umulhi(mul, x);
        return (t + ((x - t) >> s1)) >> s2;
    }
};
inline Divisor make_divisor(uint32_t d)
{
    int l = 0;
    while (l < 32 && ((uint64_t)1 << l) < d) ++l;
    return Divisor{d, (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << l) - d)) / d + 1), l > 0 ? 1u : 0u, l > 0 ? (uint32_t)l - 1u : 0u};
}

// ---- launches -----------------------------------------------------------------------------------------------------------------
struct DropoutArgs {
    const void *x, *residual;                                     // backward: dy, NULL
    const int32_t *offsets;
    void *y;
    int64_t n, ld_x;
    int c, scope, n_clouds;
    Drop drop;
};
int dropout(const DropoutArgs &a, int in_dtype, int out_dtype, hipStream_t stream);

struct GroupNormArgs {
    const void *x, *dy;
    const float *w, *b;
    const int32_t *offsets;
    void *y, *dx;
    float *dw, *db;
    float *stats;                                                 // [clouds][groups][mean, rstd]: written forward, read backward
    float *part;                                                  // workspace
    float *coef;                                                  // backward: [clouds][groups][m1, m2]
    int64_t n, ld_x;
    int c, groups, n_clouds, act;
    float eps;
    Drop drop;
};
struct GroupNormSizes { int64_t rows; int chunks; size_t slots, part, extra, bytes; };       // rows of a chunk; byte sizes
GroupNormSizes group_norm_sizes(int64_t n, int c, int n_clouds, int groups, bool backward);
int group_norm_fwd(const GroupNormArgs &a, int dtype, hipStream_t stream);
int group_norm_bwd(const GroupNormArgs &a, int dtype, hipStream_t stream);

}  // namespace pcpp
