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
    // the first cloud that ends behind `row`, `count` if none does: for a lane's own row
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
    // ... for a row that the whole wave asks for: 64 offsets at a time, so one load for up to 64 clouds
    __device__ inline int at_for_all(int64_t row) const
    {
        if (!offsets) return row < n ? 0 : 1;
        const int lane = threadIdx.x & 63;
        int lo = 0, hi = count;
        while (hi - lo > 64) {
            const int step = (hi - lo + 63) / 64, i = lo + (lane + 1) * step - 1;
            const unsigned long long behind = __ballot(i >= hi || bound(i + 1) > row);
            const int k = behind ? __ffsll((long long)behind) - 1 : 64;
            lo = lo + k * step < hi ? lo + k * step : hi;
            hi = lo + step - 1 < hi ? lo + step - 1 : hi;
        }
        const unsigned long long behind = __ballot(lo + lane >= hi || bound(lo + lane + 1) > row);
        const int k = behind ? __ffsll((long long)behind) - 1 : 64;
        return __builtin_amdgcn_readfirstlane(lo + k < hi ? lo + k : hi);
    }
};
// The clouds as a wave asks for them, all lanes the same: up to 63 are held, an offset a lane, so that all its questions cost one load
struct WaveClouds {
    Clouds clouds;
    int own = 0;
    bool held;
    __device__ inline explicit WaveClouds(const Clouds &c) : clouds(c), held(c.offsets && c.count < 64)
    {
        const int lane = threadIdx.x & 63;
        if (held) own = (int)c.bound(lane <= c.count ? lane : c.count);
    }
    __device__ inline int64_t bound(int b) const { return held ? (int64_t)__builtin_amdgcn_readlane(own, b) : clouds.bound(b); }
    __device__ inline int64_t first(int b) const { return bound(b); }
    __device__ inline int64_t end(int b) const
    {
        const int64_t a = bound(b), e = bound(b + 1);
        return e > a ? e : a;
    }
    __device__ inline int at(int64_t row) const
    {
        if (!held) return clouds.at_for_all(row);
        const int lane = threadIdx.x & 63;
        const unsigned long long behind = __ballot(lane >= 1 && lane <= clouds.count && own > row);
        return behind ? __ffsll((long long)behind) - 2 : clouds.count;
    }
};

// ---- activations --------------------------------------------------------------------------------------------------------------
__device__ inline float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * z)); }
// The normal distribution below -a, a >= 0: 2 to a polynomial of degree 10, fitted to the logarithm over 0 .. 8 by least squares for the absolute
// error (and a hundredth of it for the relative), reweighted until it was level; behind 8 it goes on falling.  In fp32 off by 1.1e-7 at most, a times
// it by 5e-8, and by 3.5e-5 of itself below 6. One exponential and no division: with the library's erff a 115 200 x 256 output took 20 us longer than
// without an activation, with exp(-a^2) t P(t), t = 1 / (1 + k a), 12.
__device__ inline float normal_tail(float a)
{
    float p = -8.52743387e-09f;
    p = __builtin_fmaf(p, a, 3.22056252e-07f);
    p = __builtin_fmaf(p, a, -5.06018932e-06f);
    p = __builtin_fmaf(p, a, 4.1338244e-05f);
    p = __builtin_fmaf(p, a, -0.000156961585f);
    p = __builtin_fmaf(p, a, -0.000257518404f);
    p = __builtin_fmaf(p, a, 0.0072662225f);
    p = __builtin_fmaf(p, a, -0.0526625291f);
    p = __builtin_fmaf(p, a, -0.459144771f);
    p = __builtin_fmaf(p, a, -1.15111411f);
    p = __builtin_fmaf(p, a, -0.999999821f);
    return __builtin_amdgcn_exp2f(p);
}
__device__ inline float tail_at(float z) { return __builtin_fabsf(z) > 14.f ? 14.f : __builtin_fabsf(z); }     // (a NaN stays; further out nothing is left)
template <int ACT> __device__ inline float activate(float z)
{
    if constexpr (ACT == PCPP_ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
    else if constexpr (ACT == PCPP_ACT_SILU) return z * logistic(z);
    else if constexpr (ACT == PCPP_ACT_GELU) {
        const float a = tail_at(z);
        return __builtin_fmaf(-a, normal_tail(a), fmaxf(z, 0.f));
    } else return z;
}
template <int ACT> __device__ inline float slope(float z)         // the derivative
{
    if constexpr (ACT == PCPP_ACT_RELU) return z > 0.f ? 1.f : (z != z ? z : 0.f);
    else if constexpr (ACT == PCPP_ACT_SILU) {
        const float s = logistic(z);
        return __builtin_fmaf(z * s, 1.f - s, s);
    } else if constexpr (ACT == PCPP_ACT_GELU) {
        const float a = tail_at(z), below = __builtin_fmaf(-0.39894228f * a, __builtin_amdgcn_exp2f(-0.72134752f * a * a), normal_tail(a));
        return z > 0.f ? 1.f - below : below;
    } else return 1.f;
}
// f(activation): a branch that all lanes take alike
template <typename F> __device__ inline void as_act(int act, F f)
{
    if (act == PCPP_ACT_NONE) f(Int<PCPP_ACT_NONE>{});
    else if (act == PCPP_ACT_SILU) f(Int<PCPP_ACT_SILU>{});
    else if (act == PCPP_ACT_GELU) f(Int<PCPP_ACT_GELU>{});
    else f(Int<PCPP_ACT_RELU>{});
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
