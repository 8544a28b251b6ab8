// Numbers in microscaled 4-bit floating point and the launches of their kernels; not part of the C ABI.
//
// An element is a sign, two bits of exponent and one of fraction: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives (code 8 and on).  32 of a row share
// a power of two, whose code is its exponent plus 127.  Two elements lie in a byte, the even one in the low half.
#pragma once

#include "pointwise.h"

namespace pcpp {

constexpr int MX_BLOCK = 32;
constexpr int64_t MX_MAX_CHANNELS = 1 << 24;                      // (a tile's rows lie within 32-bit offsets)
constexpr int64_t mx_blocks(int64_t c) { return ceil_div(c, MX_BLOCK); }
constexpr int64_t mx_row_bytes(int64_t c) { return 16 * mx_blocks(c); }
constexpr int64_t mx_scale_bytes(int64_t c) { return 4 * ceil_div(c, 4 * MX_BLOCK); }       // whole 32-bit words

// Code of a block from the bits of its largest magnitude: the smallest power of two with which nothing rounds past 6, not below 2^-126 nor
// above 2^125 (6 times the next would be Inf; the largest numbers stay at 6); 255 where a value is Inf or NaN.  To nearest, 7 steps and more round past 6; at
// random, anything above.
constexpr uint32_t MX_TOP_CODE = 252u, MX_NAN_CODE = 255u;
__device__ inline uint32_t mx_code(uint32_t amax, bool random)
{
    if (amax >= 0x7f800000u) return MX_NAN_CODE;
    const int e = (int)((amax + (random ? 0x3fffffu : 0x200000u)) >> 23) - 2;
    return e < 1 ? 1u : (e < (int)MX_TOP_CODE ? (uint32_t)e : MX_TOP_CODE);
}
__device__ inline float mx_inverse(uint32_t code) { return __uint_as_float((254u - (code < MX_TOP_CODE ? code : MX_TOP_CODE)) << 23); }

// Eight numbers, scaled already, as eight 4-bit codes, to the nearest (ties to the even fraction, past 6 to 6)
__device__ inline uint32_t mx_nearest(const float (&v)[8])
{
    uint32_t r = 0u;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], 1.f, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], 1.f, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], 1.f, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], 1.f, 3);
}
// One number, scaled already, rounded away from zero if the first sixteen bits of the remainder and `u` make a whole step: in [1, 6] the codes
// are the numbers' own exponent and fraction, below 1 they are steps of a half.
__device__ inline uint32_t mx_random(float v, uint32_t u)
{
    const uint32_t bits = __float_as_uint(v), a = bits & 0x7fffffffu;
    const uint32_t large = (a - (126u << 23) + (u << 6)) >> 22, small = ((uint32_t)(__uint_as_float(a) * 131072.f) + u) >> 16;
    const uint32_t code = a < 0x3f800000u ? small : large;
    return (code < 7u ? code : 7u) | (bits >> 28 & 8u);
}

struct MxPackArgs {
    const void *x;
    uint8_t *q, *scales, *qt, *scales_t;                          // rows, and columns; NULL: not wanted
    int64_t n, c, ld_x;
    Random random;                                                // without a state: to the nearest
};
int mx_pack(const MxPackArgs &a, int dtype, hipStream_t stream);
int mx_unpack(const uint8_t *q, const uint8_t *scales, int64_t n, int64_t c, void *x, int dtype, hipStream_t stream);

struct MxProductArgs {
    const uint8_t *a, *a_scales, *b, *b_scales;                   // [n, k], [m, k]
    const float *bias;
    void *out;                                                    // [n, m]
    float *part;                                                  // workspace: partial products
    int64_t n, m, k;
    int act;
};
size_t mx_product_workspace_bytes(int64_t n, int64_t m, int64_t k);
int mx_product(const MxProductArgs &a, int out_dtype, hipStream_t stream);

}  // namespace pcpp
