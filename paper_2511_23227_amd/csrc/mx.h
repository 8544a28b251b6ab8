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
    const uint32_t e = (amax + (random ? 0x3fffffu : 0x200000u)) >> 23, at_least = e > 3u ? e : 3u, code = (at_least < MX_TOP_CODE + 2u ? at_least : MX_TOP_CODE + 2u) - 2u;
    return amax >= 0x7f800000u ? MX_NAN_CODE : code;
}
__device__ inline float mx_step(uint32_t code) { return __uint_as_float(code << 23); }      // (255: what comes of it is left aside)

// ---- eight numbers as they lie in memory to eight 4-bit codes -----------------------------------------------------------------------
// The conversions divide by the power of two (exactly) and round to nearest (ties to the even fraction) or at random: a 32-bit fraction is added to
// what lies below the last place, here an element's sixteen bits in the upper half, so up if the remainder's first sixteen bits and they make a whole
// step.  Past 6 they give 6.  A pair of numbers shares a conversion; at random each takes its own, of which only its half is used (the second of a
// pair takes the fraction one place lower; the compiler does not hand the destination's other bytes on, so they are put together here).
typedef uint16_t v2u16 __attribute__((ext_vector_type(2)));
template <typename T> struct Pair;
template <> struct Pair<float> {
    float lo, hi;
    template <int BYTE> __device__ inline uint32_t nearest(uint32_t to, float step) const { return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(to, lo, hi, step, BYTE); }
    __device__ inline uint32_t random(uint32_t seed_lo, uint32_t seed_hi, float step) const      // in the lowest byte; what is above may be anything
    {
        const uint32_t a = __builtin_amdgcn_cvt_scalef32_sr_pk_fp4_f32(0u, v2f{lo, hi}, seed_lo, step, 0), b = __builtin_amdgcn_cvt_scalef32_sr_pk_fp4_f32(0u, v2f{lo, hi}, seed_hi, step, 0);
        return (a & 15u) | (b & ~15u);
    }
};
template <> struct Pair<bf16_t> {
    uint32_t bits;
    template <int BYTE> __device__ inline uint32_t nearest(uint32_t to, float step) const
    {
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(to, __builtin_bit_cast(v2bf, bits), step, BYTE);
    }
    // (the conversion from bf16 keeps so few bits of the remainder that small numbers never go up)
    __device__ inline uint32_t random(uint32_t seed_lo, uint32_t seed_hi, float step) const
    {
        return Pair<float>{__uint_as_float(bits << 16), __uint_as_float(bits & 0xffff0000u)}.random(seed_lo, seed_hi, step);
    }
};
// channels 2 i and 2 i + 1
template <int I> __device__ inline Pair<float> pair_of(const Eight<float> &r) { return Pair<float>{__uint_as_float(r.a[I >> 1][2 * I & 3]), __uint_as_float(r.a[I >> 1][(2 * I & 3) + 1])}; }
template <int I> __device__ inline Pair<bf16_t> pair_of(const Eight<bf16_t> &r) { return Pair<bf16_t>{r.a[0][I]}; }

// the bits of the largest magnitude as an fp32 number's (as whole numbers: a NaN is larger than any number)
__device__ inline uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ inline uint32_t larger_pair(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(v2u16, a), __builtin_bit_cast(v2u16, b)));
}
__device__ inline uint32_t largest(const Eight<float> &r)
{
    uint32_t m = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = larger(m, r.a[e >> 2][e & 3] & 0x7fffffffu);
    return m;
}
__device__ inline uint32_t largest(const Eight<bf16_t> &r)
{
    uint32_t m = r.a[0][0] & 0x7fff7fffu;
#pragma unroll
    for (int i = 1; i < 4; ++i) m = larger_pair(m, r.a[0][i] & 0x7fff7fffu);
    return larger(m << 16, m & 0xffff0000u);
}
__device__ inline uint32_t quad_largest(uint32_t m)
{
    m = larger(m, dpp<DPP_XOR1>(m));
    return larger(m, dpp<DPP_XOR2>(m));
}
// element e's sixteen bits as the fraction of the first and of the second of a pair
__device__ inline uint32_t first_seed(const uint32_t (&u)[4], int e) { return (e & 1) ? u[e >> 1] & 0xffff0000u : u[e >> 1] << 16; }
__device__ inline uint32_t second_seed(const uint32_t (&u)[4], int e) { return (e & 1) ? (u[e >> 1] & 0xffff0000u) >> 1 : u[e >> 1] << 15; }
template <bool RANDOM, typename T> __device__ inline uint32_t mx_quantise(const Eight<T> &r, uint32_t code, const uint32_t (&u)[4])
{
    const float step = mx_step(code);
    uint32_t q = 0u;
    if constexpr (RANDOM) {
        const uint32_t b0 = pair_of<0>(r).random(first_seed(u, 0), second_seed(u, 1), step), b1 = pair_of<1>(r).random(first_seed(u, 2), second_seed(u, 3), step);
        const uint32_t b2 = pair_of<2>(r).random(first_seed(u, 4), second_seed(u, 5), step), b3 = pair_of<3>(r).random(first_seed(u, 6), second_seed(u, 7), step);
        q = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b3, b2, 0x0c0c0400u), __builtin_amdgcn_perm(b1, b0, 0x0c0c0400u), 0x05040100u);
    } else {
        q = pair_of<0>(r).template nearest<0>(q, step);
        q = pair_of<1>(r).template nearest<1>(q, step);
        q = pair_of<2>(r).template nearest<2>(q, step);
        q = pair_of<3>(r).template nearest<3>(q, step);
    }
    return code == MX_NAN_CODE ? 0u : q;
}

// Channels c0 .. of a row of c; zeros past the last.  Where the row ends inside the eight the row's last eight are read and moved into place.
__device__ inline void move_down(Eight<float> &r, int by)
{
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = r.a[e >> 2][e & 3];
#pragma unroll
    for (int s = 4; s > 0; s >>= 1)
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = by & s ? (e + s < 8 ? w[e + s < 8 ? e + s : 7] : 0u) : w[e];
#pragma unroll
    for (int e = 0; e < 8; ++e) r.a[e >> 2][e & 3] = w[e];
}
__device__ inline void move_down(Eight<bf16_t> &r, int by)
{
    uint32_t w[4] = {r.a[0][0], r.a[0][1], r.a[0][2], r.a[0][3]};
#pragma unroll
    for (int s = 2; s > 0; s >>= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = by & 2 * s ? (i + s < 4 ? w[i + s < 4 ? i + s : 3] : 0u) : w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = by & 1 ? w[i] >> 16 | (i < 3 ? w[i < 3 ? i + 1 : 3] << 16 : 0u) : w[i];
    r.a[0] = v4u{w[0], w[1], w[2], w[3]};
}
template <typename T> __device__ inline void load_within(const T *row, int64_t c0, int64_t c, Eight<T> &r) { load_eight<false>(row + (c0 + 8 <= c ? c0 : c - 8), r); }
template <typename T> __device__ inline void into_place(int64_t c0, int64_t c, Eight<T> &r)
{
    if (c0 + 8 <= c) return;
    if (c0 < c) return move_down(r, (int)(c0 + 8 - c));
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.a[i] = v4u{0u, 0u, 0u, 0u};
}
template <typename T> __device__ inline void load_channels(const T *row, int64_t c0, int64_t c, Eight<T> &r)
{
    if (c >= 8) {
        load_within(row, c0, c, r);
        into_place(c0, c, r);
        return;
    }
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.a[i] = v4u{0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (c0 + e < c) {
            if constexpr (sizeof(T) == 4) r.a[e >> 2][e & 3] = __float_as_uint(row[c0 + e]);
            else r.a[0][e >> 1] |= (uint32_t)row[c0 + e] << (16 * (e & 1));
        }
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
// rows of x [n, k] as they are, rounded where they are multiplied (a and a_scales are not read)
bool mx_linear_alone(int64_t n, int64_t m, int64_t k);
int mx_linear_alone(const MxProductArgs &a, const void *x, int x_dtype, int64_t ld_x, int out_dtype, hipStream_t stream);

}  // namespace pcpp
