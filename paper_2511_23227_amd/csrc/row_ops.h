// Rows of channels in registers, shared by the kernels that take whole rows (block_norm.hip, act_pack.hip, log_probs.hip); not part
// of the C ABI.
//
// A row is held by LPR neighbouring lanes (a power of two, 4 .. 64), eight consecutive channels each.  Loads and stores move 16 or 32
// bytes per lane at whatever alignment the row has (the hardware takes global accesses at any).  Where the row ends inside a lane's
// eight channels the lane holds the row's last eight instead: the first of them are the lane before's too, come out the same there and
// are written twice, but count in no sum (Span).  So no access leaves the row and none is narrower; shifting the channels into place
// took three instructions for each, 57 us instead of 42 for the gradients between blocks of 91 channels, 99 991 rows.  Rows of fewer
// than eight channels are read and written one by one.
#pragma once

#include "mvmr_rows_common.h"

namespace pcpp {

typedef uint16_t bf16_t;                                          // a bf16 number as it lies in memory

struct __attribute__((packed, aligned(1))) Bytes16 { v4u v; };
struct __attribute__((packed, aligned(1))) Bytes8 { uint32_t v[2]; };

template <typename T> struct Eight;                               // eight channels as they lie in memory
template <> struct Eight<float> { v4u a[2]; };
template <> struct Eight<bf16_t> { v4u a[1]; };

__device__ inline float bf16_float(uint32_t bits) { return __uint_as_float(bits << 16); }
template <typename T> __device__ inline float one_float(T v);
template <> __device__ inline float one_float<float>(float v) { return v; }
template <> __device__ inline float one_float<bf16_t>(bf16_t v) { return bf16_float(v); }
template <typename T> __device__ inline T one_of(float v);
template <> __device__ inline float one_of<float>(float v) { return v; }
template <> __device__ inline bf16_t one_of<bf16_t>(float v) { return (bf16_t)(cvt_pk_bf16(v, v) & 0xffffu); }

template <typename T> __device__ inline void load_eight(const T *p, Eight<T> &r)
{
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.a[i] = reinterpret_cast<const Bytes16 *>(p)[i].v;
}
template <typename T> __device__ inline void to_floats(const Eight<T> &r, float (&v)[8])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(r.a[e >> 2][e & 3]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __uint_as_float((e & 1) ? r.a[0][e >> 1] & 0xffff0000u : r.a[0][e >> 1] << 16);
    }
}
template <typename T> __device__ inline void store_eight(T *p, const float (&v)[8])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            reinterpret_cast<Bytes16 *>(p)[i].v = v4u{__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]),
                                                      __float_as_uint(v[4 * i + 3])};
    } else {
        reinterpret_cast<Bytes16 *>(p)->v = v4u{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]), cvt_pk_bf16(v[6], v[7])};
    }
}

// The channels of a row of c that the lane at c0, c0 + 8 .. 's place holds: element e is channel at + e and its own if lo <= e < hi.
// WHOLE: c is a multiple of eight, so a lane holds its eight or none.
template <bool WHOLE> struct Span {
    int at, lo, hi;
    __device__ inline Span() {}
    __device__ inline Span(int c0, int c)
    {
        at = c0;
        lo = c0 < c ? 0 : 8;
        hi = 8;
        if (!WHOLE) {
            if (c < 8) hi = c;
            else if (c0 < c && c0 + 8 > c) at = c - 8, lo = c0 - at;
        }
    }
    __device__ inline bool any() const { return lo < 8; }
    __device__ inline bool own(int e) const { return WHOLE ? lo == 0 : e >= lo && e < hi; }
    __device__ inline bool narrow() const { return !WHOLE && hi < 8; }
};

// What a lane reads of a row, all zero without channels (and past them in narrow rows)
template <typename T, bool WHOLE> __device__ inline void row_load(const T *row, const Span<WHOLE> &s, Eight<T> &r)
{
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.a[i] = v4u{0u, 0u, 0u, 0u};
    if (!s.any()) return;
    if (!s.narrow()) {
        load_eight(row + s.at, r);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < s.hi) {
                if constexpr (sizeof(T) == 4) r.a[e >> 2][e & 3] = __float_as_uint(row[e]);
                else r.a[0][e >> 1] |= (uint32_t)row[e] << (16 * (e & 1));
            }
    }
}
template <typename T, bool WHOLE> __device__ inline void row_store(T *row, const Span<WHOLE> &s, const float (&v)[8])
{
    if (!s.any()) return;
    if (!s.narrow()) {
        store_eight(row + s.at, v);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < s.hi) row[e] = one_of<T>(v[e]);
    }
}

// Value of the lane at distance 1, 2 and, where the lanes of a quad (of eight) hold the same already, of another quad (eight).
template <int CTRL> __device__ inline uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
constexpr int DPP_XOR1 = 0xb1, DPP_XOR2 = 0x4e, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;

// op over the LPR lanes of a row, the same in all of them: pairs, quads, half rows and rows of sixteen lanes by DPP, beyond by exchanging rows
// between two copies of the register
template <int LPR, typename Op> __device__ inline float row_reduce(float v, Op op)
{
    auto with = [&](uint32_t o) { v = op(v, __uint_as_float(o)); };
    if constexpr (LPR >= 2) with(dpp<DPP_XOR1>(__float_as_uint(v)));
    if constexpr (LPR >= 4) with(dpp<DPP_XOR2>(__float_as_uint(v)));
    if constexpr (LPR >= 8) with(dpp<DPP_HALF_MIRROR>(__float_as_uint(v)));
    if constexpr (LPR >= 16) with(dpp<DPP_MIRROR>(__float_as_uint(v)));
    if constexpr (LPR >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    if constexpr (LPR >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    return v;
}
template <int LPR> __device__ inline float row_sum(float v) { return row_reduce<LPR>(v, [](float a, float b) { return a + b; }); }
template <int LPR> __device__ inline float row_max(float v) { return row_reduce<LPR>(v, [](float a, float b) { return fmaxf(a, b); }); }

// ---- eight bits: blocks of 32 channels of a row share a power of two, value = q 2^(code - 127) --------------------------------
constexpr int ACT_BLOCK = 32;
constexpr int act_code_bytes(int c) { return (int)ceil_div(c, 4 * ACT_BLOCK) * 4; }     // per row, whole 32-bit words

// Code of a block from the bits of its largest magnitude: the smallest power of two with which nothing rounds past 127 (a magnitude of
// 127.5 steps or more takes the next), not below 2^-126; 255 where a value is Inf or NaN.
__device__ inline uint32_t act_code(uint32_t amax)
{
    if (amax >= 0x7f800000u) return 255u;
    const int e = (int)((amax + 0x10000u) >> 23) - 6;
    return (uint32_t)(e < 1 ? 1 : e);
}
__device__ inline float act_step(uint32_t code) { return __uint_as_float(code << 23); }  // 255: Inf, with q = 0 a NaN

// The lane's eight channels in 8 bits; the block's four lanes are a quad.  The products are exact (a power of two), so adding 1.5 2^23
// rounds once, to nearest even, and leaves q in the low byte.
template <bool WHOLE> __device__ inline uint32_t act_quantise(const float (&v)[8], const Span<WHOLE> &s, uint32_t (&q)[2])
{
    uint32_t amax = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t b = s.own(e) ? __float_as_uint(v[e]) & 0x7fffffffu : 0u;
        amax = amax > b ? amax : b;                               // (as integers: a NaN is larger than any number)
    }
    uint32_t o = dpp<DPP_XOR1>(amax);
    amax = amax > o ? amax : o;
    o = dpp<DPP_XOR2>(amax);
    amax = amax > o ? amax : o;
    const uint32_t code = act_code(amax);
    const float scale = __uint_as_float((254u - (code < 254u ? code : 253u)) << 23);
    uint32_t b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = __float_as_uint(__builtin_fmaf(v[e], scale, 12582912.0f));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lo = __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x04000c0cu);
        q[i] = code == 255u ? 0u : lo | hi;
    }
    return code;
}
// ... stored as channels of `row` (q: [c] bytes, codes: act_code_bytes(c) bytes, the unused ones zero).  All lanes of the quad call it.
template <bool WHOLE> __device__ inline void act_store(const float (&v)[8], int8_t *row, uint8_t *codes, const Span<WHOLE> &s, int c0, int c)
{
    uint32_t q[2];
    const uint32_t code = act_quantise(v, s, q);
    if (!s.any()) return;
    if (WHOLE || (!s.narrow() && (s.lo == 0 || c0 % ACT_BLOCK != 0))) {
        *reinterpret_cast<Bytes8 *>(row + s.at) = Bytes8{{q[0], q[1]}};
    } else {                                                      // (the lane before's are of another block)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (s.own(e)) row[s.at + e] = (int8_t)(q[e >> 2] >> (8 * (e & 3)));
    }
    if (c0 % ACT_BLOCK == 0) {
        const int at = c0 / ACT_BLOCK;
        codes[at] = (uint8_t)code;
        if (c0 + ACT_BLOCK >= c)
            for (int i = at + 1; i < act_code_bytes(c); ++i) codes[i] = 0;
    }
}
// What a lane reads of a row in 8 bits, and its values.
struct Eight8 { uint32_t q[2], code, before; };                   // before: code of the channels that are the lane before's
template <bool WHOLE> __device__ inline void act_load(const int8_t *row, const uint8_t *codes, const Span<WHOLE> &s, int c0, Eight8 &r)
{
    r = Eight8{{0u, 0u}, 0u, 0u};
    if (!s.any()) return;
    r.code = codes[c0 / ACT_BLOCK];
    if (!WHOLE) r.before = codes[s.at / ACT_BLOCK];
    if (!s.narrow()) {
        const Bytes8 b = *reinterpret_cast<const Bytes8 *>(row + s.at);
        r.q[0] = b.v[0];
        r.q[1] = b.v[1];
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < s.hi) r.q[e >> 2] |= (uint32_t)(uint8_t)row[e] << (8 * (e & 3));
    }
}
template <bool WHOLE> __device__ inline void act_floats(const Eight8 &r, const Span<WHOLE> &s, float (&v)[8])
{
    const float step = act_step(r.code), before = WHOLE ? step : act_step(r.before);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)(int8_t)(r.q[e >> 2] >> (8 * (e & 3))) * (WHOLE || e >= s.lo ? step : before);
}

}  // namespace pcpp
