// Rows of channels in registers, shared by the kernels that take whole rows (block_norm.hip, act_pack.hip, log_probs.hip); not part
// of the C ABI.
//
// A row is held by LPR neighbouring lanes (a power of two, 4 .. 64), eight consecutive channels each, so a wave holds 64 / LPR rows.  It
// reads and writes them through buffer descriptors that start at its first row and end behind the tensor's last one: the lanes'
// offsets are the same for all the rows it goes through, and what lies past the tensor or past a row's channels (an offset past
// any descriptor) reads as zero and is not written, without a branch.  A tensor that is not there is an empty descriptor.  Accesses are
// 16 or 32 bytes per lane at whatever alignment the row has.
//
// Where the row ends inside a lane's eight channels (RAGGED) the lane holds the row's last eight instead: the first of them are the lane
// before's too, come out the same there and are written twice, but count in no sum.  So no access is narrower.  Gradients between
// blocks of 91 channels, 99 991 rows: 57 us with those channels shifted into place, 47 held twice, 34 with descriptors in place of branches.  Rows of fewer than eight
// channels (NARROW) are read and written one by one.
#pragma once

#include "mvmr_rows_common.h"

namespace pcpp {

typedef uint16_t bf16_t;                                          // a bf16 number as it lies in memory
typedef uint32_t v2u32 __attribute__((ext_vector_type(2)));

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

// ---- eight channels anywhere in memory, for rows that are walked (log_probs.hip) ----------------------------------------------
typedef v4u v4u_anywhere __attribute__((aligned(1)));
template <bool ONCE, typename T> __device__ inline void load_eight(const T *p, Eight<T> &r)     // ONCE: past the caches
{
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) {
        const v4u_anywhere *at = reinterpret_cast<const v4u_anywhere *>(p) + i;
        if constexpr (ONCE) r.a[i] = __builtin_nontemporal_load(at);
        else r.a[i] = *at;
    }
}
template <typename T> __device__ inline void from_floats(const float (&v)[8], Eight<T> &r)
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            r.a[i] = v4u{__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])};
    } else {
        r.a[0] = v4u{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]), cvt_pk_bf16(v[6], v[7])};
    }
}
template <bool ONCE, typename T> __device__ inline void store_eight(T *p, const float (&v)[8])
{
    Eight<T> r;
    from_floats(v, r);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) {
        v4u_anywhere *at = reinterpret_cast<v4u_anywhere *>(p) + i;
        if constexpr (ONCE) __builtin_nontemporal_store(r.a[i], at);
        else *at = r.a[i];
    }
}

// ---- rows in registers --------------------------------------------------------------------------------------------------------
constexpr int RAGGED = 0, WHOLE = 1, NARROW = 2;                  // c >= 8, a multiple of eight, < 8
// Lanes for a row of c <= 512 channels; rows of up to 1024 lie in 64 lanes, sixteen channels each.
constexpr int row_lanes(int c) { return c <= 32 ? 4 : (c <= 64 ? 8 : (c <= 128 ? 16 : (c <= 256 ? 32 : 64))); }

// The channels of a row of c that the lane whose place is c0, c0 + 8 .. holds: element e is channel at + e.
template <int MODE> struct Span {
    int at, lo, n;                                                // lo: the first element that is the lane's own, 8: none
    __device__ inline Span() {}
    __device__ inline Span(int c0, int c)
    {
        const bool ragged = MODE == RAGGED && c0 < c && c0 + 8 > c;
        at = ragged ? c - 8 : c0;
        lo = c0 < c ? c0 - at : 8;
        n = c;
    }
    __device__ inline bool any() const { return lo < 8; }
    __device__ inline bool own(int e) const { return MODE == WHOLE ? lo == 0 : (MODE == RAGGED ? e >= lo : lo == 0 && e < n); }
    // byte offset of the channels of the row that starts `first` elements behind the descriptor's start
    template <int ES> __device__ inline uint32_t offset(uint32_t first) const { return any() ? (first + (uint32_t)at) * ES : OOB_OFFSET; }
};

// rows of `pitch` elements of ES bytes from row `first` of a tensor of n rows of c channels on, as many as a wave goes through at a time
template <int ES> __device__ inline __amdgpu_buffer_rsrc_t rows_from(const void *p, int64_t first, int64_t n, int64_t pitch, int c, int rows)
{
    const int64_t left = n - first < rows ? n - first : rows;     // (> 0)
    const char *at = static_cast<const char *>(p) + first * pitch * ES;
    return make_rsrc(at, p ? (uint32_t)(((left - 1) * pitch + c) * ES) : 0u);
}

template <typename T, int MODE> __device__ inline void row_load(const __amdgpu_buffer_rsrc_t &rs, uint32_t off, const Span<MODE> &s, Eight<T> &r)
{
    if constexpr (MODE != NARROW) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i) {
            const auto v = __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(off + 16u * i), 0, 0);
            r.a[i] = v4u{v[0], v[1], v[2], v[3]};
        }
    } else {
        if constexpr (sizeof(T) == 4) r.a[1] = v4u{0u, 0u, 0u, 0u};
        r.a[0] = v4u{0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 7; ++e) {
            const uint32_t at = e < s.n ? off + (uint32_t)(e * sizeof(T)) : OOB_OFFSET;
            if constexpr (sizeof(T) == 4) r.a[e >> 2][e & 3] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, (int)at, 0, 0);
            else r.a[0][e >> 1] |= (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, (int)at, 0, 0) << (16 * (e & 1));
        }
    }
}
template <typename T, int MODE> __device__ inline void row_store(const __amdgpu_buffer_rsrc_t &rs, uint32_t off, const Span<MODE> &s, const float (&v)[8])
{
    Eight<T> r;
    from_floats(v, r);
    if constexpr (MODE != NARROW) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i) __builtin_amdgcn_raw_buffer_store_b128(r.a[i], rs, (int)(off + 16u * i), 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e) {
            const uint32_t at = e < s.n ? off + (uint32_t)(e * sizeof(T)) : OOB_OFFSET;
            if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(r.a[e >> 2][e & 3], rs, (int)at, 0, 0);
            else __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(r.a[0][e >> 1] >> (16 * (e & 1))), rs, (int)at, 0, 0);
        }
    }
}

// One element at a multiple of the descriptor's elements
template <typename T> __device__ inline uint32_t load_one(const __amdgpu_buffer_rsrc_t &rs, uint32_t at)     // as the bits of an fp32 number
{
    if constexpr (sizeof(T) == 4) return (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, (int)(at * 4u), 0, 0);
    else return (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, (int)(at * 2u), 0, 0) << 16;
}
template <typename T> __device__ inline void store_one(const __amdgpu_buffer_rsrc_t &rs, uint32_t at, float v)
{
    if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), rs, (int)(at * 4u), 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b16(one_of<bf16_t>(v), rs, (int)(at * 2u), 0, 0);
}

// Values of other lanes of a row of sixteen
template <int CTRL> __device__ inline uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
constexpr int DPP_XOR1 = 0xb1, DPP_XOR2 = 0x4e, DPP_XOR3 = 0x1b, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;
constexpr int DPP_SHL = 0x100, DPP_ROR = 0x120;                   // + n: of the lane n further on (zero past the sixteen), n back in a ring

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
// 127.5 steps or more takes the next), not below 2^-126 nor above 2^121, whose next would round such a magnitude to 2^128, an Inf; 255 where a
// value is Inf or NaN.
constexpr uint32_t ACT_TOP_CODE = 248u;
__device__ inline uint32_t act_code(uint32_t amax)
{
    if (amax >= 0x7f800000u) return 255u;
    const int e = (int)((amax + 0x10000u) >> 23) - 6;
    return e < 1 ? 1u : (e < (int)ACT_TOP_CODE ? (uint32_t)e : ACT_TOP_CODE);
}
__device__ inline float act_step(uint32_t code) { return __uint_as_float(code << 23); }  // 255: Inf, with q = 0 a NaN

// The lane's eight channels in 8 bits; the block's four lanes are a quad.  The products are exact (a power of two), so adding 1.5 2^23
// rounds once, to nearest even, and leaves q in the low byte.
template <int MODE> __device__ inline uint32_t act_quantise(const float (&v)[8], const Span<MODE> &s, uint32_t (&q)[2])
{
    uint32_t amax = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t b = MODE == WHOLE || s.own(e) ? __float_as_uint(v[e]) & 0x7fffffffu : 0u;
        amax = amax > b ? amax : b;                               // (as integers: a NaN is larger than any number)
    }
    if (MODE == WHOLE && !s.any()) amax = 0u;
    uint32_t o = dpp<DPP_XOR1>(amax);
    amax = amax > o ? amax : o;
    o = dpp<DPP_XOR2>(amax);
    amax = amax > o ? amax : o;
    const uint32_t code = act_code(amax);
    const float scale = __uint_as_float((254u - (code < 254u ? code : 253u)) << 23);
    uint32_t b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = __float_as_uint(__builtin_fmaf(v[e], scale, 12582912.0f));
    if (code == ACT_TOP_CODE) {                                   // (127.5 steps and more, which have no next power of two, stay at 127)
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = __float_as_uint(__builtin_amdgcn_fmed3f(__uint_as_float(b[e]), 12582785.0f, 12583039.0f));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lo = __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x04000c0cu);
        q[i] = code == 255u ? 0u : lo | hi;
    }
    return code;
}

// Rows in 8 bits of a wave: descriptors of q and of the codes, and where a lane's channels c0 .. lie.
struct ActRows { __amdgpu_buffer_rsrc_t q, codes; };
__device__ inline ActRows act_rows(const int8_t *q, const uint8_t *codes, int64_t first, int64_t n, int c, int rows)
{
    const int words = act_code_bytes(c);
    return ActRows{rows_from<1>(q, first, n, c, c, rows), rows_from<1>(codes, first, n, words, words, rows)};
}

// All lanes of the row call it.  The codes of 128 channels are one word, which the first of their lanes writes.
template <int LPR, int MODE>
__device__ inline void act_store(const float (&v)[8], const ActRows &to, uint32_t row, const Span<MODE> &s, int c0, int c)
{
    uint32_t q[2];
    uint32_t code = act_quantise(v, s, q);
    const uint32_t at = s.template offset<1>(row * (uint32_t)c);
    if constexpr (MODE == WHOLE) {
        __builtin_amdgcn_raw_buffer_store_b64(v2u32{q[0], q[1]}, to.q, (int)at, 0, 0);
    } else if (MODE == RAGGED && (s.lo == 0 || s.lo == 8 || c0 % ACT_BLOCK != 0)) {
        __builtin_amdgcn_raw_buffer_store_b64(v2u32{q[0], q[1]}, to.q, (int)at, 0, 0);
    } else {                                                      // (the lane before's channels are of another block)
#pragma unroll
        for (int e = 0; e < 8; ++e) __builtin_amdgcn_raw_buffer_store_b8((uint8_t)(q[e >> 2] >> (8 * (e & 3))), to.q, (int)(s.own(e) ? at + (uint32_t)e : OOB_OFFSET), 0, 0);
    }
    code = c0 / ACT_BLOCK * ACT_BLOCK < c ? code : 0u;            // (the block's first channel)
    uint32_t word = code;
    if constexpr (LPR >= 8) word |= dpp<DPP_SHL + 4>(code) << 8;
    if constexpr (LPR >= 16) word |= dpp<DPP_SHL + 8>(code) << 16 | dpp<DPP_SHL + 12>(code) << 24;
    const bool first = c0 % (4 * ACT_BLOCK) == 0 && c0 < c;
    __builtin_amdgcn_raw_buffer_store_b32(word, to.codes, (int)(first ? row * (uint32_t)act_code_bytes(c) + (uint32_t)(c0 / ACT_BLOCK) : OOB_OFFSET), 0, 0);
}
// What a lane reads of a row in 8 bits, and its values.
struct Eight8 { uint32_t q[2], code, before; };                   // before: code of the channels that are the lane before's
template <int MODE> __device__ inline void act_load(const ActRows &from, uint32_t row, const Span<MODE> &s, int c0, int c, Eight8 &r)
{
    const uint32_t at = s.template offset<1>(row * (uint32_t)c), codes = row * (uint32_t)act_code_bytes(c);
    r.code = (uint32_t)(uint8_t)__builtin_amdgcn_raw_buffer_load_b8(from.codes, (int)(s.any() ? codes + (uint32_t)(c0 / ACT_BLOCK) : OOB_OFFSET), 0, 0);
    if constexpr (MODE == RAGGED)
        r.before = (uint32_t)(uint8_t)__builtin_amdgcn_raw_buffer_load_b8(from.codes, (int)(s.any() ? codes + (uint32_t)(s.at / ACT_BLOCK) : OOB_OFFSET), 0, 0);
    if constexpr (MODE != NARROW) {
        const auto b = __builtin_amdgcn_raw_buffer_load_b64(from.q, (int)at, 0, 0);
        r.q[0] = b[0];
        r.q[1] = b[1];
    } else {
        r.q[0] = r.q[1] = 0u;
#pragma unroll
        for (int e = 0; e < 7; ++e)
            r.q[e >> 2] |= (uint32_t)(uint8_t)__builtin_amdgcn_raw_buffer_load_b8(from.q, (int)(e < c ? at + (uint32_t)e : OOB_OFFSET), 0, 0) << (8 * (e & 3));
    }
}
template <int MODE> __device__ inline void act_floats(const Eight8 &r, const Span<MODE> &s, float (&v)[8])
{
    const float step = act_step(r.code), before = MODE == RAGGED ? act_step(r.before) : step;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)(int8_t)(r.q[e >> 2] >> (8 * (e & 3))) * (MODE != RAGGED || e >= s.lo ? step : before);
}

// ---- dispatch -----------------------------------------------------------------------------------------------------------------
template <int N> struct Int { static constexpr int value = N; };
// f(lanes of a row, groups of eight channels in each, mode)
template <typename F> void with_rows(int c, F f)
{
    auto mode = [&](auto lanes, auto groups) { c % 8 == 0 ? f(lanes, groups, Int<WHOLE>{}) : f(lanes, groups, Int<RAGGED>{}); };
    if (c < 8) return f(Int<4>{}, Int<1>{}, Int<NARROW>{});
    if (c > 512) return mode(Int<64>{}, Int<2>{});
    switch (row_lanes(c)) {
    case 4: return mode(Int<4>{}, Int<1>{});
    case 8: return mode(Int<8>{}, Int<1>{});
    case 16: return mode(Int<16>{}, Int<1>{});
    case 32: return mode(Int<32>{}, Int<1>{});
    default: return mode(Int<64>{}, Int<1>{});
    }
}

}  // namespace pcpp
