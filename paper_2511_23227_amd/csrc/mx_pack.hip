// Rows to microscaled 4-bit floating point and back.
//
// Rows: a thread takes eight neighbouring channels, a quad of threads the 32 that share a power of two.  Columns (32 rows of a channel share it; the result is
// the transposed matrix, for products that sum over the rows): a wave takes 32 rows of 64 channels, a lane four rows of eight channels, so that the maximum goes
// over eight lanes; a block's 128 rows go through LDS and leave in pieces of 64 bytes of a channel.  Both forms come of one pass where both are wanted.
// Scaling by a power of two is exact, so the codes are the same in any implementation.
//
// To nearest memory bounds it: rows of 199 993 x 128 bf16 in 12.7 us (5.1 TB/s), columns of 200 000 x 128 in 17.5 (3.7), back to bf16
// 11.1 (5.9; with the values formed by hand, where the conversions take a third of the instructions, 17).  At
// random vector instructions do: 580 a wave for 2048 elements of columns (100 000 x 91 fp32 14.8 us, 2.8 TB/s), 750 for rows and columns (200 000 x
// 256 bf16 47 us, 3.3 TB/s), 20 wide multiplications of the generator for eight elements and a conversion for each element and form among them.
#include "mx.h"

namespace pcpp {

namespace {

constexpr int THREADS = 256;
constexpr int TILE_ROWS = 128, TILE_CHANNELS = 64;

// Rows `first` .. of the tensor; `threads` is a multiple of four, `per_row` of a row
template <typename T, bool RANDOM>
__global__ __launch_bounds__(THREADS) void pack_rows_kernel(const MxPackArgs a, int64_t first, uint32_t threads, const Divisor per_row)
{
    const uint32_t id = blockIdx.x * (uint32_t)THREADS + threadIdx.x;
    if (id >= threads) return;                                    // (quads stay whole)
    const uint32_t r = per_row.quotient(id), j = id - r * per_row.by;
    const int64_t row = first + r, c0 = 8 * (int64_t)j;
    Eight<T> v;
    load_channels(static_cast<const T *>(a.x) + row * a.ld_x, c0, a.c, v);
    uint32_t u[4] = {0u, 0u, 0u, 0u};
    if constexpr (RANDOM) Philox(a.random).draw((uint32_t)row * (uint32_t)ceil_div(a.c, 8) + j, u);
    const uint32_t code = mx_code(quad_largest(largest(v)), RANDOM);
    reinterpret_cast<uint32_t *>(a.q + row * mx_row_bytes(a.c))[j] = mx_quantise<RANDOM>(v, code, u);
    if (j % 4 == 0) {
        uint8_t *to = a.scales + row * mx_scale_bytes(a.c);
        to[j / 4] = (uint8_t)code;
        if (j / 4 + 1 == mx_blocks(a.c))
            for (int64_t i = j / 4 + 1; i < mx_scale_bytes(a.c); ++i) to[i] = 0;
    }
}

// over the lanes that hold other rows of the same channels: lanes 8, 16 and 32 apart
template <typename Op> __device__ inline uint32_t over_rows(uint32_t m, Op op)
{
    m = op(m, dpp<DPP_ROR + 8>(m));
    const auto a = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    m = op(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    return op(b[0], b[1]);
}
// The largest magnitudes of the lane's eight channels over its four rows and the wave's, and the four rows' pairs (0, 1), (2, 3) of a channel
template <typename T> struct Columns;
template <> struct Columns<float> {
    uint32_t most[8];
    __device__ inline explicit Columns(const Eight<float> (&v)[4])
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint32_t m = 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) m = larger(m, v[i].a[e >> 2][e & 3] & 0x7fffffffu);
            most[e] = over_rows(m, larger);
        }
    }
    __device__ inline uint32_t largest_of(int e) const { return most[e]; }
    __device__ static inline Pair<float> pair(const Eight<float> &a, const Eight<float> &b, int e)
    {
        return Pair<float>{__uint_as_float(a.a[e >> 2][e & 3]), __uint_as_float(b.a[e >> 2][e & 3])};
    }
};
template <> struct Columns<bf16_t> {
    uint32_t most[4];
    __device__ inline explicit Columns(const Eight<bf16_t> (&v)[4])
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t m = v[0].a[0][k] & 0x7fff7fffu;
#pragma unroll
            for (int i = 1; i < 4; ++i) m = larger_pair(m, v[i].a[0][k] & 0x7fff7fffu);
            most[k] = over_rows(m, larger_pair);
        }
    }
    __device__ inline uint32_t largest_of(int e) const { return (e & 1) ? most[e >> 1] & 0xffff0000u : most[e >> 1] << 16; }
    __device__ static inline Pair<bf16_t> pair(const Eight<bf16_t> &a, const Eight<bf16_t> &b, int e)
    {
        return Pair<bf16_t>{__builtin_amdgcn_perm(b.a[0][e >> 1], a.a[0][e >> 1], (e & 1) ? 0x07060302u : 0x05040100u)};
    }
};

// the 32 rows of a wave from row `first` on; nothing where they lie behind the last
template <int ES> __device__ inline __amdgpu_buffer_rsrc_t tile_rows(const void *p, int64_t first, int64_t n, int64_t pitch, int64_t c)
{
    const int64_t left = n - first < 32 ? n - first : 32;
    return make_rsrc(static_cast<const char *>(p) + first * pitch * ES, left > 0 ? (uint32_t)(((left - 1) * pitch + c) * ES) : 0u);
}

template <typename T, bool RANDOM, bool ROWS> __global__ __launch_bounds__(THREADS) void pack_columns_kernel(const MxPackArgs a, const Divisor row_tiles)
{
    __shared__ __attribute__((aligned(16))) uint8_t tile[TILE_CHANNELS][80];    // 64 bytes a channel, and a pitch that spreads the banks
    __shared__ __attribute__((aligned(8))) uint8_t codes[4][TILE_CHANNELS];    // of the waves' rows
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), rl = lane / 8, cl = lane % 8;
    const uint32_t tile_y = row_tiles.quotient(blockIdx.x), tile_x = blockIdx.x - tile_y * row_tiles.by;
    const int64_t first = (int64_t)tile_x * TILE_ROWS + 32 * wave, c0 = (int64_t)tile_y * TILE_CHANNELS + 8 * cl;      // the wave's first row, the lane's first channel
    const uint32_t row = 4u * (uint32_t)rl;
    Eight<T> v[4];
    if (a.c >= 8) {
        const __amdgpu_buffer_rsrc_t xs = tile_rows<sizeof(T)>(a.x, first, a.n, a.ld_x, a.c);
        const int64_t at = c0 + 8 <= a.c ? c0 : a.c - 8;          // (where the row ends inside the eight, its last eight, moved into place)
        const uint32_t pitch = (uint32_t)a.ld_x, off = c0 < a.c ? row * pitch + (uint32_t)at : 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < (int)(sizeof(T) / 2); ++k) {
                const auto r = __builtin_amdgcn_raw_buffer_load_b128(xs, (int)(c0 < a.c ? (off + (uint32_t)i * pitch) * (uint32_t)sizeof(T) + 16u * k : OOB_OFFSET), 0, 0);
                v[i].a[k] = v4u{r[0], r[1], r[2], r[3]};
            }
        if (a.c % 8 != 0 && c0 + 8 > a.c && c0 < a.c) {
#pragma unroll
            for (int i = 0; i < 4; ++i) move_down(v[i], (int)(c0 - at));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = first + row + i;
            load_channels(static_cast<const T *>(a.x) + (r < a.n ? r : a.n - 1) * a.ld_x, c0, r < a.n ? a.c : 0, v[i]);
        }
    }
    uint32_t u[4][4];
    if constexpr (RANDOM) {
        const Philox philox(a.random);
        const uint32_t per_row = (uint32_t)ceil_div(a.c, 8), from = ((uint32_t)first + row) * per_row + (uint32_t)(c0 / 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) philox.draw(from + (uint32_t)i * per_row, u[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) u[i][k] = 0u;
    }
    if constexpr (ROWS) {
        const uint32_t q_pitch = (uint32_t)mx_row_bytes(a.c), s_pitch = (uint32_t)mx_scale_bytes(a.c), blocks = (uint32_t)mx_blocks(a.c), block = (uint32_t)(c0 / MX_BLOCK);
        const __amdgpu_buffer_rsrc_t qs = tile_rows<1>(a.q, first, a.n, q_pitch, q_pitch), ss = tile_rows<1>(a.scales, first, a.n, s_pitch, s_pitch);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t code = mx_code(quad_largest(largest(v[i])), RANDOM), bits = mx_quantise<RANDOM>(v[i], code, u[i]), r = row + (uint32_t)i;
            __builtin_amdgcn_raw_buffer_store_b32(bits, qs, (int)(block < blocks ? r * q_pitch + (uint32_t)(c0 / 2) : OOB_OFFSET), 0, 0);
            __builtin_amdgcn_raw_buffer_store_b8((uint8_t)code, ss, (int)(block < blocks && cl % 4 == 0 ? r * s_pitch + block : OOB_OFFSET), 0, 0);
            if (blocks % 4u != 0u && block + 1u == blocks && cl % 4 == 0)                       // (the rest of the row's whole words)
                for (uint32_t k = block + 1u; k < s_pitch; ++k) __builtin_amdgcn_raw_buffer_store_b8((uint8_t)0, ss, (int)(r * s_pitch + k), 0, 0);
        }
    }
    // channel by channel: the largest of the wave's 32 rows, four codes of the lane's rows
    const Columns<T> columns(v);
    uint32_t scales[2] = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t code = mx_code(columns.largest_of(e), RANDOM);
        const float step = mx_step(code);
        const Pair<T> first = Columns<T>::pair(v[0], v[1], e), second = Columns<T>::pair(v[2], v[3], e);
        uint32_t bits = 0u;
        if constexpr (RANDOM) {
            bits = __builtin_amdgcn_perm(second.random(first_seed(u[2], e), second_seed(u[3], e), step), first.random(first_seed(u[0], e), second_seed(u[1], e), step), 0x0c0c0400u);
        } else {
            bits = first.template nearest<0>(bits, step);
            bits = second.template nearest<1>(bits, step);
        }
        if (code == MX_NAN_CODE) bits = 0u;
        *reinterpret_cast<uint16_t *>(&tile[8 * cl + e][16 * wave + 2 * rl]) = (uint16_t)bits;
        scales[e / 4] |= code << 8 * (e % 4);
    }
    if (rl == 0) *reinterpret_cast<v2u32 *>(&codes[wave][8 * cl]) = first < a.n ? v2u32{scales[0], scales[1]} : v2u32{0u, 0u};
    __syncthreads();
    const int ch = threadIdx.x / 4, part = threadIdx.x % 4;
    const int64_t channel = (int64_t)tile_y * TILE_CHANNELS + ch, block = 4 * (int64_t)tile_x + part;
    if (channel >= a.c) return;
    if (block < mx_blocks(a.n)) *reinterpret_cast<v4u *>(a.qt + channel * mx_row_bytes(a.n) + 16 * block) = *reinterpret_cast<const v4u *>(&tile[ch][16 * part]);
    if (part == 0) reinterpret_cast<uint32_t *>(a.scales_t + channel * mx_scale_bytes(a.n))[tile_x] = codes[0][ch] | (uint32_t)codes[1][ch] << 8 | (uint32_t)codes[2][ch] << 16 | (uint32_t)codes[3][ch] << 24;
}

// The values of eight codes, which the conversions multiply by the power of two, to a row's channels c0 .. up to the last
__device__ inline void store_values(float *row, int64_t c0, int64_t c, uint32_t bits, uint32_t code)
{
    const float step = mx_step(code);
    const v2f p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(bits, step, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(bits, step, 1),
                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(bits, step, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(bits, step, 3)};
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = code == MX_NAN_CODE ? __builtin_nanf("") : p[e >> 1][e & 1];
    if (c0 + 8 <= c) return store_eight<false>(row + c0, v);
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (c0 + e < c) row[c0 + e] = v[e];
}
__device__ inline void store_values(bf16_t *row, int64_t c0, int64_t c, uint32_t bits, uint32_t code)
{
    const float step = mx_step(code);
    v4u w = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(bits, step, 0)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(bits, step, 1)),
             __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(bits, step, 2)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(bits, step, 3))};
    if (code == MX_NAN_CODE) w = v4u{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
    if (c0 + 8 <= c) {
        *reinterpret_cast<v4u_anywhere *>(row + c0) = w;
        return;
    }
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (c0 + e < c) row[c0 + e] = (bf16_t)(w[e >> 1] >> 16 * (e & 1));
}

template <typename T>
__global__ __launch_bounds__(THREADS) void unpack_kernel(const uint8_t *__restrict__ q, const uint8_t *__restrict__ scales, int64_t first, uint32_t threads, int64_t c,
                                                         T *__restrict__ x, const Divisor per_row)
{
    const uint32_t id = blockIdx.x * (uint32_t)THREADS + threadIdx.x;
    if (id >= threads) return;
    const uint32_t r = per_row.quotient(id), j = id - r * per_row.by;
    const int64_t row = first + r;
    const uint32_t bits = reinterpret_cast<const uint32_t *>(q + row * mx_row_bytes(c))[j], code = scales[row * mx_scale_bytes(c) + j / 4];
    store_values(x + row * c, 8 * (int64_t)j, c, bits, code);
}

template <typename F> void with_type(int dtype, F f)
{
    if (dtype == PCPP_F32) f(float{});
    else f(bf16_t{});
}
// f(first row, rows) for pieces of whole rows of less than 2^31 threads
template <typename F> void in_pieces(int64_t n, int64_t per_row, F f)
{
    const int64_t most = ((int64_t)1 << 30) / per_row;            // (at least 256)
    for (int64_t first = 0; first < n; first += most) f(first, n - first < most ? n - first : most);
}

}  // namespace

int mx_pack(const MxPackArgs &a, int dtype, hipStream_t stream)
{
    if (!a.qt) {
        const int64_t per_row = 4 * mx_blocks(a.c);
        in_pieces(a.n, per_row, [&](int64_t first, int64_t rows) {
            const uint32_t threads = (uint32_t)(rows * per_row);
            with_type(dtype, [&](auto t) {
                const unsigned blocks = (unsigned)ceil_div(threads, THREADS);
                if (a.random.state) pack_rows_kernel<decltype(t), true><<<blocks, THREADS, 0, stream>>>(a, first, threads, make_divisor((uint32_t)per_row));
                else pack_rows_kernel<decltype(t), false><<<blocks, THREADS, 0, stream>>>(a, first, threads, make_divisor((uint32_t)per_row));
            });
        });
        PCPP_HIP_CHECK(hipGetLastError());
        return PCPP_OK;
    }
    const Divisor row_tiles = make_divisor((uint32_t)ceil_div(a.n, TILE_ROWS));
    const unsigned grid = (unsigned)(row_tiles.by * ceil_div(a.c, TILE_CHANNELS));
    with_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        if (a.random.state) {
            if (a.q) pack_columns_kernel<T, true, true><<<grid, THREADS, 0, stream>>>(a, row_tiles);
            else pack_columns_kernel<T, true, false><<<grid, THREADS, 0, stream>>>(a, row_tiles);
        } else {
            if (a.q) pack_columns_kernel<T, false, true><<<grid, THREADS, 0, stream>>>(a, row_tiles);
            else pack_columns_kernel<T, false, false><<<grid, THREADS, 0, stream>>>(a, row_tiles);
        }
    });
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

int mx_unpack(const uint8_t *q, const uint8_t *scales, int64_t n, int64_t c, void *x, int dtype, hipStream_t stream)
{
    const int64_t per_row = 4 * mx_blocks(c);
    in_pieces(n, per_row, [&](int64_t first, int64_t rows) {
        const uint32_t threads = (uint32_t)(rows * per_row);
        with_type(dtype, [&](auto t) {
            unpack_kernel<<<(unsigned)ceil_div(threads, THREADS), THREADS, 0, stream>>>(q, scales, first, threads, c, static_cast<decltype(t) *>(x),
                                                                                        make_divisor((uint32_t)per_row));
        });
    });
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

}  // namespace pcpp
