// Products of rows in microscaled 4-bit floating point: out[i, j] = act(sum_l a[i, l] b[j, l] + bias[j]).
//
// The scaled matrix instruction takes 16 x 128 elements of either side, a lane 32 of one row, which is a block, with the block's power of
// two; products and sums are fp32.  b's rows go to the instruction's rows, so that a lane ends with four neighbouring columns of one row of out.
// Where there are few tiles and many elements to sum, the sum is cut into parts, which are joined in order by a second kernel.
//
// 8192 x 8192 x 8192 takes 290 to 335 us by the numbers and the card, 3.8 to 3.3 PFLOP/s (the matrix instructions alone reach 8.5 on constant numbers and 6 to 7 on random ones, with their
// operands from LDS but no requests 4.3 to 4.8). 115 200 x 64 -> 256 with gelu takes 28 us with the rounding of x (bytes 15): the vector instructions
// of 29 million activations.  256 x 128 x 200 000 takes 21 (bytes 8), a block for each CU and a join of 4.7.
#include "mx.h"

namespace pcpp {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v4f_anywhere __attribute__((ext_vector_type(4), aligned(4)));
typedef v2u32 v2u32_anywhere __attribute__((aligned(2)));

// which bytes of the scales
template <int B_BYTE, int A_BYTE = B_BYTE> __device__ inline v4f multiply(const v4u &b, const v4u &a, v4f sum, uint32_t b_scale, uint32_t a_scale)
{
    const v8i x = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0}, y = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, sum, 4, 4, B_BYTE, (int)b_scale, A_BYTE, (int)a_scale);
}

// N neighbouring columns of a row of out, of which `left` are there
template <int N, typename T> __device__ inline void store_columns(T *to, const float (&v)[N], int64_t left)
{
    if (left >= N) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < N; i += 4) reinterpret_cast<v4u_anywhere *>(to)[i / 4] = v4u{__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3])};
        } else if constexpr (N == 8) {
            *reinterpret_cast<v4u_anywhere *>(to) = v4u{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]), cvt_pk_bf16(v[6], v[7])};
        } else {
            *reinterpret_cast<v2u32_anywhere *>(to) = v2u32{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])};
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
        if (i < left) to[i] = one_of<T>(v[i]);
}
template <int N> __device__ inline void load_bias(const float *bias, int64_t j, int64_t m, float (&v)[N])
{
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = bias && j + e < m ? bias[j + e] : 0.f;
}

// ---- tiles through LDS --------------------------------------------------------------------------------------------------------------
// A block of WA x WB waves takes 16 WA FA rows of a and 16 WB FB of b, a wave 16 FA and 16 FB of them.  A stage is 256 elements: 128 bytes of every
// row's codes, a whole cache line, moved straight into LDS, and with every second one the sixteen scales of two (a request of eight takes the caches
// as long as one of a line: 153 us for 130).  (Stages of 128 elements, three of them ahead: 8192 x 8192 x 8192 in 401 us where these took 337, before
// the order below.)
//
// What a wave does meanwhile is laid out by hand.  A stage is two instructions deep.  While the first one's products run the operands of the second
// are read; then all waves meet, the stage's place in LDS is free, and the stage after the next is requested, two requests at a time between the
// products (a compute unit takes as long for the requests as for the products).  Half way through the second one's products the next stage, requested
// one and a half stages ago, is waited for, and the operands of its first are read.
//
// A row's eight 16-byte pieces (blocks) lie in LDS at piece ^ s, s a function of the row.  The sixteen lanes whose reads share a cycle are 0-3, 12-15
// and 20-27 (or 4-11, 16-19 and 28-31; the same again 32 further on), so of an instruction's rows r 0-3 and 12-15 with one piece and 4-11 with the
// piece two on: with bit 2 of s set for rows 4-11 and its other bits from bits 3 and 1 of r they meet all banks (s = r / 2 mod 8, made for
// neighbouring lanes, doubled the cycles of every read).  b's rows go to two instructions in turn, four by four, so that a lane ends with eight
// neighbouring columns of a row of out. Lane (r, l) of an instruction has row r; over the stage's two instructions it takes the blocks 2 l and 2 l +
// 1, whose scales are one 16-bit read (the order in which blocks are summed is free).
constexpr int STAGE = 256, STAGE_BYTES = 128, STAGE_BLOCKS = 8, SCALE_BYTES = 16;         // (a row's scales of two stages)

// rows of a tensor as a descriptor in scalar registers, for inline assembly
__device__ inline v4u scalar_rows(const uint8_t *p, int64_t first, int64_t n, int64_t pitch, int rows)
{
    const int64_t left = n - first < rows ? n - first : rows;
    const uint64_t at = reinterpret_cast<uint64_t>(p) + (uint64_t)(first * pitch);
    const uint32_t bytes = (uint32_t)(left * pitch);
    return v4u{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32)),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
}
// 16 bytes a lane from its offset behind the descriptor's start to LDS byte address `lds` + 16 lane; zeros past the descriptor.  (The address travels in
// M0, which the compiler reserves and nothing else here uses.)
__device__ inline void rows_to_lds_b128(const v4u &rows, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset), "s"(rows), "s"(lds) : "memory");
}

template <int WA, int WB, int FA, int FB> struct Tile {
    static constexpr int A = 16 * WA * FA, B = 16 * WB * FB, WAVES = WA * WB, ROWS = A + B;
    static constexpr int CODES = ROWS * STAGE_BYTES, SCALES = ROWS * SCALE_BYTES, BYTES = CODES + SCALES;
    static constexpr int LOADS = ROWS / 8 / WAVES, SCALE_LOADS = ROWS / 64 / WAVES;          // of a wave for a stage's codes, for two stages' scales
    static_assert(A % 64 == 0 && ROWS % (64 * WAVES) == 0 && A % (8 * WAVES) == 0 && WAVES % 4 == 0 && LOADS == 2 * FB && FA % 2 == 0 && FB % 2 == 0, "whole loads");
};

// Which tile a block takes: the blocks of a chiplet (every eighth) take neighbouring tiles, bands of eight rows of tiles column by column, so that its cache
// serves the rows they share.
__device__ inline void tile_of(uint32_t id, uint32_t rows, uint32_t columns, uint32_t &y, uint32_t &x)
{
    const uint32_t total = rows * columns, each = total / 8u, more = total % 8u, chiplet = id % 8u, nth = id / 8u;
    const uint32_t t = chiplet * each + (chiplet < more ? chiplet : more) + nth;
    const uint32_t band = t / (8u * columns), in = t - band * 8u * columns, left = rows - 8u * band, high = left < 8u ? left : 8u;
    x = in / high;
    y = 8u * band + in - x * high;
}

// A wave of the 256 x 256 tile has a SIMD and its 512 registers to itself.  With fp32 results two registers go to scratch behind the loop, where they
// are stored; none of the waits that count requests has scratch accesses beside it (8192 x 8192 x 8192 to fp32 315 us, to bf16 325).
// PARTS: blockIdx.y's part of the sum.  ONE: the sum has one stage.  X: a's rows come as they are, in that type (uint8_t: in 4 bits), and the block rounds its own.
template <typename T, typename X, bool PARTS, bool ONE, int WA, int WB, int FA, int FB>
__global__ __launch_bounds__(64 * WA * WB, ONE ? 4 : (FA == 8 ? 1 : 2)) void tile_kernel(const MxProductArgs p, const X *__restrict__ rows, int64_t ld_rows, uint32_t tile_rows,
                                                                                         uint32_t tile_columns, int64_t stages, int64_t of_part, const Divisor per_row)
{
    constexpr bool ROUND = sizeof(X) > 1;
    static_assert(!ROUND || ONE, "rounded rows are short");
    typedef Tile<WA, WB, FA, FB> S;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), r = lane & 15, l = lane >> 4;
    uint32_t ty, tx;
    tile_of(blockIdx.x, tile_rows, tile_columns, ty, tx);
    const int64_t i0 = (int64_t)ty * S::A, j0 = (int64_t)tx * S::B;
    const uint32_t pitch = (uint32_t)mx_row_bytes(p.k), scale_pitch = (uint32_t)mx_scale_bytes(p.k), blocks = (uint32_t)mx_blocks(p.k);
    const int64_t from = PARTS ? blockIdx.y * of_part : 0, to = PARTS && from + of_part < stages ? from + of_part : stages;
    const v4u aq = scalar_rows(p.a, i0, p.n, pitch, S::A), as = scalar_rows(p.a_scales, i0, p.n, scale_pitch, S::A);
    const v4u bq = scalar_rows(p.b, j0, p.m, pitch, S::B), bs = scalar_rows(p.b_scales, j0, p.m, scale_pitch, S::B);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    // what the lane moves: a piece of rows 8 (wave + i WAVES) + lane / 8, the scales of row 64 wave + lane
    auto spread = [](uint32_t bit3, uint32_t bit2, uint32_t bit1) { return ((bit2 ^ bit3) & 1u) << 2 | (bit3 & 1u) << 1 | (bit1 & 1u); };
    const uint32_t wv = (uint32_t)wave, ln = (uint32_t)lane;
    const uint32_t a_piece = (ln & 7u) ^ spread(wv, ln >> 5, ln >> 4), b_piece = (ln & 7u) ^ spread(wv >> 1, wv, ln >> 4);
    const uint32_t a_code_at = (8u * wv + (ln >> 3)) * pitch + 16u * a_piece, b_code_at = (8u * wv + (ln >> 3)) * pitch + 16u * b_piece;
    const uint32_t scale_at = (64u * wv + ln) * scale_pitch;
    const uint32_t some_blocks = (uint64_t)blocks < 8u * (uint64_t)to ? blocks : 8u * (uint32_t)to;
    // the i-th of a wave's requests for a stage (past the part's last one: of nothing)
    auto request = [&](uint32_t stage, uint32_t to_lds, int i) {
        const bool of_a = 8 * i * S::WAVES < S::A;
        const uint32_t row = 8u * (uint32_t)i * S::WAVES - (of_a ? 0u : (uint32_t)S::A), at = row * pitch + STAGE_BYTES * stage;
        rows_to_lds_b128(of_a ? aq : bq, STAGE_BLOCKS * stage + (of_a ? a_piece : b_piece) < some_blocks ? at + (of_a ? a_code_at : b_code_at) : OOB_OFFSET,
                         to_lds + (uint32_t)(8 * (wave + i * S::WAVES)) * STAGE_BYTES);
    };
    // of two stages from an even one of the part on (behind a row's last scales the next row's, which count for nothing)
    auto request_scales = [&](uint32_t stage, uint32_t to_lds) {
#pragma unroll
        for (int i = 0; i < S::SCALE_LOADS; ++i) {
            const bool of_a = S::SCALE_LOADS > 1 ? 64 * i * S::WAVES < S::A : wave < S::A / 64;
            if (ROUND && of_a) continue;
            const uint32_t row = 64u * (uint32_t)i * S::WAVES - (of_a ? 0u : (uint32_t)S::A);
            rows_to_lds_b128(of_a ? as : bs, STAGE_BLOCKS * stage < some_blocks ? scale_at + row * scale_pitch + STAGE_BLOCKS * stage : OOB_OFFSET,
                             to_lds + 1024u * (wv + (uint32_t)i * S::WAVES));
        }
    };
    const int wa = wave / WB, wb = wave % WB;
    const int b_row = 8 * (r >> 2) + (r & 3);                     // of the even one of two instructions; the odd one's are four further on, with the same s
    const uint32_t own_s = spread((uint32_t)r >> 3, (uint32_t)r >> 2, (uint32_t)r >> 1), in_row = 16u * ((2u * (uint32_t)l) ^ own_s);
    const uint32_t read_a = (uint32_t)r * STAGE_BYTES + in_row, read_b = (uint32_t)b_row * STAGE_BYTES + in_row;
    v4f sum[FA][FB];
#pragma unroll
    for (int y = 0; y < FA; ++y)
#pragma unroll
        for (int x = 0; x < FB; ++x) sum[y][x] = v4f{0.f, 0.f, 0.f, 0.f};
    v4u va[2][FA], vb[2][FB];
    uint32_t sa[FA / 2], sb[FB / 2];                              // two rows' scales of a stage in a word
    auto read_a_rows = [&](const uint8_t *codes, int t) {
#pragma unroll
        for (int y = 0; y < FA; ++y) va[t][y] = *reinterpret_cast<const v4u *>(codes + (read_a ^ (16u * t)) + 16 * (wa * FA + y) * STAGE_BYTES);
    };
    auto read_b_row = [&](const uint8_t *codes, int t, int x) {
        vb[t][x] = *reinterpret_cast<const v4u *>(codes + S::A * STAGE_BYTES + (read_b ^ (16u * t)) + (16 * (wb * FB + (x & ~1)) + 4 * (x & 1)) * STAGE_BYTES);
    };
    auto read_scales = [&](const uint8_t *from_lds, uint32_t stage) {
        const uint8_t *scales = from_lds + 2 * l;
        auto half = [&](int row) { return (uint32_t)*reinterpret_cast<const uint16_t *>(scales + row * SCALE_BYTES); };
        const uint32_t own = STAGE_BLOCKS * stage + 2u * (uint32_t)l;    // (scales behind a row's last block may be anything)
        const uint32_t mask = ((own < blocks ? 0xffu : 0u) | (own + 1u < blocks ? 0xff00u : 0u)) * 0x10001u;
#pragma unroll
        for (int y = 0; y < FA; y += 2) sa[y / 2] = (half(16 * (wa * FA + y) + r) | half(16 * (wa * FA + y + 1) + r) << 16) & mask;
#pragma unroll
        for (int x = 0; x < FB; x += 2) sb[x / 2] = (half(S::A + 16 * (wb * FB + x) + b_row) | half(S::A + 16 * (wb * FB + x) + 4 + b_row) << 16) & mask;
    };
    auto products = [&](auto t, int x) {
        constexpr int D = decltype(t)::value;
#pragma unroll
        for (int y = 0; y < FA; ++y) {
            const v4u &b = vb[D][x], &a = va[D][y];
            if (x % 2 == 0) sum[y][x] = y % 2 == 0 ? multiply<D, D>(b, a, sum[y][x], sb[x / 2], sa[y / 2]) : multiply<D, 2 + D>(b, a, sum[y][x], sb[x / 2], sa[y / 2]);
            else sum[y][x] = y % 2 == 0 ? multiply<2 + D, D>(b, a, sum[y][x], sb[x / 2], sa[y / 2]) : multiply<2 + D, 2 + D>(b, a, sum[y][x], sb[x / 2], sa[y / 2]);
        }
    };
    // in LDS: the codes of an even and an odd stage of the part, the scales of an even and an odd pair of stages
    constexpr uint32_t SCALES_AT = (ONE ? 1 : 2) * S::CODES;
    const uint32_t first = (uint32_t)from, last = (uint32_t)to;
    request_scales(first, lds0 + SCALES_AT);
#pragma unroll
    for (int j = 0; j < (ONE ? 1 : 2); ++j)
#pragma unroll
        for (int i = ROUND ? S::A / 8 / S::WAVES : 0; i < S::LOADS; ++i) request(first + j, lds0 + j * S::CODES, i);
    if constexpr (ROUND) {
        // (what lies behind a row's last block, and rows behind the last: any codes, with scales that are masked and b's zeros, or not stored)
        const uint32_t total = (p.n - i0 < S::A ? (uint32_t)(p.n - i0) : (uint32_t)S::A) * per_row.by;
        constexpr uint32_t AT_ONCE = 4, STEP = 64 * S::WAVES;
        for (uint32_t id0 = threadIdx.x; id0 < total; id0 += AT_ONCE * STEP) {
            Eight<X> v[AT_ONCE];
            uint32_t row[AT_ONCE], j[AT_ONCE];
#pragma unroll
            for (uint32_t u = 0; u < AT_ONCE; ++u) {              // (past the last as the first, which is left)
                const uint32_t id = id0 + u * STEP < total ? id0 + u * STEP : id0;
                row[u] = per_row.quotient(id), j[u] = id - row[u] * per_row.by;
            }
            const X *x = rows + i0 * ld_rows;
            if (p.k >= 8) {
#pragma unroll
                for (uint32_t u = 0; u < AT_ONCE; ++u) load_within(x + row[u] * ld_rows, 8 * (int64_t)j[u], p.k, v[u]);
#pragma unroll
                for (uint32_t u = 0; u < AT_ONCE; ++u) into_place(8 * (int64_t)j[u], p.k, v[u]);
            } else {
#pragma unroll
                for (uint32_t u = 0; u < AT_ONCE; ++u) load_channels(x + row[u] * ld_rows, 8 * (int64_t)j[u], p.k, v[u]);
            }
#pragma unroll
            for (uint32_t u = 0; u < AT_ONCE; ++u) {
                if (id0 + u * STEP >= total) break;               // (quads stay whole)
                const uint32_t block = j[u] / 4u, none[4] = {0u, 0u, 0u, 0u}, code = mx_code(quad_largest(largest(v[u])), false), q = mx_quantise<false>(v[u], code, none);
                *reinterpret_cast<uint32_t *>(lds + row[u] * STAGE_BYTES + 16u * (block ^ spread(row[u] >> 3, row[u] >> 2, row[u] >> 1)) + 4u * (j[u] % 4u)) = q;
                if (j[u] % 4u == 0u) lds[SCALES_AT + row[u] * SCALE_BYTES + block] = (uint8_t)code;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(ONE ? 0 : S::LOADS) : "memory");
    read_a_rows(lds, 0);
    read_scales(lds + SCALES_AT, first);
#pragma unroll
    for (int x = 0; x < FB; ++x) read_b_row(lds, 0, x);
    uint32_t at = 0u;                                             // of the stage's codes in LDS
    for (uint32_t s = first; ONE ? s == first : s < last; ++s) {
        const uint32_t nth = s - first, next = S::CODES - at;
        auto scales_at = [&](uint32_t nth) { return SCALES_AT + (nth >> 1 & 1u) * S::SCALES; };
        if (!ONE && nth % 2u == 0u) request_scales(s + 2u, lds0 + scales_at(nth + 2u));
        // (no branches from here on: the compiler would move the products behind them)
        read_a_rows(lds + at, 1);
#pragma unroll
        for (int x = 0; x < FB / 2; ++x) {
            read_b_row(lds + at, 1, 2 * x);
            read_b_row(lds + at, 1, 2 * x + 1);
            products(Int<0>{}, x);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (!ONE) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        auto go_on = [&](auto t, int x, int i) {
            if constexpr (!ONE) {
                request(s + 2u, lds0 + at, i);
                request(s + 2u, lds0 + at, i + 1);
                __builtin_amdgcn_sched_barrier(0);
            }
            products(t, x);
            __builtin_amdgcn_sched_barrier(0);
        };
#pragma unroll
        for (int x = 0; x < FB / 2; ++x) go_on(Int<0>{}, FB / 2 + x, 2 * x);
#pragma unroll
        for (int x = 0; x < FB / 2; ++x) go_on(Int<1>{}, x, FB + 2 * x);
        if constexpr (!ONE) {
            asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(S::LOADS) : "memory");
            read_a_rows(lds + next, 0);
        }
#pragma unroll
        for (int x = FB / 2; x < FB; ++x) {
            if constexpr (!ONE) {
                read_b_row(lds + next, 0, 2 * x - FB);
                read_b_row(lds + next, 0, 2 * x - FB + 1);
            }
            products(Int<1>{}, x);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (!ONE) read_scales(lds + scales_at(nth + 1u) + (nth + 1u) % 2u * STAGE_BLOCKS, s + 1u);
        at = next;
    }
    if constexpr (!ONE) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (nothing of this wave is still on its way into LDS)
    as_act(PARTS ? PCPP_ACT_NONE : p.act, [&](auto act) {
#pragma unroll
        for (int x = 0; x < FB; x += 2) {
            const int64_t j = j0 + 16 * (wb * FB + x) + 8 * l;
            float bias[8];
            load_bias<8>(PARTS ? nullptr : p.bias, j, p.m, bias);
#pragma unroll
            for (int y = 0; y < FA; ++y) {
                const int64_t i = i0 + 16 * (wa * FA + y) + r;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = activate<decltype(act)::value>(sum[y][x + e / 4][e % 4] + bias[e]);
                if (i >= p.n || j >= p.m) continue;
                if constexpr (PARTS) store_columns<8>(p.part + ((int64_t)blockIdx.y * p.n + i) * p.m + j, v, p.m - j);
                else store_columns<8>(static_cast<T *>(p.out) + i * p.m + j, v, p.m - j);
            }
        }
    });
}

// Parts of a sum joined: a block takes 256 neighbouring elements of out, a wave every sixteenth part of them, then the waves' sums in order.
template <typename T> __global__ __launch_bounds__(1024) void join_kernel(const MxProductArgs p, int parts, const Divisor columns)
{
    __shared__ v4f sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t total = (uint32_t)(p.n * p.m), at = 256u * blockIdx.x + 4u * (uint32_t)lane;
    v4f v = {0.f, 0.f, 0.f, 0.f};
    if (at + 4u <= total) {
#pragma unroll 8
        for (int s = wave; s < parts; s += 16) v += *reinterpret_cast<const v4f_anywhere *>(p.part + (size_t)s * total + at);
    } else {
        for (int s = wave; s < parts; s += 16)
#pragma unroll
            for (int e = 0; e < 3; ++e) v[e] += at + e < total ? p.part[(size_t)s * total + at + e] : 0.f;
    }
    sums[wave][lane] = v;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) v += sums[w][lane];
    as_act(p.act, [&](auto act) {
        float o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t i = at + e, j = i - columns.quotient(i) * columns.by;
            o[e] = activate<decltype(act)::value>(v[e] + (p.bias ? p.bias[j] : 0.f));
        }
        if (at < total) store_columns<4>(static_cast<T *>(p.out) + at, o, (int64_t)(total - at));
    });
}

// ---- few rows -----------------------------------------------------------------------------------------------------------------------
// Up to sixteen rows of a: what counts is reading b once (1 x 16 384 x 4096: 9.8 us with the rounding of a, 3.6 TB/s; an empty kernel takes 2.3).  A
// block takes sixteen rows of b, its waves every WAVES-th stage of the sum; codes go from memory to the registers of the lanes that multiply them.  a
// comes in 4 bits or, of few elements, as it is: the block rounds it into LDS while its first rows of b are on their way.
constexpr int FEW_ROWS = 16;
constexpr int64_t FEW_ELEMENTS = 16384;                           // of a that every block rounds for itself (9 KB of LDS; 1 x 4096 x 32 768 28 us, rounded first 21)

template <typename T, typename X, int WAVES> __global__ __launch_bounds__(64 * WAVES) void few_kernel(const MxProductArgs p, const X *__restrict__ x, int64_t ld_x)
{
    constexpr bool ROUND = sizeof(X) > 1;
    __shared__ v4f sums[WAVES][64];
    extern __shared__ __attribute__((aligned(16))) uint8_t own[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), r = lane & 15, l = lane >> 4;
    const int64_t j0 = 16 * (int64_t)blockIdx.x;
    const uint32_t pitch = (uint32_t)mx_row_bytes(p.k), scale_pitch = (uint32_t)mx_scale_bytes(p.k), blocks = (uint32_t)mx_blocks(p.k), n = (uint32_t)p.n;
    const uint32_t stages = (uint32_t)ceil_div(p.k, STAGE);
    const __amdgpu_buffer_rsrc_t bq = rows_from<1>(p.b, j0, p.m, pitch, (int)pitch, 16), bs = rows_from<1>(p.b_scales, j0, p.m, scale_pitch, (int)scale_pitch, 16);
    struct Some {
        v4u q[2];
        uint32_t scales;
    };
    // two blocks of the lane's row in stage s; zeros past the last
    auto load = [&](const __amdgpu_buffer_rsrc_t &q, const __amdgpu_buffer_rsrc_t &scales, uint32_t row, uint32_t s, Some &v) {
        const uint32_t block = STAGE_BLOCKS * s + 2u * (uint32_t)l;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const auto c = __builtin_amdgcn_raw_buffer_load_b128(q, (int)(block + t < blocks ? row * pitch + 16u * (block + t) : OOB_OFFSET), 0, 0);
            v.q[t] = v4u{c[0], c[1], c[2], c[3]};
        }
        v.scales = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(scales, (int)(block < blocks ? row * scale_pitch + block : OOB_OFFSET), 0, 0);
        if (block + 1u >= blocks) v.scales &= 0xffu;              // (scales behind a row's last block may be anything)
    };
    constexpr int AHEAD = 4;
    Some b[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) load(bq, bs, (uint32_t)r, (uint32_t)(wave + i * WAVES), b[i]);
    if constexpr (ROUND) {
        const uint32_t per_row = 4u * blocks;
        for (uint32_t id = threadIdx.x; id < n * per_row; id += 64 * WAVES) {
            const uint32_t row = id / per_row, j = id - row * per_row;
            Eight<X> v;
            load_channels(x + row * ld_x, 8 * (int64_t)j, p.k, v);
            const uint32_t none[4] = {0u, 0u, 0u, 0u}, code = mx_code(quad_largest(largest(v)), false);
            reinterpret_cast<uint32_t *>(own + row * pitch)[j] = mx_quantise<false>(v, code, none);
            if (j % 4u == 0u) own[n * pitch + row * scale_pitch + j / 4u] = (uint8_t)code;
        }
        __syncthreads();
    }
    const __amdgpu_buffer_rsrc_t aq = rows_from<1>(p.a, 0, p.n, pitch, (int)pitch, 16), as = rows_from<1>(p.a_scales, 0, p.n, scale_pitch, (int)scale_pitch, 16);
    v4f sum = {0.f, 0.f, 0.f, 0.f};
    for (uint32_t s0 = (uint32_t)wave; s0 < stages; s0 += AHEAD * WAVES) {
        Some a[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const uint32_t s = s0 + i * WAVES;
            if constexpr (ROUND) {
                const uint32_t block = STAGE_BLOCKS * s + 2u * (uint32_t)l, at = (uint32_t)r < n ? (uint32_t)r : 0u;
                const bool here = (uint32_t)r < n && block < blocks, both = here && block + 1u < blocks;
                a[i].q[0] = here ? *reinterpret_cast<const v4u *>(own + at * pitch + 16u * block) : v4u{0u, 0u, 0u, 0u};
                a[i].q[1] = both ? *reinterpret_cast<const v4u *>(own + at * pitch + 16u * (block + 1u)) : v4u{0u, 0u, 0u, 0u};
                a[i].scales = here ? *reinterpret_cast<const uint16_t *>(own + n * pitch + at * scale_pitch + block) & (both ? 0xffffu : 0xffu) : 0u;
            } else {
                load(aq, as, (uint32_t)r, s, a[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            sum = multiply<0>(b[i].q[0], a[i].q[0], sum, b[i].scales, a[i].scales);
            sum = multiply<1>(b[i].q[1], a[i].q[1], sum, b[i].scales, a[i].scales);
            if (s0 + AHEAD * WAVES < stages) load(bq, bs, (uint32_t)r, s0 + (AHEAD + i) * WAVES, b[i]);
        }
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) sum += sums[w][lane];
    const int64_t j = j0 + 4 * l;
    if ((uint32_t)r >= n || j >= p.m) return;
    as_act(p.act, [&](auto act) {
        float bias[4], v[4];
        load_bias<4>(p.bias, j, p.m, bias);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = activate<decltype(act)::value>(sum[e] + bias[e]);
        store_columns<4>(static_cast<T *>(p.out) + (int64_t)r * p.m + j, v, p.m - j);
    });
}

// ... of sums up to 8192 long: the waves of one block walk the whole sum, tiles cut it over the card (16 x 256 x 4096 in 6.2 us, in parts 8.4; 16 x 256 x 16 384
// in 12.5 and 8.6, 16 x 4096 x 50 000 in 31 and 25)
bool few_rows(int64_t n, int64_t k) { return n <= FEW_ROWS && k <= 32 * STAGE; }

// How a product is cut: tiles, and parts of the sum where the tiles do not fill the card.
struct Shape {
    bool few, large;
    int64_t rows, columns, stages, parts, of_part;
};
Shape shape_of(int64_t n, int64_t m, int64_t k)
{
    Shape s{};
    s.stages = ceil_div(k, STAGE);
    s.parts = 1;
    s.few = few_rows(n, k);
    if (s.few) return s;
    s.large = ceil_div(n, 256) * ceil_div(m, 256) >= 192 && s.stages >= 4;
    const int tile = s.large ? 256 : 128;
    s.rows = ceil_div(n, tile);
    s.columns = ceil_div(m, tile);
    const int64_t tiles = s.rows * s.columns;
    if (tiles < 128 && s.stages >= 8) {                           // (a block for each CU: 256 x 128 x 200 000 in 21 us, two 27; three stages a part at least)
        s.parts = 256 / tiles;
        if (s.parts > s.stages / 3) s.parts = s.stages / 3;
    }
    s.of_part = ceil_div(s.stages, s.parts);
    s.parts = ceil_div(s.stages, s.of_part);                      // (none is empty)
    return s;
}

template <typename T, bool PARTS, bool ONE, int WA, int WB, int FA, int FB, typename X = uint8_t>
int launch_tiles(const MxProductArgs &p, const Shape &s, hipStream_t stream, const X *x = nullptr, int64_t ld_x = 0)
{
    typedef Tile<WA, WB, FA, FB> L;
    const auto kernel = tile_kernel<T, X, PARTS, ONE, WA, WB, FA, FB>;
    constexpr size_t bytes = (ONE ? 1 : 2) * (size_t)L::BYTES;
    if (int rc = raise_lds_limit(reinterpret_cast<const void *>(kernel), bytes)) return rc;
    // pieces of whole bands whose blocks a grid holds
    const int64_t most = s.columns > (1 << 22) ? 1 : (1 << 22) / s.columns;
    for (int64_t y = 0; y < s.rows; y += most) {
        MxProductArgs q = p;
        const int64_t i = y * L::A, rows = s.rows - y < most ? s.rows - y : most;
        if (!x) q.a += i * mx_row_bytes(p.k), q.a_scales += i * mx_scale_bytes(p.k);
        q.out = static_cast<T *>(p.out) + i * p.m;
        q.n = p.n - i < rows * L::A ? p.n - i : rows * L::A;
        kernel<<<dim3((unsigned)(rows * s.columns), (unsigned)s.parts), 64 * L::WAVES, bytes, stream>>>(
            q, x ? x + i * ld_x : nullptr, ld_x, (uint32_t)rows, (uint32_t)s.columns, s.stages, s.of_part, make_divisor((uint32_t)(4 * mx_blocks(p.k))));
    }
    return PCPP_OK;
}

// (more waves a block where the blocks are few)
template <typename T, typename X> void launch_few(const MxProductArgs &p, const X *x, int64_t ld_x, hipStream_t stream)
{
    const unsigned blocks = (unsigned)ceil_div(p.m, 16);
    const size_t bytes = sizeof(X) > 1 ? (size_t)(p.n * (mx_row_bytes(p.k) + mx_scale_bytes(p.k))) : 0;
    if (blocks < 256) few_kernel<T, X, 16><<<blocks, 1024, bytes, stream>>>(p, x, ld_x);
    else few_kernel<T, X, 4><<<blocks, 256, bytes, stream>>>(p, x, ld_x);
}

}  // namespace

// Which products take rows as they are, one launch less than rounding first.  Few: 1 x 64 x 16 384 in 9.1 us, 12.1.  Sums of one stage with one or
// two columns of tiles, each of which rounds the rows (115 200 x 64 -> 64 9.9 us, 13.9; 200 000 x 128 -> 256 33, 39, but -> 512 with gelu 87, 82; 100
// x 256 -> 256 7.2, 6.6).
bool few_of_x(int64_t n, int64_t k) { return n <= FEW_ROWS && n * MX_BLOCK * mx_blocks(k) <= FEW_ELEMENTS; }
bool mx_linear_alone(int64_t n, int64_t m, int64_t k) { return few_of_x(n, k) || (k <= STAGE && m <= 256); }
int mx_linear_alone(const MxProductArgs &p, const void *x, int x_dtype, int64_t ld_x, int out_dtype, hipStream_t stream)
{
    auto with = [&](auto t, auto s) -> int {
        typedef decltype(t) T;
        typedef decltype(s) X;
        const X *rows = static_cast<const X *>(x);
        if (!few_of_x(p.n, p.k)) return launch_tiles<T, false, true, 2, 2, 4, 4>(p, shape_of(p.n, p.m, p.k), stream, rows, ld_x);
        launch_few<T>(p, rows, ld_x, stream);
        return PCPP_OK;
    };
    const int rc = x_dtype == PCPP_F32 ? (out_dtype == PCPP_F32 ? with(float{}, float{}) : with(bf16_t{}, float{}))
                                       : (out_dtype == PCPP_F32 ? with(float{}, bf16_t{}) : with(bf16_t{}, bf16_t{}));
    if (rc != PCPP_OK) return rc;
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

size_t mx_product_workspace_bytes(int64_t n, int64_t m, int64_t k)
{
    const Shape s = shape_of(n, m, k);
    return s.parts > 1 ? align_up((size_t)s.parts * (size_t)n * (size_t)m * sizeof(float)) : 0;
}

int mx_product(const MxProductArgs &p, int out_dtype, hipStream_t stream)
{
    const Shape s = shape_of(p.n, p.m, p.k);
    auto with = [&](auto t) -> int {
        typedef decltype(t) T;
        if (s.few) {
            const uint8_t *none = nullptr;
            launch_few<T>(p, none, 0, stream);
            return PCPP_OK;
        }
        if (s.parts > 1) {
            if (int rc = launch_tiles<float, true, false, 2, 2, 4, 4>(p, s, stream)) return rc;
            join_kernel<T><<<(unsigned)ceil_div(p.n * p.m, 256), 1024, 0, stream>>>(p, (int)s.parts, make_divisor((uint32_t)p.m));
            return PCPP_OK;
        }
        if (s.large) return launch_tiles<T, false, false, 2, 2, 8, 8>(p, s, stream);
        return s.stages == 1 ? launch_tiles<T, false, true, 2, 2, 4, 4>(p, s, stream) : launch_tiles<T, false, false, 2, 2, 4, 4>(p, s, stream);
    };
    if (int rc = out_dtype == PCPP_F32 ? with(float{}) : with(bf16_t{})) return rc;
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

}  // namespace pcpp
