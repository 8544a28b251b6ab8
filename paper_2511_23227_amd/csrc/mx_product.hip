// Products of rows in microscaled 4-bit floating point: out[i, j] = act(sum_l a[i, l] b[j, l] + bias[j]).
//
// The scaled matrix instruction takes 16 x 128 elements of either side, a lane 32 of one row, which is a block, with the block's power of
// two; products and sums are fp32.  b's rows go to the instruction's rows, so that a lane ends with four neighbouring columns of one row of out.
// Where there are few tiles and many elements to sum, the sum is cut into parts, which are joined in order by a second kernel.
#include "mx.h"

namespace pcpp {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v4f_anywhere __attribute__((ext_vector_type(4), aligned(4)));
typedef v2u32 v2u32_anywhere __attribute__((aligned(2)));

constexpr int THREADS = 256;

// BYTE: which byte of the scales
template <int BYTE> __device__ inline v4f multiply(const v4u &b, const v4u &a, v4f sum, uint32_t b_scale, uint32_t a_scale)
{
    const v8i x = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0}, y = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, sum, 4, 4, BYTE, (int)b_scale, BYTE, (int)a_scale);
}

// four neighbouring columns of a row of out, of which `left` are there
template <typename T> __device__ inline void store_four(T *to, const float (&v)[4], int64_t left)
{
    if (left >= 4) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<v4f_anywhere *>(to) = v4f{v[0], v[1], v[2], v[3]};
        else *reinterpret_cast<v2u32_anywhere *>(to) = v2u32{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])};
        return;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < left) to[i] = one_of<T>(v[i]);
}
template <typename T> __device__ inline void finish_four(const MxProductArgs &p, int64_t i, int64_t j, const float (&v)[4])
{
    float o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = v[e] + (p.bias && j + e < p.m ? p.bias[j + e] : 0.f);
    auto each = [&](auto act) {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = activate<decltype(act)::value>(o[e]);
    };
    if (p.act == PCPP_ACT_RELU) each(Int<PCPP_ACT_RELU>{});
    else if (p.act == PCPP_ACT_SILU) each(Int<PCPP_ACT_SILU>{});
    else if (p.act == PCPP_ACT_GELU) each(Int<PCPP_ACT_GELU>{});
    store_four(static_cast<T *>(p.out) + i * p.m + j, o, p.m - j);
}

// ---- tiles through LDS --------------------------------------------------------------------------------------------------------------
// A block of WA x WB waves takes 16 WA FA rows of a and 16 WB FB of b, a wave 16 FA and 16 FB of them.  A stage is 256 elements: of every row 128 bytes of
// codes and two words of scales, moved straight into LDS, the next stage while the matrix cores work on this one.
//
// A row's eight 16-byte pieces (blocks) lie in LDS at piece ^ (row / 2 mod 8), so that sixteen lanes reading one piece of sixteen rows meet all banks.
// Lane (r, l) of an instruction has row r; over the stage's two instructions it takes the blocks 2 l and 2 l + 1, whose scales are one 16-bit read (the order in
// which blocks are summed is free).
constexpr int STAGE = 256, STAGE_BYTES = 128, STAGE_BLOCKS = 8;

// rows of a tensor as a descriptor in scalar registers, for inline assembly
__device__ inline v4u scalar_rows(const uint8_t *p, int64_t first, int64_t n, int64_t pitch, int rows)
{
    const int64_t left = n - first < rows ? n - first : rows;
    const uint64_t at = reinterpret_cast<uint64_t>(p) + (uint64_t)(first * pitch);
    const uint32_t bytes = (uint32_t)(left * pitch);
    return v4u{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32)),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
}
// 16 (4) bytes a lane from its offset behind the descriptor's start to LDS byte address `lds` + 16 (4) lane; zeros past the descriptor.  (The address travels in
// M0, which the compiler reserves and nothing else here uses.)
__device__ inline void rows_to_lds_b128(const v4u &rows, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset), "s"(rows), "s"(lds) : "memory");
}
__device__ inline void rows_to_lds_b32(const v4u &rows, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(offset), "s"(rows), "s"(lds) : "memory");
}

template <int WA, int WB, int FA, int FB> struct Tile {
    static constexpr int A = 16 * WA * FA, B = 16 * WB * FB, WAVES = WA * WB, ROWS = A + B;
    static constexpr int SCALES_AT = ROWS * STAGE_BYTES, BYTES = ROWS * (STAGE_BYTES + STAGE_BLOCKS);
    static constexpr int CODE_LOADS = ROWS / 8 / WAVES, SCALE_LOADS = ROWS / 32 / WAVES;     // of a wave for a stage
    static_assert(A % (16 * WAVES) == 0 && B % (16 * WAVES) == 0 && A % (32 * WAVES) == 0 && B % (32 * WAVES) == 0, "whole loads");
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

template <typename T, bool PARTS, int WA, int WB, int FA, int FB>
__global__ __launch_bounds__(64 * WA * WB, WA *WB == 8 ? 2 : 1) void tile_kernel(const MxProductArgs p, uint32_t tile_rows, uint32_t tile_columns, int64_t stages, int64_t of_part)
{
    typedef Tile<WA, WB, FA, FB> S;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), r = lane & 15, l = lane >> 4;
    uint32_t ty, tx;
    tile_of(blockIdx.x, tile_rows, tile_columns, ty, tx);
    const int64_t i0 = (int64_t)ty * S::A, j0 = (int64_t)tx * S::B;
    const uint32_t pitch = (uint32_t)mx_row_bytes(p.k), scale_pitch = (uint32_t)mx_scale_bytes(p.k), blocks = (uint32_t)mx_blocks(p.k), words = scale_pitch / 4u;
    const v4u aq = scalar_rows(p.a, i0, p.n, pitch, S::A), as = scalar_rows(p.a_scales, i0, p.n, scale_pitch, S::A);
    const v4u bq = scalar_rows(p.b, j0, p.m, pitch, S::B), bs = scalar_rows(p.b_scales, j0, p.m, scale_pitch, S::B);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    // what the lane moves: piece `piece` of rows 8 (wave + i WAVES) + lane / 8, word lane % 2 of rows 32 (wave + i WAVES) + lane / 2
    const uint32_t piece = (uint32_t)(lane & 7) ^ ((4u * (uint32_t)wave + (uint32_t)(lane >> 4)) & 7u);
    const uint32_t code_at = (8u * (uint32_t)wave + (uint32_t)(lane >> 3)) * pitch + 16u * piece, word_at = (32u * (uint32_t)wave + (uint32_t)(lane >> 1)) * scale_pitch + 4u * (uint32_t)(lane & 1);
    auto request = [&](int64_t stage, uint32_t buffer) {
        const uint32_t to = lds0 + buffer * S::BYTES, block0 = STAGE_BLOCKS * (uint32_t)stage, word = 2u * (uint32_t)stage + (uint32_t)(lane & 1);
        const bool some = block0 + piece < blocks;
#pragma unroll
        for (int i = 0; i < S::CODE_LOADS; ++i) {
            const bool of_a = 8 * i * S::WAVES < S::A;
            const uint32_t row = 8u * (uint32_t)i * S::WAVES - (of_a ? 0u : (uint32_t)S::A);
            rows_to_lds_b128(of_a ? aq : bq, some ? code_at + row * pitch + 16u * block0 : OOB_OFFSET, to + (uint32_t)(8 * (wave + i * S::WAVES)) * STAGE_BYTES);
        }
#pragma unroll
        for (int i = 0; i < S::SCALE_LOADS; ++i) {
            const bool of_a = 32 * i * S::WAVES < S::A;
            const uint32_t row = 32u * (uint32_t)i * S::WAVES - (of_a ? 0u : (uint32_t)S::A);
            rows_to_lds_b32(of_a ? as : bs, word < words ? word_at + row * scale_pitch + 8u * (uint32_t)stage : OOB_OFFSET,
                            to + S::SCALES_AT + (uint32_t)(32 * (wave + i * S::WAVES)) * STAGE_BLOCKS);
        }
    };
    const int wa = wave / WB, wb = wave % WB;
    const uint32_t read_at = (uint32_t)r * STAGE_BYTES + 16u * ((2u * (uint32_t)l) ^ ((uint32_t)r >> 1 & 7u));
    v4f sum[FA][FB];
#pragma unroll
    for (int y = 0; y < FA; ++y)
#pragma unroll
        for (int x = 0; x < FB; ++x) sum[y][x] = v4f{0.f, 0.f, 0.f, 0.f};
    const int64_t from = PARTS ? blockIdx.y * of_part : 0, to = PARTS && from + of_part < stages ? from + of_part : stages;
    request(from, 0u);
    for (int64_t s = from; s < to; ++s) {
        const uint32_t buffer = (uint32_t)(s - from) & 1u;
        // this stage has arrived, and all waves are done with the one before, whose place the next one takes
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (s + 1 < to) request(s + 1, buffer ^ 1u);
        const uint8_t *codes = lds + buffer * S::BYTES, *scales = codes + S::SCALES_AT;
        const uint32_t left = blocks - STAGE_BLOCKS * (uint32_t)s, own = 2u * (uint32_t)l;   // (scales behind a row's last block may be anything)
        const uint32_t mask = (own < left ? 0xffu : 0u) | (own + 1u < left ? 0xff00u : 0u);
        uint32_t sa[FA], sb[FB];
#pragma unroll
        for (int y = 0; y < FA; ++y) sa[y] = *reinterpret_cast<const uint16_t *>(scales + (16 * (wa * FA + y) + r) * STAGE_BLOCKS + 2 * l) & mask;
#pragma unroll
        for (int x = 0; x < FB; ++x) sb[x] = *reinterpret_cast<const uint16_t *>(scales + (S::A + 16 * (wb * FB + x) + r) * STAGE_BLOCKS + 2 * l) & mask;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint8_t *at = codes + (read_at ^ (16u * t));
            v4u va[FA], vb[FB];
#pragma unroll
            for (int x = 0; x < FB; ++x) vb[x] = *reinterpret_cast<const v4u *>(at + (S::A + 16 * (wb * FB + x)) * STAGE_BYTES);
#pragma unroll
            for (int y = 0; y < FA; ++y) va[y] = *reinterpret_cast<const v4u *>(at + 16 * (wa * FA + y) * STAGE_BYTES);
#pragma unroll
            for (int y = 0; y < FA; ++y)
#pragma unroll
                for (int x = 0; x < FB; ++x) sum[y][x] = t == 0 ? multiply<0>(vb[x], va[y], sum[y][x], sb[x], sa[y]) : multiply<1>(vb[x], va[y], sum[y][x], sb[x], sa[y]);
        }
    }
#pragma unroll
    for (int y = 0; y < FA; ++y)
#pragma unroll
        for (int x = 0; x < FB; ++x) {
            const int64_t i = i0 + 16 * (wa * FA + y) + r, j = j0 + 16 * (wb * FB + x) + 4 * l;
            if (i >= p.n || j >= p.m) continue;
            const float v[4] = {sum[y][x][0], sum[y][x][1], sum[y][x][2], sum[y][x][3]};
            if constexpr (PARTS) store_four(p.part + ((int64_t)blockIdx.y * p.n + i) * p.m + j, v, p.m - j);
            else finish_four<T>(p, i, j, v);
        }
}

template <typename T> __global__ __launch_bounds__(THREADS) void join_kernel(const MxProductArgs p, int parts)
{
    const int64_t fours = ceil_div(p.m, 4);
    const int64_t id = (int64_t)blockIdx.x * THREADS + threadIdx.x;
    if (id >= p.n * fours) return;
    const int64_t i = id / fours, j = 4 * (id - i * fours);
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < parts; ++s) {
        const float *from = p.part + ((int64_t)s * p.n + i) * p.m + j;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += j + e < p.m ? from[e] : 0.f;
    }
    finish_four<T>(p, i, j, v);
}

// How a product is cut: tiles, and parts of the sum where the tiles do not fill the card.
struct Shape {
    bool large;
    int64_t rows, columns, stages, parts, of_part;
};
Shape shape_of(int64_t n, int64_t m, int64_t k)
{
    Shape s{};
    s.stages = ceil_div(k, STAGE);
    s.large = ceil_div(n, 256) * ceil_div(m, 256) >= 192 && s.stages >= 4;
    const int tile = s.large ? 256 : 128;
    s.rows = ceil_div(n, tile);
    s.columns = ceil_div(m, tile);
    s.parts = 1;
    const int64_t tiles = s.rows * s.columns;
    if (tiles < 256 && s.stages >= 8) {
        s.parts = ceil_div(512, tiles);
        if (s.parts > s.stages / 4) s.parts = s.stages / 4;
    }
    s.of_part = ceil_div(s.stages, s.parts);
    s.parts = ceil_div(s.stages, s.of_part);                      // (none is empty)
    return s;
}

template <typename T, bool PARTS, int WA, int WB, int FA, int FB> int launch_tiles(const MxProductArgs &p, const Shape &s, hipStream_t stream)
{
    typedef Tile<WA, WB, FA, FB> L;
    const auto kernel = tile_kernel<T, PARTS, WA, WB, FA, FB>;
    const size_t bytes = (size_t)(s.of_part > 1 ? 2 : 1) * L::BYTES;
    if (int rc = raise_lds_limit(reinterpret_cast<const void *>(kernel), 2 * L::BYTES)) return rc;
    // pieces of whole bands whose blocks a grid holds
    const int64_t most = s.columns > (1 << 22) ? 1 : (1 << 22) / s.columns;
    for (int64_t y = 0; y < s.rows; y += most) {
        MxProductArgs q = p;
        const int64_t i = y * L::A, rows = s.rows - y < most ? s.rows - y : most;
        q.a += i * mx_row_bytes(p.k);
        q.a_scales += i * mx_scale_bytes(p.k);
        q.out = static_cast<T *>(p.out) + i * p.m;
        q.n = p.n - i < rows * L::A ? p.n - i : rows * L::A;
        kernel<<<dim3((unsigned)(rows * s.columns), (unsigned)s.parts), 64 * L::WAVES, bytes, stream>>>(q, (uint32_t)rows, (uint32_t)s.columns, s.stages, s.of_part);
    }
    return PCPP_OK;
}

}  // namespace

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
        if (s.parts > 1) {
            if (int rc = launch_tiles<float, true, 2, 2, 4, 4>(p, s, stream)) return rc;
            join_kernel<T><<<(unsigned)ceil_div(p.n * ceil_div(p.m, 4), THREADS), THREADS, 0, stream>>>(p, (int)s.parts);
            return PCPP_OK;
        }
        return s.large ? launch_tiles<T, false, 4, 2, 4, 8>(p, s, stream) : launch_tiles<T, false, 2, 2, 4, 4>(p, s, stream);
    };
    if (int rc = out_dtype == PCPP_F32 ? with(float{}) : with(bf16_t{})) return rc;
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

}  // namespace pcpp
