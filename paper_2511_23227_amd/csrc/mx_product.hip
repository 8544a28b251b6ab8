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
constexpr int STEP = 128;                                         // elements of a sum that an instruction takes
constexpr int BLOCK_ROWS = 128;                                         // rows of a and of b that a block takes

__device__ inline v4f multiply(const v4u &b, const v4u &a, v4f sum, uint32_t b_scale, uint32_t a_scale)
{
    const v8i x = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0}, y = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, sum, 4, 4, 0, (int)b_scale, 0, (int)a_scale);
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

// Rows of one side from `first` on: descriptors of codes and scales that end behind the tensor's last row
struct Side {
    __amdgpu_buffer_rsrc_t q, scales;
    __device__ inline Side(const uint8_t *at, const uint8_t *scales_at, int64_t first, int64_t n, int64_t k, int rows)
        : q(rows_from<1>(at, first, n, mx_row_bytes(k), (int)mx_row_bytes(k), rows)),
          scales(rows_from<1>(scales_at, first, n, mx_scale_bytes(k), (int)mx_scale_bytes(k), rows))
    {
    }
};

// A block takes 128 rows of a and of b, a wave 64 of each; blockIdx.z a part of the sum (PARTS).
template <typename T, bool PARTS> __global__ __launch_bounds__(THREADS) void product_kernel(const MxProductArgs p, int64_t steps, int64_t steps_of_part)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), r = lane & 15, l = lane >> 4;
    const int64_t i0 = (int64_t)blockIdx.y * BLOCK_ROWS + 64 * (wave >> 1), j0 = (int64_t)blockIdx.x * BLOCK_ROWS + 64 * (wave & 1);
    if (i0 >= p.n || j0 >= p.m) return;
    const Side a(p.a, p.a_scales, i0, p.n, p.k, 64), b(p.b, p.b_scales, j0, p.m, p.k, 64);
    const uint32_t pitch = (uint32_t)mx_row_bytes(p.k), scale_pitch = (uint32_t)mx_scale_bytes(p.k), blocks = (uint32_t)mx_blocks(p.k);
    v4f sum[4][4];
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int x = 0; x < 4; ++x) sum[y][x] = v4f{0.f, 0.f, 0.f, 0.f};
    const int64_t from = PARTS ? blockIdx.z * steps_of_part : 0, to = PARTS && from + steps_of_part < steps ? from + steps_of_part : steps;
    for (int64_t s = from; s < to; ++s) {
        const uint32_t block = 4u * (uint32_t)s + (uint32_t)l;
        v4u aq[4], bq[4];
        uint32_t as[4], bs[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const uint32_t row = 16u * x + (uint32_t)r;
            const uint32_t at = block < blocks ? row * pitch + 16u * block : OOB_OFFSET, scale_at = block < blocks ? row * scale_pitch + block : OOB_OFFSET;
            const auto av = __builtin_amdgcn_raw_buffer_load_b128(a.q, (int)at, 0, 0), bv = __builtin_amdgcn_raw_buffer_load_b128(b.q, (int)at, 0, 0);
            aq[x] = v4u{av[0], av[1], av[2], av[3]};
            bq[x] = v4u{bv[0], bv[1], bv[2], bv[3]};
            as[x] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(a.scales, (int)scale_at, 0, 0);
            bs[x] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(b.scales, (int)scale_at, 0, 0);
        }
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int x = 0; x < 4; ++x) sum[y][x] = multiply(bq[x], aq[y], sum[y][x], bs[x], as[y]);
    }
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int64_t i = i0 + 16 * y + r, j = j0 + 16 * x + 4 * l;
            if (i >= p.n || j >= p.m) continue;
            const float v[4] = {sum[y][x][0], sum[y][x][1], sum[y][x][2], sum[y][x][3]};
            if constexpr (PARTS) store_four(p.part + ((int64_t)blockIdx.z * p.n + i) * p.m + j, v, p.m - j);
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

struct Shape { int64_t rows, columns, steps, parts; };
Shape shape_of(int64_t n, int64_t m, int64_t k)
{
    Shape s{ceil_div(n, BLOCK_ROWS), ceil_div(m, BLOCK_ROWS), ceil_div(k, STEP), 1};
    const int64_t tiles = s.rows * s.columns;
    if (tiles < 512 && s.steps >= 16) {
        s.parts = ceil_div(1024, tiles);
        if (s.parts > s.steps / 8) s.parts = s.steps / 8;
        if (s.parts > 256) s.parts = 256;
        s.parts = ceil_div(s.steps, ceil_div(s.steps, s.parts));  // (none is empty)
    }
    return s;
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
    auto with = [&](auto t) {
        typedef decltype(t) T;
        for (int64_t y = 0; y < s.rows; y += 65535) {             // (a grid's second extent)
            MxProductArgs q = p;
            const int64_t i = y * BLOCK_ROWS, rows = s.rows - y < 65535 ? s.rows - y : 65535;
            q.a += i * mx_row_bytes(p.k);
            q.a_scales += i * mx_scale_bytes(p.k);
            q.out = static_cast<T *>(p.out) + i * p.m;
            q.n = p.n - i;
            const dim3 grid((unsigned)s.columns, (unsigned)rows, (unsigned)s.parts);
            const int64_t of_part = ceil_div(s.steps, s.parts);
            if (s.parts > 1) product_kernel<T, true><<<grid, THREADS, 0, stream>>>(q, s.steps, of_part);
            else product_kernel<T, false><<<grid, THREADS, 0, stream>>>(q, s.steps, of_part);
        }
        if (s.parts > 1) join_kernel<T><<<(unsigned)ceil_div(p.n * ceil_div(p.m, 4), THREADS), THREADS, 0, stream>>>(p, (int)s.parts);
    };
    if (out_dtype == PCPP_F32) with(float{});
    else with(bf16_t{});
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

}  // namespace pcpp
