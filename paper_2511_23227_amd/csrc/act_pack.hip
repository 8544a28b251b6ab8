// Activations in 8 bits, for a backward pass that needs them later: pack and unpack.  Blocks of 32 channels of a row share a power of
// two, so a value in 8 bits is a bf16 number exactly and what reads the rows (mvmr_weight.hip, block_norm.hip) rounds nothing again.
//
// Rows in registers (row_ops.h), one wave 64 / LPR rows.  Both kernels are bound by memory: 199 993 x 128 bf16, 77 MB each, 15 us.

#include "row_ops.h"

namespace pcpp {

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int64_t MAX_BLOCKS = 1 << 22;                            // (a grid has fewer than 2^32 threads)

template <typename T, int LPR, int G, int MODE>
__global__ __launch_bounds__(THREADS) void pack_kernel(const T *__restrict__ x, int64_t n, int c, int8_t *__restrict__ q, uint8_t *__restrict__ codes)
{
    constexpr int ROWS = 64 / LPR;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t row = (uint32_t)(lane / LPR);
    for (int64_t first = ((int64_t)blockIdx.x * WAVES + wave) * ROWS; first < n; first += (int64_t)gridDim.x * WAVES * ROWS) {
        const __amdgpu_buffer_rsrc_t xs = rows_from<sizeof(T)>(x, first, n, c, c, ROWS);
        const ActRows to = act_rows(q, codes, first, n, c, ROWS);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int c0 = 8 * (lane % LPR) + 8 * LPR * g;
            const Span<MODE> span(c0, c);
            Eight<T> raw;
            row_load<T>(xs, span.template offset<sizeof(T)>(row * (uint32_t)c), span, raw);
            float v[8];
            to_floats(raw, v);
            act_store<LPR>(v, to, row, span, c0, c);
        }
    }
}

template <typename T, int LPR, int G, int MODE>
__global__ __launch_bounds__(THREADS) void unpack_kernel(const int8_t *__restrict__ q, const uint8_t *__restrict__ codes, int64_t n, int c,
                                                         T *__restrict__ x)
{
    constexpr int ROWS = 64 / LPR;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t row = (uint32_t)(lane / LPR);
    for (int64_t first = ((int64_t)blockIdx.x * WAVES + wave) * ROWS; first < n; first += (int64_t)gridDim.x * WAVES * ROWS) {
        const __amdgpu_buffer_rsrc_t xs = rows_from<sizeof(T)>(x, first, n, c, c, ROWS);
        const ActRows from = act_rows(q, codes, first, n, c, ROWS);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int c0 = 8 * (lane % LPR) + 8 * LPR * g;
            const Span<MODE> span(c0, c);
            Eight8 raw;
            act_load(from, row, span, c0, c, raw);
            float v[8];
            act_floats(raw, span, v);
            row_store<T>(xs, span.template offset<sizeof(T)>(row * (uint32_t)c), span, v);
        }
    }
}

template <typename F> void with_type(int dtype, F f)
{
    if (dtype == PCPP_F32) f(float{});
    else f(bf16_t{});
}
unsigned blocks_for(int64_t n, int lpr)
{
    const int64_t b = ceil_div(n, WAVES * 64 / lpr);
    return (unsigned)(b < MAX_BLOCKS ? b : MAX_BLOCKS);
}

}  // namespace

int act_pack(const void *x, int dtype, int64_t n, int c, int8_t *q, uint8_t *codes, hipStream_t stream)
{
    with_type(dtype, [&](auto t) {
        with_rows(c, [&](auto lpr, auto g, auto mode) {
            typedef decltype(t) T;
            pack_kernel<T, decltype(lpr)::value, decltype(g)::value, decltype(mode)::value>
                <<<blocks_for(n, decltype(lpr)::value), THREADS, 0, stream>>>(static_cast<const T *>(x), n, c, q, codes);
        });
    });
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

int act_unpack(const int8_t *q, const uint8_t *codes, int64_t n, int c, void *x, int dtype, hipStream_t stream)
{
    with_type(dtype, [&](auto t) {
        with_rows(c, [&](auto lpr, auto g, auto mode) {
            typedef decltype(t) T;
            unpack_kernel<T, decltype(lpr)::value, decltype(g)::value, decltype(mode)::value>
                <<<blocks_for(n, decltype(lpr)::value), THREADS, 0, stream>>>(q, codes, n, c, static_cast<T *>(x));
        });
    });
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

}  // namespace pcpp
