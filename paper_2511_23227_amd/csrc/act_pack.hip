// Activations in 8 bits, for a backward pass that needs them later: pack and unpack.  Blocks of 32 channels of a row share a power of
// two, so a value in 8 bits is a bf16 number exactly and what reads the rows (mvmr_weight.hip, block_norm.hip) rounds nothing again.
//
// One lane takes eight channels, a quad of lanes a block; a thread block takes whole rows.  Both kernels are bound by memory.

#include "row_ops.h"

namespace pcpp {

namespace {

constexpr int THREADS = 256;
constexpr int64_t MAX_BLOCKS = 1 << 22;                            // (a grid has fewer than 2^32 threads)

unsigned blocks_for(int64_t n, int rows)
{
    const int64_t b = ceil_div(n, rows);
    return (unsigned)(b < MAX_BLOCKS ? b : MAX_BLOCKS);
}

// Lanes of a row: whole quads, so that the four lanes of a block of channels are one quad of the wave.
__host__ __device__ inline int row_lanes(int c) { return (int)ceil_div(c, ACT_BLOCK) * 4; }

template <typename T, bool WHOLE>
__global__ __launch_bounds__(THREADS) void pack_kernel(const T *__restrict__ x, int64_t n, int c, int8_t *__restrict__ q, uint8_t *__restrict__ codes)
{
    const int lanes = row_lanes(c), rows = THREADS / lanes;
    const int r = (int)threadIdx.x / lanes, c0 = 8 * ((int)threadIdx.x % lanes);
    if (r >= rows) return;                                        // (whole quads, here and below)
    const Span<WHOLE> span(c0, c);
    for (int64_t row = (int64_t)blockIdx.x * rows + r; row < n; row += (int64_t)gridDim.x * rows) {
        Eight<T> raw;
        row_load<T>(x + row * c, span, raw);
        float v[8];
        to_floats(raw, v);
        act_store(v, q + row * c, codes + row * act_code_bytes(c), span, c0, c);
    }
}

template <typename T, bool WHOLE>
__global__ __launch_bounds__(THREADS) void unpack_kernel(const int8_t *__restrict__ q, const uint8_t *__restrict__ codes, int64_t n, int c,
                                                         T *__restrict__ x)
{
    const int lanes = row_lanes(c), rows = THREADS / lanes;
    const int r = (int)threadIdx.x / lanes, c0 = 8 * ((int)threadIdx.x % lanes);
    if (r >= rows) return;
    const Span<WHOLE> span(c0, c);
    for (int64_t row = (int64_t)blockIdx.x * rows + r; row < n; row += (int64_t)gridDim.x * rows) {
        Eight8 raw;
        act_load(q + row * c, codes + row * act_code_bytes(c), span, c0, raw);
        float v[8];
        act_floats(raw, span, v);
        row_store(x + row * c, span, v);
    }
}

}  // namespace

int act_pack(const void *x, int dtype, int64_t n, int c, int8_t *q, uint8_t *codes, hipStream_t stream)
{
    const unsigned blocks = blocks_for(n, THREADS / row_lanes(c));
    auto launch = [&](auto kernel, auto *p) { kernel<<<blocks, THREADS, 0, stream>>>(p, n, c, q, codes); };
    if (dtype == PCPP_F32) launch(c % 8 == 0 ? pack_kernel<float, true> : pack_kernel<float, false>, static_cast<const float *>(x));
    else launch(c % 8 == 0 ? pack_kernel<bf16_t, true> : pack_kernel<bf16_t, false>, static_cast<const bf16_t *>(x));
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

int act_unpack(const int8_t *q, const uint8_t *codes, int64_t n, int c, void *x, int dtype, hipStream_t stream)
{
    const unsigned blocks = blocks_for(n, THREADS / row_lanes(c));
    auto launch = [&](auto kernel, auto *p) { kernel<<<blocks, THREADS, 0, stream>>>(q, codes, n, c, p); };
    if (dtype == PCPP_F32) launch(c % 8 == 0 ? unpack_kernel<float, true> : unpack_kernel<float, false>, static_cast<float *>(x));
    else launch(c % 8 == 0 ? unpack_kernel<bf16_t, true> : unpack_kernel<bf16_t, false>, static_cast<bf16_t *>(x));
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

}  // namespace pcpp
