// Dropout of a branch with the residual behind it, and the branch's gradient:
//
//   forward    y = residual + k x 65536 / (65536 - t),   k = 1 where the element's (row's, cloud's) sixteen random bits are t = round(65536 p) or more
//   backward   dx = k dy 65536 / (65536 - t)             the same kernel without a residual
//
// The bits come from a counter (philox.h) and are formed again where they are needed: no mask is stored.  A thread takes eight
// neighbouring channels, which share a counter.  Where a row ends inside a thread's eight channels it takes the row's last eight instead,
// some of which are the thread before's too: their bits come from that thread, and both write the same.
//
// Memory bounds it: 1 000 000 x 256 bf16 in 166 us, 6.2 TB/s; 99 991 x 91 bf16 onto an fp32 residual in 15.1 us, 6.0 TB/s.  The ten rounds of the
// generator hide behind it (138 vector instructions a wave in all).
#include "pointwise.h"

namespace pcpp {

namespace {

constexpr int THREADS = 256;

// S: type of what is read, T: of the residual and of what is written
template <typename S, typename T, bool RESIDUAL, int MODE>
__global__ __launch_bounds__(THREADS) void dropout_kernel(const DropoutArgs a, const Divisor per_row, const uint32_t groups)
{
    const uint32_t id = blockIdx.x * (uint32_t)THREADS + threadIdx.x;
    const uint32_t group = id < groups ? id : groups - 1u, row = per_row.quotient(group);
    const int c0 = 8 * (int)(group - row * per_row.by);
    const bool tail = MODE == RAGGED && c0 + 8 > a.c;
    const int at = tail ? a.c - 8 : c0;
    const S *x = static_cast<const S *>(a.x) + (int64_t)row * a.ld_x + at;
    const int64_t to = (int64_t)row * a.c + at;
    Eight<S> xr;
    Eight<T> rr;
    float v[8], r[8];
    if constexpr (MODE != NARROW) {
        load_eight<false>(x, xr);
        if constexpr (RESIDUAL) load_eight<false>(static_cast<const T *>(a.residual) + to, rr);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e) {
            v[e] = e < a.c ? one_float(x[e]) : 0.f;
            if constexpr (RESIDUAL) r[e] = e < a.c ? one_float(static_cast<const T *>(a.residual)[to + e]) : 0.f;
        }
        v[7] = r[7] = 0.f;
    }
    const Philox philox(a.drop.random);
    uint32_t bits;
    bool live = id < groups;
    if (a.scope == PCPP_DROP_ELEMENTS) {
        bits = kept(philox, group, a.drop.threshold);
        if constexpr (MODE == RAGGED) {
            uint32_t before = __shfl_up(bits, 1);
            if (tail && (threadIdx.x & 63) == 0) before = kept(philox, group - 1u, a.drop.threshold);
            if (tail) bits = before >> (8 - (c0 - at)) | bits << (c0 - at);
        }
    } else {
        uint32_t which = row;
        if (a.scope == PCPP_DROP_CLOUDS) {
            const Clouds clouds{a.offsets, a.n_clouds, a.n};
            which = (uint32_t)clouds.at(row);
            live = live && which < (uint32_t)a.n_clouds && (int64_t)row >= clouds.bound(0);
        }
        bits = kept(philox, which, a.drop.threshold) & 1u ? 0xffu : 0u;
    }
    if constexpr (MODE != NARROW) {
        to_floats(xr, v);
        if constexpr (RESIDUAL) to_floats(rr, r);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float k = bits >> e & 1u ? v[e] : 0.f;              // (an Inf or NaN that is dropped leaves nothing)
        v[e] = RESIDUAL ? __builtin_fmaf(k, a.drop.scale, r[e]) : k * a.drop.scale;
    }
    if (!live) return;
    T *y = static_cast<T *>(a.y) + to;
    if constexpr (MODE != NARROW) {
        store_eight<false>(y, v);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < a.c) y[e] = one_of<T>(v[e]);
    }
}

}  // namespace

int dropout(const DropoutArgs &a, int in_dtype, int out_dtype, hipStream_t stream)
{
    const uint32_t per_row = (uint32_t)ceil_div(a.c, 8), groups = (uint32_t)(a.n * per_row);
    const unsigned blocks = (unsigned)ceil_div(groups, THREADS);
    auto launch = [&](auto s, auto t) {
        typedef decltype(s) S;
        typedef decltype(t) T;
        auto with = [&](auto mode) {
            constexpr int MODE = decltype(mode)::value;
            if (a.residual) dropout_kernel<S, T, true, MODE><<<blocks, THREADS, 0, stream>>>(a, make_divisor(per_row), groups);
            else dropout_kernel<S, T, false, MODE><<<blocks, THREADS, 0, stream>>>(a, make_divisor(per_row), groups);
        };
        a.c < 8 ? with(Int<NARROW>{}) : (a.c % 8 == 0 ? with(Int<WHOLE>{}) : with(Int<RAGGED>{}));
    };
    if (in_dtype == PCPP_F32) out_dtype == PCPP_F32 ? launch(float{}, float{}) : launch(float{}, bf16_t{});
    else out_dtype == PCPP_F32 ? launch(bf16_t{}, float{}) : launch(bf16_t{}, bf16_t{});
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

}  // namespace pcpp
