// What lies between two blocks of a residual network, in one pass over the rows: norm behind the block, gate, residual, norm in front of
// the next block; and its gradients.
//
//   n(v) = (v - mean v) rstd (LAYER), v rstd (RMS), v (NONE);  rstd = 1 / sqrt(mean (v - mean v)^2 + eps)
//   forward    r = scale x + sigmoid(gate) w_post n(f),   h = w_pre n(r)
//   backward   y = w_pre dh,  d = dr + rstd (y - [mean y] - n(r) mean(y n(r)))     what flows to r, [..] with LAYER only
//              dx = scale d,  du = sigmoid(gate) d,  dgate = du (1 - sigmoid(gate)) w_post n(f)  (summed over the row for a gate per row)
//              z = w_post du,  df = rstd (z - [mean z] - n(f) mean(z n(f)))
//              dw_pre = sum over rows dh n(r),  dw_post = sum over rows du n(f)
//
// Bound by memory: every tensor is read or written once.  Backward, 1 000 000 x 256 bf16 with a gate for every channel 815 us = 5.0 TB/s (a 2 GiB
// copy reaches 4.9), 99 991 x 91 35.7 us = 4.4; forward, 115 200 x 64 bf16 beside an fp32 stream with 8-bit copies 23.3 us = 5.1, 100 000 x 32 fp32 11.1 us =
// 4.6, three rows 2.4 us, which is an empty launch's.  A row stays in the registers of 4 .. 64 lanes (row_ops.h), all sums over it
// are taken there in 32 bits, and what the backward pass needs of the row's statistics it takes from the row again, which costs no
// memory.  h is formed from r before r is rounded, and the 8-bit copy of h before h is rounded: one rounding each.  The blocks
// walk the rows with the weights in registers; the weights' gradients are summed there too, then over the lanes and waves of a block,
// then over the blocks by a second kernel, always in the same order.

#include "block_norm.h"
#include "row_ops.h"

namespace pcpp {

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int MAX_BLOCKS = 2048;                                  // forward: eight blocks for each CU
constexpr int MAX_BWD_BLOCKS = 1024;                              // backward: as many partial sums of the weights' gradients

__device__ inline float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * g)); }
// ... and what it leaves of one, to its own last bits (all of it where exp(-g) passes 2^126, so that no infinity meets a zero; a NaN stays)
__device__ inline float sigmoid(float g, float &rest)
{
    const float t = -1.44269504f * g, e = __builtin_amdgcn_exp2f(t), s = __builtin_amdgcn_rcpf(1.f + e);
    rest = t > 126.f ? 1.f : e * s;
    return s;
}

// The row's mean (LAYER; else 0) subtracted from v in place, and 1 / sqrt(mean v^2 + eps).
template <int LPR, int G, int MODE>
__device__ inline float centre_row(float (&v)[G][8], int kind, const Span<MODE> (&own)[G], float inv_c, float eps)
{
    if (kind == PCPP_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += MODE == WHOLE || own[g].own(e) ? v[g][e] : 0.f;
        const float mean = row_sum<LPR>(s) * inv_c;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const float m = own[g].any() ? mean : 0.f;            // (no channels: zeros stay)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[g][e] -= m;
        }
    }
    float s = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float m = MODE == WHOLE || own[g].own(e) ? v[g][e] : 0.f;
            s = __builtin_fmaf(m, m, s);
        }
    return __builtin_amdgcn_rsqf(row_sum<LPR>(s) * inv_c + eps);
}

// the channels' weights, ones without; zero where there is no channel
template <int G, int MODE>
__device__ inline void load_weights(const float *w, const Span<MODE> (&own)[G], int c, float (&v)[G][8])
{
    const __amdgpu_buffer_rsrc_t rs = make_rsrc(w, w ? 4u * (uint32_t)c : 0u);
#pragma unroll
    for (int g = 0; g < G; ++g) {
        Eight<float> r;
        row_load<float>(rs, own[g].template offset<4>(0u), own[g], r);
        to_floats(r, v[g]);
        if (!w) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[g][e] = own[g].any() && (MODE != NARROW || e < c) ? 1.f : 0.f;
        }
    }
}

// S: type of the residual stream, T: of the block's tensors.  A row lies in LPR lanes, G times eight channels each.  FULL: a gate for
// every channel.
template <typename S, typename T, int LPR, int G, int MODE, bool FULL>
__global__ __launch_bounds__(THREADS) void block_fwd_kernel(const BlockNormFwd a)
{
    constexpr int ROWS = 64 / LPR, SS = sizeof(S), TS = sizeof(T);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), c = a.c;
    const uint32_t row = (uint32_t)(lane / LPR);
    int c0[G];
    Span<MODE> own[G];
#pragma unroll
    for (int g = 0; g < G; ++g) c0[g] = 8 * (lane % LPR) + 8 * LPR * g, own[g] = Span<MODE>(c0[g], c);
    float wp[G][8], wn[G][8];
    load_weights(a.w_post, own, c, wp);
    load_weights(a.w_pre, own, c, wn);
    for (int64_t first = ((int64_t)blockIdx.x * WAVES + wave) * ROWS; first < a.n; first += (int64_t)gridDim.x * WAVES * ROWS) {
        const __amdgpu_buffer_rsrc_t xs = rows_from<SS>(a.x, first, a.n, c, c, ROWS), fs = rows_from<TS>(a.f, first, a.n, a.ld_f, c, ROWS);
        const __amdgpu_buffer_rsrc_t gs = rows_from<TS>(a.gate, first, a.n, a.ld_gate, a.gate_cols, ROWS);
        Eight<S> xr[G];
        Eight<T> fr[G], gr[G];
        uint32_t row_gate = 0u;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            row_load<S>(xs, own[g].template offset<SS>(row * (uint32_t)c), own[g], xr[g]);
            row_load<T>(fs, own[g].template offset<TS>(row * (uint32_t)a.ld_f), own[g], fr[g]);
            if constexpr (FULL) row_load<T>(gs, own[g].template offset<TS>(row * (uint32_t)a.ld_gate), own[g], gr[g]);
        }
        if constexpr (!FULL) row_gate = load_one<T>(gs, row * (uint32_t)a.ld_gate);
        float r[G][8];
#pragma unroll
        for (int g = 0; g < G; ++g) to_floats(xr[g], r[g]);
        if (a.f) {
            float f[G][8];
#pragma unroll
            for (int g = 0; g < G; ++g) to_floats(fr[g], f[g]);
            if (a.f_codes.q) {
                const ActRows to = act_rows(a.f_codes.q, a.f_codes.e, first, a.n, c, ROWS);
#pragma unroll
                for (int g = 0; g < G; ++g) act_store<LPR>(f[g], to, row, own[g], c0[g], c);
            }
            float rstd = 1.f;
            if (a.post != PCPP_NORM_NONE) rstd = centre_row<LPR>(f, a.post, own, a.inv_c, a.eps);
            const float s1 = a.gate_cols == 1 ? sigmoid(__uint_as_float(row_gate)) : 1.f;
            const __amdgpu_buffer_rsrc_t rs = rows_from<SS>(a.r, first, a.n, c, c, ROWS);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float s[8];
                if constexpr (FULL) to_floats(gr[g], s);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float sg = FULL ? sigmoid(s[e]) : s1;
                    r[g][e] = __builtin_fmaf(sg, wp[g][e] * (f[g][e] * rstd), a.scale * r[g][e]);
                }
                row_store<S>(rs, own[g].template offset<SS>(row * (uint32_t)c), own[g], r[g]);
            }
        }
        if (a.pre != PCPP_NORM_NONE) {
            const float rstd = centre_row<LPR>(r, a.pre, own, a.inv_c, a.eps);
            const __amdgpu_buffer_rsrc_t hs = rows_from<TS>(a.h, first, a.n, c, c, ROWS);
#pragma unroll
            for (int g = 0; g < G; ++g) {
#pragma unroll
                for (int e = 0; e < 8; ++e) r[g][e] = wn[g][e] * (r[g][e] * rstd);
                row_store<T>(hs, own[g].template offset<TS>(row * (uint32_t)c), own[g], r[g]);
            }
            if (a.h_codes.q) {
                const ActRows to = act_rows(a.h_codes.q, a.h_codes.e, first, a.n, c, ROWS);
#pragma unroll
                for (int g = 0; g < G; ++g) act_store<LPR>(r[g], to, row, own[g], c0[g], c);
            }
        }
    }
}

template <typename S, typename T, int LPR, int G, int MODE, bool FULL>
__global__ __launch_bounds__(THREADS) void block_bwd_kernel(const BlockNormBwd a)
{
    constexpr int ROWS = 64 / LPR, SS = sizeof(S), TS = sizeof(T);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), c = a.c;
    const uint32_t row = (uint32_t)(lane / LPR);
    const bool pre = a.pre != PCPP_NORM_NONE, post = a.post != PCPP_NORM_NONE;
    int c0[G];
    Span<MODE> own[G];
#pragma unroll
    for (int g = 0; g < G; ++g) c0[g] = 8 * (lane % LPR) + 8 * LPR * g, own[g] = Span<MODE>(c0[g], c);
    float wp[G][8], wn[G][8], dwp[G][8], dwn[G][8];
    load_weights(a.w_post, own, c, wp);
    load_weights(a.w_pre, own, c, wn);
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) dwp[g][e] = dwn[g][e] = 0.f;
    for (int64_t first = ((int64_t)blockIdx.x * WAVES + wave) * ROWS; first < a.n; first += (int64_t)gridDim.x * WAVES * ROWS) {
        const bool live = first + row < a.n;                      // (rows past the last are zeros; eps may be zero too)
        Eight<S> drr[G], rr[G];
        Eight<T> dhr[G], fr[G], gr[G];
        Eight8 qr[G];
        uint32_t row_gate = 0u;
        const __amdgpu_buffer_rsrc_t drs = rows_from<SS>(a.dr, first, a.n, c, c, ROWS), rs = rows_from<SS>(a.r, first, a.n, c, c, ROWS);
        const __amdgpu_buffer_rsrc_t dhs = rows_from<TS>(a.dh, first, a.n, c, c, ROWS), gs = rows_from<TS>(a.gate, first, a.n, a.ld_gate, a.gate_cols, ROWS);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            row_load<S>(drs, own[g].template offset<SS>(row * (uint32_t)c), own[g], drr[g]);
            row_load<S>(rs, own[g].template offset<SS>(row * (uint32_t)c), own[g], rr[g]);
            row_load<T>(dhs, own[g].template offset<TS>(row * (uint32_t)c), own[g], dhr[g]);
            if constexpr (FULL) row_load<T>(gs, own[g].template offset<TS>(row * (uint32_t)a.ld_gate), own[g], gr[g]);
        }
        if constexpr (!FULL) row_gate = load_one<T>(gs, row * (uint32_t)a.ld_gate);
        if (a.f_codes.q) {
            const ActRows from = act_rows(a.f_codes.q, a.f_codes.e, first, a.n, c, ROWS);
#pragma unroll
            for (int g = 0; g < G; ++g) act_load(from, row, own[g], c0[g], c, qr[g]);
        } else {
            const __amdgpu_buffer_rsrc_t fs = rows_from<TS>(a.f, first, a.n, a.ld_f, c, ROWS);
#pragma unroll
            for (int g = 0; g < G; ++g) row_load<T>(fs, own[g].template offset<TS>(row * (uint32_t)a.ld_f), own[g], fr[g]);
        }

        // through the norm in front of the next block (without one dh and r are zero, and rstd)
        float d[G][8], r[G][8], y[G][8];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            to_floats(rr[g], r[g]);
            to_floats(dhr[g], y[g]);
        }
        float rstd = centre_row<LPR>(r, a.pre, own, a.inv_c, a.eps);
        rstd = pre && live ? rstd : 0.f;
        float sy = 0.f, syn = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                r[g][e] *= rstd;                                  // n(r)
                dwn[g][e] = __builtin_fmaf(y[g][e], r[g][e], dwn[g][e]);
                y[g][e] *= wn[g][e];
                const float m = MODE != RAGGED || own[g].own(e) ? y[g][e] : 0.f;    // (the weights are zero where there is no channel)
                sy += m;
                syn = __builtin_fmaf(m, r[g][e], syn);
            }
        const float my = a.pre == PCPP_NORM_LAYER ? row_sum<LPR>(sy) * a.inv_c : 0.f, myn = row_sum<LPR>(syn) * a.inv_c;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            to_floats(drr[g], d[g]);
#pragma unroll
            for (int e = 0; e < 8; ++e) d[g][e] = __builtin_fmaf(rstd, y[g][e] - my - r[g][e] * myn, d[g][e]);
        }
        if (a.dx) {
            const __amdgpu_buffer_rsrc_t xs = rows_from<SS>(a.dx, first, a.n, c, c, ROWS);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = a.scale * d[g][e];
                row_store<S>(xs, own[g].template offset<SS>(row * (uint32_t)c), own[g], o);
            }
        }
        if (!a.df) continue;

        // through the gate and the norm behind the block
        float f[G][8];
        if (a.f_codes.q) {
#pragma unroll
            for (int g = 0; g < G; ++g) act_floats(qr[g], own[g], f[g]);
        } else {
#pragma unroll
            for (int g = 0; g < G; ++g) to_floats(fr[g], f[g]);
        }
        rstd = 1.f;
        if (post) rstd = centre_row<LPR>(f, a.post, own, a.inv_c, a.eps);
        rstd = live ? rstd : 0.f;
        float rest1 = 0.f;
        const float s1 = a.gate_cols == 1 ? sigmoid(__uint_as_float(row_gate), rest1) : 1.f;
        float sz = 0.f, szn = 0.f, sg1 = 0.f;
        const __amdgpu_buffer_rsrc_t dgs = rows_from<TS>(a.dgate, first, a.n, a.gate_cols, a.gate_cols, ROWS);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float s[8];
            if constexpr (FULL) to_floats(gr[g], s);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float rest = 0.f;
                const float sg = FULL ? sigmoid(s[e], rest) : s1;
                const float du = d[g][e] * sg;
                f[g][e] *= rstd;                                  // n(f)
                dwp[g][e] = __builtin_fmaf(du, f[g][e], dwp[g][e]);
                d[g][e] = wp[g][e] * du;                          // z
                const float m = MODE != RAGGED || own[g].own(e) ? d[g][e] : 0.f;
                sz += m;
                if constexpr (FULL) {
                    szn = __builtin_fmaf(m, f[g][e], szn);
                    s[e] = rest * (d[g][e] * f[g][e]);
                } else {
                    sg1 = __builtin_fmaf(m, f[g][e], sg1);
                }
            }
            if constexpr (FULL) row_store<T>(dgs, own[g].template offset<TS>(row * (uint32_t)c), own[g], s);
        }
        if constexpr (!FULL) {
            sg1 = row_sum<LPR>(sg1);                              // sum z n(f): the gate's gradient and the norm's
            store_one<T>(dgs, lane % LPR == 0 && a.gate_cols ? row : OOB_OFFSET / TS, rest1 * sg1);
            szn = sg1;
        } else {
            szn = row_sum<LPR>(szn);
        }
        const float mz = a.post == PCPP_NORM_LAYER ? row_sum<LPR>(sz) * a.inv_c : 0.f, mzn = post ? szn * a.inv_c : 0.f;
        const __amdgpu_buffer_rsrc_t dfs = rows_from<TS>(a.df, first, a.n, c, c, ROWS);
#pragma unroll
        for (int g = 0; g < G; ++g) {
#pragma unroll
            for (int e = 0; e < 8; ++e) d[g][e] = rstd * (d[g][e] - mz - f[g][e] * mzn);
            row_store<T>(dfs, own[g].template offset<TS>(row * (uint32_t)c), own[g], d[g]);
        }
    }

    // the weights' gradients: over the rows that the wave's lanes hold, then over the waves
    __shared__ float sums[WAVES][2][G * 8 * LPR];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float p = dwp[g][e], n = dwn[g][e];
#pragma unroll
            for (int m = LPR; m < 64; m <<= 1) {
                p += __shfl_xor(p, m);
                n += __shfl_xor(n, m);
            }
            if (lane < LPR && own[g].own(e)) {
                sums[wave][0][own[g].at + e] = p;
                sums[wave][1][own[g].at + e] = n;
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * c; i += THREADS) {
        const int which = i >= c, ch = which ? i - c : i;
        float v = sums[0][which][ch];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += sums[w][which][ch];
        a.part[(size_t)blockIdx.x * 2 * c + i] = v;
    }
}

// Sums of the blocks' partial sums [blocks][2][c]: a block takes sixteen columns, a thread every 64th row of one; then the four threads of a
// wave and the waves, in order.  (64 columns a block and every 16th row: 5.2 us for 1024 blocks of 91 channels, 3.9 so.)
__global__ __launch_bounds__(1024) void weight_sums_kernel(const float *__restrict__ part, int blocks, int c, float *__restrict__ dw_post,
                                                           float *__restrict__ dw_pre)
{
    __shared__ float sums[16][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, column = lane & 15;
    const int i = (int)blockIdx.x * 16 + column;
    float v = 0.f;
    if (i < 2 * c) {
#pragma unroll 16
        for (int b = 4 * wave + (lane >> 4); b < blocks; b += 64) v += part[(size_t)b * 2 * c + i];
    }
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
    if (lane < 16) sums[wave][column] = v;
    __syncthreads();
    if (threadIdx.x >= 16 || i >= 2 * c) return;
    v = sums[0][column];
#pragma unroll
    for (int w = 1; w < 16; ++w) v += sums[w][column];
    float *to = i < c ? dw_post : dw_pre;
    if (to) to[i < c ? i : i - c] = v;
}

int blocks_for(int64_t n, int c, int most)
{
    const int64_t b = ceil_div(n, WAVES * 64 / row_lanes(c));
    return (int)(b < most ? b : most);
}

template <typename F> void with_types(int stream_dtype, int dtype, F f)
{
    if (stream_dtype == PCPP_F32 && dtype == PCPP_F32) f(float{}, float{});
    else if (stream_dtype == PCPP_F32) f(float{}, bf16_t{});
    else f(bf16_t{}, bf16_t{});
}

}  // namespace

int block_norm_fwd(const BlockNormFwd &a, int stream_dtype, int dtype, hipStream_t stream)
{
    const unsigned blocks = (unsigned)blocks_for(a.n, a.c, MAX_BLOCKS);
    with_types(stream_dtype, dtype, [&](auto s, auto t) {
        with_rows(a.c, [&](auto lpr, auto g, auto mode) {
            constexpr int LPR = decltype(lpr)::value, G = decltype(g)::value, MODE = decltype(mode)::value;
            if (a.gate_cols > 1) block_fwd_kernel<decltype(s), decltype(t), LPR, G, MODE, true><<<blocks, THREADS, 0, stream>>>(a);
            else block_fwd_kernel<decltype(s), decltype(t), LPR, G, MODE, false><<<blocks, THREADS, 0, stream>>>(a);
        });
    });
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

size_t block_norm_bwd_workspace_bytes(int64_t n, int c) { return align_up((size_t)blocks_for(n, c, MAX_BWD_BLOCKS) * 2 * c * sizeof(float)); }

int block_norm_bwd(const BlockNormBwd &a, int stream_dtype, int dtype, hipStream_t stream)
{
    const int blocks = blocks_for(a.n, a.c, MAX_BWD_BLOCKS);
    with_types(stream_dtype, dtype, [&](auto s, auto t) {
        with_rows(a.c, [&](auto lpr, auto g, auto mode) {
            constexpr int LPR = decltype(lpr)::value, G = decltype(g)::value, MODE = decltype(mode)::value;
            if (a.gate_cols > 1) block_bwd_kernel<decltype(s), decltype(t), LPR, G, MODE, true><<<(unsigned)blocks, THREADS, 0, stream>>>(a);
            else block_bwd_kernel<decltype(s), decltype(t), LPR, G, MODE, false><<<(unsigned)blocks, THREADS, 0, stream>>>(a);
        });
    });
    PCPP_HIP_CHECK(hipGetLastError());
    if (!a.dw_post && !a.dw_pre) return PCPP_OK;
    weight_sums_kernel<<<(unsigned)ceil_div(2 * a.c, 16), 1024, 0, stream>>>(a.part, blocks, a.c, a.dw_post, a.dw_pre);
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

}  // namespace pcpp
