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
// Bound by memory: every tensor is read or written once.  A row stays in the registers of 4 .. 64 lanes (row_ops.h), all sums over it
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

// The row's mean (LAYER; else 0) subtracted from v in place, and 1 / sqrt(mean v^2 + eps).
template <int LPR, int G, bool WHOLE>
__device__ inline float centre_row(float (&v)[G][8], int kind, const Span<WHOLE> (&own)[G], float inv_c, float eps)
{
    if (kind == PCPP_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += WHOLE || own[g].own(e) ? v[g][e] : 0.f;
        const float mean = row_sum<LPR>(s) * inv_c;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[g][e] = !WHOLE || own[g].any() ? v[g][e] - mean : 0.f;
    }
    float s = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float m = WHOLE || own[g].own(e) ? v[g][e] : 0.f;
            s = __builtin_fmaf(m, m, s);
        }
    return __builtin_amdgcn_rsqf(row_sum<LPR>(s) * inv_c + eps);
}

// the channels' weights, ones without; zero where there is no channel
template <int G, bool WHOLE>
__device__ inline void load_weights(const float *w, const Span<WHOLE> (&own)[G], float (&v)[G][8])
{
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[g][e] = own[g].any() && (WHOLE || e < own[g].hi) ? (w ? w[own[g].at + e] : 1.f) : 0.f;
}

// S: type of the residual stream, T: of the block's tensors.  A row lies in LPR lanes, G times eight channels each.
template <typename S, typename T, int LPR, int G, bool WHOLE>
__global__ __launch_bounds__(THREADS) void block_fwd_kernel(const BlockNormFwd a)
{
    constexpr int ROWS = THREADS / LPR, NEXT = 8 * LPR;
    const int c = a.c, c0 = 8 * ((int)threadIdx.x % LPR);
    Span<WHOLE> own[G];
#pragma unroll
    for (int g = 0; g < G; ++g) own[g] = Span<WHOLE>(c0 + NEXT * g, c);
    float wp[G][8], wn[G][8];
    load_weights(a.w_post, own, wp);
    load_weights(a.w_pre, own, wn);
    // (a row's lanes leave the loop together, and nothing in it reads another row's lanes)
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR; row < a.n; row += (int64_t)gridDim.x * ROWS) {
        Eight<S> xr[G];
        Eight<T> fr[G], gr[G];
        float row_gate = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) row_load<S>(static_cast<const S *>(a.x) + row * c, own[g], xr[g]);
        if (a.f) {
#pragma unroll
            for (int g = 0; g < G; ++g) row_load<T>(static_cast<const T *>(a.f) + row * a.ld_f, own[g], fr[g]);
            if (a.gate_cols > 1) {
#pragma unroll
                for (int g = 0; g < G; ++g) row_load<T>(static_cast<const T *>(a.gate) + row * a.ld_gate, own[g], gr[g]);
            } else if (a.gate_cols == 1) {
                row_gate = one_float<T>(static_cast<const T *>(a.gate)[row * a.ld_gate]);
            }
        }
        float r[G][8];
#pragma unroll
        for (int g = 0; g < G; ++g) to_floats(xr[g], r[g]);
        if (a.f) {
            float f[G][8];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                to_floats(fr[g], f[g]);
                if (a.f_codes.q) act_store(f[g], a.f_codes.q + row * c, a.f_codes.e + row * act_code_bytes(c), own[g], c0 + NEXT * g, c);
            }
            float rstd = 1.f;
            if (a.post != PCPP_NORM_NONE) rstd = centre_row<LPR>(f, a.post, own, a.inv_c, a.eps);
            const float s1 = a.gate_cols == 1 ? sigmoid(row_gate) : 1.f;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float s[8];
                if (a.gate_cols > 1) to_floats(gr[g], s);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float sg = a.gate_cols > 1 ? sigmoid(s[e]) : s1;
                    r[g][e] = __builtin_fmaf(sg, wp[g][e] * (f[g][e] * rstd), a.scale * r[g][e]);
                }
            }
#pragma unroll
            for (int g = 0; g < G; ++g) row_store(static_cast<S *>(a.r) + row * c, own[g], r[g]);
        }
        if (a.pre != PCPP_NORM_NONE) {
            const float rstd = centre_row<LPR>(r, a.pre, own, a.inv_c, a.eps);
#pragma unroll
            for (int g = 0; g < G; ++g) {
#pragma unroll
                for (int e = 0; e < 8; ++e) r[g][e] = wn[g][e] * (r[g][e] * rstd);
                row_store(static_cast<T *>(a.h) + row * c, own[g], r[g]);
                if (a.h_codes.q) act_store(r[g], a.h_codes.q + row * c, a.h_codes.e + row * act_code_bytes(c), own[g], c0 + NEXT * g, c);
            }
        }
    }
}

template <typename S, typename T, int LPR, int G, bool WHOLE>
__global__ __launch_bounds__(THREADS) void block_bwd_kernel(const BlockNormBwd a)
{
    constexpr int ROWS = THREADS / LPR, NEXT = 8 * LPR;
    const int c = a.c, c0 = 8 * ((int)threadIdx.x % LPR);
    const bool pre = a.pre != PCPP_NORM_NONE, post = a.post != PCPP_NORM_NONE, branch = a.df != nullptr;
    Span<WHOLE> own[G];
#pragma unroll
    for (int g = 0; g < G; ++g) own[g] = Span<WHOLE>(c0 + NEXT * g, c);
    float wp[G][8], wn[G][8], dwp[G][8], dwn[G][8];
    load_weights(a.w_post, own, wp);
    load_weights(a.w_pre, own, wn);
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) dwp[g][e] = dwn[g][e] = 0.f;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR; row < a.n; row += (int64_t)gridDim.x * ROWS) {
        Eight<S> drr[G], rr[G];
        Eight<T> dhr[G], fr[G], gr[G];
        Eight8 qr[G];
        float row_gate = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (a.dr) row_load<S>(static_cast<const S *>(a.dr) + row * c, own[g], drr[g]);
            if (pre) {
                row_load<T>(static_cast<const T *>(a.dh) + row * c, own[g], dhr[g]);
                row_load<S>(static_cast<const S *>(a.r) + row * c, own[g], rr[g]);
            }
            if (branch) {
                if (a.f_codes.q) act_load(a.f_codes.q + row * c, a.f_codes.e + row * act_code_bytes(c), own[g], c0 + NEXT * g, qr[g]);
                else if (a.f) row_load<T>(static_cast<const T *>(a.f) + row * a.ld_f, own[g], fr[g]);
                if (a.gate_cols > 1) row_load<T>(static_cast<const T *>(a.gate) + row * a.ld_gate, own[g], gr[g]);
            }
        }
        if (branch && a.gate_cols == 1) row_gate = one_float<T>(static_cast<const T *>(a.gate)[row * a.ld_gate]);

        float d[G][8];
        if (a.dr) {
#pragma unroll
            for (int g = 0; g < G; ++g) to_floats(drr[g], d[g]);
        } else {
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int e = 0; e < 8; ++e) d[g][e] = 0.f;
        }
        if (pre) {
            float r[G][8], y[G][8];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                to_floats(rr[g], r[g]);
                to_floats(dhr[g], y[g]);
            }
            const float rstd = centre_row<LPR>(r, a.pre, own, a.inv_c, a.eps);
            float sy = 0.f, syn = 0.f;
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    r[g][e] *= rstd;                              // n(r)
                    dwn[g][e] = __builtin_fmaf(y[g][e], r[g][e], dwn[g][e]);
                    y[g][e] *= wn[g][e];
                    const float m = WHOLE || own[g].own(e) ? y[g][e] : 0.f;
                    sy += m;
                    syn = __builtin_fmaf(m, r[g][e], syn);
                }
            const float my = a.pre == PCPP_NORM_LAYER ? row_sum<LPR>(sy) * a.inv_c : 0.f, myn = row_sum<LPR>(syn) * a.inv_c;
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int e = 0; e < 8; ++e) d[g][e] = __builtin_fmaf(rstd, y[g][e] - my - r[g][e] * myn, d[g][e]);
        }
        if (a.dx) {
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = a.scale * d[g][e];
                row_store(static_cast<S *>(a.dx) + row * c, own[g], o);
            }
        }
        if (!branch) continue;
        float f[G][8];
        const bool has_f = a.f_codes.q || a.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (a.f_codes.q) {
                act_floats(qr[g], own[g], f[g]);
            } else if (a.f) {
                to_floats(fr[g], f[g]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) f[g][e] = 0.f;
            }
        }
        float rstd = 1.f;
        if (post && has_f) rstd = centre_row<LPR>(f, a.post, own, a.inv_c, a.eps);
        const float s1 = a.gate_cols == 1 ? sigmoid(row_gate) : 1.f;
        float sz = 0.f, szn = 0.f, sg1 = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float s[8];
            if (a.gate_cols > 1) to_floats(gr[g], s);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float sg = a.gate_cols > 1 ? sigmoid(s[e]) : s1;
                const float nf = f[g][e] * rstd;
                const float du = d[g][e] * sg;
                dwp[g][e] = __builtin_fmaf(du, nf, dwp[g][e]);
                d[g][e] = wp[g][e] * du;                          // z (zero where there is no channel, as the weights are)
                s[e] = (1.f - sg) * (d[g][e] * nf);
                const float m = WHOLE || own[g].own(e) ? d[g][e] : 0.f;
                sg1 += WHOLE || own[g].own(e) ? s[e] : 0.f;
                sz += m;
                szn = __builtin_fmaf(m, nf, szn);
                f[g][e] = nf;
            }
            if (a.gate_cols > 1) row_store(static_cast<T *>(a.dgate) + row * c, own[g], s);
        }
        if (a.gate_cols == 1) {
            sg1 = row_sum<LPR>(sg1);
            if (c0 == 0) static_cast<T *>(a.dgate)[row] = one_of<T>(sg1);
        }
        if (post) {
            const float mz = a.post == PCPP_NORM_LAYER ? row_sum<LPR>(sz) * a.inv_c : 0.f, mzn = row_sum<LPR>(szn) * a.inv_c;
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int e = 0; e < 8; ++e) d[g][e] = rstd * (d[g][e] - mz - f[g][e] * mzn);
        }
#pragma unroll
        for (int g = 0; g < G; ++g) row_store(static_cast<T *>(a.df) + row * c, own[g], d[g]);
    }

    // the weights' gradients: over the rows that the wave's lanes hold, then over the waves
    __shared__ float sums[WAVES][2][G * 8 * LPR];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
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

// Sums of the blocks' partial sums [blocks][2][c]: wave w of sixteen adds the rows w, w + 16, ..., then the waves' sums in order of w.
__global__ __launch_bounds__(1024) void weight_sums_kernel(const float *__restrict__ part, int blocks, int c, float *__restrict__ dw_post,
                                                           float *__restrict__ dw_pre)
{
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int i = (int)blockIdx.x * 64 + lane;
    float v = 0.f;
    if (i < 2 * c) {
#pragma unroll 8
        for (int b = wave; b < blocks; b += 16) v += part[(size_t)b * 2 * c + i];
    }
    sums[wave][lane] = v;
    __syncthreads();
    if (wave != 0 || i >= 2 * c) return;
    v = sums[0][lane];
#pragma unroll
    for (int w = 1; w < 16; ++w) v += sums[w][lane];
    float *to = i < c ? dw_post : dw_pre;
    if (to) to[i < c ? i : i - c] = v;
}

int bwd_blocks(int64_t n, int lpr)
{
    const int64_t b = ceil_div(n, THREADS / lpr);
    return (int)(b < MAX_BWD_BLOCKS ? b : MAX_BWD_BLOCKS);
}

// Lanes for a row of c channels: eight each, sixteen past 512.
int row_lpr(int c)
{
    int lpr = 4;
    while (lpr < 64 && 8 * lpr < c) lpr *= 2;
    return lpr;
}

template <typename F> void with_types(int stream_dtype, int dtype, F f)
{
    if (stream_dtype == PCPP_F32 && dtype == PCPP_F32) f(float{}, float{});
    else if (stream_dtype == PCPP_F32) f(float{}, bf16_t{});
    else f(bf16_t{}, bf16_t{});
}
template <int N> struct Int { static constexpr int value = N; };
template <typename F> void with_shape(int c, F f)
{
    auto whole = [&](auto lpr, auto g) {
        if (c % 8 == 0) f(lpr, g, std::true_type{});
        else f(lpr, g, std::false_type{});
    };
    if (c > 512) return whole(Int<64>{}, Int<2>{});
    switch (row_lpr(c)) {
    case 4: return whole(Int<4>{}, Int<1>{});
    case 8: return whole(Int<8>{}, Int<1>{});
    case 16: return whole(Int<16>{}, Int<1>{});
    case 32: return whole(Int<32>{}, Int<1>{});
    default: return whole(Int<64>{}, Int<1>{});
    }
}

}  // namespace

int block_norm_fwd(const BlockNormFwd &a, int stream_dtype, int dtype, hipStream_t stream)
{
    const int64_t want = ceil_div(a.n, THREADS / row_lpr(a.c));
    const unsigned blocks = (unsigned)(want < MAX_BLOCKS ? want : MAX_BLOCKS);
    with_types(stream_dtype, dtype, [&](auto s, auto t) {
        with_shape(a.c, [&](auto lpr, auto g, auto whole) {
            block_fwd_kernel<decltype(s), decltype(t), decltype(lpr)::value, decltype(g)::value, decltype(whole)::value>
                <<<blocks, THREADS, 0, stream>>>(a);
        });
    });
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

size_t block_norm_bwd_workspace_bytes(int64_t n, int c) { return align_up((size_t)bwd_blocks(n, row_lpr(c)) * 2 * c * sizeof(float)); }

int block_norm_bwd(const BlockNormBwd &a, int stream_dtype, int dtype, hipStream_t stream)
{
    const int blocks = bwd_blocks(a.n, row_lpr(a.c));
    with_types(stream_dtype, dtype, [&](auto s, auto t) {
        with_shape(a.c, [&](auto lpr, auto g, auto whole) {
            block_bwd_kernel<decltype(s), decltype(t), decltype(lpr)::value, decltype(g)::value, decltype(whole)::value>
                <<<(unsigned)blocks, THREADS, 0, stream>>>(a);
        });
    });
    PCPP_HIP_CHECK(hipGetLastError());
    if (!a.dw_post && !a.dw_pre) return PCPP_OK;
    weight_sums_kernel<<<(unsigned)ceil_div(2 * a.c, 64), 1024, 0, stream>>>(a.part, blocks, a.c, a.dw_post, a.dw_pre);
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

}  // namespace pcpp
