// Group norm with an activation and dropout behind it, channels last, over the clouds of a batch; and its gradients.
//
//   over the rows of a cloud and the channels of a group:  v = (x - mean) rstd,  rstd = 1 / sqrt(mean (x - mean)^2 + eps)
//   forward    z = w v + b,  y = drop(act(z))
//   backward   dz = drop(dy) act'(z),  dw = sum dz v,  db = sum dz,  dx = rstd (w dz - m1 - v m2),
//              m1, m2 = means over the cloud's rows and the group's channels of w dz and of w dz v
//
// Rows are cut into chunks, whatever clouds they belong to; a block takes a chunk and in it one cloud after the other.  What it finds for
// (chunk i, cloud b) goes to slot i + b: along the rows either the chunk or the cloud goes on, so no two have the same slot.  So the host needs to know
// nothing of the clouds but their number, and every sum has one order.
//
// Statistics: a lane sums x - k and (x - k)^2, k the range's first row, which cannot lose what the variance is made of unless that row lies
// thousands of deviations off; channels, chunks and clouds are joined by their means and sums of squares about them.  x - mean is formed before anything
// is multiplied by it: a channel that is constant in its cloud has v = 0 whatever its size (with z = x (w rstd) + (b - mean w rstd) it was off by 2^-24
// mean rstd, with x = 1e5 and eps = 1e-5 by 2).
//
// Forward x is read twice, backward x and dy are, since nothing can be written before the last row of a cloud is known; the second pass goes from the
// end on, where the caches still have rows.  1 000 000 x 256 bf16 takes 316 us forward (1.5 GB moved at 4.9 TB/s) and 511 backward with dropout (2.6
// GB, 5.0 TB/s: memory, with the generator's and the activation's 43 000 vector instructions a wave for each pass beside it); 99 991 x 91 fp32 44
// backward (4.1 TB/s; three launches).  115 200 x 64 takes 27 forward where its bytes take 9: two kernels of 9.5 and 19.  Of the second about 8 are
// the vector instructions of gelu and dropout (2500 a wave), the rest a chain of the first loads and the statistics joined over 56 chunks, which two
// waves a SIMD do not hide (blocks of half and a quarter of the rows for it: as long, and 2 us more).
#include "pointwise.h"

namespace pcpp {

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;

// A lane's channels.  ALIKE: the groups are of whole eights, so a lane's eight channels are of one group and have one mean.
template <int LPR, int G, int MODE> struct Lane {
    int c0[G];
    Span<MODE> own[G];
    uint32_t row;                                                 // of the wave's rows
    __device__ inline explicit Lane(int c)
    {
        const int lane = threadIdx.x & 63;
        row = (uint32_t)(lane / LPR);
#pragma unroll
        for (int g = 0; g < G; ++g) c0[g] = 8 * (lane % LPR) + 8 * LPR * g, own[g] = Span<MODE>(c0[g], c);
    }
    template <typename T> __device__ inline uint32_t offset(int g, uint32_t row_at, int64_t pitch) const
    {
        return own[g].template offset<sizeof(T)>(row_at * (uint32_t)pitch);
    }
};
__device__ inline int wave_of() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

template <int G, int MODE>
__device__ inline void load_affine(const float *w, float without, const Span<MODE> (&own)[G], int c, float (&v)[G][8])
{
    const __amdgpu_buffer_rsrc_t rs = make_rsrc(w, w ? 4u * (uint32_t)c : 0u);
#pragma unroll
    for (int g = 0; g < G; ++g) {
        Eight<float> r;
        row_load<float>(rs, own[g].template offset<4>(0u), own[g], r);
        to_floats(r, v[g]);
        if (!w) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[g][e] = without;
        }
    }
}

// Which of the lane's elements stay; `at` is the lane's row in the tensor.  All lanes of a row call it.
template <int LPR, int G, int MODE>
__device__ inline void keep_bits(const Philox &philox, uint32_t at, int c, uint32_t threshold, const Lane<LPR, G, MODE> &lane, uint32_t (&bits)[G])
{
    const uint32_t first = at * (uint32_t)((c + 7) / 8);
#pragma unroll
    for (int g = 0; g < G; ++g) bits[g] = kept(philox, first + (uint32_t)lane.c0[g] / 8u, threshold);
    if constexpr (MODE == RAGGED) {
        // (some of the last eight channels are the lane before's)
        uint32_t before[G];
        const int l = threadIdx.x & 63;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            before[g] = __shfl_up(bits[g], 1);
            if (g > 0) {
                const uint32_t last = __shfl(bits[g > 0 ? g - 1 : 0], l + LPR - 1);
                before[g] = l % LPR == 0 ? last : before[g];
            }
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int lo = lane.own[g].lo;
            if (lo > 0 && lo < 8) bits[g] = before[g] >> (8 - lo) | bits[g] << lo;
        }
    }
}
// Zero for what goes (not scaled)
template <int LPR, int G, int MODE>
__device__ inline void drop_rows(const Philox &philox, uint32_t at, int c, const Drop &drop, const Lane<LPR, G, MODE> &lane, float (&v)[G][8])
{
    if constexpr (MODE == RAGGED) {
        uint32_t bits[G];
        keep_bits(philox, at, c, drop.threshold, lane, bits);
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[g][e] = bits[g] >> e & 1u ? v[g][e] : 0.f;
    } else {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            uint32_t x[4];
            philox.draw(at * (uint32_t)((c + 7) / 8) + (uint32_t)lane.c0[g] / 8u, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[g][e] = half_of(x, e) >= drop.threshold ? v[g][e] : 0.f;
        }
    }
}

// v over the lanes of a wave that hold the same channels of other rows: every LPR-th lane
template <int LPR> __device__ inline float rows_sum(float v)
{
    auto ring = [&](auto by) { v += __uint_as_float(dpp<DPP_ROR + decltype(by)::value>(__float_as_uint(v))); };
    if constexpr (LPR <= 4) ring(Int<4>{});
    if constexpr (LPR <= 8) ring(Int<8>{});
    if constexpr (LPR <= 16) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    if constexpr (LPR <= 32) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    return v;
}

// Two sums for every channel over the rows of a wave's lanes, then over the waves: [2][CP] in `total`.  (CP: channels in whole lanes)
template <int LPR, int G, int MODE, int CP>
__device__ inline void channel_sums(const float (&p)[G][8], const float (&q)[G][8], const Lane<LPR, G, MODE> &lane, int c, float (*sums)[2][CP], float (*total)[CP])
{
    const int l = threadIdx.x & 63, wave = wave_of();
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = rows_sum<LPR>(p[g][e]), b = rows_sum<LPR>(q[g][e]);
            if (l < LPR && lane.own[g].own(e)) {
                sums[wave][0][lane.own[g].at + e] = a;
                sums[wave][1][lane.own[g].at + e] = b;
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * c; i += THREADS) {
        const int which = i >= c, ch = which ? i - c : i;
        float v = sums[0][which][ch];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += sums[w][which][ch];
        total[which][ch] = v;
    }
    __syncthreads();
}

// v and that of the lane's partner, N neighbouring lanes having the same
template <int N> __device__ inline float lanes_sum(float v)
{
    if constexpr (N < 16) {
        constexpr int CTRL = N == 1 ? DPP_XOR1 : (N == 2 ? DPP_XOR2 : (N == 4 ? DPP_HALF_MIRROR : DPP_MIRROR));
        return v + __uint_as_float(dpp<CTRL>(__float_as_uint(v)));
    } else if constexpr (N == 16) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return __uint_as_float(p[0]) + __uint_as_float(p[1]);
    } else {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
}

// For every group f(group, lane among `per`, per, sum over those lanes, whether it is one) by neighbouring lanes of a wave
template <typename F> __device__ inline void for_groups(int groups, int width, F f)
{
    int per = 64;
    while (per > 1 && (per * groups > THREADS || per >= 2 * width)) per >>= 1;
    const int lane = (int)threadIdx.x % per;
    auto sum = [&](float v) {
        if (per >= 2) v = lanes_sum<1>(v);
        if (per >= 4) v = lanes_sum<2>(v);
        if (per >= 8) v = lanes_sum<4>(v);
        if (per >= 16) v = lanes_sum<8>(v);
        if (per >= 32) v = lanes_sum<16>(v);
        return per >= 64 ? lanes_sum<32>(v) : v;
    };
    for (int g0 = 0; g0 < groups; g0 += THREADS / per) {
        const int g = g0 + (int)threadIdx.x / per;                // (past the last: as the last, without an effect)
        f(g < groups ? g : groups - 1, lane, per, sum, g < groups);
    }
}

// Mean and sum of squares about it of every group over rows [lo, hi), not empty: f(group, mean, squares), by one thread each.
template <typename T, int LPR, int G, int MODE, int CP, typename F>
__device__ inline void range_statistics(const GroupNormArgs &a, int64_t lo, int64_t hi, const Lane<LPR, G, MODE> &lane, float (*sums)[2][CP], float (*total)[CP],
                                        float *shift, F f)
{
    constexpr int ROWS = 64 / LPR, STEP = WAVES * ROWS, AT_ONCE = sizeof(T) * G > 4 ? 2 : 4;
    const int c = a.c;
    float k[G][8], s[G][8], q[G][8];
    const __amdgpu_buffer_rsrc_t ks = rows_from<sizeof(T)>(a.x, lo, hi, a.ld_x, c, 1);
#pragma unroll
    for (int g = 0; g < G; ++g) {
        Eight<T> raw;
        row_load<T>(ks, lane.template offset<T>(g, 0u, 0), lane.own[g], raw);
        to_floats(raw, k[g]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[g][e] = q[g][e] = 0.f;
            if ((int)threadIdx.x < LPR && lane.own[g].own(e)) shift[lane.own[g].at + e] = k[g][e];
        }
    }
    for (int64_t first = lo + (int64_t)wave_of() * ROWS; first < hi; first += AT_ONCE * STEP) {
        const __amdgpu_buffer_rsrc_t xs = rows_from<sizeof(T)>(a.x, first, hi, a.ld_x, c, AT_ONCE * STEP);
        Eight<T> raw[AT_ONCE][G];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
            for (int g = 0; g < G; ++g) row_load<T>(xs, lane.template offset<T>(g, (uint32_t)(u * STEP) + lane.row, a.ld_x), lane.own[g], raw[u][g]);
        auto add = [&](auto all) {
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const bool live = decltype(all)::value || first + u * STEP + lane.row < hi;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    float v[8];
                    to_floats(raw[u][g], v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float d = live ? v[e] - k[g][e] : 0.f;
                        s[g][e] += d;
                        q[g][e] = __builtin_fmaf(d, d, q[g][e]);
                    }
                }
            }
        };
        if (first + (AT_ONCE - 1) * STEP + ROWS <= hi) add(Int<1>{});
        else add(Int<0>{});
    }
    channel_sums<LPR, G, MODE, CP>(s, q, lane, c, sums, total);
    const float rows = (float)(hi - lo), inv = 1.f / rows;
    for (int ch = threadIdx.x; ch < c; ch += THREADS) {
        const float sum = total[0][ch], off = sum * inv, m2 = total[1][ch] - sum * off;
        total[0][ch] = shift[ch] + off;
        total[1][ch] = m2 < 0.f ? 0.f : m2;                       // (a NaN stays)
    }
    __syncthreads();
    const int width = c / a.groups;
    for_groups(a.groups, width, [&](int group, int l, int per, auto sum, bool write) {
        float mean = 0.f, m2 = 0.f, about = 0.f;
        const float pivot = total[0][group * width];
        for (int i = l; i < width; i += per) {
            mean += total[0][group * width + i] - pivot;
            m2 += total[1][group * width + i];
        }
        mean = sum(mean) / (float)width;
        for (int i = l; i < width; i += per) {
            const float d = total[0][group * width + i] - pivot - mean;
            about = __builtin_fmaf(d, d, about);
        }
        m2 = sum(m2) + rows * sum(about);
        if (write && l == 0) f(group, pivot + mean, m2);
    });
    __syncthreads();                                              // (the sums are free again)
}

// One of the two numbers of a group for each of the lane's channels; pairs: [groups][2] of a cloud
template <bool ALIKE, int LPR, int G, int MODE>
__device__ inline void lane_pairs(const float *pairs, const Divisor &width, const Lane<LPR, G, MODE> &lane, float (&first)[G][ALIKE ? 1 : 8], float (&second)[G][ALIKE ? 1 : 8])
{
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < (ALIKE ? 1 : 8); ++e) {
            const bool there = lane.own[g].any() && (MODE != NARROW || e < lane.own[g].n);
            const uint32_t group = there ? width.quotient((uint32_t)(lane.own[g].at + e)) : 0u;
            first[g][e] = pairs[2u * group];
            second[g][e] = pairs[2u * group + 1u];
        }
}

// y of rows [lo, hi), not empty: z = (x - mean) by + b.  The weights and the first rows are on their way while `statistics` finds the cloud's, the next ones while some are
// written.
template <bool ALIKE, typename T, int LPR, int G, int MODE, typename F>
__device__ inline void apply_range(const GroupNormArgs &a, int64_t lo, int64_t hi, const Lane<LPR, G, MODE> &lane, const Divisor &width, const Philox &philox, F statistics)
{
    constexpr int ROWS = 64 / LPR, STEP = WAVES * ROWS, AT_ONCE = sizeof(T) * G > 4 ? 1 : 2;
    const int c = a.c;
    Eight<T> raw[AT_ONCE][G];
    auto load = [&](int64_t first, Eight<T> (&to)[AT_ONCE][G]) {
        if (first >= hi) return;
        const __amdgpu_buffer_rsrc_t xs = rows_from<sizeof(T)>(a.x, first, hi, a.ld_x, c, AT_ONCE * STEP);
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
            for (int g = 0; g < G; ++g) row_load<T>(xs, lane.template offset<T>(g, (uint32_t)(u * STEP) + lane.row, a.ld_x), lane.own[g], to[u][g]);
    };
    int64_t first = lo + (int64_t)wave_of() * ROWS;
    load(first, raw);
    float by[G][8], b[G][8], mean[G][ALIKE ? 1 : 8], rstd[G][ALIKE ? 1 : 8];
    load_affine(a.w, 1.f, lane.own, a.c, by);
    load_affine(a.b, 0.f, lane.own, a.c, b);
    lane_pairs<ALIKE>(statistics(), width, lane, mean, rstd);
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) by[g][e] *= rstd[g][ALIKE ? 0 : e];
    for (; first < hi; first += AT_ONCE * STEP) {
        Eight<T> next[AT_ONCE][G];
        load(first + AT_ONCE * STEP, next);
        const __amdgpu_buffer_rsrc_t ys = rows_from<sizeof(T)>(a.y, first, hi, c, c, AT_ONCE * STEP);
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const uint32_t row = (uint32_t)(u * STEP) + lane.row;
            float v[G][8];
#pragma unroll
            for (int g = 0; g < G; ++g) to_floats(raw[u][g], v[g]);
            as_act(a.act, [&](auto act) {
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[g][e] = activate<decltype(act)::value>(__builtin_fmaf(v[g][e] - mean[g][ALIKE ? 0 : e], by[g][e], b[g][e]));
            });
            if (a.drop.threshold) {
                drop_rows(philox, (uint32_t)first + row, c, a.drop, lane, v);
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[g][e] *= a.drop.scale;
            }
#pragma unroll
            for (int g = 0; g < G; ++g) row_store<T>(ys, lane.template offset<T>(g, row, c), lane.own[g], v[g]);
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
            for (int g = 0; g < G; ++g) raw[u][g] = next[u][g];
    }
}

// What the gradients' two passes know of a lane's channels.  v = (x - mean) rstd, z = (x - mean) by + b
template <bool ALIKE, int G> struct Known {
    float mean[G][ALIKE ? 1 : 8], rstd[G][ALIKE ? 1 : 8], by[G][8], b[G][8];
    template <int LPR, int MODE>
    __device__ inline void load(const GroupNormArgs &a, const Lane<LPR, G, MODE> &lane, const float *stats, const Divisor &width)
    {
        load_affine(a.w, 1.f, lane.own, a.c, by);
        load_affine(a.b, 0.f, lane.own, a.c, b);
        lane_pairs<ALIKE>(stats, width, lane, mean, rstd);
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) by[g][e] *= rstd[g][ALIKE ? 0 : e];
    }
};

// Rows of x and dy on their way
template <typename T, int G> struct Rows {
    Eight<T> x[G], dy[G];
    template <int LPR, int MODE>
    __device__ inline void load(const GroupNormArgs &a, int64_t first, int64_t hi, const Lane<LPR, G, MODE> &lane)
    {
        if (first >= hi) return;
        const __amdgpu_buffer_rsrc_t xs = rows_from<sizeof(T)>(a.x, first, hi, a.ld_x, a.c, 64 / LPR), ds = rows_from<sizeof(T)>(a.dy, first, hi, a.c, a.c, 64 / LPR);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            row_load<T>(xs, lane.template offset<T>(g, lane.row, a.ld_x), lane.own[g], x[g]);
            row_load<T>(ds, lane.template offset<T>(g, lane.row, a.c), lane.own[g], dy[g]);
        }
    }
    // x - mean and what flows to z, without the scale of the dropout, which is zero in rows past the last
    template <bool ALIKE, int LPR, int MODE>
    __device__ inline void gradient(const GroupNormArgs &a, const Known<ALIKE, G> &known, uint32_t at, const Lane<LPR, G, MODE> &lane, const Philox &philox, float (&xv)[G][8],
                                    float (&d)[G][8]) const
    {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            to_floats(x[g], xv[g]);
            to_floats(dy[g], d[g]);
        }
        if (a.drop.threshold) drop_rows(philox, at, a.c, a.drop, lane, d);
        as_act(a.act, [&](auto act) {
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    xv[g][e] -= known.mean[g][ALIKE ? 0 : e];
                    if constexpr (decltype(act)::value != PCPP_ACT_NONE) d[g][e] *= slope<decltype(act)::value>(__builtin_fmaf(xv[g][e], known.by[g][e], known.b[g][e]));
                }
        });
    }
};

// Sums of dz and dz v of every channel over rows [lo, hi), not empty: [2][CP] in `total`
template <bool ALIKE, typename T, int LPR, int G, int MODE, int CP>
__device__ inline void range_gradients(const GroupNormArgs &a, int64_t lo, int64_t hi, const Lane<LPR, G, MODE> &lane, const float *stats, const Divisor &width,
                                       const Philox &philox, float (*sums)[2][CP], float (*total)[CP])
{
    constexpr int ROWS = 64 / LPR, STEP = WAVES * ROWS;
    int64_t first = lo + (int64_t)wave_of() * ROWS;
    Rows<T, G> rows, next;                                        // (one on its way while the other is in use)
    rows.load(a, first, hi, lane);
    Known<ALIKE, G> known;
    known.load(a, lane, stats, width);
    float s[G][8], q[G][8];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[g][e] = q[g][e] = 0.f;
    for (; first < hi; first += STEP) {
        next.load(a, first + STEP, hi, lane);
        float x[G][8], d[G][8];
        rows.gradient(a, known, (uint32_t)first + lane.row, lane, philox, x, d);
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s[g][e] += d[g][e];
                q[g][e] = __builtin_fmaf(d[g][e], x[g][e], q[g][e]);
            }
        rows = next;
    }
    const float scale = a.drop.threshold ? a.drop.scale : 1.f;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[g][e] *= scale, q[g][e] *= scale * known.rstd[g][ALIKE ? 0 : e];
    channel_sums<LPR, G, MODE, CP>(s, q, lane, a.c, sums, total);
}

// m1 and m2 of every group of a cloud of `rows` rows from its channels' sums: [groups][2] in `coef`
template <int CP> __device__ inline void group_means(const GroupNormArgs &a, const float (*total)[CP], double rows, float *coef)
{
    const int width = a.c / a.groups;
    const float inv = (float)(1.0 / (rows * (double)width));
    for_groups(a.groups, width, [&](int group, int l, int per, auto sum, bool write) {
        float m1 = 0.f, m2 = 0.f;
        for (int i = group * width + l; i < (group + 1) * width; i += per) {
            const float w = a.w ? a.w[i] : 1.f;
            m1 = __builtin_fmaf(w, total[0][i], m1);
            m2 = __builtin_fmaf(w, total[1][i], m2);
        }
        m1 = sum(m1);
        m2 = sum(m2);
        if (write && l == 0) coef[2 * group] = m1 * inv, coef[2 * group + 1] = m2 * inv;
    });
    __syncthreads();
}

// dx of rows [lo, hi), not empty:  rstd (w dz - m1 - v m2) = dz (w rstd) + (x - mean) (-rstd^2 m2) - rstd m1.  `means` finds m1 and m2.
template <bool ALIKE, typename T, int LPR, int G, int MODE, typename F>
__device__ inline void gradient_range(const GroupNormArgs &a, int64_t lo, int64_t hi, const Lane<LPR, G, MODE> &lane, const float *stats, const Divisor &width,
                                      const Philox &philox, F means)
{
    constexpr int ROWS = 64 / LPR, STEP = WAVES * ROWS, N = ALIKE ? 1 : 8;
    int64_t first = lo + (int64_t)wave_of() * ROWS;
    Rows<T, G> rows, next;
    rows.load(a, first, hi, lane);
    Known<ALIKE, G> known;
    known.load(a, lane, stats, width);
    float m1[G][N], m2[G][N], of_d[G][8];
    lane_pairs<ALIKE>(means(), width, lane, m1, m2);
    const float scale = a.drop.threshold ? a.drop.scale : 1.f;
#pragma unroll
    for (int g = 0; g < G; ++g) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            m1[g][e] *= -known.rstd[g][e];
            m2[g][e] *= -known.rstd[g][e] * known.rstd[g][e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) of_d[g][e] = known.by[g][e] * scale;
    }
    for (; first < hi; first += STEP) {
        next.load(a, first + STEP, hi, lane);
        const __amdgpu_buffer_rsrc_t os = rows_from<sizeof(T)>(a.dx, first, hi, a.c, a.c, ROWS);
        float x[G][8], d[G][8];
        rows.gradient(a, known, (uint32_t)first + lane.row, lane, philox, x, d);
#pragma unroll
        for (int g = 0; g < G; ++g) {
#pragma unroll
            for (int e = 0; e < 8; ++e) d[g][e] = __builtin_fmaf(d[g][e], of_d[g][e], __builtin_fmaf(x[g][e], m2[g][ALIKE ? 0 : e], m1[g][ALIKE ? 0 : e]));
            row_store<T>(os, lane.template offset<T>(g, lane.row, a.c), lane.own[g], d[g]);
        }
        rows = next;
    }
}

// A chunk's rows and the clouds in it
struct Chunk {
    int64_t lo, hi;
    int first, last;
    __device__ inline Chunk(const WaveClouds &of, int64_t rows, int i)
    {
        const int64_t n = of.clouds.n;
        lo = (int64_t)i * rows;
        hi = lo + rows < n ? lo + rows : n;
        const int end = of.clouds.count - 1;                      // (rows behind the last cloud: it has none of them)
        first = of.at(lo), last = of.at(hi - 1);
        first = first < end ? first : end;
        last = last < end ? last : end;
    }
    __device__ inline bool range(const WaveClouds &clouds, int b, int64_t &from, int64_t &to) const
    {
        const int64_t f = clouds.first(b), e = clouds.end(b);
        from = f > lo ? f : lo;
        to = e < hi ? e : hi;
        return from < to;
    }
};

template <typename T, int LPR, int G, int MODE> __global__ __launch_bounds__(THREADS) void chunk_statistics_kernel(const GroupNormArgs a, int64_t rows)
{
    constexpr int CP = 8 * LPR * G;
    __shared__ float sums[WAVES][2][CP], total[2][CP], shift[CP];
    const WaveClouds clouds(Clouds{a.offsets, a.n_clouds, a.n});
    const Chunk chunk(clouds, rows, (int)blockIdx.x);
    const Lane<LPR, G, MODE> lane(a.c);
    for (int b = chunk.first; b <= chunk.last; ++b) {
        float *to = a.part + ((size_t)blockIdx.x + (size_t)b) * 2 * a.groups;
        int64_t lo, hi;
        if (!chunk.range(clouds, b, lo, hi)) continue;            // (nothing reads the slot)
        range_statistics<T, LPR, G, MODE, CP>(a, lo, hi, lane, sums, total, shift, [&](int g, float mean, float m2) { to[2 * g] = mean, to[2 * g + 1] = m2; });
    }
}

// Sums of a cloud's chunks' means and squares about a pivot
struct Joined {
    float s, q, m;
    __device__ inline void add(const GroupNormArgs &a, int64_t rows, int64_t lo, int64_t hi, const float *part, float pivot, int i)
    {
        const int64_t from = (int64_t)i * rows > lo ? (int64_t)i * rows : lo, to = (int64_t)(i + 1) * rows < hi ? (int64_t)(i + 1) * rows : hi;
        const float *at = part + (size_t)i * 2 * a.groups;
        const float cnt = (float)(to - from), d = at[0] - pivot;
        s = __builtin_fmaf(cnt, d, s);
        q = __builtin_fmaf(cnt * d, d, q);
        m += at[1];
    }
    __device__ inline void finish(const GroupNormArgs &a, int64_t rows_of_cloud, float pivot, float &mean, float &rstd) const
    {
        const float n = (float)rows_of_cloud, width = (float)(a.c / a.groups), off = s / n, between = q - s * off, m2 = m + width * (between < 0.f ? 0.f : between);
        mean = pivot + off;
        rstd = 1.f / sqrtf(m2 / (n * width) + a.eps);
    }
};

// The chunks of a cloud joined: a block takes sixteen groups, a thread every 64th chunk of one.
__global__ __launch_bounds__(1024) void cloud_statistics_kernel(const GroupNormArgs a, int64_t rows)
{
    __shared__ float sums[64][16][3];
    const Clouds clouds{a.offsets, a.n_clouds, a.n};
    const int b = (int)blockIdx.x, gl = threadIdx.x & 15, sl = threadIdx.x >> 4, group = (int)blockIdx.y * 16 + gl;
    const int64_t lo = clouds.first(b), hi = clouds.end(b);
    float *to = a.stats + ((size_t)b * a.groups + group) * 2;
    if (lo >= hi) {
        if (sl == 0 && group < a.groups) to[0] = to[1] = 0.f;
        return;
    }
    const int i0 = (int)(lo / rows), i1 = (int)((hi - 1) / rows);
    const float *part = a.part + ((size_t)b * a.groups + group) * 2;
    Joined v{0.f, 0.f, 0.f};
    float pivot = 0.f;
    if (group < a.groups) {
        pivot = part[(size_t)i0 * 2 * a.groups];
#pragma unroll 4
        for (int i = i0 + sl; i <= i1; i += 64) v.add(a, rows, lo, hi, part, pivot, i);
    }
    sums[sl][gl][0] = v.s;
    sums[sl][gl][1] = v.q;
    sums[sl][gl][2] = v.m;
    for (int step = 32; step > 0; step >>= 1) {
        __syncthreads();
        if (sl < step) {
#pragma unroll
            for (int k = 0; k < 3; ++k) sums[sl][gl][k] += sums[sl + step][gl][k];
        }
    }
    if (sl != 0 || group >= a.groups) return;
    float mean, rstd;
    Joined{sums[0][gl][0], sums[0][gl][1], sums[0][gl][2]}.finish(a, hi - lo, pivot, mean, rstd);
    to[0] = mean, to[1] = rstd;
}

// JOIN: every block joins the chunks of its clouds for itself, the first of a cloud writes the result
template <bool JOIN, bool ALIKE, typename T, int LPR, int G, int MODE>
__global__ __launch_bounds__(THREADS) void apply_kernel(const GroupNormArgs a, int64_t rows, const Divisor chunk_rows, const Divisor width)
{
    constexpr int CP = 8 * LPR * G;
    __shared__ float stats[JOIN ? 2 * CP : 1];
    const WaveClouds clouds(Clouds{a.offsets, a.n_clouds, a.n});
    const Chunk chunk(clouds, rows, (int)(gridDim.x - 1 - blockIdx.x));         // (from the end on: what was read last is still in the caches)
    const Lane<LPR, G, MODE> lane(a.c);
    const Philox philox(a.drop.random);
    if constexpr (JOIN) {
        if (blockIdx.x == 0)                                      // clouds without rows, which no chunk has
            for (int i = threadIdx.x; i < a.n_clouds; i += THREADS)
                if (clouds.clouds.first(i) >= clouds.clouds.end(i))
                    for (int k = 0; k < 2 * a.groups; ++k) a.stats[(size_t)i * 2 * a.groups + k] = 0.f;
    }
    for (int i = chunk.first; i <= chunk.last; ++i) {
        int64_t lo, hi;
        if (!chunk.range(clouds, i, lo, hi)) continue;
        apply_range<ALIKE, T>(a, lo, hi, lane, width, philox, [&]() -> const float * {
            if constexpr (!JOIN) return a.stats + (size_t)i * a.groups * 2;
            const int64_t first = clouds.first(i), end = clouds.end(i);
            const int i0 = (int)chunk_rows.quotient((uint32_t)first), i1 = (int)chunk_rows.quotient((uint32_t)(end - 1));
            __syncthreads();                                      // (the last cloud's are in use no more)
            for_groups(a.groups, i1 - i0 + 1, [&](int group, int l, int per, auto sum, bool write) {
                const float *part = a.part + ((size_t)i * a.groups + group) * 2;
                const float pivot = part[(size_t)i0 * 2 * a.groups];
                Joined v{0.f, 0.f, 0.f};
#pragma unroll 4
                for (int k = i0 + l; k <= i1; k += per) v.add(a, rows, first, end, part, pivot, k);
                v.s = sum(v.s), v.q = sum(v.q), v.m = sum(v.m);
                float mean, rstd;
                v.finish(a, end - first, pivot, mean, rstd);
                if (write && l == 0) {
                    stats[2 * group] = mean, stats[2 * group + 1] = rstd;
                    if (lo == first) a.stats[((size_t)i * a.groups + group) * 2] = mean, a.stats[((size_t)i * a.groups + group) * 2 + 1] = rstd;
                }
            });
            __syncthreads();
            return stats;
        });
    }
}

// Few rows: a block takes a cloud from its statistics to y.
template <typename T, int LPR, int G, int MODE> __global__ __launch_bounds__(THREADS) void small_forward_kernel(const GroupNormArgs a, const Divisor width)
{
    constexpr int CP = 8 * LPR * G;
    __shared__ float sums[WAVES][2][CP], total[2][CP], shift[CP], stats[2 * CP];
    const Clouds clouds{a.offsets, a.n_clouds, a.n};
    const Lane<LPR, G, MODE> lane(a.c);
    const Philox philox(a.drop.random);
    const int64_t lo = clouds.first((int)blockIdx.x), hi = clouds.end((int)blockIdx.x);
    float *to = a.stats ? a.stats + (size_t)blockIdx.x * a.groups * 2 : nullptr;
    if (lo >= hi) {
        if (to)
            for (int i = threadIdx.x; i < 2 * a.groups; i += THREADS) to[i] = 0.f;
        return;
    }
    const float count = (float)(hi - lo) * (float)(a.c / a.groups);
    range_statistics<T, LPR, G, MODE, CP>(a, lo, hi, lane, sums, total, shift, [&](int g, float mean, float m2) {
        const float rstd = 1.f / sqrtf(m2 / count + a.eps);
        stats[2 * g] = mean, stats[2 * g + 1] = rstd;
        if (to) to[2 * g] = mean, to[2 * g + 1] = rstd;
    });
    apply_range<false, T>(a, lo, hi, lane, width, philox, [&] { return stats; });
}

template <bool ALIKE, typename T, int LPR, int G, int MODE>
__global__ __launch_bounds__(THREADS) void chunk_gradients_kernel(const GroupNormArgs a, int64_t rows, const Divisor width)
{
    constexpr int CP = 8 * LPR * G;
    __shared__ float sums[WAVES][2][CP], total[2][CP];
    const WaveClouds clouds(Clouds{a.offsets, a.n_clouds, a.n});
    const Chunk chunk(clouds, rows, (int)blockIdx.x);
    const Lane<LPR, G, MODE> lane(a.c);
    const Philox philox(a.drop.random);
    for (int i = chunk.first; i <= chunk.last; ++i) {
        int64_t lo, hi;
        if (!chunk.range(clouds, i, lo, hi)) continue;            // (nothing reads the slot)
        range_gradients<ALIKE, T, LPR, G, MODE, CP>(a, lo, hi, lane, a.stats + (size_t)i * a.groups * 2, width, philox, sums, total);
        float *to = a.part + ((size_t)blockIdx.x + (size_t)i) * 2 * a.c;
        for (int k = threadIdx.x; k < 2 * a.c; k += THREADS) to[k] = total[k >= a.c][k >= a.c ? k - a.c : k];
        __syncthreads();
    }
}

// The chunks of a cloud summed, channel by channel, to a.coef [clouds][2][c]: a block takes sixteen columns, a thread every 64th chunk.
__global__ __launch_bounds__(1024) void cloud_gradients_kernel(const GroupNormArgs a, int64_t rows)
{
    __shared__ float sums[64][16];
    const Clouds clouds{a.offsets, a.n_clouds, a.n};
    const int b = (int)blockIdx.x, cl = threadIdx.x & 15, sl = threadIdx.x >> 4, column = (int)blockIdx.y * 16 + cl;
    const int64_t lo = clouds.first(b), hi = clouds.end(b);
    float v = 0.f;
    if (lo < hi && column < 2 * a.c) {
        const int i0 = (int)(lo / rows), i1 = (int)((hi - 1) / rows);
        const float *part = a.part + (size_t)b * 2 * a.c + column;
#pragma unroll 8
        for (int i = i0 + sl; i <= i1; i += 64) v += part[(size_t)i * 2 * a.c];
    }
    sums[sl][cl] = v;
    for (int step = 32; step > 0; step >>= 1) {
        __syncthreads();
        if (sl < step) sums[sl][cl] += sums[sl + step][cl];
    }
    if (sl == 0 && column < 2 * a.c) a.coef[(size_t)b * 2 * a.c + column] = sums[0][cl];
}

// dx, and in blocks behind the chunks' the weights' gradients: the clouds' sums joined, sixteen columns a block
template <bool ALIKE, typename T, int LPR, int G, int MODE>
__global__ __launch_bounds__(THREADS) void gradient_kernel(const GroupNormArgs a, int64_t rows, int chunks, const Divisor width)
{
    constexpr int CP = 8 * LPR * G;
    __shared__ float total[2][CP], coef[2 * CP], parts[16][16];
    const WaveClouds clouds(Clouds{a.offsets, a.n_clouds, a.n});
    if ((int)blockIdx.x >= chunks) {
        const int column = ((int)blockIdx.x - chunks) * 16 + (threadIdx.x & 15), sl = threadIdx.x >> 4;
        float v = 0.f;
        if (column < 2 * a.c) {
#pragma unroll 4
            for (int b = sl; b < a.n_clouds; b += 16) v += a.coef[(size_t)b * 2 * a.c + column];
        }
        parts[sl][threadIdx.x & 15] = v;
        __syncthreads();
        if (sl != 0 || column >= 2 * a.c) return;
        for (int i = 1; i < 16; ++i) v += parts[i][threadIdx.x & 15];
        float *to = column < a.c ? a.db : a.dw;                   // (sums of dz, sums of dz v)
        if (to) to[column < a.c ? column : column - a.c] = v;
        return;
    }
    const Chunk chunk(clouds, rows, chunks - 1 - (int)blockIdx.x);
    const Lane<LPR, G, MODE> lane(a.c);
    const Philox philox(a.drop.random);
    for (int i = chunk.first; i <= chunk.last; ++i) {
        int64_t lo, hi;
        if (!chunk.range(clouds, i, lo, hi)) continue;
        gradient_range<ALIKE, T>(a, lo, hi, lane, a.stats + (size_t)i * a.groups * 2, width, philox, [&] {
            const float *from = a.coef + (size_t)i * 2 * a.c;
            for (int k = threadIdx.x; k < 2 * a.c; k += THREADS) total[k >= a.c][k >= a.c ? k - a.c : k] = from[k];
            __syncthreads();
            group_means<CP>(a, total, (double)(clouds.end(i) - clouds.first(i)), coef);
            return coef;
        });
        __syncthreads();
    }
}

// Few rows: a block takes a cloud.  The weights' gradients are written by the only one or, of several clouds, joined by gradient_kernel's last blocks.
template <typename T, int LPR, int G, int MODE> __global__ __launch_bounds__(THREADS) void small_backward_kernel(const GroupNormArgs a, const Divisor width)
{
    constexpr int CP = 8 * LPR * G;
    __shared__ float sums[WAVES][2][CP], total[2][CP], coef[2 * CP];
    const Clouds clouds{a.offsets, a.n_clouds, a.n};
    const Lane<LPR, G, MODE> lane(a.c);
    const Philox philox(a.drop.random);
    const int64_t lo = clouds.first((int)blockIdx.x), hi = clouds.end((int)blockIdx.x);
    const float *stats = a.stats + (size_t)blockIdx.x * a.groups * 2;
    if (lo < hi) {
        range_gradients<false, T, LPR, G, MODE, CP>(a, lo, hi, lane, stats, width, philox, sums, total);
        if (a.dx) {
            gradient_range<false, T>(a, lo, hi, lane, stats, width, philox, [&] {
                group_means<CP>(a, total, (double)(hi - lo), coef);
                return coef;
            });
        }
    }
    for (int k = threadIdx.x; k < 2 * a.c; k += THREADS) {
        const int which = k >= a.c, ch = which ? k - a.c : k;
        const float v = lo < hi ? total[which][ch] : 0.f;
        float *only = which ? a.dw : a.db;
        if (a.n_clouds > 1) a.coef[(size_t)blockIdx.x * 2 * a.c + k] = v;
        else if (only) only[ch] = v;
    }
}

template <typename F> void with_kernel(int dtype, int c, F f)
{
    with_rows(c, [&](auto lpr, auto g, auto mode) { dtype == PCPP_F32 ? f(float{}, lpr, g, mode) : f(bf16_t{}, lpr, g, mode); });
}
// ... and whether a lane's channels are of one group
template <typename F> void with_kernel(int dtype, int c, int groups, F f)
{
    with_kernel(dtype, c, [&](auto t, auto lpr, auto g, auto mode) {
        if constexpr (decltype(mode)::value == WHOLE) {
            if (c / groups % 8 == 0) return f(t, lpr, g, mode, Int<1>{});
        }
        f(t, lpr, g, mode, Int<0>{});
    });
}

int64_t rows_at_once(int c) { return WAVES * 64 / row_lanes(c); }
// A block to a cloud, from its statistics to its rows, in place of passes over chunks: where a cloud has ten steps of a block or fewer on average.
// (256 x 64 of one cloud, eight steps: 8.1 us forward and 12.8 backward, by chunks 10.0 and 14.3; 1000 x 16, sixteen: 11.0 and 19.9, 10.6 and 15.3.
// Eighty steps in all at most, for clouds of very different sizes.)
bool block_a_cloud(int64_t n, int c, int n_clouds)
{
    const int64_t steps = ceil_div(n, rows_at_once(c));
    return steps <= 80 && steps <= 10 * (int64_t)n_clouds;
}
// Whether the blocks that write y join the chunks' statistics for themselves: that saves a launch and costs each a read of their clouds' (8 groups,
// 115 200 x 64 of one cloud: 19.4 us for 20.7; 16 groups 23.7 for 21.6; 30 000 x 64, 235 chunks of 16 groups: 13.6 for 15.0).  All chunks count, as if
// one cloud had them; of several clouds, whose blocks read less, some take the launch that need not.
bool join_in_place(const GroupNormSizes &s, int groups) { return (int64_t)s.chunks * groups <= 4096; }

}  // namespace

// part: what the blocks find, for every slot; extra: forward the statistics where the caller does not want them, backward the clouds' sums
GroupNormSizes group_norm_sizes(int64_t n, int c, int n_clouds, int groups, bool backward)
{
    GroupNormSizes s{};
    const int64_t step = rows_at_once(c);
    // (two blocks for each CU; four make 5 of 43 us more of 99 991 x 91, one takes a third more of 1 000 000 x 256.  More for very many clouds, which
    // a block takes one by one.)
    const int64_t most = n_clouds > 512 ? n_clouds : 512, of_cloud = ceil_div(ceil_div(n, n_clouds), step), least = of_cloud < 4 ? (of_cloud > 1 ? of_cloud : 1) : 4;
    s.rows = ceil_div(ceil_div(n, most), step) * step;
    if (s.rows < least * step) s.rows = least * step;
    s.chunks = (int)ceil_div(n > 0 ? n : 1, s.rows);
    s.slots = (size_t)s.chunks + (size_t)n_clouds - 1;
    const bool small = block_a_cloud(n, c, n_clouds);
    s.part = small ? 0 : align_up(s.slots * 2 * (size_t)(backward ? c : groups) * sizeof(float));
    s.extra = small && !(backward && n_clouds > 1) ? 0 : align_up((size_t)n_clouds * 2 * (size_t)(backward ? c : groups) * sizeof(float));
    s.bytes = s.part + s.extra;
    return s;
}

int group_norm_fwd(const GroupNormArgs &a, int dtype, hipStream_t stream)
{
    const Divisor width = make_divisor((uint32_t)(a.c / a.groups));
    if (block_a_cloud(a.n, a.c, a.n_clouds)) {
        with_kernel(dtype, a.c, [&](auto t, auto lpr, auto g, auto mode) {
            small_forward_kernel<decltype(t), decltype(lpr)::value, decltype(g)::value, decltype(mode)::value><<<(unsigned)a.n_clouds, THREADS, 0, stream>>>(a, width);
        });
        PCPP_HIP_CHECK(hipGetLastError());
        return PCPP_OK;
    }
    const GroupNormSizes s = group_norm_sizes(a.n, a.c, a.n_clouds, a.groups, false);
    const bool join = join_in_place(s, a.groups);
    with_kernel(dtype, a.c, [&](auto t, auto lpr, auto g, auto mode) {
        chunk_statistics_kernel<decltype(t), decltype(lpr)::value, decltype(g)::value, decltype(mode)::value>
            <<<(unsigned)s.chunks, THREADS, 0, stream>>>(a, s.rows);
    });
    PCPP_HIP_CHECK(hipGetLastError());
    if (!join) {
        cloud_statistics_kernel<<<dim3((unsigned)a.n_clouds, (unsigned)ceil_div(a.groups, 16)), 1024, 0, stream>>>(a, s.rows);
        PCPP_HIP_CHECK(hipGetLastError());
    }
    with_kernel(dtype, a.c, a.groups, [&](auto t, auto lpr, auto g, auto mode, auto alike) {
        constexpr int LPR = decltype(lpr)::value, G = decltype(g)::value, MODE = decltype(mode)::value;
        constexpr bool ALIKE = decltype(alike)::value;
        if (join) apply_kernel<true, ALIKE, decltype(t), LPR, G, MODE><<<(unsigned)s.chunks, THREADS, 0, stream>>>(a, s.rows, make_divisor((uint32_t)s.rows), width);
        else apply_kernel<false, ALIKE, decltype(t), LPR, G, MODE><<<(unsigned)s.chunks, THREADS, 0, stream>>>(a, s.rows, make_divisor((uint32_t)s.rows), width);
    });
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

int group_norm_bwd(const GroupNormArgs &a, int dtype, hipStream_t stream)
{
    const Divisor width = make_divisor((uint32_t)(a.c / a.groups));
    const int sums = a.dw || a.db ? (int)ceil_div(2 * a.c, 16) : 0;
    if (block_a_cloud(a.n, a.c, a.n_clouds)) {
        with_kernel(dtype, a.c, [&](auto t, auto lpr, auto g, auto mode) {
            small_backward_kernel<decltype(t), decltype(lpr)::value, decltype(g)::value, decltype(mode)::value><<<(unsigned)a.n_clouds, THREADS, 0, stream>>>(a, width);
        });
        PCPP_HIP_CHECK(hipGetLastError());
        if (sums && a.n_clouds > 1) {
            with_kernel(dtype, a.c, [&](auto t, auto lpr, auto g, auto mode) {
                gradient_kernel<false, decltype(t), decltype(lpr)::value, decltype(g)::value, decltype(mode)::value><<<(unsigned)sums, THREADS, 0, stream>>>(a, 0, 0, width);
            });
            PCPP_HIP_CHECK(hipGetLastError());
        }
        return PCPP_OK;
    }
    const GroupNormSizes s = group_norm_sizes(a.n, a.c, a.n_clouds, a.groups, true);
    with_kernel(dtype, a.c, a.groups, [&](auto t, auto lpr, auto g, auto mode, auto alike) {
        chunk_gradients_kernel<(bool)decltype(alike)::value, decltype(t), decltype(lpr)::value, decltype(g)::value, decltype(mode)::value>
            <<<(unsigned)s.chunks, THREADS, 0, stream>>>(a, s.rows, width);
    });
    PCPP_HIP_CHECK(hipGetLastError());
    cloud_gradients_kernel<<<dim3((unsigned)a.n_clouds, (unsigned)ceil_div(2 * a.c, 16)), 1024, 0, stream>>>(a, s.rows);
    PCPP_HIP_CHECK(hipGetLastError());
    const int chunks = a.dx ? s.chunks : 0;
    with_kernel(dtype, a.c, a.groups, [&](auto t, auto lpr, auto g, auto mode, auto alike) {
        gradient_kernel<(bool)decltype(alike)::value, decltype(t), decltype(lpr)::value, decltype(g)::value, decltype(mode)::value>
            <<<(unsigned)(chunks + sums), THREADS, 0, stream>>>(a, s.rows, chunks, width);
    });
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

}  // namespace pcpp
