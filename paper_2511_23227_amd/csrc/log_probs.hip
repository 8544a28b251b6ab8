// Log probabilities of given classes, entropy and the most probable classes of every row of logits, and the gradient of the logits.
//
//   m = max x, S = sum exp(x - m), T = sum exp(x - m) (x - m)        one pass over the row, in 32 bits; when the maximum grows by g,
//                                                                     S and T become S exp(-g) and exp(-g) (T - g S)
//   log p_j = (x_j - m) - log S,  entropy = log S - T / S             (m and log S apart: their sum would lose log S beside a large m)
//   d_j = d_log_prob (1[j = label] - p_j) - d_entropy p_j (log p_j + entropy)
//
// A masked class has x = -inf (or the type's lowest value): its terms are zero.  A row without any class has log probabilities -inf,
// entropy 0 and no gradient.  A row that holds a NaN or +inf has NaN everywhere but in its indices.
//
// Bound by memory, and in bf16 nearly as much by the exponentials.  Rows of up to 512 classes lie in the registers of a few lanes;
// longer ones are walked by a thread block, or, where there are few rows, by several, whose sums a second kernel joins.
// The most probable classes are kept as a list, sorted over the lanes of a wave, of 64-bit keys: the value in an order-preserving
// form above the complement of the index, so that of equal values the lowest index is the largest key.  Hardly any element of a long
// row passes the list's last entry, and only one that does costs more than the comparison.

#include "log_probs.h"
#include "row_ops.h"

namespace pcpp {

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int64_t MAX_BLOCKS = 1 << 22;                            // (a grid has fewer than 2^32 threads)
constexpr int SMALL = 512;                                        // classes of the rows that lie in registers
constexpr float LOG2E = 1.44269504f;
typedef unsigned long long key_t64;

__device__ inline float exp_of(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }

// A logarithm of a probability beside the probability, in products of the two: below -104 the probability is zero, and so has the product to
// be, for -inf too.
__device__ inline float bounded(float log_p) { return fmaxf(log_p, -1e4f); }

__device__ inline uint32_t ordered(float x)                       // same order as the values; -0 is 0, a NaN is -inf
{
    const uint32_t b = __float_as_uint(x != x ? -__builtin_inff() : x + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ inline float from_ordered(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? o ^ 0x80000000u : ~o); }
__device__ inline key_t64 key_of(float x, uint32_t index) { return (key_t64)ordered(x) << 32 | (uint32_t)~index; }
__device__ inline uint32_t key_index(key_t64 k) { return ~(uint32_t)k; }
__device__ inline float key_value(key_t64 k) { return from_ordered((uint32_t)(k >> 32)); }

__device__ inline key_t64 lane_of(key_t64 k, int lane)
{
    return (key_t64)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)k, lane);
}

template <int D> __device__ inline uint32_t lane_xor(uint32_t v, int lane)   // the value of lane ^ D
{
    if constexpr (D == 1) return dpp<DPP_XOR1>(v);
    if constexpr (D == 2) return dpp<DPP_XOR2>(v);
    if constexpr (D == 4) return dpp<DPP_XOR3>(dpp<DPP_HALF_MIRROR>(v));              // xor 7, then xor 3
    if constexpr (D == 8) return dpp<DPP_ROR + 8>(v);                                   // rotation of sixteen lanes by eight
    if constexpr (D == 16) {
        const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return (lane & 16) ? p[0] : p[1];
    }
    if constexpr (D == 32) {
        const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return (lane & 32) ? p[0] : p[1];
    }
    return v;
}
template <int D> __device__ inline key_t64 lane_xor(key_t64 k, int lane)
{
    return (key_t64)lane_xor<D>((uint32_t)(k >> 32), lane) << 32 | lane_xor<D>((uint32_t)k, lane);
}
// The larger of the pair (lane, lane ^ D) to its lower lane, or to its upper one where `up`.  (K: keys of 32 or 64 bits)
template <int D, typename K> __device__ inline K exchange(K k, int lane, bool up)
{
    const K o = lane_xor<D>(k, lane);
    return ((lane & D) != 0) == up ? (k > o ? k : o) : (k > o ? o : k);
}
// lanes' keys that rise and then fall (or the other way round), into descending order
template <typename K> __device__ inline K bitonic_merge(K k, int lane)
{
    k = exchange<32>(k, lane, false);
    k = exchange<16>(k, lane, false);
    k = exchange<8>(k, lane, false);
    k = exchange<4>(k, lane, false);
    k = exchange<2>(k, lane, false);
    return exchange<1>(k, lane, false);
}
template <typename K> __device__ inline K sort_lanes(K k, int lane)               // any keys, into descending order
{
    bool up = lane & 2;
    k = exchange<1>(k, lane, up);
    up = lane & 4;
    k = exchange<1>(exchange<2>(k, lane, up), lane, up);
    up = lane & 8;
    k = exchange<1>(exchange<2>(exchange<4>(k, lane, up), lane, up), lane, up);
    up = lane & 16;
    k = exchange<1>(exchange<2>(exchange<4>(exchange<8>(k, lane, up), lane, up), lane, up), lane, up);
    up = lane & 32;
    k = exchange<1>(exchange<2>(exchange<4>(exchange<8>(exchange<16>(k, lane, up), lane, up), lane, up), lane, up), lane, up);
    return bitonic_merge(k, lane);
}
// the 64 largest of two lists in descending order
__device__ inline key_t64 merge_lists(key_t64 a, key_t64 b, int lane)
{
    b = lane_xor<32>(lane_xor<16>((key_t64)dpp<DPP_MIRROR>((uint32_t)(b >> 32)) << 32 | dpp<DPP_MIRROR>((uint32_t)b), lane), lane);
    return bitonic_merge(a > b ? a : b, lane);
}

// The largest keys seen by a wave: lane j holds the (j + 1)-th, 0 where there are fewer.
struct TopList {
    key_t64 mine = 0, last = 0;                                   // last: keys up to it do not belong to the n_top largest
    int n_top;
    __device__ inline void insert(key_t64 k, int lane)            // k: the same in all lanes, larger than `last`
    {
        const int at = __popcll(__ballot(mine > k));
        const key_t64 before = (key_t64)dpp<0x138>((uint32_t)(mine >> 32)) << 32 | dpp<0x138>((uint32_t)mine);   // of the lane before
        mine = lane < at ? mine : (lane == at ? k : before);
        const key_t64 l = lane_of(mine, n_top - 1);
        if (l > last) last = l;
    }
    // A bound in front of the first offers, from every lane's largest value: the n_top-th largest of these is reached by n_top keys, so that
    // hardly more than n_top of the first keys are candidates.
    __device__ inline void expect(float largest, int lane)
    {
        const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)sort_lanes(ordered(largest), lane), n_top - 1);
        if (o > ordered(-__builtin_inff())) raise((key_t64)o << 32);
    }
    __device__ inline void raise(key_t64 reached)                 // n_top keys of the row reach it
    {
        if (reached > last) last = reached - 1;
    }
    // Several values of every lane at once; mask(e): the lanes whose value v[e] may belong, index(e): its class.  A few are put into the list
    // one by one; more are gathered 64 at a time (`room`: 64 keys of LDS, the wave's own), sorted and merged, 28 exchanges of lanes for 64, where
    // one insertion takes as long as three.
    template <int N, typename Mask, typename Index>
    __device__ inline void offer(const float (&v)[N], Mask mask, Index index, key_t64 *room, int lane)
    {
        int n = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) n += __popcll(mask(e));
        if (n <= 6) {
#pragma unroll
            for (int e = 0; e < N; ++e)
                for (key_t64 left = mask(e); left; left &= left - 1) {
                    const int from = __ffsll((long long)left) - 1;
                    const key_t64 k = key_of(__uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v[e]), from)),
                                             (uint32_t)__builtin_amdgcn_readlane((int)index(e), from));
                    if (k > last) insert(k, lane);
                }
            return;
        }
        n = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const key_t64 all = mask(e);
            if (!all) continue;
            const key_t64 k = key_of(v[e], index(e));
            bool in = (all >> lane & 1) && k > last;
            key_t64 m = __ballot(in);
            if (n + __popcll(m) > 64) {
                merge(room, n, lane);
                n = 0;
                in = in && k > last;
                m = __ballot(in);
            }
            if (in) room[n + __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u))] = k;
            n += __popcll(m);
        }
        merge(room, n, lane);
    }
    __device__ inline void merge(const key_t64 *room, int n, int lane)
    {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");    // (the lanes' writes before the reads, and these before the next writes)
        __builtin_amdgcn_wave_barrier();
        const key_t64 k = lane < n ? room[lane] : 0;
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        mine = merge_lists(mine, sort_lanes(k, lane), lane);
        const key_t64 l = lane_of(mine, n_top - 1);
        if (l > last) last = l;
    }
};

// sums of a part of a row
struct Sums {
    float m, s, t;
    __device__ inline void join(float om, float os, float ot)
    {
        const float nm = fmaxf(m, om);
        if (nm == -__builtin_inff()) {                            // no class on either side (a NaN is kept)
            s += os;
            return;
        }
        const float a = bounded(m - nm), b = bounded(om - nm), ea = exp_of(a), eb = exp_of(b);
        t = ea * (t + a * s) + eb * (ot + b * os);
        s = ea * s + eb * os;
        m = nm;
    }
};
__device__ inline Sums join_lanes(Sums v, int lanes)
{
    for (int d = 1; d < lanes; d <<= 1) {
        const float om = __shfl_xor(v.m, d), os = __shfl_xor(v.s, d), ot = __shfl_xor(v.t, d);
        v.join(om, os, ot);
    }
    return v;
}

// what a row's sums say; NaN in S reaches everything
__device__ inline float row_results(const LogProbsFwd &a, int64_t row, const Sums &v, float x_label, bool labelled)
{
    const bool empty = v.s == 0.f;
    const float log_s = __builtin_amdgcn_logf(v.s) * 0.693147181f;
    if (a.max_log_sum) *reinterpret_cast<float2 *>(a.max_log_sum + 2 * row) = float2{v.m, empty ? 0.f : log_s};
    if (a.entropy) a.entropy[row] = empty ? 0.f : log_s - v.t / v.s;
    if (a.log_prob) {
        const float lp = empty ? -__builtin_inff() : (x_label - v.m) - log_s;
        a.log_prob[row] = labelled ? lp : 0.f;
    }
    return log_s;
}
__device__ inline float top_value(const Sums &v, float x, float log_s) { return v.s == 0.f ? -__builtin_inff() : (x - v.m) - log_s; }

// op over the LPR lanes of a row, the same in all of them
template <int LPR, typename Op> __device__ inline uint32_t row_best(uint32_t v, Op op)
{
    return __float_as_uint(row_reduce<LPR>(__uint_as_float(v), [&](float a, float b) { return __uint_as_float(op(__float_as_uint(a), __float_as_uint(b))); }));
}

// ---- rows in registers: LPR lanes a row, lane l holding the classes l + LPR e ------------------------------------------------
template <typename T, int LPR>
__global__ __launch_bounds__(THREADS) void small_fwd_kernel(const LogProbsFwd a)
{
    constexpr int ROWS = THREADS / LPR, E = 8;
    const int l = (int)threadIdx.x % LPR;
    const int v = (int)a.v;
    // (a row's lanes leave together)
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR; row < a.n; row += (int64_t)gridDim.x * ROWS) {
        const T *x = static_cast<const T *>(a.logits) + row * a.ld;
        float xs[E];
#pragma unroll
        for (int e = 0; e < E; ++e) xs[e] = l + LPR * e < v ? one_float<T>(x[l + LPR * e]) : -__builtin_inff();
        const int label = a.labels ? a.labels[row] : -1;
        const bool labelled = label >= 0 && label < v;
        Sums u{-__builtin_inff(), 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < E; ++e) u.m = fmaxf(u.m, xs[e]);
        u.m = row_max<LPR>(u.m);
        const float m0 = u.m == -__builtin_inff() ? 0.f : u.m;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float d = xs[e] - m0, p = exp_of(d);
            u.s += p;
            u.t = __builtin_fmaf(p, bounded(d), u.t);
        }
        u.s = row_sum<LPR>(u.s);
        u.t = row_sum<LPR>(u.t);
        if (l == 0) row_results(a, row, u, labelled ? one_float<T>(x[label]) : 0.f, labelled);
        const float log_s = __builtin_amdgcn_logf(u.s) * 0.693147181f;
        // one class after the other: the largest of the lane's, then of the row's lanes; of equal ones the lowest index
        if (a.n_top == 0) continue;
        uint32_t value[E], mine = 0u, at = 0u;                     // 0: no class, or taken already; at: class of the lane's largest
#pragma unroll
        for (int e = 0; e < E; ++e) {
            value[e] = l + LPR * e < v ? ordered(xs[e]) : 0u;
            if (value[e] > mine) mine = value[e], at = (uint32_t)(l + LPR * e);
        }
        for (int k = 0; k < a.n_top; ++k) {
            const uint32_t best = row_best<LPR>(mine, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
            const uint32_t index = row_best<LPR>(mine == best ? at : ~0u, [](uint32_t p, uint32_t q) { return p < q ? p : q; });
            if (at == index && mine == best) {                     // (one lane)
                a.top_log_prob[row * a.n_top + k] = top_value(u, from_ordered(best), log_s);
                a.top_index[row * a.n_top + k] = (int32_t)index;
                mine = 0u;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if ((uint32_t)(l + LPR * e) == index) value[e] = 0u;
                    if (value[e] > mine) mine = value[e], at = (uint32_t)(l + LPR * e);
                }
            }
        }
    }
}

// ---- long rows ------------------------------------------------------------------------------------------------------------
// Classes [from, to) of a row by a thread block.  A lane takes twice eight classes a step, and has the next step's on their way meanwhile.
constexpr int DEEP = 2;

// the lane's classes at + 512 j .. at + 512 j + 7 as they lie in memory, -inf behind the end
// ONCE: by way of no cache
template <typename T, bool ONCE> __device__ inline void load_step(const T *x, int64_t at, int64_t to, Eight<T> (&r)[DEEP])
{
    constexpr uint32_t NOTHING = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
#pragma unroll
    for (int j = 0; j < DEEP; ++j) {
        const int64_t p = at + 512 * j;
        if (p + 8 <= to) {
            load_eight<ONCE>(x + p, r[j]);
        } else {
#pragma unroll
            for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r[j].a[i] = v4u{NOTHING, NOTHING, NOTHING, NOTHING};
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (p + e < to) {
                    if constexpr (sizeof(T) == 4) r[j].a[e >> 2][e & 3] = __float_as_uint(x[p + e]);
                    else r[j].a[0][e >> 1] = (e & 1) ? (r[j].a[0][e >> 1] & 0xffffu) | (uint32_t)x[p + e] << 16 : 0xff800000u | x[p + e];
                }
        }
    }
}

// reached: LDS of the block, the largest key so far that n_top keys of one of its waves reach; zero at the start
template <typename T, bool TOP, bool ONCE>
__device__ inline void walk(const T *x, int64_t from, int64_t to, Sums &u, TopList &list, key_t64 *room, key_t64 *reached, int lane, int wave)
{
    constexpr int N = 8 * DEEP, WAVE = 64 * N;
    u = Sums{-__builtin_inff(), 0.f, 0.f};
    // (the wave goes round together, so that the list sees all lanes)
    int64_t base = from + wave * WAVE;
    Eight<T> r[DEEP];
    if (base < to) load_step<T, ONCE>(x, base + lane * 8, to, r);
    for (; base < to; base += WAVES * WAVE) {
        const int64_t at = base + lane * 8;
        float v[N];
#pragma unroll
        for (int j = 0; j < DEEP; ++j) to_floats(r[j], *reinterpret_cast<float (*)[8]>(v + 8 * j));
        if (base + WAVES * WAVE < to) load_step<T, ONCE>(x, at + WAVES * WAVE, to, r);
        const key_t64 others = TOP ? *reinterpret_cast<volatile key_t64 *>(reached) : 0;
        float m = v[0];
#pragma unroll
        for (int e = 1; e < N; ++e) m = fmaxf(m, v[e]);
        if (m > u.m) {
            if (u.m > -__builtin_inff()) {
                const float g = bounded(u.m - m), a = exp_of(g);
                u.t = a * (u.t + g * u.s);
                u.s *= a;
            }
            u.m = m;
        }
        const float m0 = u.m == -__builtin_inff() ? 0.f : u.m;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float d = v[e] - m0, p = exp_of(d);
            u.s += p;
            u.t = __builtin_fmaf(p, bounded(d), u.t);
        }
        if (!TOP) continue;
        list.raise((key_t64)(uint32_t)__builtin_amdgcn_readfirstlane((int)(others >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)others));
        if (list.last == 0) list.expect(m, lane);
        const float bound = list.last ? key_value(list.last) : -__builtin_inff();
        if (!__ballot(!(m < bound))) continue;
        const key_t64 before = list.last;
        list.offer(v, [&](int e) { return __ballot(!(v[e] < bound) && at + 512 * (e / 8) + e % 8 < to); },
                   [&](int e) { return (uint32_t)(at + 512 * (e / 8) + e % 8); }, room, lane);
        if (list.last > before && lane == 0) atomicMax(reached, list.last);
    }
}

struct Partial { float m, s, t, unused; };

// The sums and lists of a block's N waves (a power of two), pair by pair; both end in wave 0.
template <int N, bool TOP>
__device__ inline void join_waves(Sums &u, TopList &list, Sums *sums, key_t64 (*keys)[64], int lane, int wave)
{
    u = join_lanes(u, 64);
    if (lane == 0) sums[wave] = u;
    if (TOP) keys[wave][lane] = list.mine;
    __syncthreads();
    if (wave == 0) {
        u = join_lanes(sums[lane % N], N);                         // (in all lanes)
    }
    if (TOP) {
#pragma unroll
        for (int half = N / 2; half > 0; half >>= 1) {
            if (wave < half) {
                list.mine = merge_lists(list.mine, keys[wave + half][lane], lane);
                keys[wave][lane] = list.mine;
            }
            if (half > 1) __syncthreads();
        }
    }
}

__device__ inline void store_top(const LogProbsFwd &a, int64_t row, const Sums &u, const TopList &list, float log_s, int lane)
{
    if (lane >= a.n_top) return;
    a.top_log_prob[row * a.n_top + lane] = top_value(u, key_value(list.mine), log_s);
    a.top_index[row * a.n_top + lane] = (int32_t)key_index(list.mine);
}

template <typename T, bool TOP, bool ONCE>
__global__ __launch_bounds__(THREADS) void long_fwd_kernel(const LogProbsFwd a, int splits, int64_t per, Partial *parts, key_t64 *keys)
{
    __shared__ Sums wave_sums[WAVES];
    __shared__ key_t64 wave_keys[TOP ? WAVES : 1][64], room[TOP ? WAVES : 1][64], reached;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    for (int64_t block = blockIdx.x; block < a.n * splits; block += gridDim.x) {
        const int64_t row = block / splits;
        const int split = (int)(block % splits);
        const T *x = static_cast<const T *>(a.logits) + row * a.ld;
        const int64_t from = split * per, to = from + per < a.v ? from + per : a.v;
        Sums u;
        TopList list;
        list.n_top = a.n_top;
        if (TOP) {
            if (threadIdx.x == 0) reached = 0;
            __syncthreads();
        }
        walk<T, TOP, ONCE>(x, from, to, u, list, room[TOP ? wave : 0], &reached, lane, wave);
        join_waves<WAVES, TOP>(u, list, wave_sums, wave_keys, lane, wave);
        if (wave == 0 && splits == 1) {
            const int64_t label = a.labels ? a.labels[row] : -1;
            const bool labelled = label >= 0 && label < a.v;
            const float log_s = __builtin_amdgcn_logf(u.s) * 0.693147181f;
            if (lane == 0) row_results(a, row, u, labelled ? one_float<T>(x[label]) : 0.f, labelled);
            if (TOP) store_top(a, row, u, list, log_s, lane);
        } else if (wave == 0) {
            if (lane == 0) parts[block] = Partial{u.m, u.s, u.t, 0.f};
            if (TOP && lane < a.n_top) keys[block * a.n_top + lane] = list.mine;      // (0 past the end of a short list)
        }
        __syncthreads();                                           // (the next row's sums go where these lay)
    }
}

// One block a row: the sums and lists of its splits, the lists by the waves in turn, then pair by pair.
constexpr int JOIN_WAVES = 16;
template <typename T, bool TOP>
__global__ __launch_bounds__(JOIN_WAVES * 64) void join_fwd_kernel(const LogProbsFwd a, int splits, const Partial *parts, const key_t64 *keys)
{
    __shared__ Sums wave_sums[JOIN_WAVES];
    __shared__ key_t64 wave_keys[TOP ? JOIN_WAVES : 1][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t row = blockIdx.x;                               // (few rows: they were split)
    const T *x = static_cast<const T *>(a.logits) + row * a.ld;
    Sums u{-__builtin_inff(), 0.f, 0.f};
    for (int s = threadIdx.x; s < splits; s += JOIN_WAVES * 64) {
        const Partial p = parts[row * splits + s];
        u.join(p.m, p.s, p.t);
    }
    TopList list;
    list.n_top = a.n_top;
    if (TOP)
        for (int s = wave; s < splits; s += JOIN_WAVES)
            list.mine = merge_lists(list.mine, lane < a.n_top ? keys[(row * splits + s) * a.n_top + lane] : 0, lane);
    join_waves<JOIN_WAVES, TOP>(u, list, wave_sums, wave_keys, lane, wave);
    if (wave != 0) return;
    const int64_t label = a.labels ? a.labels[row] : -1;
    const bool labelled = label >= 0 && label < a.v;
    const float log_s = __builtin_amdgcn_logf(u.s) * 0.693147181f;
    if (lane == 0) row_results(a, row, u, labelled ? one_float<T>(x[label]) : 0.f, labelled);
    if (TOP) store_top(a, row, u, list, log_s, lane);
}

// ---- gradient --------------------------------------------------------------------------------------------------------------
struct RowGrad { float m, log_s, h, dl, dh; int64_t label; };
__device__ inline RowGrad row_grad(const LogProbsBwd &a, int64_t row)
{
    RowGrad g;
    const int64_t label = a.labels ? a.labels[row] : -1;
    g.label = label >= 0 && label < a.v ? label : -1;
    g.m = a.max_log_sum[2 * row];
    g.log_s = a.max_log_sum[2 * row + 1];
    const bool empty = g.m == -__builtin_inff() && g.log_s == 0.f;
    if (empty) g.m = 0.f;                                          // (every x is -inf: p = 0)
    g.dl = a.d_log_prob && g.label >= 0 && !empty ? a.d_log_prob[row] : 0.f;
    g.dh = a.d_entropy && !empty ? a.d_entropy[row] : 0.f;
    g.h = a.d_entropy ? a.entropy[row] : 0.f;
    return g;
}
__device__ inline float grad_of(const RowGrad &g, float x, bool hit)
{
    const float lp = (x - g.m) - g.log_s, p = exp_of(lp);
    return (hit ? g.dl : 0.f) - p * g.dl - g.dh * (p * (bounded(lp) + g.h));
}

template <typename T, int LPR>
__global__ __launch_bounds__(THREADS) void small_bwd_kernel(const LogProbsBwd a)
{
    constexpr int ROWS = THREADS / LPR, E = 8;
    const int l = (int)threadIdx.x % LPR;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR; row < a.n; row += (int64_t)gridDim.x * ROWS) {
        const T *x = static_cast<const T *>(a.logits) + row * a.ld;
        T *d = static_cast<T *>(a.d_logits) + row * a.ld_d;
        const RowGrad g = row_grad(a, row);
        float xs[E];
#pragma unroll
        for (int e = 0; e < E; ++e) xs[e] = l + LPR * e < a.v ? one_float<T>(x[l + LPR * e]) : 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (l + LPR * e < a.v) d[l + LPR * e] = one_of<T>(grad_of(g, xs[e], l + LPR * e == g.label));
    }
}

template <typename T, bool ONCE>
__global__ __launch_bounds__(THREADS) void long_bwd_kernel(const LogProbsBwd a, int chunks, int64_t per)
{
    for (int64_t block = blockIdx.x; block < a.n * chunks; block += gridDim.x) {
        const int64_t row = block / chunks, from = block % chunks * per;
        const int64_t to = from + per < a.v ? from + per : a.v;
        const T *x = static_cast<const T *>(a.logits) + row * a.ld;
        T *d = static_cast<T *>(a.d_logits) + row * a.ld_d;
        const RowGrad g = row_grad(a, row);
        for (int64_t at = from + threadIdx.x * 8; at < to; at += THREADS * 8) {
            if (at + 8 <= to) {
                Eight<T> raw;
                load_eight<ONCE>(x + at, raw);
                float v[8];
                to_floats(raw, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = grad_of(g, v[e], at + e == g.label);
                store_eight(d + at, v);
            } else {
                for (int64_t j = at; j < to; ++j) d[j] = one_of<T>(grad_of(g, one_float<T>(x[j]), j == g.label));
            }
        }
    }
}

// Blocks of a long row: one, unless there are too few rows to occupy the device; then pieces of at least 4096 classes.
constexpr int64_t WANTED_BLOCKS = 1024;
struct Split { int splits; int64_t per; };
Split split_of(int64_t n, int64_t v)
{
    int64_t s = n > 0 ? WANTED_BLOCKS / n : 1;
    const int64_t most = ceil_div(v, 4096);
    if (s > most) s = most;
    if (s < 1) s = 1;
    const int64_t per = (ceil_div(v, s) + 7) / 8 * 8;
    return Split{(int)ceil_div(v, per), per};
}

// Logits that fill more than half of the memory's cache (256 MB) are read past the caches.  Forward and gradient with / without, us: 4096 x 32 768
// bf16 (268 MB) 132 / 165, 2000 x 20 000 fp32 (160 MB) 99 / 105, bf16 (80 MB) 53 / 49.
template <typename T> bool read_once(int64_t n, int64_t v) { return n * v * (int64_t)sizeof(T) > (int64_t)128 << 20; }

unsigned grid_of(int64_t blocks) { return (unsigned)(blocks < MAX_BLOCKS ? blocks : MAX_BLOCKS); }

template <typename F> void with_lanes(int64_t v, F f)
{
    if (v <= 32) return f(std::integral_constant<int, 4>{});
    if (v <= 64) return f(std::integral_constant<int, 8>{});
    if (v <= 128) return f(std::integral_constant<int, 16>{});
    if (v <= 256) return f(std::integral_constant<int, 32>{});
    return f(std::integral_constant<int, 64>{});
}

template <typename T>
int launch_fwd(const LogProbsFwd &a, void *workspace, hipStream_t stream)
{
    if (a.v <= SMALL) {
        with_lanes(a.v, [&](auto lanes) {
            constexpr int LPR = decltype(lanes)::value;
            small_fwd_kernel<T, LPR><<<grid_of(ceil_div(a.n, THREADS / LPR)), THREADS, 0, stream>>>(a);
        });
        PCPP_HIP_CHECK(hipGetLastError());
        return PCPP_OK;
    }
    const Split s = split_of(a.n, a.v);
    Partial *parts = static_cast<Partial *>(workspace);
    key_t64 *keys = reinterpret_cast<key_t64 *>(static_cast<char *>(workspace) + align_up((size_t)a.n * s.splits * sizeof(Partial)));
    const bool once = read_once<T>(a.n, a.v);
    auto kernel = a.n_top > 0 ? (once ? long_fwd_kernel<T, true, true> : long_fwd_kernel<T, true, false>)
                              : (once ? long_fwd_kernel<T, false, true> : long_fwd_kernel<T, false, false>);
    kernel<<<grid_of(a.n * s.splits), THREADS, 0, stream>>>(a, s.splits, s.per, parts, keys);
    PCPP_HIP_CHECK(hipGetLastError());
    if (s.splits == 1) return PCPP_OK;
    auto join = a.n_top > 0 ? join_fwd_kernel<T, true> : join_fwd_kernel<T, false>;
    join<<<(unsigned)a.n, JOIN_WAVES * 64, 0, stream>>>(a, s.splits, parts, keys);
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

template <typename T>
int launch_bwd(const LogProbsBwd &a, hipStream_t stream)
{
    if (a.v <= SMALL) {
        with_lanes(a.v, [&](auto lanes) {
            constexpr int LPR = decltype(lanes)::value;
            small_bwd_kernel<T, LPR><<<grid_of(ceil_div(a.n, THREADS / LPR)), THREADS, 0, stream>>>(a);
        });
    } else {
        const Split s = split_of(a.n, a.v);
        auto kernel = read_once<T>(a.n, a.v) ? long_bwd_kernel<T, true> : long_bwd_kernel<T, false>;
        kernel<<<grid_of(a.n * s.splits), THREADS, 0, stream>>>(a, s.splits, s.per);
    }
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

}  // namespace

size_t log_probs_workspace_bytes(int64_t n, int64_t v, int n_top)
{
    if (v <= SMALL) return 0;
    const Split s = split_of(n, v);
    if (s.splits == 1) return 0;
    return align_up((size_t)n * s.splits * sizeof(Partial)) + align_up((size_t)n * s.splits * n_top * sizeof(key_t64));
}

int log_probs_fwd(const LogProbsFwd &a, int dtype, void *workspace, hipStream_t stream)
{
    return dtype == PCPP_F32 ? launch_fwd<float>(a, workspace, stream) : launch_fwd<bf16_t>(a, workspace, stream);
}

int log_probs_bwd(const LogProbsBwd &a, int dtype, hipStream_t stream)
{
    return dtype == PCPP_F32 ? launch_bwd<float>(a, stream) : launch_bwd<bf16_t>(a, stream);
}

}  // namespace pcpp
