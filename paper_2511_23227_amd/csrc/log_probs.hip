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
// Bound by memory, and in bf16 nearly as much by the exponentials: 4096 x 32 768 bf16 46 us = 5.8 TB/s, the gradient 102 us = 5.3; 115 200 x 17 fp32 with three
// alternatives 8.5 us, one row of 131 072 bf16 with twenty 9.1 + 4.3.  Rows of up to 512 classes lie in the registers of a few lanes;
// longer ones are walked, by a wave or by a block of four, or, where there are few rows, by several blocks whose sums a second kernel
// joins.
//
// The most probable classes.  A key is the value in an order-preserving form above the complement of the index, so that of equal
// values the lowest index is the largest key, and no two are equal.  The n_top-th largest of the lanes' maxima so far is a bound that n_top
// keys reach; it is close to the n_top-th largest key (of 64 maxima the 20th is about the 24th of all).  So only keys that pass it are
// looked at: they go to a pool in LDS, and at the end every one that passes the last bound counts how many are larger, which is its place.
// Rows whose order defeats the bound (their largest values in a few lanes) fill the pool; it is then sorted 64 keys at a time over the
// lanes and merged into a list.

#include "log_probs.h"
#include "row_ops.h"

namespace pcpp {

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int64_t MAX_BLOCKS = 1 << 22;                            // (a grid has fewer than 2^32 threads)
constexpr int SMALL = 512;                                        // classes of the rows that lie in registers
constexpr float LOG2E = 1.44269504f;
typedef unsigned long long key_t64;

// The rounding of x log2(e) puts the power off by about |x| 2^-24 of itself, 5e-7 at -10, 3e-6 at -60, where a class has no weight in a sum; in a
// gradient it shows in such classes' own elements.  The product's second term would take two more instructions an element, in passes that these bound
// nearly as much as memory.  Powers below 2^-126 are zero.
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

// The largest key that `n_top` of the wave's (N in each lane, as values in order) reach; not the largest such where some more reach it too, 0 where
// fewer are not 0.
template <int N> __device__ inline uint32_t bound_of(const uint32_t (&o)[N], int n_top)
{
    uint32_t bound = 0u;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t at = bound | 1u << bit;
        int n = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) n += __popcll(__ballot(o[e] >= at));
        if (n >= n_top) {
            bound = at;
            if (n <= n_top + 4) break;
        }
    }
    return bound;
}

// What a wave keeps of the keys that it has seen.
constexpr int POOL = 256;
struct TopKeys {
    key_t64 list = 0, last = 0;                                   // list: lane j its (j + 1)-th largest; last: keys up to it do not belong
    key_t64 *pool;                                                // LDS, the wave's own
    int n = 0, n_top;
    bool listed = false;

    // (the lanes' writes before the reads, and these before the next writes)
    __device__ static inline void settle()
    {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    __device__ inline void raise(uint32_t bound) { if (bound && (key_t64)bound << 32 > last) last = ((key_t64)bound << 32) - 1; }
    __device__ static inline uint32_t before(key_t64 m) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u)); }
    // the lanes' keys k where `in`
    __device__ inline void push(key_t64 k, bool in, int lane)
    {
        in = in && k > last;
        key_t64 m = __ballot(in);
        if (n + __popcll(m) > POOL) {
            flush(pool, lane);
            in = in && k > last;
            m = __ballot(in);
        }
        if (in) pool[n + before(m)] = k;
        n += __popcll(m);
    }
    __device__ inline void merge(key_t64 k, int lane)             // the lanes' keys, in any order
    {
        k = sort_lanes(k, lane);
        list = listed ? merge_lists(list, k, lane) : k;
        listed = true;
        const key_t64 l = lane_of(list, n_top - 1);
        if (l > last) last = l;
    }
    __device__ inline void flush(const key_t64 *from, int lane)   // the n keys there into the list
    {
        settle();
        for (int i = 0; i < n; i += 64) merge(i + lane < n ? from[i + lane] : 0, lane);
        settle();
        n = 0;
    }
    // Keys there that still belong, to the front of the pool behind those that it holds (at or in front of `from`).
    __device__ inline void gather(const key_t64 *from, int count, int lane)
    {
        settle();
        for (int i = 0; i < count; i += 64) {
            const key_t64 k = i + lane < count ? from[i + lane] : 0;
            const bool in = k > last;
            const key_t64 m = __ballot(in);
            settle();
            if (in) pool[n + before(m)] = k;
            n += __popcll(m);
        }
        settle();
    }
    // put(place, key) for the n_top largest of the pool and the list, each in one lane
    template <typename Put> __device__ inline void finish(int lane, Put put)
    {
        if (!listed && n <= 64) {
            const key_t64 k = lane < n ? pool[lane] : 0;
            int place = 0;
            int j = 0;
            for (; j + 4 <= n; j += 4) {                          // (four reads under way)
                const key_t64 k0 = pool[j], k1 = pool[j + 1], k2 = pool[j + 2], k3 = pool[j + 3];
                place += (k0 > k) + (k1 > k) + (k2 > k) + (k3 > k);
            }
            for (; j < n; ++j) place += pool[j] > k;
            if (lane < n && place < n_top) put(place, k);
        } else {
            flush(pool, lane);
            if (lane < n_top) put(lane, list);
        }
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
// the sums of the LPR lanes of a row, in all of them
template <int LPR> __device__ inline Sums join_lanes(Sums v)
{
    const float m = row_max<LPR>(v.m), d = m == -__builtin_inff() ? 0.f : bounded(v.m - m), e = exp_of(d);
    return Sums{m, row_sum<LPR>(e * v.s), row_sum<LPR>(e * (v.t + d * v.s))};
}

// what a row's sums say; NaN in S reaches everything
__device__ inline float log_of(float s) { return __builtin_amdgcn_logf(s) * 0.693147181f; }
__device__ inline void row_results(const LogProbsFwd &a, int64_t row, const Sums &v, float log_s, float x_label, bool labelled)
{
    const bool empty = v.s == 0.f;
    if (a.max_log_sum) *reinterpret_cast<float2 *>(a.max_log_sum + 2 * row) = float2{v.m, empty ? 0.f : log_s};
    if (a.entropy) a.entropy[row] = empty ? 0.f : log_s - v.t / v.s;
    if (a.log_prob) {
        const float lp = empty ? -__builtin_inff() : (x_label - v.m) - log_s;
        a.log_prob[row] = labelled ? lp : 0.f;
    }
}
__device__ inline float top_value(const Sums &v, float x, float log_s) { return v.s == 0.f ? -__builtin_inff() : (x - v.m) - log_s; }

// op over the LPR lanes of a row, the same in all of them
template <int LPR, typename Op> __device__ inline uint32_t row_best(uint32_t v, Op op)
{
    return __float_as_uint(row_reduce<LPR>(__uint_as_float(v), [&](float a, float b) { return __uint_as_float(op(__float_as_uint(a), __float_as_uint(b))); }));
}

// ---- rows in registers ---------------------------------------------------------------------------------------------------------
// One class after the other: the largest of the lanes', of equal ones the lowest index.  For rows in fewer than 64 lanes, that is up to 256 classes; n_top
// may be larger than the lanes' number.  So / by the pool with a row in a whole wave, 200 000 rows in bf16, us a call: three alternatives of 32 classes
// 10 / 107, of 64 17 / 111, 128 30 / 116, 129 67 / 131, 256 66 / 128; five of 256 84 / 131; twenty of 32 44 / 190, 64 55 / 208, 128 106 / 258, 129
// 234 / 372, but of 200 230 / 171 and of 256 231 / 151, which a line by n_top as well would give to the pool.  On the other side, twenty of 400: 519 /
// 158.
template <int LPR, typename Put> __device__ inline void take_in_turn(uint32_t (&value)[8], int at, int n_top, Put put)
{
    uint32_t mine = 0u, index = 0u;                                // 0: none left
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (value[e] > mine) mine = value[e], index = (uint32_t)(at + e);
    for (int k = 0; k < n_top; ++k) {
        const uint32_t best = row_best<LPR>(mine, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
        const uint32_t first = row_best<LPR>(mine == best ? index : ~0u, [](uint32_t p, uint32_t q) { return p < q ? p : q; });
        if (index == first && mine == best) {                      // (one lane)
            put(k, best, index);
            mine = 0u;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if ((uint32_t)(at + e) == first) value[e] = 0u;
                if (value[e] > mine) mine = value[e], index = (uint32_t)(at + e);
            }
        }
    }
}

template <typename T, int LPR, int MODE, bool TOP>
__global__ __launch_bounds__(THREADS) void small_fwd_kernel(const LogProbsFwd a)
{
    constexpr int ROWS = 64 / LPR, TS = sizeof(T);
    __shared__ key_t64 pool[TOP && LPR == 64 ? WAVES : 1][POOL];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), v = (int)a.v;
    const Span<MODE> own(8 * (lane % LPR), v);
    const uint32_t in_wave = (uint32_t)(lane / LPR), off = own.template offset<TS>(in_wave * (uint32_t)a.ld);
    for (int64_t first = ((int64_t)blockIdx.x * WAVES + wave) * ROWS; first < a.n; first += (int64_t)gridDim.x * WAVES * ROWS) {
        const int64_t row = first + in_wave;
        const bool live = row < a.n;
        const __amdgpu_buffer_rsrc_t xs = rows_from<TS>(a.logits, first, a.n, a.ld, v, ROWS);
        Eight<T> raw;
        row_load<T>(xs, off, own, raw);
        const int label = a.labels && live ? a.labels[row] : -1;
        const bool labelled = label >= 0 && label < v;
        const float x_label = __uint_as_float(load_one<T>(xs, labelled ? in_wave * (uint32_t)a.ld + (uint32_t)label : OOB_OFFSET / TS));
        float x[8];
        to_floats(raw, x);
        Sums u{-__builtin_inff(), 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = own.own(e) ? x[e] : -__builtin_inff();
            u.m = fmaxf(u.m, x[e]);
        }
        const float lane_m = u.m;
        u.m = row_max<LPR>(u.m);
        const float m0 = u.m == -__builtin_inff() ? 0.f : u.m;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = x[e] - m0, p = exp_of(d);
            u.s += p;
            u.t = __builtin_fmaf(p, bounded(d), u.t);
        }
        u.s = row_sum<LPR>(u.s);
        u.t = row_sum<LPR>(u.t);
        const float log_s = log_of(u.s);
        if (live && lane % LPR == 0) row_results(a, row, u, log_s, x_label, labelled);
        if constexpr (TOP) {
            auto put = [&](int k, uint32_t value, uint32_t index) {
                if (!live) return;
                a.top_log_prob[row * a.n_top + k] = top_value(u, from_ordered(value), log_s);
                a.top_index[row * a.n_top + k] = (int32_t)index;
            };
            if constexpr (LPR == 64) {
                TopKeys keys;
                keys.pool = pool[wave];
                keys.n_top = a.n_top;
                const uint32_t largest[1] = {lane_m > -__builtin_inff() ? ordered(lane_m) : 0u};
                keys.raise(bound_of(largest, a.n_top));
#pragma unroll
                for (int e = 0; e < 8; ++e) keys.push(key_of(x[e], (uint32_t)(own.at + e)), own.own(e), lane);
                TopKeys::settle();
                keys.finish(lane, [&](int k, key_t64 key) { put(k, (uint32_t)(key >> 32), key_index(key)); });
                TopKeys::settle();
            } else {
                uint32_t value[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) value[e] = own.own(e) ? ordered(x[e]) : 0u;
                take_in_turn<LPR>(value, own.at, a.n_top, put);
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

// W: waves that walk the row
template <typename T, int W, bool TOP, bool ONCE>
__device__ inline void walk(const T *x, int64_t from, int64_t to, Sums &u, TopKeys &keys, int lane, int wave)
{
    constexpr int N = 8 * DEEP, WAVE = 64 * N;
    u = Sums{-__builtin_inff(), 0.f, 0.f};
    // (the wave goes round together, so that the pool sees all lanes)
    int64_t base = from + wave * WAVE;
    Eight<T> r[DEEP];
    if (base < to) load_step<T, ONCE>(x, base + lane * 8, to, r);
    for (; base < to; base += W * WAVE) {
        const int64_t at = base + lane * 8;
        float v[N];
#pragma unroll
        for (int j = 0; j < DEEP; ++j) to_floats(r[j], *reinterpret_cast<float (*)[8]>(v + 8 * j));
        if (base + W * WAVE < to) load_step<T, ONCE>(x, at + W * WAVE, to, r);
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
        auto bound = [&] { return keys.last ? key_value(keys.last) : -__builtin_inff(); };
        if (!__ballot(!(m < bound()))) continue;
        const uint32_t largest[1] = {u.m > -__builtin_inff() ? ordered(u.m) : 0u};
        keys.raise(bound_of(largest, keys.n_top));
        const float b = bound();
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int64_t index = at + 512 * (e / 8) + e % 8;
            const bool in = !(v[e] < b) && index < to;
            if (__ballot(in)) keys.push(key_of(v[e], (uint32_t)index), in, lane);
        }
    }
}

struct Partial { float m, s, t, unused; };

// LDS of a block's N waves
template <int N> struct Joint {
    Sums sums[N];
    uint32_t largest[N][64];
    int count[N];
    bool listed[N];
    key_t64 last[N], list[N][64];
};

// The sums of a block's N waves, in wave 0.
template <int N> __device__ inline void join_sums(Sums &u, Sums *sums, int lane, int wave)
{
    if (lane == 0) sums[wave] = u;
    __syncthreads();
    if (wave == 0) u = join_lanes<N>(sums[lane % N]);               // (in all lanes)
}

// What N waves keep of a row, into wave 0's; pools: the waves' pools one behind the other.  largest: the lane's value, in order.
template <int N>
__device__ inline void join_keys(TopKeys &keys, Joint<N> &joint, key_t64 (*pools)[POOL], uint32_t largest, int lane, int wave)
{
    joint.largest[wave][lane] = largest;
    if (keys.listed) joint.list[wave][lane] = keys.list;
    if (lane == 0) {
        joint.count[wave] = keys.n;
        joint.listed[wave] = keys.listed;
        joint.last[wave] = keys.last;
    }
    __syncthreads();
    if (wave != 0) return;
    uint32_t o[N];
#pragma unroll
    for (int w = 0; w < N; ++w) o[w] = joint.largest[w][lane];
    keys.raise(bound_of(o, keys.n_top));
#pragma unroll
    for (int w = 1; w < N; ++w) {
        const key_t64 l = joint.last[w];
        if (l > keys.last) keys.last = l - 1;                     // (wave w may hold the key itself)
    }
    keys.n = 0;
#pragma unroll
    for (int w = 0; w < N; ++w) keys.gather(pools[w], joint.count[w], lane);
#pragma unroll
    for (int w = 1; w < N; ++w)
        if (joint.listed[w]) {
            keys.list = keys.listed ? merge_lists(keys.list, joint.list[w][lane], lane) : joint.list[w][lane];
            keys.listed = true;
        }
}

// W waves a row, or a part of it
template <typename T, int W, bool TOP, bool ONCE>
__global__ __launch_bounds__(THREADS) void long_fwd_kernel(const LogProbsFwd a, int splits, int64_t per, Partial *parts, key_t64 *split_keys)
{
    constexpr int ROWS = WAVES / W;
    __shared__ Joint<W> joint;
    __shared__ key_t64 pools[TOP ? WAVES : 1][POOL];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    // (W = 1: no barriers, so the waves need not go round together)
    for (int64_t block = (int64_t)blockIdx.x * ROWS + wave / W; block < a.n * splits; block += (int64_t)gridDim.x * ROWS) {
        const int64_t row = block / splits;
        const int split = (int)(block % splits);
        const T *x = static_cast<const T *>(a.logits) + row * a.ld;
        const int64_t from = split * per, to = from + per < a.v ? from + per : a.v;
        Sums u;
        TopKeys keys;
        keys.n_top = a.n_top;
        keys.pool = pools[TOP ? wave : 0];
        walk<T, W, TOP, ONCE>(x, from, to, u, keys, lane, wave % W);
        const float lane_m = u.m;
        u = join_lanes<64>(u);
        if constexpr (W > 1) {
            join_sums<W>(u, joint.sums, lane, wave);
            if (TOP) join_keys<W>(keys, joint, pools, lane_m > -__builtin_inff() ? ordered(lane_m) : 0u, lane, wave);
        } else if (TOP) {
            const uint32_t largest[1] = {lane_m > -__builtin_inff() ? ordered(lane_m) : 0u};
            keys.raise(bound_of(largest, a.n_top));
            const int n = keys.n;
            keys.n = 0;
            keys.gather(keys.pool, n, lane);
        }
        if (wave % W == 0) {
            if (splits == 1) {
                const int64_t label = a.labels ? a.labels[row] : -1;
                const bool labelled = label >= 0 && label < a.v;
                const float log_s = log_of(u.s);
                if (lane == 0) row_results(a, row, u, log_s, labelled ? one_float<T>(x[label]) : 0.f, labelled);
                if (TOP)
                    keys.finish(lane, [&](int k, key_t64 key) {
                        a.top_log_prob[row * a.n_top + k] = top_value(u, key_value(key), log_s);
                        a.top_index[row * a.n_top + k] = (int32_t)key_index(key);
                    });
            } else {
                if (lane == 0) parts[block] = Partial{u.m, u.s, u.t, 0.f};
                if (TOP) {
                    key_t64 *to_keys = split_keys + block * a.n_top;
                    const int held = keys.listed ? 64 : keys.n;
                    if (lane >= held && lane < a.n_top) to_keys[lane] = 0;            // (a short part has fewer)
                    keys.finish(lane, [&](int k, key_t64 key) { to_keys[k] = key; });
                }
            }
        }
        if constexpr (W > 1) __syncthreads();                      // (the next row's sums and keys go where these lay)
        else if (TOP) TopKeys::settle();
    }
}

// One block a row: the sums and lists of its splits, the lists by the waves in turn, then pair by pair.
constexpr int JOIN_WAVES = 16;
template <typename T, bool TOP>
__global__ __launch_bounds__(JOIN_WAVES * 64) void join_fwd_kernel(const LogProbsFwd a, int splits, const Partial *parts, const key_t64 *keys)
{
    __shared__ Sums sums[JOIN_WAVES];
    __shared__ key_t64 lists[TOP ? JOIN_WAVES : 1][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t row = blockIdx.x;                               // (few rows: they were split)
    const T *x = static_cast<const T *>(a.logits) + row * a.ld;
    Sums u{-__builtin_inff(), 0.f, 0.f};
    for (int s = threadIdx.x; s < splits; s += JOIN_WAVES * 64) {
        const Partial p = parts[row * splits + s];
        u.join(p.m, p.s, p.t);
    }
    u = join_lanes<64>(u);
    key_t64 list = 0;
    if (TOP) {
        for (int s = wave; s < splits; s += JOIN_WAVES) {
            const key_t64 k = lane < a.n_top ? keys[(row * splits + s) * a.n_top + lane] : 0;
            list = s == wave ? k : merge_lists(list, k, lane);
        }
        lists[wave][lane] = list;
    }
    join_sums<JOIN_WAVES>(u, sums, lane, wave);
    if (TOP) {
        for (int half = JOIN_WAVES / 2; half > 0; half >>= 1) {
            if (wave < half) {
                if (wave + half < splits) lists[wave][lane] = list = merge_lists(list, lists[wave + half][lane], lane);
            }
            __syncthreads();
        }
    }
    if (wave != 0) return;
    const int64_t label = a.labels ? a.labels[row] : -1;
    const bool labelled = label >= 0 && label < a.v;
    const float log_s = log_of(u.s);
    if (lane == 0) row_results(a, row, u, log_s, labelled ? one_float<T>(x[label]) : 0.f, labelled);
    if (TOP && lane < a.n_top) {
        a.top_log_prob[row * a.n_top + lane] = top_value(u, key_value(list), log_s);
        a.top_index[row * a.n_top + lane] = (int32_t)key_index(list);
    }
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

template <typename T, int LPR, int MODE>
__global__ __launch_bounds__(THREADS) void small_bwd_kernel(const LogProbsBwd a)
{
    constexpr int ROWS = 64 / LPR, TS = sizeof(T);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), v = (int)a.v;
    const Span<MODE> own(8 * (lane % LPR), v);
    const uint32_t in_wave = (uint32_t)(lane / LPR), off = own.template offset<TS>(in_wave * (uint32_t)a.ld);
    const uint32_t off_d = own.template offset<TS>(in_wave * (uint32_t)a.ld_d);
    for (int64_t first = ((int64_t)blockIdx.x * WAVES + wave) * ROWS; first < a.n; first += (int64_t)gridDim.x * WAVES * ROWS) {
        const int64_t row = first + in_wave < a.n ? first + in_wave : a.n - 1;      // (rows past the last are not written)
        const __amdgpu_buffer_rsrc_t xs = rows_from<TS>(a.logits, first, a.n, a.ld, v, ROWS), ds = rows_from<TS>(a.d_logits, first, a.n, a.ld_d, v, ROWS);
        Eight<T> raw;
        row_load<T>(xs, off, own, raw);
        const RowGrad g = row_grad(a, row);
        float x[8];
        to_floats(raw, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = grad_of(g, x[e], own.at + e == g.label);
        row_store<T>(ds, off_d, own, x);
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
                store_eight<ONCE>(d + at, v);
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

// A row by a wave on its own rather than by a block's four: no barrier, and the alternatives' pool is not joined, but a fourth of the waves.
// By a wave / by four, bf16, us a call, one behind the other: five alternatives, 8000 x 8000 44 / 63, 2000 x 5000 15.5 / 20.4, 2000 x 16 000 32 / 29; twenty, 1100 x
// 16 000 38 / 24; none, forward and gradient of 30 000 x 3000 107 / 107, of 4096 x 32 768 134 / 130.  (Twenty alternatives of very many long rows,
// 5000 x 20 000 69 / 82, would gain as well; but then how many rows there are would change a row's last bits from 1024 rows on.)
bool row_by_wave(int64_t n, int64_t v, bool top) { return n >= 1024 && v <= (top ? 8192 : 4096); }

// Logits of more than 64 MB, a quarter of the memory's cache, are read past the caches, and their gradient is written past them.  Forward and gradient so /
// by way of the caches, us: 268 MB (4096 x 32 768 bf16) 143 / 164 (reads alone 152), 120 MB 73 / 76, 80 MB 52.7 / 54.5, 40 MB 27.9 / 24.6.
template <typename T> bool read_once(int64_t n, int64_t v) { return n * v * (int64_t)sizeof(T) > (int64_t)64 << 20; }

unsigned grid_of(int64_t blocks) { return (unsigned)(blocks < MAX_BLOCKS ? blocks : MAX_BLOCKS); }

// Rows in registers: up to 512 classes, and pitches with which a wave's sixteen rows lie within 32-bit offsets
bool in_registers(int64_t v, int64_t ld) { return v <= SMALL && ld < 1 << 24; }

template <typename T>
int launch_fwd(const LogProbsFwd &a, void *workspace, hipStream_t stream)
{
    const bool top = a.n_top > 0;
    if (in_registers(a.v, a.ld)) {
        with_rows((int)a.v, [&](auto lanes, auto, auto mode) {
            constexpr int LPR = decltype(lanes)::value, MODE = decltype(mode)::value;
            auto kernel = top ? small_fwd_kernel<T, LPR, MODE, true> : small_fwd_kernel<T, LPR, MODE, false>;
            kernel<<<grid_of(ceil_div(a.n, THREADS / LPR)), THREADS, 0, stream>>>(a);
        });
        PCPP_HIP_CHECK(hipGetLastError());
        return PCPP_OK;
    }
    const Split s = split_of(a.n, a.v);
    Partial *parts = static_cast<Partial *>(workspace);
    key_t64 *keys = reinterpret_cast<key_t64 *>(static_cast<char *>(workspace) + align_up((size_t)a.n * s.splits * sizeof(Partial)));
    const bool once = read_once<T>(a.n, a.v), wave = row_by_wave(a.n, a.v, top);
    auto pick = [&](auto w) {
        constexpr int W = decltype(w)::value;
        auto kernel = top ? (once ? long_fwd_kernel<T, W, true, true> : long_fwd_kernel<T, W, true, false>)
                          : (once ? long_fwd_kernel<T, W, false, true> : long_fwd_kernel<T, W, false, false>);
        kernel<<<grid_of(ceil_div(a.n * s.splits, WAVES / W)), THREADS, 0, stream>>>(a, s.splits, s.per, parts, keys);
    };
    if (wave) pick(Int<1>{});
    else pick(Int<WAVES>{});
    PCPP_HIP_CHECK(hipGetLastError());
    if (s.splits == 1) return PCPP_OK;
    auto join = top ? join_fwd_kernel<T, true> : join_fwd_kernel<T, false>;
    join<<<(unsigned)a.n, JOIN_WAVES * 64, 0, stream>>>(a, s.splits, parts, keys);
    PCPP_HIP_CHECK(hipGetLastError());
    return PCPP_OK;
}

template <typename T>
int launch_bwd(const LogProbsBwd &a, hipStream_t stream)
{
    if (in_registers(a.v, a.ld > a.ld_d ? a.ld : a.ld_d)) {
        with_rows((int)a.v, [&](auto lanes, auto, auto mode) {
            constexpr int LPR = decltype(lanes)::value;
            small_bwd_kernel<T, LPR, decltype(mode)::value><<<grid_of(ceil_div(a.n, THREADS / LPR)), THREADS, 0, stream>>>(a);
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
    if (v <= SMALL) return 0;                                     // (of one block a row, whatever the pitch)
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
