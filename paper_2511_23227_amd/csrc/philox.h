// Random numbers by counter (Philox 4x32 with ten rounds: Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011),
// for dropout and for rounding at random.  Not part of the C ABI.
//
// The numbers are a function of a program's state (seed, step) in device memory, the operator's site and the element's place, so a
// backward pass and a captured graph form them again and no mask is stored.  Eight neighbouring channels of a row share a counter and take
// sixteen bits each of its 128.  Ten rounds cost 20 wide multiplications, 2.5 an element; 32 bits an element would cost twice that.
#pragma once

#include "pcpp_internal.h"

namespace pcpp {

struct Random {                                                   // what the host hands to a kernel
    const int64_t *state;                                         // device: seed, step; NULL: no random numbers
    uint32_t site;
};
struct Philox {                                                   // what a kernel holds of it, the same in all lanes
    uint32_t key[2], site, step[2];
    __device__ inline Philox(const Random &r) : key{0u, 0u}, site(r.site), step{0u, 0u}
    {
        if (r.state) {
            const uint64_t seed = (uint64_t)r.state[0], at = (uint64_t)r.state[1];
            key[0] = (uint32_t)seed, key[1] = (uint32_t)(seed >> 32);
            step[0] = (uint32_t)at, step[1] = (uint32_t)(at >> 32);
        }
    }
    // the four words of the eight channels with number `group` (row * ceil(c / 8) + channel / 8): channel 2 i has the low half of
    // word i, channel 2 i + 1 the high half
    __device__ inline void draw(uint32_t group, uint32_t (&x)[4]) const
    {
        uint32_t k0 = key[0], k1 = key[1];
        x[0] = group, x[1] = site, x[2] = step[0], x[3] = step[1];
#pragma unroll
        for (int r = 0; r < 10; ++r) {
            const uint64_t a = (uint64_t)0xD2511F53u * x[0], b = (uint64_t)0xCD9E8D57u * x[2];
            const uint32_t x1 = x[1], x3 = x[3];
            x[0] = __builtin_amdgcn_bitop3_b32((uint32_t)(b >> 32), x1, k0, 0x96);                // (0x96: exclusive or of the three)
            x[1] = (uint32_t)b;
            x[2] = __builtin_amdgcn_bitop3_b32((uint32_t)(a >> 32), x3, k1, 0x96);
            x[3] = (uint32_t)a;
            k0 += 0x9E3779B9u;
            k1 += 0xBB67AE85u;
        }
    }
};
__device__ inline uint32_t half_of(const uint32_t (&x)[4], int e) { return (e & 1) ? x[e >> 1] >> 16 : x[e >> 1] & 0xffffu; }

// Dropout: an element goes where its sixteen bits are below the threshold round(65536 p); what stays is multiplied by 65536 / (65536 - threshold).
struct Drop {
    uint32_t threshold;                                           // 0: nothing is dropped, 65536: everything
    float scale;
    Random random;
};
inline Drop make_drop(float p, const int64_t *state, uint32_t site)
{
    Drop d;
    d.threshold = (uint32_t)(65536.0 * (double)p + 0.5);
    d.scale = d.threshold < 65536u ? (float)(65536.0 / (65536.0 - (double)d.threshold)) : 0.f;
    d.random = Random{state, site};
    return d;
}
// bit e: element e of the eight stays
__device__ inline uint32_t kept(const Philox &f, uint32_t group, uint32_t threshold)
{
    uint32_t x[4], bits = 0u;
    f.draw(group, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) bits |= (half_of(x, e) >= threshold ? 1u : 0u) << e;
    return bits;
}

}  // namespace pcpp
