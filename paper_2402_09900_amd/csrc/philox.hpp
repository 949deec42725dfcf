// philox.hpp -- dropout's random numbers: Philox4x32-10, the counter-based generator of
// Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3" (SC 2011),
// from the paper's description.  The mask is a function of (seed, step, site, row,
// column) and is formed again wherever it is needed; nothing of it is stored.
//
// One block, counter (column / 8, row, step, site) and key = seed, is 128 bits: eight
// 16-bit numbers, the upper halves of the 32-bit numbers of eight columns.  An
// element is kept if its number is not below the limit, p 2^32; its lower half, from
// the block of the same counter with the first word's top bit set, matters only where
// the upper half equals the limit's (once in 65536 elements), so a second block is
// formed only by wavefronts that hold such an element: 32 bits of resolution at the
// price of 16.  (Beside memory that is next to free: 32768 x 2048 bf16, the norm takes 97 us
// with dropout and 93 without, dropout into a residual 6.2 TB/s.)
#pragma once

#include "scan_common.hpp"
#include "kernels.hpp"

namespace memoroid {

__device__ __forceinline__ void philox_block(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int n = 0; n < 10; ++n) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * c[0], p1 = (uint64_t)0xCD9E8D57u * c[2];
        const uint32_t c0 = (uint32_t)(p1 >> 32) ^ c[1] ^ k0, c2 = (uint32_t)(p0 >> 32) ^ c[3] ^ k1;
        c[1] = (uint32_t)p1;
        c[3] = (uint32_t)p0;
        c[0] = c0;
        c[2] = c2;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

// The call's part of the counter and the key, in scalar registers
struct DropKey {
    uint32_t k0, k1, step, site, hi, lo;     // hi, lo: halves of the limit (hi may be 2^16: nothing stays)
    float scale;
};
__device__ __forceinline__ DropKey drop_key(const DropArgs& a) {
    DropKey k;
    const uint64_t seed = (uint64_t)a.rng[0];
    k.k0 = __builtin_amdgcn_readfirstlane((uint32_t)seed);
    k.k1 = __builtin_amdgcn_readfirstlane((uint32_t)(seed >> 32));
    k.step = __builtin_amdgcn_readfirstlane((uint32_t)(uint64_t)a.rng[1]);
    k.site = a.site;
    k.hi = (uint32_t)(a.limit >> 16);
    k.lo = (uint32_t)a.limit & 0xFFFFu;
    k.scale = a.scale;
    return k;
}

// For each element e of the octet (column / 8 = block): stays(e, whether it stays)
template <class F>
__device__ __forceinline__ void each_kept(const DropKey& k, uint32_t block, uint32_t row, F stays) {
    uint32_t c[4] = {block, row, k.step, k.site};
    philox_block(c, k.k0, k.k1);
    bool tie = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t u = e & 1 ? c[e >> 1] >> 16 : c[e >> 1] & 0xFFFFu;
        tie = tie || u == k.hi;
    }
    uint32_t l[4] = {~0u, ~0u, ~0u, ~0u};    // no tie: any lower half
    if (k.lo != 0 && tie) {
        l[0] = block | 0x80000000u;
        l[1] = row;
        l[2] = k.step;
        l[3] = k.site;
        philox_block(l, k.k0, k.k1);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t u = e & 1 ? c[e >> 1] >> 16 : c[e >> 1] & 0xFFFFu;
        const uint32_t x = e & 1 ? l[e >> 1] >> 16 : l[e >> 1] & 0xFFFFu;
        stays(e, u > k.hi || (u == k.hi && x >= k.lo));
    }
}
// v[e] -> scale v[e] where element e stays, else 0
__device__ __forceinline__ void drop_octet(float (&v)[8], const DropKey& k, uint32_t block, uint32_t row) {
    each_kept(k, block, row, [&](int e, bool stays) { v[e] = stays ? v[e] * k.scale : 0.0f; });
}

}  // namespace memoroid
