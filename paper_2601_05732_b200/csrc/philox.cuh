// Counter-based random bits for dropout: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as
// 1, 2, 3", 2011).  A group of 8 consecutive elements shares one counter, (group index, offset), and takes 16 bits each
// of its four words, the low half first; the key is the seed.  A mask is therefore a function of (seed, offset, element)
// and is computed again wherever it is needed instead of being stored.
//
// 16 bits a mask bit halve the arithmetic of 32 (ten rounds, about 90 instructions, for 8 elements): with 32 the integer
// pipe, not the memory, would bound a bf16 dropout.  The price is that p counts as rounded to a multiple of 2^-16; the
// factor 1 / (1 - p) uses the rounded p, so the expectation is exact.
#pragma once
#include "common.cuh"

namespace mhcl {

// Host side: threshold of p in units of 2^-16 (65536 would drop everything: refused by the callers).
inline int drop_threshold(float p) { return (int)((double)p * 65536.0 + 0.5); }
inline float drop_factor(int threshold) { return (float)(65536.0 / (65536 - threshold)); }

#ifdef __CUDACC__
// The four words of group `g` under rng = (seed, offset).
__device__ __forceinline__ uint4 philox_group(uint64_t g, uint64_t seed, uint64_t offset) {
    uint32_t c0 = (uint32_t)g, c1 = (uint32_t)(g >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}
// f[e] <- f[e] * factor where element e of the group stays, 0 (whatever f[e] is) where it is dropped.
__device__ __forceinline__ void drop8(float* f, uint64_t g, uint64_t seed, uint64_t offset, uint32_t threshold, float factor) {
    const uint4 w = philox_group(g, seed, offset);
    const uint32_t r[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[2 * e] = (r[e] & 0xFFFFu) >= threshold ? f[2 * e] * factor : 0.f;
        f[2 * e + 1] = (r[e] >> 16) >= threshold ? f[2 * e + 1] * factor : 0.f;
    }
}
#endif

}  // namespace mhcl
