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
#include "kernels.h"

namespace mhcl {

// Host side: threshold of p in units of 2^-16 (65536 would drop everything: refused by the callers).
inline int drop_threshold(float p) { return (int)((double)p * 65536.0 + 0.5); }
inline float drop_factor(int threshold) { return (float)(65536.0 / (65536 - threshold)); }

#ifdef __CUDACC__
// The generator of one kernel.  The round keys are made anew for each group (18 additions): kept, they cost 20 registers
// a thread, and the warps that those displace were worth more (dropout of 134 M elements: 98 -> 92.5 us in a short run).
struct Philox {
    uint32_t s0, s1, o0, o1;
    __device__ __forceinline__ Philox(const uint64_t* rng, bool use) {     // rng is read only if it is to be used
        const uint64_t seed = use ? ld_dep(rng) : 0, offset = use ? ld_dep(rng + 1) : 0;
        s0 = (uint32_t)seed; s1 = (uint32_t)(seed >> 32);
        o0 = (uint32_t)offset; o1 = (uint32_t)(offset >> 32);
    }
    // the four words of group `g`
    __device__ __forceinline__ uint4 operator()(uint64_t g) const {
        uint32_t c0 = (uint32_t)g, c1 = (uint32_t)(g >> 32), c2 = o0, c3 = o1, k0 = s0, k1 = s1;
        asm volatile("" : "+r"(k0), "+r"(k1));                             // keeps the compiler from hoisting the keys
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
};
// f[e] (packed pairs) <- f where the element stays, 0 (whatever f is) where it is dropped; the caller multiplies by the
// factor together with what else it has.  `thr_hi` is the threshold in the upper half-word: the upper 16 bits of a word are
// compared as they lie, the lower ones shifted up.
__device__ __forceinline__ void drop8(uint64_t* f, const uint4& w, uint32_t thr_hi, float dropped = 0.f) {
    const uint32_t r[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float lo, hi;
        unpack2f(f[e], lo, hi);
        f[e] = pack2f((r[e] << 16) >= thr_hi ? lo : dropped, r[e] >= thr_hi ? hi : dropped);
    }
}
// The same for a gradient and its gate, of which nothing may be left where the element is dropped (0 times NaN): x = e^-a
// becomes infinite there, which closes the gate.
__device__ __forceinline__ void drop8(uint64_t* f, uint64_t* x, const uint4& w, uint32_t thr_hi) {
    drop8(f, w, thr_hi);
    drop8(x, w, thr_hi, INFINITY);
}
#endif

}  // namespace mhcl
