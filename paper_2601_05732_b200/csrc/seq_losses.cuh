// Losses of whole sequences on the per-token losses that the cross entropy leaves (nll = -log probability of a token), and their
// gradients with respect to these (included by ce_kernels.cu).  A token counts where its target is not negative and it lies in a
// sequence; sequence s holds the tokens starts[s] .. starts[s+1].
//
// Policy:      x = nll_old - nll, r = e^x, A the advantage;  pg = max(-A r, -A clip(r, 1 - lo, 1 + hi))
//              d = nll - nll_ref,  kl = e^d - d - 1;  loss_s = w sum (pg + b kl),  w = 1 or 1 / (tokens that count)
//              dnll = dloss_s w ([not clipped] A r + b (e^d - 1))
// Preference:  R_s = w sum (nll_ref - nll);  pair p of sequences 2 p (chosen), 2 p + 1 (rejected):
//              x = beta (R_c - R_r) - margin;  loss_p = (1 - e) softplus(-x) + e softplus(x)
//              dnll = -+ beta w dloss_p (e - sigmoid(-x)) over the chosen and the rejected tokens
//
// Each warp walks a range of its own, 128 tokens a step (four a lane), with running sums of the sequence it is in: no exchange but
// where a sequence ends, whatever the lengths.  A sequence inside one range is complete there; one that crosses ranges leaves a
// piece in each, which seq_join_k adds up in order: the same bits from run to run.  What a gradient takes from a whole sequence
// (1 / n, the pair's slope) is put on by a last pass.  Steps in which several sequences end are added up by runs and a scan along
// the lanes, all of their sequences at once (sequences of two tokens: 128 000 tokens 28 us against 135 one by one).
// Sums: four tokens in fp32, from there in 64 bits.
//
// What bounds it: HBM for large batches, 24 bytes a token with reference and gradient (16.8 M tokens, 2048 sequences, on one B200: the
// sums 73 us at 5.5 TB/s, the join 5, the last pass 18 within L2; 98 for the call), start and drain in between (8.4 M tokens
// of 4096 pairs 37 us for 134 MB), and the latency of dependent phases below some 500 000 tokens (9 to 10 us).
#pragma once

#include <stddef.h>

#include "seq_index.h"

namespace mhcl {

enum SeqOp { SEQ_POLICY = 0, SEQ_PAIR = 1 };
constexpr int kSeqStep = 128;                 // tokens of a warp's step
constexpr int kScaleSteps = 4, kScaleRange = kScaleSteps * kSeqStep;      // of the last pass
constexpr int kSeqBlock = 256;
// Blocks an SM and steps in a warp's ring, and with them ranges at most: as many as are under way at once (of a B200's 148 SMs:
// the plan gives the scratch's size, so it does not look at the device).  The policy loss takes some 110 registers: two
// blocks 100 us for 16.8 M tokens, four of 64 registers, which spill, 108.
__host__ __device__ constexpr int seq_blocks(int op) { return op == SEQ_POLICY ? 2 : 4; }
__host__ __device__ constexpr int seq_stages(int op) { return op == SEQ_POLICY ? 4 : 3; }
constexpr int seq_ranges(int op) { return 148 * seq_blocks(op) * (kSeqBlock / 32); }
// Up to so many tokens and sequences one block does it all in one launch, with what its warps exchange in shared memory, or one
// cluster of eight (with the gradient, on the device: 1000 tokens 4.1 us, 4096 with the cluster 6.4, 16384 6.9, 32768 8.3; three
// launches 7.9 there, but the host takes 9 to 10 to make them; at 65536 the cluster's eight SMs take 11.7 against 8.4).
constexpr int kSeqOne = 16 * kSeqStep, kSeqOneS = 511;
constexpr int kSeqCluster = 32768, kSeqClusterS = 16384, kSeqClusterWarps = 8 * 16;
inline bool seq_one(int64_t T, int64_t S) { return T <= kSeqOne && S <= kSeqOneS; }
inline bool seq_cluster(int64_t T, int64_t S) { return T <= kSeqCluster && S <= kSeqClusterS; }

struct SeqSum { double a, b; int n, c; };     // policy: pg, kl, tokens, clipped ones; preference: log ratio, -, tokens, -

struct SeqArgs {
    int T, S, W, range;                       // W ranges of `range` tokens, a multiple of kSeqStep
    uint64_t per_range;                       // 2^40 over the steps of a range, rounded up: seq_range_of
    const float *nll, *old, *ref, *adv, *dloss;
    const int64_t *target, *starts;
    int mean;
    double edge[2];                           // the borders of x under a positive advantage and of -x under a negative one,
    float edge32[2], close[2];                // in fp32, and how close to it only 64 bits tell the side (below 0: never)
    float held[2];                            // the borders of r
    double kl_weight, beta, margin, smoothing;
    float kl_slope;                           // kl_weight in fp32
    float *loss, *stats, *dnll;               // stats: [S][3], or the rewards [P][2]
    SeqSum *whole, *head, *tail;              // [S] complete ones; [W] the pieces at the ranges' begins and ends
    float* coef;                              // [S] what a gradient takes from its whole sequence
    float* raw;                               // [T] the gradient without that (policy)
    int* hint;                                // the sequence at every kScaleRange-th token
    uint8_t* bits;                            // which of four tokens each have a target (preference)
    int* status;
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Where a sequence begins, cut to the tokens there are; behind the last, at their end.
__device__ __forceinline__ int seq_start(const SeqArgs& a, int i) {
    if (i > a.S) return a.T;
    const int64_t v = a.starts[i];
    return v < 0 ? 0 : v > a.T ? a.T : (int)v;
}
// The sequence that a warp is in (-1 before the first, S behind the last) and where it ends.  The lanes hold the next 32 starts
// and the values c0, c1 of these sequences, so that a boundary costs no load.
struct SeqWalk {
    int base, bound, s, next;
    float c0, c1, v0, v1;
    // whatever the starts hold, s stays within -1 .. S and next grows
    __device__ __forceinline__ void take(int j, int cur) {
        s = base + j;
        next = max(__shfl_sync(0xffffffffu, bound, j), cur + 1);
        v0 = __shfl_sync(0xffffffffu, c0, j);
        v1 = __shfl_sync(0xffffffffu, c1, j);
    }
    // the sequence `to` is known, or found: eight probes a lane and round
    __device__ __forceinline__ void enter(const SeqArgs& a, int to, int cur, const float* p0, const float* p1) {
        const int lane = threadIdx.x & 31, i = to + lane;
        const bool in = i >= 0 && i < a.S;
        base = to;
        bound = seq_start(a, to + 1 + lane);
        c0 = p0 && in ? p0[i] : 0.f;
        c1 = p1 && in ? p1[i] : 0.f;
        take(0, cur);
    }
    __device__ __forceinline__ void locate(const SeqArgs& a, int cur, const float* p0, const float* p1) {
        const int lane = threadIdx.x & 31;
        int at = 0, n = a.S + 1;                              // starts <= cur: all before `at`, none from at + n on
        while (n > 32) {
            const int step = (n + 255) >> 8;
            int k = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = (e * 32 + lane + 1) * step - 1;
                k += i < n && seq_start(a, at + i) <= cur;
            }
            k = __reduce_add_sync(0xffffffffu, k);
            at += k * step;
            n = step == 1 ? 0 : min(step - 1, n - k * step);
        }
        at += __popc(__ballot_sync(0xffffffffu, lane < n && seq_start(a, at + lane) <= cur));
        enter(a, at - 1, cur, p0, p1);
    }
    __device__ __forceinline__ void advance(const SeqArgs& a, int cur, const float* p0, const float* p1) {
        const int j = __popc(__ballot_sync(0xffffffffu, bound <= cur));
        if (j == 32) locate(a, cur, p0, p1);
        else take(j, cur);
    }
};

// Four fp32 of a lane, as two pairs.
struct Quad { uint64_t lo, hi; };
__device__ __forceinline__ void seq_store(float* p, int t, int T, const float (&v)[4]) {
    if (t + 4 <= T) {
        *reinterpret_cast<float4*>(p + t) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (t + i < T) p[t + i] = v[i];
    }
}
__device__ __forceinline__ void seq_unpack(const Quad& q, float (&v)[4]) { unpack2f(q.lo, v[0], v[1]); unpack2f(q.hi, v[2], v[3]); }
__device__ __forceinline__ Quad operator-(const Quad& a, const Quad& b) {      // rounded once
    const uint64_t m = pack2f(-1.f, -1.f);
    return {fma2(b.lo, m, a.lo), fma2(b.hi, m, a.hi)};
}
// What is read once leaves L2 first: a gradient that is scaled at the end should still be there.
__device__ __forceinline__ uint64_t seq_once() {
    uint64_t p;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}
// The steps of a warp come through a ring of its own in shared memory, STAGES - 1 of them under way: registers for a step ahead
// spilled, and a spilled load is waited for.  A lane copies just what it will read, so that nothing is waited for between lanes.
__device__ __forceinline__ void seq_copy16(uint32_t to, const void* p, uint64_t policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(to), "l"(p), "l"(policy) : "memory");
}
// Element i of 4 or 8 bytes where one is left there.
template <typename V>
__device__ __forceinline__ void seq_copy(uint32_t to, const V* p, int i, int left) {
    if (left <= 0) return;
    if (sizeof(V) == 8) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(p + i) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(p + i) : "memory");
}
__device__ __forceinline__ Quad seq_read(uint32_t at) {
    Quad q;
    asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(q.lo), "=l"(q.hi) : "r"(at) : "memory");
    return q;
}
// Bytes of a step: four targets a lane, and four fp32 a lane of each tensor.
__host__ __device__ constexpr int seq_tensors(int op, bool ref, bool each) { return 1 + (op == SEQ_POLICY) + ref + each; }
__host__ __device__ constexpr int seq_stage(int op, bool ref, bool each) { return 512 * (2 + seq_tensors(op, ref, each)); }
// Bytes of a warp: the ring, and the 128 ints of seq_ids.
__host__ __device__ constexpr int seq_bytes(int op, bool ref, bool each, int stages) { return stages * seq_stage(op, ref, each) + 512; }
// Those of a lane's four tokens that lie in cur .. end.
__device__ __forceinline__ uint32_t seq_within(int t, int cur, int end) {
    const int lo = max(cur - t, 0), hi = min(end - t, 4);
    return hi > lo ? (1u << hi) - (1u << lo) : 0u;
}

// Steps in which at least so many sequences end are added up all at once, by lanes, instead of sequence by sequence.
constexpr int kSeqDense = 3;
__device__ __forceinline__ bool seq_dense(const SeqWalk& k, int base, int stop) {
    return __popc(__ballot_sync(0xffffffffu, k.bound > base && k.bound < stop)) >= kSeqDense;
}
// The sequence of each of a lane's four tokens (S behind the last): where one starts its number is put into `ids` (128 ints of the
// warp's own), the largest where several do, and each token takes the largest up to it.  False where more than 256 start in the step.
__device__ __forceinline__ bool seq_ids(const SeqArgs& a, int s, int base, int stop, uint32_t ids, int (&id)[4]) {
    const int lane = threadIdx.x & 31;
    __syncwarp();
    sts128(ids + lane * 16, make_uint4(~0u, ~0u, ~0u, ~0u));
    __syncwarp();
    bool more = true;
#pragma unroll 1
    for (int c = 0; c < 8 && more; ++c) {
        const int64_t i = (int64_t)s + 1 + c * 32 + lane;
        const int at = i <= a.S ? seq_start(a, (int)i) : 0x7FFFFFFF;
        if (at >= base && at < stop) asm volatile("red.shared.max.s32 [%0], %1;" ::"r"(ids + (at - base) * 4), "r"((int)i) : "memory");
        more = __all_sync(0xffffffffu, at < stop);
    }
    __syncwarp();
    const uint4 v = lds128(ids + lane * 16);
    id[0] = (int)v.x;
    id[1] = max(id[0], (int)v.y);
    id[2] = max(id[1], (int)v.z);
    id[3] = max(id[2], (int)v.w);
    int top = id[3];
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int y = __shfl_up_sync(0xffffffffu, top, o);
        if (lane >= o) top = max(top, y);
    }
    int before = __shfl_up_sync(0xffffffffu, top, 1);
    before = lane ? max(before, s) : s;
#pragma unroll
    for (int i = 0; i < 4; ++i) id[i] = max(id[i], before);
    return !more;
}

// e^q: q log2 e with the part of it that fp32 leaves out, so that only ex2's 2^-22 and two roundings are left of the error.  Where
// the result is neither 0 nor infinite that part is below 2^-17; of a large q it is anything (of an infinite one NaN), and 1 + it
// must stay above 0: it is held within 0.01.
__device__ __forceinline__ uint64_t exp_pair(uint64_t q) {
    const float low = (float)(1.4426950408889634 - (double)kLog2e);
    const uint64_t l = pack2f(kLog2e, kLog2e), n = pack2f(kLn2, kLn2), one = pack2f(1.f, 1.f);
    const uint64_t t = mul2(q, l), minus = mul2(t, pack2f(-1.f, -1.f));
    float a, b;
    unpack2f(mul2(fma2(q, pack2f(low, low), fma2(q, l, minus)), n), a, b);
    return mul2(ex2_pair(t), add2(one, pack2f(fmaxf(fminf(a, 0.01f), -0.01f), fmaxf(fminf(b, 0.01f), -0.01f))));
}
// e^d - 1 - d by its series: for |d| < 1 the terms from d^12 / 12! on are below 2^-27 of it (5.3e-9 towards d = -1).
__device__ __forceinline__ uint64_t exp_series(uint64_t d) {
    const float c[10] = {1.f / 39916800, 1.f / 3628800, 1.f / 362880, 1.f / 40320, 1.f / 5040, 1.f / 720, 1.f / 120, 1.f / 24, 1.f / 6, 1.f / 2};
    uint64_t h = pack2f(c[0], c[0]);
#pragma unroll
    for (int i = 1; i < 10; ++i) h = fma2(h, d, pack2f(c[i], c[i]));
    return mul2(mul2(d, d), h);
}

// What the border on an advantage's side asks for (none where it is 0 or NaN: then neither term is the larger).
struct SeqSide {
    float adv, sign, held, edge, close;
    int side;
    __device__ __forceinline__ void choose(const SeqArgs& a, float x) {
        adv = x;
        side = x < 0.f;
        sign = side ? -1.f : 1.f;
        held = side ? a.held[1] : a.held[0];
        const bool there = fabsf(x) > 0.f;
        edge = there ? (side ? a.edge32[1] : a.edge32[0]) : INFINITY;
        close = there ? (side ? a.close[1] : a.close[0]) : -1.f;
    }
};
// `ready` is called between the first copies and the first look at the starts; `first` is where the walk begins.
template <int OP, bool REF, bool EACH, int STAGES, typename F>          // EACH: an advantage for each token
__device__ __forceinline__ void seq_sums(const SeqArgs& a, int w, uint32_t ring, F ready, SeqWalk& first) {
    const int lane = threadIdx.x & 31, lo = w * a.range, hi = a.T - lo < a.range ? a.T : lo + a.range;
    const float* p0 = OP == SEQ_POLICY && !EACH ? a.adv : nullptr;
    const float* p1 = OP == SEQ_POLICY && a.dnll && !a.mean ? a.dloss : nullptr;       // a gradient that needs nothing else
    const uint64_t once = seq_once();
    constexpr int STAGE = seq_stage(OP, REF, EACH);
    const bool pairs = ((uintptr_t)a.target & 15) == 0;           // targets need not lie on 16 bytes
    auto fetch = [&](int from, int ahead, int slot) {
        if (seq_before(from, ahead, hi)) {
            const int base = from + ahead;
            const uint32_t to = ring + slot * STAGE + lane * 16;
            const int t = base + lane * 4;
            if (seq_whole(base, kSeqStep, a.T)) {                 // the usual case
                if (pairs) {
                    seq_copy16(to + lane * 16, a.target + t, once);
                    seq_copy16(to + lane * 16 + 16, a.target + t + 2, once);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) seq_copy(to + lane * 16 + i * 8, a.target + t, i, 1);
                }
                seq_copy16(to + 1024, a.nll + t, once);
                if (OP == SEQ_POLICY) seq_copy16(to + 1536, a.old + t, once);
                if (REF) seq_copy16(to + 512 * (3 + (OP == SEQ_POLICY)), a.ref + t, once);
                if (EACH) seq_copy16(to + STAGE - 512, a.adv + t, once);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    seq_copy(to + lane * 16 + i * 8, a.target + t, i, a.T - t - i);
                    seq_copy(to + 1024 + i * 4, a.nll + t, i, a.T - t - i);
                    if (OP == SEQ_POLICY) seq_copy(to + 1536 + i * 4, a.old + t, i, a.T - t - i);
                    if (REF) seq_copy(to + 512 * (3 + (OP == SEQ_POLICY)) + i * 4, a.ref + t, i, a.T - t - i);
                    if (EACH) seq_copy(to + STAGE - 512 + i * 4, a.adv + t, i, a.T - t - i);
                }
            }
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < (STAGES > 1 ? STAGES - 1 : 1); ++i) fetch(lo, i * kSeqStep, i);
    SeqWalk k;
    SeqSide z;
    float slope = 0.f, kl_slope = 0.f;
    auto arrive = [&] {                                           // at the next sequence
        if (OP != SEQ_POLICY) return;
        if (!EACH) z.choose(a, k.v0);
        slope = a.mean ? 1.f : k.v1;
        kl_slope = a.kl_slope * slope;
    };
    ready();
    k.locate(a, lo, p0, p1);
    first = k;
    arrive();
    bool began = k.s >= 0 && seq_start(a, k.s) >= lo;
    double sa = 0, sb = 0;
    int sn = 0, sc = 0;
    auto flush = [&](SeqSum* to) {
        const double x = warp_sum(sa), y = REF && OP == SEQ_POLICY ? warp_sum(sb) : 0.0;
        const int n = __reduce_add_sync(0xffffffffu, sn), c = OP == SEQ_POLICY ? __reduce_add_sync(0xffffffffu, sc) : 0;
        if (lane == 0) { to->a = x; to->b = y; to->n = n; to->c = c; }
        sa = sb = 0;
        sn = sc = 0;
    };
    bool open = true;
    int slot = 0;
    for (int base = lo; base < hi; base += kSeqStep) {
        const int t = base + lane * 4, stop = min(base + kSeqStep, hi);
        cp_async_wait<(STAGES > 1 ? STAGES - 2 : 0)>();
        const uint32_t at = ring + slot * STAGE;
        const uint4 u = lds128(at + lane * 32), v = lds128(at + lane * 32 + 16);         // the halves with the sign
        uint32_t mine = ~(u.y >> 31 | u.w >> 31 << 1 | v.y >> 31 << 2 | v.w >> 31 << 3) & 15u;
        if (!seq_whole(base, kSeqStep, a.T)) mine &= seq_within(t, 0, a.T);       // behind the last token there is nothing
        Quad nll = {0, 0}, old = {0, 0}, ref = {0, 0}, adv = {0, 0};
        nll = seq_read(at + 1024 + lane * 16);
        if (OP == SEQ_POLICY) old = seq_read(at + 1536 + lane * 16);
        if (REF) ref = seq_read(at + 512 * (3 + (OP == SEQ_POLICY)) + lane * 16);
        if (EACH) adv = seq_read(at + STAGE - 512 + lane * 16);
        if (STAGES > 1) {                                         // into the slot of the step before
            fetch(base, (STAGES - 1) * kSeqStep, slot == 0 ? STAGES - 1 : slot - 1);
            slot = slot + 1 == STAGES ? 0 : slot + 1;
        }
        const bool none = !__any_sync(0xffffffffu, mine), whole = __all_sync(0xffffffffu, mine == 15u);
        uint64_t q[2] = {0, 0}, r[2] = {0, 0}, e1[2] = {0, 0}, e2[2] = {0, 0};
        float A[4], g[4] = {0.f, 0.f, 0.f, 0.f};
        if (a.hint && lane == 0 && base % kScaleRange == 0) a.hint[base / kScaleRange] = k.s;
        if (OP == SEQ_PAIR && a.bits) a.bits[t / 4] = (uint8_t)mine;
        if (none) {
        } else if (OP == SEQ_POLICY) {
            const Quad x = old - nll;
            q[0] = x.lo; q[1] = x.hi;
            r[0] = exp_pair(x.lo); r[1] = exp_pair(x.hi);
            if (REF) {
                const Quad d = nll - ref;
                e2[0] = exp_series(d.lo); e2[1] = exp_series(d.hi);
                e1[0] = add2(d.lo, e2[0]); e1[1] = add2(d.hi, e2[1]);
                float f[4];
                seq_unpack(d, f);
                if (!(fmaxf(fmaxf(fabsf(f[0]), fabsf(f[1])), fmaxf(fabsf(f[2]), fabsf(f[3]))) < 1.f)) {
                    float u[4], v[4];
                    seq_unpack({e1[0], e1[1]}, u);
                    seq_unpack({e2[0], e2[1]}, v);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(fabsf(f[i]) < 1.f)) { u[i] = expf(f[i]) - 1.f; v[i] = u[i] == INFINITY ? u[i] : u[i] - f[i]; }
                    e1[0] = pack2f(u[0], u[1]); e1[1] = pack2f(u[2], u[3]);
                    e2[0] = pack2f(v[0], v[1]); e2[1] = pack2f(v[2], v[3]);
                }
            }
            if (EACH) seq_unpack(adv, A);
        } else if (REF) {
            const Quad x = ref - nll;
            q[0] = x.lo; q[1] = x.hi;
        } else {
            q[0] = mul2(nll.lo, pack2f(-1.f, -1.f)); q[1] = mul2(nll.hi, pack2f(-1.f, -1.f));
        }
        // adds up the tokens of `in`; ALL: every token of the step
        auto tokens = [&](uint32_t in, auto ALL) {
            constexpr bool all = decltype(ALL)::value;
            sn += all ? 4 : __popc(in);
            float x[4], v[4], y[4], d[4];
            seq_unpack({q[0], q[1]}, x);
            float pa = 0.f, pb = 0.f;
            if (OP == SEQ_POLICY) {
                seq_unpack({r[0], r[1]}, v);
                seq_unpack({e1[0], e1[1]}, d);
                seq_unpack({e2[0], e2[1]}, y);
                bool cut[4];
                float nearest = INFINITY;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (EACH) z.choose(a, A[i]);
                    const float o = x[i] * z.sign - z.edge;
                    cut[i] = o > 0.f;
                    nearest = EACH ? fminf(nearest, fabsf(o) - z.close) : fminf(nearest, fabsf(o));
                }
                if (nearest <= (EACH ? 0.f : z.close)) {          // x is rounded; next to a border that may move it across
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (EACH) z.choose(a, A[i]);
                        if (!(fabsf(x[i] * z.sign - z.edge) <= z.close) || t + i >= a.T) continue;
                        cut[i] = ((double)a.old[t + i] - (double)a.nll[t + i]) * (double)z.sign > (z.side ? a.edge[1] : a.edge[0]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (EACH) z.choose(a, A[i]);
                    const bool there = all || (in >> i & 1u);
                    const float term = EACH ? z.adv * (cut[i] ? z.held : v[i]) : cut[i] ? z.held : v[i];
                    if (cut[i] && there) ++sc;
                    pa += there ? term : 0.f;
                    float grad = cut[i] ? 0.f : v[i] * (z.adv * slope);
                    if (REF) {
                        pb += there ? y[i] : 0.f;
                        grad = fmaf(kl_slope, d[i], grad);
                    }
                    g[i] = there ? grad : g[i];
                }
                // a lane without tokens here takes no advantage either: it need not be finite
                if (EACH) pa = -pa;
                else pa = all || in ? pa * -z.adv : 0.f;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) pa += all || (in >> i & 1u) ? x[i] : 0.f;
            }
            sa += (double)pa;
            if (REF && OP == SEQ_POLICY) sb += (double)pb;
        };
        // Many sequences end here: a lane adds up runs of its own four tokens, a scan along the lanes joins what crosses them, and
        // the lane of a sequence's last token has its sums.
        auto dense = [&] {
            int id[4];
            if (!seq_ids(a, k.s, base, stop, ring + STAGES * STAGE, id)) return false;
            const double ca = warp_sum(sa), cb = warp_sum(sb);    // what the first sequence brings along
            const int cn = __reduce_add_sync(0xffffffffu, sn), cc = __reduce_add_sync(0xffffffffu, sc);
            const int begin = k.s;
            auto emit = [&](int s, double x, double y, int n) {   // n: tokens, and clipped ones from bit 16 on
                if (s < 0 || s >= a.S) return;
                const bool carried = s == begin;
                SeqSum* to = carried && !began ? a.head + w : a.whole + s;
                to->a = x + (carried ? ca : 0.0);
                to->b = y + (carried ? cb : 0.0);
                to->n = (n & 0xFFFF) + (carried ? cn : 0);
                to->c = (n >> 16) + (carried ? cc : 0);
            };
            float x[4], v[4], y[4], d[4];
            seq_unpack({q[0], q[1]}, x);
            if (OP == SEQ_POLICY) {
                seq_unpack({r[0], r[1]}, v);
                seq_unpack({e1[0], e1[1]}, d);
                seq_unpack({e2[0], e2[1]}, y);
            }
            float ra = 0.f, rb = 0.f, fa = 0.f, fb = 0.f;         // of the run, and of the lane's first if it is not the last
            int rn = 0, fn = 0;
            bool several = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool valid = id[i] >= 0 && id[i] < a.S, there = valid && (mine >> i & 1u);
                if (i > 0 && id[i] != id[i - 1]) {
                    if (several) { emit(id[i - 1], ra, rb, rn); } else { fa = ra; fb = rb; fn = rn; several = true; }
                    ra = rb = 0.f;
                    rn = 0;
                }
                if (OP == SEQ_POLICY) {
                    z.choose(a, EACH ? A[i] : there ? a.adv[id[i]] : 0.f);
                    const float by = a.mean ? 1.f : there && p1 ? p1[id[i]] : 0.f, o = x[i] * z.sign - z.edge;
                    bool cut = o > 0.f;
                    if (there && fabsf(o) <= z.close)
                        cut = ((double)a.old[t + i] - (double)a.nll[t + i]) * (double)z.sign > (z.side ? a.edge[1] : a.edge[0]);
                    float grad = cut ? 0.f : v[i] * (z.adv * by);
                    if (REF) grad = fmaf(a.kl_slope * by, d[i], grad);
                    if (there) {
                        ra -= z.adv * (cut ? z.held : v[i]);
                        if (REF) rb += y[i];
                        rn += 1 + (cut ? 0x10000 : 0);
                        g[i] = grad;
                    }
                } else if (there) {
                    ra += x[i];
                    rn += 1;
                }
            }
            const int prior = __shfl_up_sync(0xffffffffu, id[3], 1);
            bool head = several || lane == 0 || id[0] != prior;   // the lane's last run begins in it
            double xa = ra, xb = rb;
            int xn = rn;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const double ya = __shfl_up_sync(0xffffffffu, xa, o), yb = REF && OP == SEQ_POLICY ? __shfl_up_sync(0xffffffffu, xb, o) : 0.0;
                const int yn = __shfl_up_sync(0xffffffffu, xn, o);
                const bool yh = __shfl_up_sync(0xffffffffu, (int)head, o) != 0;
                if (lane >= o && !head) { xa += ya; xb += yb; xn += yn; head = yh; }
            }
            const double pa = __shfl_up_sync(0xffffffffu, xa, 1), pb = __shfl_up_sync(0xffffffffu, xb, 1);
            const int pn = __shfl_up_sync(0xffffffffu, xn, 1), after = __shfl_down_sync(0xffffffffu, id[0], 1);
            if (several) {
                const bool on = lane > 0 && id[0] == prior;
                emit(id[0], fa + (on ? pa : 0.0), fb + (on ? pb : 0.0), fn + (on ? pn : 0));
            }
            if (lane < 31 && after != id[3]) emit(id[3], xa, xb, xn);
            // the last sequence stays open, unless it ends with the step
            const int last = __shfl_sync(0xffffffffu, id[3], 31);
            const bool same = last == begin;
            sa = lane == 31 ? xa + (same ? ca : 0.0) : 0.0;
            sb = lane == 31 ? xb + (same ? cb : 0.0) : 0.0;
            sn = lane == 31 ? (xn & 0xFFFF) + (same ? cn : 0) : 0;
            sc = lane == 31 ? (xn >> 16) + (same ? cc : 0) : 0;
            began = began || !same;
            k.enter(a, last, stop, p0, p1);
            if (__shfl_sync(0xffffffffu, k.bound, 0) <= stop) {
                if (last >= 0 && last < a.S) flush(began ? a.whole + last : a.head + w);
                open = stop < hi;
                if (open) k.advance(a, stop, p0, p1);
                began = true;
            }
            arrive();
            return true;
        };
        const bool done = __builtin_expect(seq_dense(k, base, stop), 0) && dense();
        for (int cur = done ? stop : base; cur < stop;) {
            const int end = min(k.next, stop);
            if (!none && k.s >= 0 && k.s < a.S) {
                if (whole && end - cur == kSeqStep) tokens(15u, std::true_type());
                else tokens(mine & seq_within(t, cur, end), std::false_type());
            }
            if (k.next <= stop) {                                 // the sequence ends here
                if (k.s >= 0 && k.s < a.S) flush(began ? a.whole + k.s : a.head + w);
                open = end < hi;
                if (open) { k.advance(a, end, p0, p1); arrive(); }
                began = true;
            }
            cur = end;
        }
        if (OP == SEQ_POLICY && a.dnll) seq_store(a.raw, t, a.T, g);
    }
    if (open && k.s >= 0 && k.s < a.S) flush(began ? a.tail + w : a.head + w);
}

// The range of token t.  Steps are below 2^24 and those of a range below 2^13, so the quotient by 2^40 is exact.
__device__ __forceinline__ int seq_range_of(const SeqArgs& a, int t) { return (int)((uint64_t)(t / kSeqStep) * a.per_range >> 40); }
// 1 / n to 2^-44 by one step of Newton's method, in a few instructions (a division in 64 bits takes some 400 cycles, and a join
// little else).
__device__ __forceinline__ double seq_share(int n) {
    if (n == 0) return 0.0;
    float f;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(f) : "f"((float)n));
    const double w = f;                                           // to 2^-22: a step squares the error
    return w * (2.0 - (double)n * w);
}
// The sums of sequence s over a team of threads: half a warp, a warp or a block of 256.  Member 0 gets them.
template <int TEAM>
__device__ __forceinline__ SeqSum seq_total(const SeqArgs& a, int s, int member) {
    const int64_t from = a.starts[s], to = a.starts[s + 1];
    const int b = seq_start(a, s), e = seq_start(a, s + 1);
    SeqSum t = {0.0, 0.0, 0, 0};
    if (member == 0 && (from < 0 || from > to || to > a.T)) report_index(a.status, MHCLITE_OP_SEQUENCES, s, from);
    if (b >= e) return t;
    const int w0 = seq_range_of(a, b), w1 = seq_range_of(a, e - 1);
    if (w0 == w1) return a.whole[s];
#pragma unroll 4
    for (int w = w0 + member; w <= w1; w += TEAM) {
        const SeqSum p = w == w0 ? a.tail[w] : a.head[w];
        t.a += p.a; t.b += p.b; t.n += p.n; t.c += p.c;
    }
    const uint32_t team = TEAM == 16 ? 0xffffu << (threadIdx.x & 16) : 0xffffffffu;
    __syncwarp(team);
#pragma unroll
    for (int o = TEAM < 32 ? TEAM / 2 : 16; o > 0; o >>= 1) {
        t.a += __shfl_xor_sync(team, t.a, o);
        t.b += __shfl_xor_sync(team, t.b, o);
        t.n += __shfl_xor_sync(team, t.n, o);
        t.c += __shfl_xor_sync(team, t.c, o);
    }
    if (TEAM > 32) {
        __shared__ SeqSum part[TEAM > 32 ? TEAM / 32 : 1];
        __syncthreads();                                          // from the sequence before
        if ((member & 31) == 0) part[member >> 5] = t;
        __syncthreads();
        t = part[0];
        for (int i = 1; i < TEAM / 32; ++i) { t.a += part[i].a; t.b += part[i].b; t.n += part[i].n; t.c += part[i].c; }
    }
    return t;
}
// What item i (a sequence, or a pair of them) gives from its sums.
template <int OP>
__device__ __forceinline__ void seq_give(const SeqArgs& a, int i, const SeqSum& c, const SeqSum& r, float dloss) {
    if (OP == SEQ_POLICY) {
        const double w = a.mean ? seq_share(c.n) : 1.0;
        a.loss[i] = (float)(w * (c.a + a.kl_weight * c.b));
        float* stats = a.stats + 3 * (int64_t)i;
        stats[0] = (float)c.n; stats[1] = (float)c.c; stats[2] = (float)(w * c.b);
        if (a.dnll && a.mean) a.coef[i] = (float)(w * dloss);
    } else {
        const double wc = a.mean ? seq_share(c.n) : 1.0, wr = a.mean ? seq_share(r.n) : 1.0;
        const double rc = a.beta * wc * c.a, rr = a.beta * wr * r.a, x = rc - rr - a.margin;
        const double m = exp(-fabs(x)), soft = log1p(m);          // softplus(-|x|)
        const double share = x > 0 ? a.smoothing : a.smoothing - 1.0;
        a.loss[i] = (float)(share == 0 ? soft : soft + share * x);
        a.stats[2 * i] = (float)rc;
        a.stats[2 * i + 1] = (float)rr;
        if (a.dnll) {
            const double dx = dloss * (a.smoothing - (x > 0 ? m : 1.0) / (1.0 + m));
            a.coef[2 * i] = (float)(-a.beta * wc * dx);
            a.coef[2 * i + 1] = (float)(a.beta * wr * dx);
        }
    }
}
template <int OP, int TEAM>
__device__ __forceinline__ void seq_item(const SeqArgs& a, int i, int member) {
    const float dloss = a.dnll && member == 0 ? a.dloss[i] : 0.f;       // fetched beside the sums
    SeqSum c, r = {0.0, 0.0, 0, 0};
    if (OP == SEQ_POLICY) {
        c = seq_total<TEAM>(a, i, member);
    } else if (TEAM == 32) {                                      // both sequences side by side, half a warp each
        c = seq_total<16>(a, 2 * i + (member >> 4), member & 15);
        __syncwarp();
        r.a = __shfl_down_sync(0xffffffffu, c.a, 16);
        r.n = __shfl_down_sync(0xffffffffu, c.n, 16);
    } else {
        c = seq_total<TEAM>(a, 2 * i, member);
        r = seq_total<TEAM>(a, 2 * i + 1, member);
    }
    if (member == 0) seq_give<OP>(a, i, c, r, dloss);
}
// The sums of a sequence that lies in one range (or is empty); false where there are pieces to add up.
__device__ __forceinline__ bool seq_complete(const SeqArgs& a, int s, SeqSum& t) {
    const int64_t from = a.starts[s], to = a.starts[s + 1];
    const int b = seq_start(a, s), e = seq_start(a, s + 1);
    if (from < 0 || from > to || to > a.T) report_index(a.status, MHCLITE_OP_SEQUENCES, s, from);
    t = {0.0, 0.0, 0, 0};
    if (b >= e) return true;
    if (seq_range_of(a, b) != seq_range_of(a, e - 1)) return false;
    t = a.whole[s];
    return true;
}
// All items, spread over `warps` warps; where there are more, over their lanes too: a lane alone where a sequence is complete, the
// warp where there are pieces.
template <int OP>
__device__ __forceinline__ void seq_items(const SeqArgs& a, int warp, int warps) {
    const int lane = threadIdx.x & 31, items = OP == SEQ_PAIR ? a.S / 2 : a.S;
    if (items <= warps) {
        if (warp < items) seq_item<OP, 32>(a, warp, lane);
        return;
    }
    for (int64_t first = warp; first < items; first += (int64_t)warps * 32) {
        const int64_t i = first + (int64_t)lane * warps;
        bool left = i < items;
        if (left) {
            SeqSum c, r = {0.0, 0.0, 0, 0};
            const float dloss = a.dnll ? a.dloss[i] : 0.f;
            if (OP == SEQ_POLICY ? seq_complete(a, (int)i, c) : seq_complete(a, 2 * (int)i, c) && seq_complete(a, 2 * (int)i + 1, r)) {
                seq_give<OP>(a, (int)i, c, r, dloss);
                left = false;
            }
        }
        for (uint32_t todo = __ballot_sync(0xffffffffu, left); todo; todo &= todo - 1)
            seq_item<OP, 32>(a, (int)(first + (int64_t)(__ffs(todo) - 1) * warps), lane);
    }
}
// A step of the last pass: the raw gradient x, or which tokens count (`mine`), times what the sequences give.
template <int OP, bool DENSE>
__device__ __forceinline__ void seq_scale_step(const SeqArgs& a, SeqWalk& k, int base, int hi, const float4& raw, uint32_t mine, uint32_t ids) {
    const int t = base + (threadIdx.x & 31) * 4, stop = min(base + kSeqStep, hi);
    const float x[4] = {raw.x, raw.y, raw.z, raw.w};
    float g[4] = {0.f, 0.f, 0.f, 0.f};
    int id[4];
    const bool done = DENSE && seq_dense(k, base, stop) && seq_ids(a, k.s, base, stop, ids, id);
    if (done) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float by = id[e] >= 0 && id[e] < a.S ? a.coef[id[e]] : 0.f;
            if (OP == SEQ_POLICY) g[e] = x[e] == 0.f ? 0.f : x[e] * by;
            else g[e] = mine >> e & 1u ? by : 0.f;
        }
        if (stop < hi) {
            k.enter(a, __shfl_sync(0xffffffffu, id[3], 31), stop, a.coef, nullptr);
            if (__shfl_sync(0xffffffffu, k.bound, 0) <= stop) k.advance(a, stop, a.coef, nullptr);
        }
    }
    for (int cur = done ? stop : base; cur < stop;) {
        const int end = min(k.next, stop);
        if (k.s >= 0 && k.s < a.S) {
            const uint32_t in = seq_within(t, cur, end);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (!(in >> e & 1u)) continue;
                if (OP == SEQ_POLICY) g[e] = x[e] == 0.f ? 0.f : x[e] * k.v0;              // tokens that do not count stay 0
                else g[e] = mine >> e & 1u ? k.v0 : 0.f;
            }
        }
        if (k.next <= stop && end < hi) k.advance(a, end, a.coef, nullptr);
        cur = end;
    }
    seq_store(a.dnll, t, a.T, g);
}
template <int OP>
__device__ __forceinline__ void seq_scale_load(const SeqArgs& a, int base, float4& raw, uint32_t& mine) {
    const int t = base + (threadIdx.x & 31) * 4;
    if (OP == SEQ_PAIR) {
        mine = a.bits[t / 4];
    } else if (seq_whole(base, kSeqStep, a.T)) {
        raw = *reinterpret_cast<const float4*>(a.raw + t);
    } else {
        raw = make_float4(t < a.T ? a.raw[t] : 0.f, t + 1 < a.T ? a.raw[t + 1] : 0.f, t + 2 < a.T ? a.raw[t + 2] : 0.f, 0.f);
        if (t + 3 < a.T) raw.w = a.raw[t + 3];
    }
}
// The last pass over the gradient, four steps a warp.  All that seq_sums left is fetched before the wait for the join, behind which
// its results are there.
template <int OP>
__device__ __forceinline__ void seq_scale(const SeqArgs& a, int w, uint32_t ids) {
    const int lane = threadIdx.x & 31, lo = w * kScaleRange, hi = a.T - lo < kScaleRange ? a.T : lo + kScaleRange;
    float4 v[kScaleSteps] = {};
    uint32_t mine[kScaleSteps] = {};
    const int first = a.hint[w];
#pragma unroll
    for (int i = 0; i < kScaleSteps; ++i)
        if (seq_before(lo, i * kSeqStep, hi)) seq_scale_load<OP>(a, lo + i * kSeqStep, v[i], mine[i]);
    pdl_wait();
    SeqWalk k;
    k.enter(a, first, lo, a.coef, nullptr);
    if (k.next >= hi && seq_whole(lo, kScaleRange, a.T) && k.v0 - k.v0 == 0.f) {               // the usual case: one sequence, or none (then v0 is 0)
#pragma unroll
        for (int i = 0; i < kScaleSteps; ++i) {
            float4* to = reinterpret_cast<float4*>(a.dnll + lo + i * kSeqStep) + lane;
            if (OP == SEQ_POLICY) *to = make_float4(v[i].x * k.v0, v[i].y * k.v0, v[i].z * k.v0, v[i].w * k.v0);
            else *to = make_float4(mine[i] & 1u ? k.v0 : 0.f, mine[i] & 2u ? k.v0 : 0.f, mine[i] & 4u ? k.v0 : 0.f, mine[i] & 8u ? k.v0 : 0.f);
        }
        return;
    }
    if (seq_dense(k, lo, hi)) {
#pragma unroll
        for (int i = 0; i < kScaleSteps; ++i)
            if (seq_before(lo, i * kSeqStep, hi)) seq_scale_step<OP, true>(a, k, lo + i * kSeqStep, hi, v[i], mine[i], ids);
        return;
    }
#pragma unroll
    for (int i = 0; i < kScaleSteps; ++i)
        if (seq_before(lo, i * kSeqStep, hi)) seq_scale_step<OP, false>(a, k, lo + i * kSeqStep, hi, v[i], mine[i], ids);
}
__device__ __forceinline__ int seq_scale_warps(const SeqArgs& a) { return (a.T - 1) / kScaleRange + 1; }      // T > 0

template <int OP, bool REF, bool EACH>
__global__ void __launch_bounds__(kSeqBlock, seq_blocks(OP)) seq_sum_k(const SeqArgs a) {
    extern __shared__ __align__(16) unsigned char sm_raw[];
    pdl_wait();
    pdl_launch();
    const int warp = threadIdx.x >> 5, w = blockIdx.x * (kSeqBlock / 32) + warp;
    SeqWalk first;
    if (w < a.W) seq_sums<OP, REF, EACH, seq_stages(OP)>(a, w, smem_u32(sm_raw) + warp * seq_bytes(OP, REF, EACH, seq_stages(OP)), [] {}, first);
}
template <int OP, int TEAM>
__global__ void __launch_bounds__(kSeqBlock) seq_join_k(const SeqArgs a) {
    pdl_wait();
    pdl_launch();
    const int items = OP == SEQ_PAIR ? a.S / 2 : a.S;
    if (TEAM == 1) seq_items<OP>(a, blockIdx.x * (kSeqBlock / 32) + (threadIdx.x >> 5), gridDim.x * (kSeqBlock / 32));
    else
        for (int i = blockIdx.x * (kSeqBlock / TEAM) + threadIdx.x / TEAM; i < items; i += gridDim.x * (kSeqBlock / TEAM)) seq_item<OP, TEAM>(a, i, threadIdx.x % TEAM);
}
// The join's blocks let this kernel begin behind their own wait for seq_sum_k, so what that left may be read before the wait for
// the join.
template <int OP>
__global__ void __launch_bounds__(kSeqBlock) seq_scale_k(const SeqArgs a) {
    __shared__ alignas(16) int ids[kSeqBlock / 32][kSeqStep];
    const int w = blockIdx.x * (kSeqBlock / 32) + (threadIdx.x >> 5);
    if (w < seq_scale_warps(a)) seq_scale<OP>(a, w, smem_u32(ids[threadIdx.x >> 5]));
}
// Few tokens: the three one after another in one launch, of one block, which keeps what its warps exchange, and the starts, in
// shared memory, or (CLUSTER) of eight.
static_assert(kSeqOneS < 512, "a thread a start");
struct SeqShared {
    alignas(16) float raw[kSeqOne];                               // stored by fours
    int64_t starts[kSeqOneS + 1];
    SeqSum whole[kSeqOneS], head[16], tail[16];
    float coef[kSeqOneS], adv[kSeqOneS], dloss[kSeqOneS];
    uint8_t bits[kSeqOne / 4];
};
constexpr int kSeqShared = sizeof(SeqShared);
static_assert(alignof(SeqShared) == 16 && kSeqShared % 16 == 0 && offsetof(SeqShared, raw) % 16 == 0, "16-byte accesses");
template <int OP, bool REF, bool EACH, bool CLUSTER>
__global__ void __launch_bounds__(512) seq_one_k(const SeqArgs args) {
    extern __shared__ __align__(16) unsigned char sm_raw[];
    constexpr int STAGES = CLUSTER ? 4 : 1;
    SeqArgs a = args;
    const int warps = gridDim.x * (blockDim.x >> 5), in = threadIdx.x >> 5, warp = in * gridDim.x + blockIdx.x, lane = threadIdx.x & 31;
    const int items = OP == SEQ_PAIR ? a.S / 2 : a.S;
    const uint32_t ring = smem_u32(sm_raw) + (CLUSTER ? 0 : kSeqShared) + in * seq_bytes(OP, REF, EACH, STAGES);
    const bool scaled = a.dnll && !(OP == SEQ_POLICY && !a.mean);
    pdl_wait();
    pdl_launch();
    auto together = [] {
        __syncwarp();
        if (CLUSTER) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        else __syncthreads();
    };
    SeqShared* sh = reinterpret_cast<SeqShared*>(sm_raw);
    auto ready = [&] {
        if (CLUSTER) return;
        const int i = threadIdx.x;                                // at most 511 sequences, 512 threads
        const int64_t start = i <= a.S ? args.starts[i] : 0;
        // without tokens the advantages are not looked at, and need not be there
        const float adv = OP == SEQ_POLICY && !EACH && a.T > 0 && i < a.S ? args.adv[i] : 0.f, dloss = a.dnll && i < items ? args.dloss[i] : 0.f;
        if (i <= a.S) sh->starts[i] = start;
        if (i < a.S) { sh->adv[i] = adv; sh->dloss[i] = dloss; }
        a.starts = sh->starts; a.whole = sh->whole; a.head = sh->head; a.tail = sh->tail; a.coef = sh->coef;
        if (OP == SEQ_POLICY && !EACH) a.adv = sh->adv;           // for steps in which many sequences end: the walk has taken args.adv
        if (a.dnll) a.dloss = sh->dloss;
        if (scaled) a.raw = sh->raw;
        if (a.bits) a.bits = sh->bits;
        __syncthreads();
    };
    SeqWalk k;
    if (warp < a.W) seq_sums<OP, REF, EACH, STAGES>(a, warp, ring, ready, k);
    else ready();
    together();
    seq_items<OP>(a, warp, warps);
    if (!scaled || a.T == 0) return;
    together();
    if (warp >= a.W) return;
    const int lo = warp * a.range, hi = min(lo + a.range, a.T);       // each warp its own tokens again
    k.enter(a, k.base, lo, a.coef, nullptr);
    for (int base = lo; base < hi; base += kSeqStep) {
        float4 raw = {};
        uint32_t mine = 0;
        seq_scale_load<OP>(a, base, raw, mine);
        seq_scale_step<OP, true>(a, k, base, hi, raw, mine, ring);
    }
}

// ---- host side -------------------------------------------------------------------------------------------------------
static size_t plan_seq(int op, SeqArgs& a, void* base) {
    char* b = (char*)base;
    size_t off = 0;
    auto take = [&](size_t n) { char* at = b + off; off += (n + 255) & ~(size_t)255; return at; };
    const int steps = (a.T + kSeqStep - 1) / kSeqStep;
    const int most = seq_cluster(a.T, a.S) ? kSeqClusterWarps : seq_ranges(op);
    a.range = (steps + most - 1) / most * kSeqStep;
    if (a.range == 0) a.range = kSeqStep;
    a.W = (int)(((int64_t)a.T + a.range - 1) / a.range);
    const int each = a.range / kSeqStep;
    a.per_range = (((uint64_t)1 << 40) + each - 1) / each;
    a.whole = (SeqSum*)take((size_t)a.S * sizeof(SeqSum));
    a.head = (SeqSum*)take((size_t)a.W * sizeof(SeqSum));
    a.tail = (SeqSum*)take((size_t)a.W * sizeof(SeqSum));
    a.coef = (float*)take((size_t)a.S * 4);
    a.bits = (uint8_t*)take((size_t)steps * 32);
    a.hint = (int*)take((size_t)(steps + kScaleSteps - 1) / kScaleSteps * 4);
    a.raw = a.dnll;
    return off;
}
size_t seq_scratch_bytes(int64_t T, int64_t S) {
    if (seq_one(T, S)) return 0;
    SeqArgs a = {};
    a.T = (int)T;
    a.S = (int)S;
    const size_t p = plan_seq(SEQ_POLICY, a, nullptr), q = plan_seq(SEQ_PAIR, a, nullptr);
    return p > q ? p : q;
}

template <int OP, bool REF, bool EACH>
static void launch_seq(const mhclite_ctx* c, SeqArgs& a, void* scratch, cudaStream_t s) {
    plan_seq(OP, a, scratch);
    a.status = c->op_status;
    const bool scaled = a.dnll && !(OP == SEQ_POLICY && !a.mean);
    if (!scaled || seq_cluster(a.T, a.S)) a.hint = nullptr;
    if (OP == SEQ_POLICY || !scaled) a.bits = nullptr;
    const int items = OP == SEQ_PAIR ? a.S / 2 : a.S, blocks = (a.W + kSeqBlock / 32 - 1) / (kSeqBlock / 32), most = c->sm_count * 16;
    if (seq_cluster(a.T, a.S)) {                                  // every case of one block is one of these
        c->launches += 1;
        constexpr int one = kSeqShared + 16 * seq_bytes(OP, REF, EACH, 1), eight = 16 * seq_bytes(OP, REF, EACH, 4);
        if (seq_one(a.T, a.S)) {
            static SmemOnce once;
            smem_limit(once, seq_one_k<OP, REF, EACH, false>, c->device, one);
            launch_after(seq_one_k<OP, REF, EACH, false>, dim3(1), dim3(512), one, s, a);
        } else {
            static SmemOnce once;
            smem_limit(once, seq_one_k<OP, REF, EACH, true>, c->device, eight);
            launch_cluster_after(seq_one_k<OP, REF, EACH, true>, dim3(8), dim3(512), 8, eight, s, a);
        }
        return;
    }
    c->launches += blocks > 0 ? 2 : 1;
    constexpr int ring = kSeqBlock / 32 * seq_bytes(OP, REF, EACH, seq_stages(OP));
    static SmemOnce once;
    smem_limit(once, seq_sum_k<OP, REF, EACH>, c->device, ring);
    if (blocks > 0) launch_after(seq_sum_k<OP, REF, EACH>, dim3(blocks), dim3(kSeqBlock), ring, s, a);
    // a block where sequences have more pieces on average than a warp adds up at a time, a warp each as long as there are enough
    // warps under way, then a lane each
    if (a.W > (int64_t)items * 32) launch_after(seq_join_k<OP, kSeqBlock>, dim3(items), dim3(kSeqBlock), 0, s, a);
    else if (items <= most * 8) launch_after(seq_join_k<OP, 32>, dim3((items + 7) / 8), dim3(kSeqBlock), 0, s, a);
    else launch_after(seq_join_k<OP, 1>, dim3(most), dim3(kSeqBlock), 0, s, a);
    if (!scaled) return;
    c->launches += 1;
    const int scale = (a.T - 1) / kScaleRange + 1;
    launch_after(seq_scale_k<OP>, dim3((scale + kSeqBlock / 32 - 1) / (kSeqBlock / 32)), dim3(kSeqBlock), 0, s, a);
}

// A border of x: its value, in fp32, and how close to that a log ratio rounded to fp32 has to be for its side to be in doubt
// (a few units in the last place; where there is no border, never).
static void seq_border(SeqArgs& a, int side, double edge, double held) {
    a.edge[side] = edge;
    a.edge32[side] = (float)edge;
    a.close[side] = isinf(edge) ? -1.f : fabsf((float)edge) * 2.4e-7f + 1e-40f;
    a.held[side] = (float)held;
}
void launch_policy_loss(const mhclite_ctx* c, int64_t T, int64_t S, const float* nll, const float* nll_old, const float* nll_ref,
                        const int64_t* target, const int64_t* starts, const float* adv, int token_adv, double clip_low, double clip_high,
                        double kl_weight, int mean, const float* dloss, float* loss, float* stats, float* dnll, void* scratch, cudaStream_t s) {
    SeqArgs a = {};
    a.T = (int)T; a.S = (int)S; a.nll = nll; a.old = nll_old; a.ref = nll_ref; a.adv = adv; a.dloss = dloss; a.target = target; a.starts = starts;
    a.mean = mean; a.kl_weight = kl_weight; a.kl_slope = (float)kl_weight; a.loss = loss; a.stats = stats; a.dnll = dnll;
    seq_border(a, 0, log1p(clip_high), 1.0 + clip_high);
    seq_border(a, 1, -log1p(-clip_low), 1.0 - clip_low);
    if (nll_ref) token_adv ? launch_seq<SEQ_POLICY, true, true>(c, a, scratch, s) : launch_seq<SEQ_POLICY, true, false>(c, a, scratch, s);
    else token_adv ? launch_seq<SEQ_POLICY, false, true>(c, a, scratch, s) : launch_seq<SEQ_POLICY, false, false>(c, a, scratch, s);
}
void launch_preference_loss(const mhclite_ctx* c, int64_t T, int64_t P, const float* nll, const float* nll_ref, const int64_t* target,
                            const int64_t* starts, double beta, double margin, double smoothing, int mean, const float* dloss, float* loss,
                            float* reward, float* dnll, void* scratch, cudaStream_t s) {
    SeqArgs a = {};
    a.T = (int)T; a.S = (int)(2 * P); a.nll = nll; a.ref = nll_ref; a.dloss = dloss; a.target = target; a.starts = starts; a.mean = mean;
    a.beta = beta; a.margin = margin; a.smoothing = smoothing; a.loss = loss; a.stats = reward; a.dnll = dnll;
    if (nll_ref) launch_seq<SEQ_PAIR, true, false>(c, a, scratch, s);
    else launch_seq<SEQ_PAIR, false, false>(c, a, scratch, s);
}

}  // namespace mhcl
