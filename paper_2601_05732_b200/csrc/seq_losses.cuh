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
// (1 / n, the pair's slope) is put on by a last pass.
// Sums: four tokens in fp32, from there in 64 bits.
#pragma once

namespace mhcl {

enum SeqOp { SEQ_POLICY = 0, SEQ_PAIR = 1 };
constexpr int kSeqStep = 128;                 // tokens of a warp's step
constexpr int kSeqWarps = 148 * 32;           // ranges at most (the plan gives the scratch's size, so it does not look at the device)
constexpr int kSeqBlock = 256;
constexpr int kSeqOne = 32 * kSeqStep;        // up to here one block does it all in one launch

struct SeqSum { double a, b; int n, c; };     // policy: pg, kl, tokens, clipped ones; preference: log ratio, -, tokens, -

struct SeqArgs {
    int T, S, W, range;                       // W ranges of `range` tokens, a multiple of kSeqStep
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
    uint4* bits;                              // [steps] which tokens have a target (preference)
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
    __device__ __forceinline__ void locate(const SeqArgs& a, int cur, const float* p0, const float* p1) {
        const int lane = threadIdx.x & 31;
        int at = 0, n = a.S + 1;                              // starts <= cur: all before `at`, none from at + n on
        while (n > 32) {
            const int step = (n + 31) / 32, i = (lane + 1) * step - 1;
            const int k = __popc(__ballot_sync(0xffffffffu, i < n && seq_start(a, at + i) <= cur));
            at += k * step;
            n = min(step, n - k * step);
        }
        base = at + __popc(__ballot_sync(0xffffffffu, lane < n && seq_start(a, at + lane) <= cur)) - 1;
        bound = seq_start(a, base + 1 + lane);
        const int i = base + lane;
        const bool in = i >= 0 && i < a.S;
        c0 = p0 && in ? p0[i] : 0.f;
        c1 = p1 && in ? p1[i] : 0.f;
        take(0, cur);
    }
    __device__ __forceinline__ void advance(const SeqArgs& a, int cur, const float* p0, const float* p1) {
        const int j = __popc(__ballot_sync(0xffffffffu, bound <= cur));
        if (j == 32) locate(a, cur, p0, p1);
        else take(j, cur);
    }
};

// Four fp32 of a lane, as two pairs; zeros behind the last token.
struct Quad { uint64_t lo, hi; };
__device__ __forceinline__ Quad seq_load(const float* p, int t, int T, uint64_t policy) {
    float v[4];
    if (t + 4 <= T) {
        asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v4.f32 {%0, %1, %2, %3}, [%4], %5;"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "l"(p + t), "l"(policy));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = t + i < T ? p[t + i] : 0.f;
    }
    return {pack2f(v[0], v[1]), pack2f(v[2], v[3])};
}
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
// Which of a step's tokens have a target.  The lanes read side by side (targets need not lie on 16 bytes), and of each target only
// the half that has the sign, and vote.
struct Targets { int sign[4]; };
__device__ __forceinline__ Targets seq_targets(const int64_t* target, int base, int T) {
    Targets v;
    const int t = base + (threadIdx.x & 31);
#pragma unroll
    for (int i = 0; i < 4; ++i) v.sign[i] = t + i * 32 < T ? reinterpret_cast<const int*>(target + t + i * 32)[1] : -1;
    return v;
}
__device__ __forceinline__ uint4 seq_votes(const Targets& v) {
    return make_uint4(__ballot_sync(0xffffffffu, v.sign[0] >= 0), __ballot_sync(0xffffffffu, v.sign[1] >= 0),
                      __ballot_sync(0xffffffffu, v.sign[2] >= 0), __ballot_sync(0xffffffffu, v.sign[3] >= 0));
}
__device__ __forceinline__ uint32_t seq_mine(const uint4& b) {
    const int lane = threadIdx.x & 31;
    const uint32_t lo = lane & 8 ? b.y : b.x, hi = lane & 8 ? b.w : b.z;
    return (lane & 16 ? hi : lo) >> ((lane & 7) * 4) & 15u;
}
// Those of a lane's four tokens that lie in cur .. end.
__device__ __forceinline__ uint32_t seq_within(int t, int cur, int end) {
    const int lo = max(cur - t, 0), hi = min(end - t, 4);
    return hi > lo ? (1u << hi) - (1u << lo) : 0u;
}

// e^q: q log2 e with the part of it that fp32 leaves out, so that only ex2's 2^-22 and two roundings are left of the error.
__device__ __forceinline__ uint64_t exp_pair(uint64_t q) {
    const float low = (float)(1.4426950408889634 - (double)kLog2e);
    const uint64_t l = pack2f(kLog2e, kLog2e), n = pack2f(kLn2, kLn2), one = pack2f(1.f, 1.f);
    const uint64_t t = mul2(q, l), minus = mul2(t, pack2f(-1.f, -1.f));
    float a, b;
    unpack2f(mul2(fma2(q, pack2f(low, low), fma2(q, l, minus)), n), a, b);
    return mul2(ex2_pair(t), add2(one, pack2f(fminf(a, 0.01f), fminf(b, 0.01f))));      // of an infinite q the rest is NaN: it goes
}
// e^d - 1 - d by its series: for |d| < 1 the terms from d^12 / 12! on are below 2^-28 of it.
__device__ __forceinline__ uint64_t exp_series(uint64_t d) {
    const float c[10] = {1.f / 39916800, 1.f / 3628800, 1.f / 362880, 1.f / 40320, 1.f / 5040, 1.f / 720, 1.f / 120, 1.f / 24, 1.f / 6, 1.f / 2};
    uint64_t h = pack2f(c[0], c[0]);
#pragma unroll
    for (int i = 1; i < 10; ++i) h = fma2(h, d, pack2f(c[i], c[i]));
    return mul2(mul2(d, d), h);
}

template <int OP, bool REF, bool EACH>                       // EACH: an advantage for each token
__device__ __forceinline__ void seq_sums(const SeqArgs& a, int w) {
    const int lane = threadIdx.x & 31, lo = w * a.range, hi = a.T - lo < a.range ? a.T : lo + a.range;
    const float* p0 = OP == SEQ_POLICY && !EACH ? a.adv : nullptr;
    const float* p1 = OP == SEQ_POLICY && a.dnll && !a.mean ? a.dloss : nullptr;       // a gradient that needs nothing else
    const uint64_t once = seq_once();
    Targets target;
    Quad nll, old = {0, 0}, ref = {0, 0}, adv = {0, 0};
    auto fetch = [&](int base) {
        const int t = base + lane * 4;
        target = seq_targets(a.target, base, a.T);
        nll = seq_load(a.nll, t, a.T, once);
        if (OP == SEQ_POLICY) old = seq_load(a.old, t, a.T, once);
        if (REF) ref = seq_load(a.ref, t, a.T, once);
        if (EACH) adv = seq_load(a.adv, t, a.T, once);
    };
    fetch(lo);
    SeqWalk k;
    k.locate(a, lo, p0, p1);
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
    for (int base = lo; base < hi; base += kSeqStep) {
        const int t = base + lane * 4, stop = min(base + kSeqStep, hi);
        const uint4 votes = seq_votes(target);
        const uint32_t mine = seq_mine(votes);
        float q[4], r[4], e1[4], e2[4], A[4], g[4] = {0.f, 0.f, 0.f, 0.f};
        const Quad n0 = nll, o0 = old;
        if (OP == SEQ_POLICY) {
            const Quad x = old - nll;
            seq_unpack(x, q);
            seq_unpack({exp_pair(x.lo), exp_pair(x.hi)}, r);
            if (REF) {
                const Quad d = nll - ref, y = {exp_series(d.lo), exp_series(d.hi)};
                seq_unpack({add2(d.lo, y.lo), add2(d.hi, y.hi)}, e1);
                seq_unpack(y, e2);
                float f[4];
                seq_unpack(d, f);
                if (!(fmaxf(fmaxf(fabsf(f[0]), fabsf(f[1])), fmaxf(fabsf(f[2]), fabsf(f[3]))) < 1.f)) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(fabsf(f[i]) < 1.f)) { e1[i] = expf(f[i]) - 1.f; e2[i] = e1[i] == INFINITY ? e1[i] : e1[i] - f[i]; }
                }
            }
            if (EACH) seq_unpack(adv, A);
        } else {
            if (a.bits && lane == 0) a.bits[base / kSeqStep] = votes;
            if (REF) {
                seq_unpack(ref - nll, q);
            } else {
                seq_unpack(nll, q);
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = -q[i];
            }
        }
        if (base + kSeqStep < hi) fetch(base + kSeqStep);
        for (int cur = base; cur < stop;) {
            const int end = min(k.next, stop);
            if (k.s >= 0 && k.s < a.S) {
                const uint32_t in = mine & seq_within(t, cur, end);
                sn += __popc(in);
                float pa = 0.f, pb = 0.f;
                if (OP == SEQ_POLICY) {
                    const float slope = a.mean ? 1.f : k.v1, kl_slope = a.kl_slope * slope;
                    float held = 0.f, edge = 0.f, close = 0.f, sign = 1.f, adv_i = k.v0;
                    int side = 0;
                    auto choose = [&](float x) {                  // 0: no border
                        adv_i = x;
                        side = x < 0.f;
                        sign = x < 0.f ? -1.f : 1.f;
                        held = a.held[side];
                        edge = x != 0.f ? a.edge32[side] : INFINITY;
                        close = x != 0.f ? a.close[side] : -1.f;
                    };
                    if (!EACH) choose(k.v0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (EACH) choose(A[i]);
                        const float x = q[i] * sign;
                        bool cut = x > edge;
                        if (fabsf(x - edge) <= close) {           // q is rounded; next to a border that may move it across
                            float on[4], ox[4];
                            seq_unpack(n0, on);
                            seq_unpack(o0, ox);
                            cut = ((double)ox[i] - (double)on[i]) * (double)sign > a.edge[side];
                        }
                        const bool there = in >> i & 1u;
                        sc += cut && there;
                        pa -= there ? adv_i * (cut ? held : r[i]) : 0.f;
                        float grad = cut ? 0.f : adv_i * slope * r[i];
                        if (REF) {
                            pb += there ? e2[i] : 0.f;
                            grad = fmaf(kl_slope, e1[i], grad);
                        }
                        if (there) g[i] = grad;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) pa += in >> i & 1u ? q[i] : 0.f;
                }
                sa += (double)pa;
                if (REF && OP == SEQ_POLICY) sb += (double)pb;
            }
            if (k.next <= stop) {                                 // the sequence ends here
                if (k.s >= 0 && k.s < a.S) flush(began ? a.whole + k.s : a.head + w);
                open = end < hi;
                if (open) k.advance(a, end, p0, p1);
                began = true;
            }
            cur = end;
        }
        if (OP == SEQ_POLICY && a.dnll) seq_store(a.dnll, t, a.T, g);
    }
    if (open && k.s >= 0 && k.s < a.S) flush(began ? a.tail + w : a.head + w);
}

// The sums of sequence s over a team of threads (a warp or a block of 256): all threads of the team get them.
template <int TEAM>
__device__ __forceinline__ SeqSum seq_total(const SeqArgs& a, int s, int member) {
    const int b = seq_start(a, s), e = seq_start(a, s + 1);
    SeqSum t = {0.0, 0.0, 0, 0};
    if (member == 0 && (a.starts[s] < 0 || a.starts[s] > a.starts[s + 1] || a.starts[s + 1] > a.T))
        report_index(a.status, MHCLITE_OP_SEQUENCES, s, a.starts[s]);
    if (b >= e) return t;
    const int w0 = b / a.range, w1 = (e - 1) / a.range;
    if (w0 == w1) return a.whole[s];
#pragma unroll 4
    for (int w = w0 + member; w <= w1; w += TEAM) {
        const SeqSum p = w == w0 ? a.tail[w] : a.head[w];
        t.a += p.a; t.b += p.b; t.n += p.n; t.c += p.c;
    }
    t.a = warp_sum(t.a); t.b = warp_sum(t.b);
    t.n = __reduce_add_sync(0xffffffffu, t.n); t.c = __reduce_add_sync(0xffffffffu, t.c);
    if (TEAM > 32) {
        __shared__ SeqSum part[TEAM / 32];
        __syncthreads();                                          // from the sequence before
        if ((member & 31) == 0) part[member >> 5] = t;
        __syncthreads();
        t = part[0];
        for (int i = 1; i < TEAM / 32; ++i) { t.a += part[i].a; t.b += part[i].b; t.n += part[i].n; t.c += part[i].c; }
    }
    return t;
}
// What item i (a sequence, or a pair of them) gives.
template <int OP, int TEAM>
__device__ __forceinline__ void seq_item(const SeqArgs& a, int i, int member) {
    if (OP == SEQ_POLICY) {
        const SeqSum t = seq_total<TEAM>(a, i, member);
        if (member != 0) return;
        const double w = a.mean ? (t.n ? 1.0 / t.n : 0.0) : 1.0;
        a.loss[i] = (float)(w * (t.a + a.kl_weight * t.b));
        a.stats[3 * i] = (float)t.n;
        a.stats[3 * i + 1] = (float)t.c;
        a.stats[3 * i + 2] = (float)(w * t.b);
        if (a.dnll && a.mean) a.coef[i] = (float)(w * a.dloss[i]);
    } else {
        const SeqSum c = seq_total<TEAM>(a, 2 * i, member), r = seq_total<TEAM>(a, 2 * i + 1, member);
        if (member != 0) return;
        const double wc = a.mean ? (c.n ? 1.0 / c.n : 0.0) : 1.0, wr = a.mean ? (r.n ? 1.0 / r.n : 0.0) : 1.0;
        const double rc = a.beta * wc * c.a, rr = a.beta * wr * r.a, x = rc - rr - a.margin;
        const double m = exp(-fabs(x)), soft = log1p(m);          // softplus(-|x|)
        const double share = x > 0 ? a.smoothing : a.smoothing - 1.0;
        a.loss[i] = (float)(share == 0 ? soft : soft + share * x);
        a.stats[2 * i] = (float)rc;
        a.stats[2 * i + 1] = (float)rr;
        if (a.dnll) {
            const double dx = a.dloss[i] * (a.smoothing - (x > 0 ? m : 1.0) / (1.0 + m));
            a.coef[2 * i] = (float)(-a.beta * wc * dx);
            a.coef[2 * i + 1] = (float)(a.beta * wr * dx);
        }
    }
}
// The last pass over the gradient: four steps of tokens times what their sequences give, all of them fetched first.
constexpr int kScaleSteps = 4, kScaleRange = kScaleSteps * kSeqStep;
template <int OP>
__device__ __forceinline__ void seq_scale(const SeqArgs& a, int w) {
    const int lane = threadIdx.x & 31, lo = w * kScaleRange, hi = a.T - lo < kScaleRange ? a.T : lo + kScaleRange;
    Quad v[kScaleSteps];
    uint32_t mine[kScaleSteps];
    const uint64_t once = seq_once();
#pragma unroll
    for (int i = 0; i < kScaleSteps; ++i) {
        const int base = lo + i * kSeqStep;
        if (base >= hi) break;
        if (OP == SEQ_POLICY) v[i] = seq_load(a.dnll, base + lane * 4, a.T, once);
        else mine[i] = seq_mine(a.bits[base / kSeqStep]);
    }
    SeqWalk k;
    k.locate(a, lo, a.coef, nullptr);
#pragma unroll
    for (int i = 0; i < kScaleSteps; ++i) {
        const int base = lo + i * kSeqStep;
        if (base >= hi) break;
        const int t = base + lane * 4, stop = min(base + kSeqStep, hi);
        float x[4], g[4] = {0.f, 0.f, 0.f, 0.f};
        if (OP == SEQ_POLICY) seq_unpack(v[i], x);
        for (int cur = base; cur < stop;) {
            const int end = min(k.next, stop);
            if (k.s >= 0 && k.s < a.S) {
                const uint32_t in = seq_within(t, cur, end);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (!(in >> e & 1u)) continue;
                    if (OP == SEQ_POLICY) g[e] = x[e] == 0.f ? 0.f : x[e] * k.v0;          // tokens that do not count stay 0
                    else g[e] = mine[i] >> e & 1u ? k.v0 : 0.f;
                }
            }
            if (k.next <= stop && end < hi) k.advance(a, end, a.coef, nullptr);
            cur = end;
        }
        seq_store(a.dnll, t, a.T, g);
    }
}
__device__ __forceinline__ int seq_scale_warps(const SeqArgs& a) { return (a.T - 1) / kScaleRange + 1; }      // T > 0

// Four blocks an SM: as many ranges as are under way at once.
template <int OP, bool REF, bool EACH>
__global__ void __launch_bounds__(kSeqBlock, 4) seq_sum_k(const SeqArgs a) {
    pdl_wait();
    pdl_launch();
    const int w = blockIdx.x * (kSeqBlock / 32) + (threadIdx.x >> 5);
    if (w < a.W) seq_sums<OP, REF, EACH>(a, w);
}
template <int OP, int TEAM>
__global__ void __launch_bounds__(kSeqBlock) seq_join_k(const SeqArgs a) {
    pdl_wait();
    pdl_launch();
    const int items = OP == SEQ_PAIR ? a.S / 2 : a.S, member = threadIdx.x % TEAM;
    for (int i = blockIdx.x * (kSeqBlock / TEAM) + threadIdx.x / TEAM; i < items; i += gridDim.x * (kSeqBlock / TEAM)) seq_item<OP, TEAM>(a, i, member);
}
template <int OP>
__global__ void __launch_bounds__(kSeqBlock) seq_scale_k(const SeqArgs a) {
    pdl_wait();
    pdl_launch();
    const int w = blockIdx.x * (kSeqBlock / 32) + (threadIdx.x >> 5);
    if (w < seq_scale_warps(a)) seq_scale<OP>(a, w);
}
// A handful of tokens: the three one after another in one block.
template <int OP, bool REF, bool EACH>
__global__ void __launch_bounds__(1024) seq_one_k(const SeqArgs a) {
    pdl_wait();
    pdl_launch();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, items = OP == SEQ_PAIR ? a.S / 2 : a.S;
    if (warp < a.W) seq_sums<OP, REF, EACH>(a, warp);
    __syncthreads();
    for (int i = warp; i < items; i += 32) seq_item<OP, 32>(a, i, lane);
    if (!a.dnll || (OP == SEQ_POLICY && !a.mean)) return;
    __syncthreads();
    if (warp < seq_scale_warps(a)) seq_scale<OP>(a, warp);
}

// ---- host side -------------------------------------------------------------------------------------------------------
static size_t plan_seq(SeqArgs& a, void* base) {
    char* b = (char*)base;
    size_t off = 0;
    auto take = [&](size_t n) { char* at = b + off; off += (n + 255) & ~(size_t)255; return at; };
    const int steps = (a.T + kSeqStep - 1) / kSeqStep;
    a.range = (int)((steps + (int64_t)kSeqWarps - 1) / kSeqWarps) * kSeqStep;
    if (a.range == 0) a.range = kSeqStep;
    a.W = (int)(((int64_t)a.T + a.range - 1) / a.range);
    a.whole = (SeqSum*)take((size_t)a.S * sizeof(SeqSum));
    a.head = (SeqSum*)take((size_t)a.W * sizeof(SeqSum));
    a.tail = (SeqSum*)take((size_t)a.W * sizeof(SeqSum));
    a.coef = (float*)take((size_t)a.S * 4);
    a.bits = (uint4*)take((size_t)steps * 16);
    return off;
}
size_t seq_scratch_bytes(int64_t T, int64_t S) {
    SeqArgs a = {};
    a.T = (int)T;
    a.S = (int)S;
    return plan_seq(a, nullptr);
}

template <int OP, bool REF, bool EACH>
static void launch_seq(const mhclite_ctx* c, SeqArgs& a, void* scratch, cudaStream_t s) {
    plan_seq(a, scratch);
    a.status = c->op_status;
    if (OP == SEQ_POLICY || !a.dnll) a.bits = nullptr;
    const int items = OP == SEQ_PAIR ? a.S / 2 : a.S, blocks = (a.W + kSeqBlock / 32 - 1) / (kSeqBlock / 32), most = c->sm_count * 16;
    if (a.T <= kSeqOne) {
        c->launches += 1;
        launch_after(seq_one_k<OP, REF, EACH>, dim3(1), dim3(1024), 0, s, a);
        return;
    }
    c->launches += 2;
    launch_after(seq_sum_k<OP, REF, EACH>, dim3(blocks), dim3(kSeqBlock), 0, s, a);
    // a warp adds up 32 pieces at a time: a block where sequences have more of them on average
    const int warps = (items + kSeqBlock / 32 - 1) / (kSeqBlock / 32);
    if (a.W > (int64_t)items * 32) launch_after(seq_join_k<OP, kSeqBlock>, dim3(items), dim3(kSeqBlock), 0, s, a);
    else launch_after(seq_join_k<OP, 32>, dim3(warps < most ? warps : most), dim3(kSeqBlock), 0, s, a);
    if (!a.dnll || (OP == SEQ_POLICY && !a.mean)) return;
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
