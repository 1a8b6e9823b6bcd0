// The seam between the mixing step and the caller's sublayer: the norm that opens the sublayer,
//   v = u r w,   r = (mean_c u^2 + eps)^-1/2,
// and what closes it,
//   y = s drop(sigmoid(a) o r w),
// with their gradients; and dropout on its own.  drop(z) is z / (1 - p) where the element stays and 0 where not
// (philox.cuh).  All of them move bf16 rows once and are bound by HBM; everything between load and store is fp32.
//
// A row belongs to a team of warps, VPT 16-byte vectors a lane.  Teams are persistent: each lane copies its own vectors of
// the team's next rows into shared memory (cp.async, STAGES - 1 rows ahead, 25 to 144 KB in flight on an SM), so a row's
// latency, its sum over the team and its arithmetic overlap the arrival of the rows behind it, and a tensor is read once.
// A lane reads back only what it copied itself: the ring needs no barrier.  The gradients keep the column sums (dw) of
// their rows in registers and leave one partial row a block; colsum_k adds the blocks up in a fixed order, so results are
// the same bit for bit from run to run.
#include "common.cuh"
#include "kernels.h"
#include "mma.cuh"
#include "philox.cuh"
#include "tc.cuh"

#include <float.h>

namespace mhcl {

constexpr int kMaxTeamWarps = 16;
__host__ __device__ constexpr int fwd_stages(int vpt) { return vpt == 4 ? 2 : 4; }
__host__ __device__ constexpr int bwd_stages(int vpt) { return vpt == 4 ? 2 : 4; }

// The threads' places: `wpr` warps a team, `lt` the thread's index in its team.
struct Team {
    int wpr, threads, teams, team, lt;
    __device__ __forceinline__ explicit Team(int wpr_) : wpr(wpr_), threads(wpr_ * 32) {
        teams = blockDim.x / threads; team = threadIdx.x / threads; lt = threadIdx.x - team * threads;
    }
};
// Sum over the team's warps; every thread of the team gets it.  `slot` alternates so that one barrier a sum is enough.
__device__ __forceinline__ float team_sum(float v, float* red, int& slot, const Team& tm) {
    v = warp_sum(v);
    if (tm.wpr == 1) return v;
    float* r = red + slot * kMaxTeamWarps + tm.team * tm.wpr;
    if ((threadIdx.x & 31) == 0) r[tm.lt >> 5] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(tm.team + 1), "r"(tm.threads) : "memory");
    float s = 0.f;
    for (int i = 0; i < tm.wpr; ++i) s += r[i];
    slot ^= 1;
    return s;
}
// Copies this lane's vectors of one row into a stage: [vector][thread] of 16 bytes.
template <int VPT>
__device__ __forceinline__ void fetch_row(uint32_t to, const uint4* row, const Team& tm, int nv) {
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int v = tm.lt + k * tm.threads;
        cp_async16(to + k * blockDim.x * 16, row + (v < nv ? v : 0), v < nv ? 16 : 0);
    }
}

// A gate's pair a as x = e^-a = 2^(-a log2 e), from which sigma(a) = 1 / (1 + x) and 1 - sigma(a) = x sigma(a), both without
// cancellation (1 - sigma formed by subtraction has no digit left from a = 17 on).  x overflows to infinity for a far below 0;
// its reciprocal is 0, and so is the product, formed with the largest finite number in its place.  The approximate exponential
// and reciprocal are off by 2^-22, against the results' rounding to bf16 by 2^-8.
__device__ __forceinline__ uint64_t exp_minus2(uint64_t a) {
    float x, y;
    unpack2f(mul2(a, pack2f(-1.4426950408889634f, -1.4426950408889634f)), x, y);
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(x));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(y));
    return pack2f(x, y);
}
__device__ __forceinline__ uint64_t sigmoid_of_exp2(uint64_t xy) {
    float x, y;
    unpack2f(add2(xy, pack2f(1.f, 1.f)), x, y);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(x));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(y));
    return pack2f(x, y);
}
__device__ __forceinline__ uint64_t sigmoid2(uint64_t a) { return sigmoid_of_exp2(exp_minus2(a)); }
__device__ __forceinline__ uint64_t finite2(uint64_t xy) {
    float x, y;
    unpack2f(xy, x, y);
    return pack2f(fminf(x, FLT_MAX), fminf(y, FLT_MAX));
}
__device__ __forceinline__ uint64_t both(float x) { return pack2f(x, x); }
// the 8 weights of a vector, as packed pairs
__device__ __forceinline__ void load_w(const float4* w, int v, uint64_t* o) {
    const ulonglong2 a = ld_dep((const ulonglong2*)w + 2 * v), b = ld_dep((const ulonglong2*)w + 2 * v + 1);
    o[0] = a.x; o[1] = a.y; o[2] = b.x; o[3] = b.y;
}

struct DropArgs {
    const uint64_t* rng;      // device (seed, offset); null: no dropout
    uint32_t threshold;       // in units of 2^-16
    float factor;
};

// The arithmetic runs on packed pairs (two fp32 operations an instruction): with gate and dropout a vector of 8 elements
// takes 204 instructions forward and 348 backward (counted), and with scalar ones the issue slots, not HBM, bounded the kernels.
template <int VPT, bool BIG, bool GATE, bool DROP>
__global__ void __launch_bounds__(BIG ? 512 : 256, BIG ? 1 : VPT == 4 ? 2 : 3)
block_fwd_k(int64_t T, int C, int wpr, const uint4* x, const uint4* gate, const float4* w,
            const float* scale, float eps, DropArgs da, uint4* out, float* rstd) {
    constexpr int STAGES = fwd_stages(VPT), NT = GATE ? 2 : 1;
    extern __shared__ __align__(16) float sm[];
    __shared__ float red[2 * kMaxTeamWarps];
    pdl_wait();
    pdl_launch();
    const Team tm(wpr);
    const int nv = C >> 3;
    const uint32_t vec = blockDim.x * 16, ring = smem_u32(sm) + threadIdx.x * 16, stage = NT * VPT * vec;
    const int64_t t0 = (int64_t)blockIdx.x * tm.teams + tm.team, step = (int64_t)gridDim.x * tm.teams;
    auto fetch = [&](int64_t t, int s) {
        if (t < T) {
            fetch_row<VPT>(ring + s * stage, x + t * nv, tm, nv);
            if (GATE) fetch_row<VPT>(ring + s * stage + VPT * vec, gate + t * nv, tm, nv);
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) fetch(t0 + i * step, i);
    int slot = 0, cur = 0;
    const float s = scale ? ld_dep(scale) : 1.f;
    const float sf = DROP ? s * da.factor : s;
    const Philox rng(DROP ? da.rng : nullptr, DROP);
    uint64_t wf[VPT][4];
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int v = tm.lt + k * tm.threads;
        load_w(w, v < nv ? v : 0, wf[k]);
    }
    for (int64_t t = t0; t < T; t += step) {
        cp_async_wait<STAGES - 2>();
        fetch(t + (STAGES - 1) * step, cur == 0 ? STAGES - 1 : cur - 1);       // into the stage of the row before
        const uint32_t at = ring + cur * stage;
        cur = cur == STAGES - 1 ? 0 : cur + 1;
        uint64_t f[VPT][4], ss2 = 0;
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            unpack8x2(lds128(at + k * vec), f[k]);
#pragma unroll
            for (int e = 0; e < 4; ++e) ss2 = fma2(f[k][e], f[k][e], ss2);
        }
        float a0, a1;
        unpack2f(ss2, a0, a1);
        const float r = rsqrtf(team_sum(a0 + a1, red, slot, tm) / (float)C + eps);
        if (tm.lt == 0) rstd[t] = r;
        const uint64_t rs2 = both(r * sf);
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            const int v = tm.lt + k * tm.threads;
            if (v >= nv) continue;
            uint64_t g[4];
            if (GATE) unpack8x2(lds128(at + (VPT + k) * vec), g);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[k][e] = mul2(mul2(f[k][e], rs2), wf[k][e]);
                if (GATE) f[k][e] = mul2(f[k][e], sigmoid2(g[e]));
            }
            if (DROP) drop8(f[k], rng((uint64_t)(t * nv + v)), da.threshold << 16);
            st_stream(out + t * nv + v, pack8x2(f[k]));
        }
    }
    cp_async_wait<0>();
}

// With d = drop'(dy), z = d sig, oh = o r, e = s z w (the gradient with respect to oh):
//   do = r (e - oh mean(e oh)),  da = e oh (1 - sig),  dw = s sum_t z oh,  ds = sum z w oh.
// s is applied once to each result.  The scale's sum runs over all T C elements and may cancel: it is added up in 64 bits
// from the rows on.
template <int VPT, bool GATE, bool DROP>
__global__ void __launch_bounds__(512, 1)
block_bwd_k(int64_t T, int C, int wpr, const uint4* x, const uint4* gate, const float4* w,
            const float* scale, const float* rstd, DropArgs da, const uint4* dy,
            uint4* dx, uint4* dgate, float* dw_part, double* ds_part,
            float* dw, float* ds, int accumulate) {
    constexpr int STAGES = bwd_stages(VPT), NT = GATE ? 3 : 2;
    extern __shared__ __align__(16) float sm[];                    // the ring, then [teams][C] column sums
    __shared__ float red[2 * kMaxTeamWarps];
    __shared__ double dred[kMaxTeamWarps];
    pdl_wait();
    pdl_launch();
    const Team tm(wpr);
    const int nv = C >> 3;
    const uint32_t vec = blockDim.x * 16, ring = smem_u32(sm) + threadIdx.x * 16, stage = NT * VPT * vec;
    const int64_t t0 = (int64_t)blockIdx.x * tm.teams + tm.team, step = (int64_t)gridDim.x * tm.teams;
    auto fetch = [&](int64_t t, int s) {
        if (t < T) {
            fetch_row<VPT>(ring + s * stage, x + t * nv, tm, nv);
            fetch_row<VPT>(ring + s * stage + VPT * vec, dy + t * nv, tm, nv);
            if (GATE) fetch_row<VPT>(ring + s * stage + 2 * VPT * vec, gate + t * nv, tm, nv);
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) fetch(t0 + i * step, i);
    int slot = 0, cur = 0;
    const float s = scale ? ld_dep(scale) : 1.f;
    // dropout's factor rides on the weights, and on s in the column sums
    const uint64_t s2 = both(s), fac2 = both(da.factor);
    const Philox rng(DROP ? da.rng : nullptr, DROP);
    uint64_t acc[VPT][4], wf[VPT][4];
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int v = tm.lt + k * tm.threads;
        load_w(w, v < nv ? v : 0, wf[k]);
#pragma unroll
        for (int e = 0; e < 4; ++e) { acc[k][e] = 0; if (DROP) wf[k][e] = mul2(wf[k][e], fac2); }
    }
    double dsum = 0.0;
    float r_next = t0 < T ? ld_dep(rstd + t0) : 0.f;
    for (int64_t t = t0; t < T; t += step) {
        const float r = r_next;
        if (t + step < T) r_next = ld_dep(rstd + t + step);
        cp_async_wait<STAGES - 2>();
        fetch(t + (STAGES - 1) * step, cur == 0 ? STAGES - 1 : cur - 1);       // into the stage of the row before
        const uint32_t at = ring + cur * stage;
        cur = cur == STAGES - 1 ? 0 : cur + 1;
        const uint64_t r2 = both(r);
        uint64_t ds2 = 0;
        uint64_t zw[VPT][4];                                       // z w
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            const int v = tm.lt + k * tm.threads;
            if (v >= nv) continue;
            uint64_t f[4], g[4], dg[4];
            unpack8x2(lds128(at + k * vec), f);
            unpack8x2(lds128(at + (VPT + k) * vec), zw[k]);
            if (GATE) unpack8x2(lds128(at + (2 * VPT + k) * vec), g);
            if (GATE)
#pragma unroll
                for (int e = 0; e < 4; ++e) g[e] = exp_minus2(g[e]);
            if (DROP && GATE) drop8(zw[k], g, rng((uint64_t)(t * nv + v)), da.threshold << 16);
            if (DROP && !GATE) drop8(zw[k], rng((uint64_t)(t * nv + v)), da.threshold << 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint64_t oh = mul2(f[e], r2);
                const uint64_t sg = GATE ? sigmoid_of_exp2(g[e]) : 0;
                if (GATE) zw[k][e] = mul2(zw[k][e], sg);
                acc[k][e] = fma2(zw[k][e], oh, acc[k][e]);
                zw[k][e] = mul2(zw[k][e], wf[k][e]);
                if (GATE) {
                    const uint64_t q = mul2(zw[k][e], oh);
                    ds2 = add2(ds2, q);
                    dg[e] = mul2(mul2(q, s2), mul2(finite2(g[e]), sg));    // 1 - sig
                } else {
                    ds2 = fma2(zw[k][e], oh, ds2);
                }
            }
            if (GATE) st_stream(dgate + t * nv + v, pack8x2(dg));
        }
        float m0, m1;
        unpack2f(ds2, m0, m1);
        const float m = team_sum(m0 + m1, red, slot, tm);          // sum_c of e oh / s: the row's part of ds
        if (tm.lt == 0) dsum += (double)m;
        const uint64_t rs2 = both(r * s), c2 = both(-r * (m / (float)C));
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            const int v = tm.lt + k * tm.threads;
            if (v >= nv) continue;
            uint64_t f[4];
            unpack8x2(lds128(at + k * vec), f);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = mul2(fma2(f[e], c2, zw[k][e]), rs2);
            st_stream(dx + t * nv + v, pack8x2(f));
        }
    }
    cp_async_wait<0>();
    __syncthreads();
    // column sums of the block: the teams' rows through shared memory, in a fixed order
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int v = tm.lt + k * tm.threads;
        if (v < nv)
#pragma unroll
            for (int e = 0; e < 4; ++e) *(uint64_t*)(sm + tm.team * C + v * 8 + 2 * e) = acc[k][e];
    }
    if (tm.lt == 0) dred[tm.team] = dsum;
    __syncthreads();
    for (int c = threadIdx.x; c < C; c += blockDim.x) {
        float a = 0.f;
        for (int i = 0; i < tm.teams; ++i) a += sm[i * C + c];
        a *= DROP ? s * da.factor : s;
        if (gridDim.x == 1) dw[c] = accumulate ? dw[c] + a : a;        // few rows: nothing to join
        else dw_part[(int64_t)blockIdx.x * C + c] = a;
    }
    if (ds && threadIdx.x == 0) {
        double a = 0.0;
        for (int i = 0; i < tm.teams; ++i) a += dred[i];
        if (gridDim.x == 1) ds[0] = accumulate ? (float)(ds[0] + a) : (float)a;
        else ds_part[blockIdx.x] = a;
    }
}

// dw[c] (+)= sum over the blocks' partial rows, ds (+)= sum of their scalars; a block takes 32 columns, its 32 warps a
// range of the partial rows each (latency is all it costs: few rows a warp, loaded together).
__global__ void __launch_bounds__(1024) colsum_k(int C, int parts, const float* dw_part,
                                                 const double* ds_part, float* dw,
                                                 float* ds, int accumulate) {
    __shared__ float red[32][33];
    __shared__ double dred[32];
    pdl_wait();
    pdl_launch();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    const int per = (parts + 31) / 32, p0 = warp * per, p1 = min(parts, p0 + per);
    float a = 0.f;
    if (c < C)
#pragma unroll 10
        for (int p = p0; p < p1; ++p) a += dw_part[(int64_t)p * C + c];
    red[warp][lane] = a;
    if (ds && blockIdx.x == 0) {
        double d = p0 + lane < p1 ? ds_part[p0 + lane] : 0.0;  // per <= 32: at most 1024 parts
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
        if (lane == 0) dred[warp] = d;
    }
    __syncthreads();
    if (warp == 0 && c < C) {
        a = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) a += red[i][lane];
        dw[c] = accumulate ? dw[c] + a : a;
    }
    if (ds && blockIdx.x == 0 && threadIdx.x == 32) {
        double d = 0.0;
        for (int i = 0; i < 32; ++i) d += dred[i];
        ds[0] = accumulate ? (float)(ds[0] + d) : (float)d;
    }
}

// A thread takes four groups of 8 elements 256 apart: their loads are in flight together, and the round keys are made
// once for the four.
constexpr int kDropGroups = 4;
__global__ void __launch_bounds__(256) dropout_k(int64_t count, const __nv_bfloat16* x, DropArgs da,
                                                 __nv_bfloat16* y) {
    pdl_wait();
    pdl_launch();
    const Philox rng(da.rng, true);
    const uint32_t thr = da.threshold << 16;
    const uint64_t fac2 = both(da.factor);
    const int64_t full = count >> 3, g0 = (int64_t)blockIdx.x * (256 * kDropGroups) + threadIdx.x;
    uint4 v[kDropGroups];
#pragma unroll
    for (int k = 0; k < kDropGroups; ++k)
        if (g0 + k * 256 < full) v[k] = ld_dep_stream(x + (g0 + k * 256) * 8);
#pragma unroll
    for (int k = 0; k < kDropGroups; ++k) {
        const int64_t g = g0 + k * 256;
        uint64_t f[4];
        if (g < full) {
            unpack8x2(v[k], f);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = mul2(f[e], fac2);
            drop8(f, rng((uint64_t)g), thr);
            st_stream(y + g * 8, pack8x2(f));
        } else if (g * 8 < count) {                        // the last, partial group
            const int m = (int)(count - g * 8);
            float s[8];
            for (int e = 0; e < 8; ++e) s[e] = e < m ? __bfloat162float(x[g * 8 + e]) : 0.f;
            for (int e = 0; e < 4; ++e) f[e] = mul2(pack2f(s[2 * e], s[2 * e + 1]), fac2);
            drop8(f, rng((uint64_t)g), thr);
            for (int e = 0; e < 4; ++e) unpack2f(f[e], s[2 * e], s[2 * e + 1]);
            for (int e = 0; e < m; ++e) y[g * 8 + e] = __float2bfloat16_rn(s[e]);
        }
    }
}

// ---- host side -----------------------------------------------------------------------------------------------------
// Vectors a lane and warps a team for C channels, with as many warps as the row fills, and about 256 threads a block forward
// (up to 512 for long rows), about 512 backward, which leaves half as many partial rows to join (1536 channels, without a
// gate: 512 rows 8.1 -> 6.6 us, 8192 rows 19.6 -> 18.0).  Four vectors a lane forward: less of a row's fixed work a vector (16384 x 2048 with gate and dropout:
// the two norms 67 -> 61 us), and backward without a gate where a row fills its warps (each 42 -> 40 us; 1536 channels would
// leave a quarter of the lanes idle: 36 -> 39 us for 4099 rows).  With a gate, two backward while a team has at most 16
// warps, since its third tensor takes the registers (four: 72 -> 76 us).
struct RowPlan { int vpt, wpr, threads, teams; };
enum RowUse { ROW_FWD, ROW_BWD, ROW_BWD_GATED };
static RowPlan plan_row(int C, RowUse use) {
    const int nv = C / 8;
    const bool full = nv * 10 >= (nv + 127) / 128 * 128 * 9;
    const bool two = use != ROW_FWD && (use == ROW_BWD_GATED || !full) && nv <= 64 * kMaxTeamWarps;
    RowPlan p;
    p.vpt = nv <= 32 ? 1 : nv <= 64 || two ? 2 : 4;
    p.wpr = (nv + 32 * p.vpt - 1) / (32 * p.vpt);
    const int most = use == ROW_FWD ? 8 : kMaxTeamWarps;
    p.teams = p.wpr < most ? most / p.wpr : 1;
    p.threads = p.teams * p.wpr * 32;
    return p;
}
// Blocks: as many as are resident, or as there are rows for.
static int row_blocks(const RowPlan& p, int64_t T, int sm_count, int per_sm) {
    const int64_t need = (T + p.teams - 1) / p.teams, cap = (int64_t)sm_count * per_sm;
    return (int)(need < cap ? need : cap);
}

static DropArgs drop_args(float p, const uint64_t* rng) {
    DropArgs d;
    d.threshold = (uint32_t)drop_threshold(p);
    d.factor = drop_factor((int)d.threshold);
    d.rng = p > 0.f ? rng : nullptr;
    return d;
}

// (one block while its teams have at most two rows each: its column sums are then the result, without a second launch)
int block_parts(int64_t T, int C, int sm_count, bool gate) {
    const RowPlan p = plan_row(C, gate ? ROW_BWD_GATED : ROW_BWD);
    return T <= 2 * p.teams ? 1 : row_blocks(p, T, sm_count, 1);
}

void launch_block_fwd(const mhclite_ctx* c, int64_t T, const void* x, const void* gate, const float* w, const float* scale,
                      float eps, float p_drop, const uint64_t* rng, void* out, float* rstd, cudaStream_t s) {
    const RowPlan p = plan_row(c->C, ROW_FWD);
    const int grid = row_blocks(p, T, c->sm_count, p.threads > 256 ? 1 : p.vpt == 4 ? 2 : 3), smem = p.threads * 16 * p.vpt * (gate ? 2 : 1) * fwd_stages(p.vpt);
    const DropArgs da = drop_args(p_drop, rng);
    c->launches += 1;
#define MHCL_FWD(V, B)                                                                                                  \
    if (p.vpt == V && (p.threads > 256) == B) {                                                                                                \
        auto k = gate ? (da.rng ? block_fwd_k<V, B, true, true> : block_fwd_k<V, B, true, false>)                             \
                      : (da.rng ? block_fwd_k<V, B, false, true> : block_fwd_k<V, B, false, false>);                          \
        if (smem > 40 * 1024) { static SmemOnce once[2][2]; smem_limit(once[gate != nullptr][da.rng != nullptr], k, c->device, 226 * 1024); }               \
        launch_after(k, dim3(grid), dim3(p.threads), smem, s, T, c->C, p.wpr, (const uint4*)x, (const uint4*)gate, (const float4*)w, scale, \
                     eps, da, (uint4*)out, rstd);                                                                       \
    }
    MHCL_FWD(1, false) MHCL_FWD(2, false) MHCL_FWD(4, false) MHCL_FWD(4, true)
#undef MHCL_FWD
}

void launch_block_bwd(const mhclite_ctx* c, int64_t T, const void* x, const void* gate, const float* w, const float* scale,
                      const float* rstd, float p_drop, const uint64_t* rng, const void* dy, void* dx, void* dgate, float* dw,
                      float* dscale, int accumulate, float* dw_part, double* ds_part, cudaStream_t s) {
    const RowPlan p = plan_row(c->C, gate ? ROW_BWD_GATED : ROW_BWD);
    const int parts = block_parts(T, c->C, c->sm_count, gate != nullptr);
    int smem = p.threads * 16 * p.vpt * (gate ? 3 : 2) * bwd_stages(p.vpt);
    if (smem < p.teams * c->C * 4) smem = p.teams * c->C * 4;
    const DropArgs da = drop_args(p_drop, rng);
    c->launches += 1;
#define MHCL_BWD(V)                                                                                                     \
    if (p.vpt == V) {                                                                                                                          \
        auto k = gate ? (da.rng ? block_bwd_k<V, true, true> : block_bwd_k<V, true, false>)                             \
                      : (da.rng ? block_bwd_k<V, false, true> : block_bwd_k<V, false, false>);                          \
        if (smem > 40 * 1024) { static SmemOnce once[2][2]; smem_limit(once[gate != nullptr][da.rng != nullptr], k, c->device, 226 * 1024); }               \
        launch_after(k, dim3(parts), dim3(p.threads), smem, s, T, c->C, p.wpr, (const uint4*)x, (const uint4*)gate, (const float4*)w, \
                     scale, rstd, da, (const uint4*)dy, (uint4*)dx, (uint4*)dgate, dw_part, ds_part, dw, dscale, accumulate); \
    }
    MHCL_BWD(1) MHCL_BWD(2) MHCL_BWD(4)
#undef MHCL_BWD
    if (parts == 1) return;
    c->launches += 1;
    launch_after(colsum_k, dim3((c->C + 31) / 32), dim3(1024), 0, s, c->C, parts, dw_part, ds_part, dw, dscale, accumulate);
}

void launch_dropout(const mhclite_ctx* c, int64_t count, const void* x, float p, const uint64_t* rng, void* y, cudaStream_t s) {
    const int64_t groups = (count + 7) / 8, per = 256 * kDropGroups;
    DropArgs da = drop_args(p, rng);
    da.rng = rng;                                          // read for p = 0 too (everything stays)
    c->launches += 1;
    launch_after(dropout_k, dim3((unsigned)((groups + per - 1) / per)), dim3(256), 0, s, count, (const __nv_bfloat16*)x, da, (__nv_bfloat16*)y);
}

}  // namespace mhcl
