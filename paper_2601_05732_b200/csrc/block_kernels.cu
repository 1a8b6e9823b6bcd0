// The seam between the mixing step and the caller's sublayer: the norm that opens the sublayer,
//   v = u r w,   r = (mean_c u^2 + eps)^-1/2,
// and what closes it,
//   y = s drop(sigmoid(a) o r w),
// with their gradients; and dropout on its own.  drop(z) is z / (1 - p) where the element stays and 0 where not
// (philox.cuh).  All of them move bf16 rows once and are bound by HBM; everything between load and store is fp32.
//
// A row is held by a team of WPR warps in registers (VPT 16-byte vectors a lane, packed), so each tensor is read once:
// the row's sum comes first, then the outputs from the same registers.  Teams of one warp need no block-wide step.
// The gradients run persistent teams over the rows, keep the column sums (dw) of their rows in registers and leave one
// partial row a block; colsum_k adds the blocks up in a fixed order, so results are the same bit for bit from run to run.
#include "common.cuh"
#include "kernels.h"
#include "philox.cuh"

namespace mhcl {

constexpr int kBlockThreads = 256;

// Sum over the team's warps; every thread of the team gets it.  `slot` alternates so that one barrier a sum is enough.
template <int WPR>
__device__ __forceinline__ float team_sum(float v, float* red, int& slot) {
    v = warp_sum(v);
    if (WPR == 1) return v;
    const int warp = threadIdx.x >> 5, team = warp / WPR, w = warp % WPR;
    float* r = red + (slot * (blockDim.x >> 5)) + team * WPR;
    if ((threadIdx.x & 31) == 0) r[w] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(WPR * 32) : "memory");
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < WPR; ++i) s += r[i];
    slot ^= 1;
    return s;
}

// sigmoid of a pair: 1 / (1 + 2^(-a log2 e)); 2^x overflows to infinity for a far below 0, whose reciprocal is 0.
__device__ __forceinline__ uint64_t sigmoid2(uint64_t a) {
    float x, y;
    unpack2f(mul2(a, pack2f(-1.4426950408889634f, -1.4426950408889634f)), x, y);
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(x));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(y));
    unpack2f(add2(pack2f(x, y), pack2f(1.f, 1.f)), x, y);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(x));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(y));
    return pack2f(x, y);
}
__device__ __forceinline__ uint64_t both(float x) { return pack2f(x, x); }
// the 8 weights of a vector, as packed pairs
__device__ __forceinline__ void load_w(const float4* __restrict__ w, int v, uint64_t* o) {
    const ulonglong2 a = __ldg((const ulonglong2*)w + 2 * v), b = __ldg((const ulonglong2*)w + 2 * v + 1);
    o[0] = a.x; o[1] = a.y; o[2] = b.x; o[3] = b.y;
}

struct DropArgs {
    const uint64_t* rng;      // device (seed, offset); null: no dropout
    uint32_t threshold;       // in units of 2^-16
    float factor;
};

// The arithmetic runs on packed pairs (two fp32 operations an instruction): with gate and dropout a vector of 8 elements
// takes some 170 instructions forward and 230 backward, and with scalar ones the issue slots, not HBM, bounded the kernels.
template <int VPT, int WPR, bool GATE, bool DROP>
__global__ void __launch_bounds__(WPR * 32 > kBlockThreads ? WPR * 32 : kBlockThreads, WPR * 32 > kBlockThreads ? 1 : 3)
block_fwd_k(int64_t T, int C, const uint4* __restrict__ x, const uint4* __restrict__ gate, const float4* __restrict__ w,
            const float* __restrict__ scale, float eps, DropArgs da, uint4* __restrict__ out, float* __restrict__ rstd) {
    __shared__ float red[2 * 16];
    const int nv = C >> 3, lt = threadIdx.x % (WPR * 32), teams = blockDim.x / (WPR * 32);
    const int64_t t = (int64_t)blockIdx.x * teams + threadIdx.x / (WPR * 32);
    if (t >= T) return;                                    // whole teams leave
    int slot = 0;
    uint4 xv[VPT], gv[VPT];
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int v = lt + k * WPR * 32;
        xv[k] = v < nv ? ld_stream(x + t * nv + v) : make_uint4(0, 0, 0, 0);
        if (GATE) gv[k] = v < nv ? ld_stream(gate + t * nv + v) : make_uint4(0, 0, 0, 0);
    }
    uint64_t ss2 = 0;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        uint64_t f[4];
        unpack8x2(xv[k], f);
#pragma unroll
        for (int e = 0; e < 4; ++e) ss2 = fma2(f[e], f[e], ss2);
    }
    float s0, s1;
    unpack2f(ss2, s0, s1);
    const float r = rsqrtf(team_sum<WPR>(s0 + s1, red, slot) / (float)C + eps);
    if (lt == 0) rstd[t] = r;
    const float s = scale ? __ldg(scale) : 1.f;
    const uint64_t r2 = both(r), s2 = both(s), fac2 = both(da.factor);
    const Philox rng(DROP ? da.rng : nullptr, DROP);
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int v = lt + k * WPR * 32;
        if (v >= nv) continue;
        uint64_t f[4], g[4], wf[4];
        unpack8x2(xv[k], f);
        load_w(w, v, wf);
        if (GATE) unpack8x2(gv[k], g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[e] = mul2(mul2(f[e], r2), wf[e]);
            if (GATE) f[e] = mul2(f[e], sigmoid2(g[e]));
        }
        if (DROP) drop8(f, rng((uint64_t)(t * nv + v)), da.threshold << 16, fac2);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = mul2(f[e], s2);
        st_stream(out + t * nv + v, pack8x2(f));
    }
}

// With d = drop'(dy), z = d sig, oh = o r, e = s z w (the gradient with respect to oh):
//   do = r (e - oh mean(e oh)),  da = e oh (1 - sig),  dw = s sum_t z oh,  ds = sum z w oh.
// s is applied once to each result.  The scale's sum runs over all T C elements and may cancel: it is added up in 64 bits
// from the rows on.
template <int VPT, int WPR, bool GATE, bool DROP>
__global__ void __launch_bounds__(WPR * 32 > kBlockThreads ? WPR * 32 : kBlockThreads, WPR * 32 > kBlockThreads ? 1 : 2)
block_bwd_k(int64_t T, int C, const uint4* __restrict__ x, const uint4* __restrict__ gate, const float4* __restrict__ w,
            const float* __restrict__ scale, const float* __restrict__ rstd, DropArgs da, const uint4* __restrict__ dy,
            uint4* __restrict__ dx, uint4* __restrict__ dgate, float* __restrict__ dw_part, double* __restrict__ ds_part) {
    extern __shared__ float sm[];                          // [teams][C] column sums
    __shared__ float red[2 * 16];
    __shared__ double dred[16];
    const int nv = C >> 3, lt = threadIdx.x % (WPR * 32), teams = blockDim.x / (WPR * 32), team = threadIdx.x / (WPR * 32);
    int slot = 0;
    const float s = scale ? __ldg(scale) : 1.f;
    const uint64_t s2 = both(s), fac2 = both(da.factor), minus1 = both(-1.f);
    const Philox rng(DROP ? da.rng : nullptr, DROP);
    uint64_t acc[VPT][4];
#pragma unroll
    for (int k = 0; k < VPT; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[k][e] = 0;
    double dsum = 0.0;
    for (int64_t t = (int64_t)blockIdx.x * teams + team; t < T; t += (int64_t)gridDim.x * teams) {
        uint4 xv[VPT], gv[VPT], yv[VPT];
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            const int v = lt + k * WPR * 32;
            if (v < nv) {
                xv[k] = ld_stream(x + t * nv + v);
                yv[k] = ld_stream(dy + t * nv + v);
                if (GATE) gv[k] = ld_stream(gate + t * nv + v);
            }
        }
        const float r = __ldg(rstd + t);
        const uint64_t r2 = both(r);
        uint64_t ds2 = 0;
        uint64_t zw[VPT][4];                               // z w
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            const int v = lt + k * WPR * 32;
            if (v >= nv) continue;
            uint64_t f[4], g[4], wf[4], dg[4];
            unpack8x2(xv[k], f);
            unpack8x2(yv[k], zw[k]);
            load_w(w, v, wf);
            if (GATE) unpack8x2(gv[k], g);
            if (DROP) drop8(zw[k], rng((uint64_t)(t * nv + v)), da.threshold << 16, fac2);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint64_t oh = mul2(f[e], r2);
                if (GATE) { g[e] = sigmoid2(g[e]); zw[k][e] = mul2(zw[k][e], g[e]); }
                acc[k][e] = fma2(zw[k][e], oh, acc[k][e]);
                zw[k][e] = mul2(zw[k][e], wf[e]);
                const uint64_t q = mul2(zw[k][e], oh);
                ds2 = add2(ds2, q);
                if (GATE) dg[e] = mul2(mul2(q, s2), fma2(g[e], minus1, both(1.f)));
            }
            if (GATE) st_stream(dgate + t * nv + v, pack8x2(dg));
        }
        float m0, m1;
        unpack2f(ds2, m0, m1);
        const float m = team_sum<WPR>(m0 + m1, red, slot);         // sum_c of e oh / s: the row's part of ds
        if (lt == 0) dsum += (double)m;
        const uint64_t rs2 = both(r * s), c2 = both(-r * (m / (float)C));
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            const int v = lt + k * WPR * 32;
            if (v >= nv) continue;
            uint64_t f[4];
            unpack8x2(xv[k], f);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = mul2(fma2(f[e], c2, zw[k][e]), rs2);
            st_stream(dx + t * nv + v, pack8x2(f));
        }
    }
    // column sums of the block: the teams' rows through shared memory, in a fixed order
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int v = lt + k * WPR * 32;
        if (v < nv)
#pragma unroll
            for (int e = 0; e < 4; ++e) *(uint64_t*)(sm + team * C + v * 8 + 2 * e) = acc[k][e];
    }
    if (lt == 0) dred[team] = dsum;
    __syncthreads();
    for (int c = threadIdx.x; c < C; c += blockDim.x) {
        float a = 0.f;
        for (int i = 0; i < teams; ++i) a += sm[i * C + c];
        dw_part[(int64_t)blockIdx.x * C + c] = a * s;
    }
    if (ds_part && threadIdx.x == 0) {
        double a = 0.0;
        for (int i = 0; i < teams; ++i) a += dred[i];
        ds_part[blockIdx.x] = a;
    }
}

// dw[c] (+)= sum over the blocks' partial rows, ds (+)= sum of their scalars; a block takes 32 columns, its 8 warps a
// range of the partial rows each.
__global__ void __launch_bounds__(256) colsum_k(int C, int parts, const float* __restrict__ dw_part,
                                                const double* __restrict__ ds_part, float* __restrict__ dw,
                                                float* __restrict__ ds, int accumulate) {
    __shared__ float red[8][33];
    __shared__ double dred[8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    const int per = (parts + 7) / 8, p0 = warp * per, p1 = min(parts, p0 + per);
    float a = 0.f;
    if (c < C)
        for (int p = p0; p < p1; ++p) a += dw_part[(int64_t)p * C + c];
    red[warp][lane] = a;
    if (ds && blockIdx.x == 0) {
        double d = 0.0;
        for (int p = p0 + lane; p < p1; p += 32) d += ds_part[p];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
        if (lane == 0) dred[warp] = d;
    }
    __syncthreads();
    if (warp == 0 && c < C) {
        a = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) a += red[i][lane];
        dw[c] = accumulate ? dw[c] + a : a;
    }
    if (ds && blockIdx.x == 0 && threadIdx.x == 0) {
        double d = 0.0;
        for (int i = 0; i < 8; ++i) d += dred[i];
        ds[0] = accumulate ? (float)(ds[0] + d) : (float)d;
    }
}

// A thread takes four groups of 8 elements 256 apart: their loads are in flight together, and the round keys are made
// once for the four.
constexpr int kDropGroups = 4;
__global__ void __launch_bounds__(256) dropout_k(int64_t count, const __nv_bfloat16* __restrict__ x, DropArgs da,
                                                 __nv_bfloat16* __restrict__ y) {
    const Philox rng(da.rng, true);
    const uint32_t thr = da.threshold << 16;
    const uint64_t fac2 = both(da.factor);
    const int64_t full = count >> 3, g0 = (int64_t)blockIdx.x * (256 * kDropGroups) + threadIdx.x;
    uint4 v[kDropGroups];
#pragma unroll
    for (int k = 0; k < kDropGroups; ++k)
        if (g0 + k * 256 < full) v[k] = ld_stream(x + (g0 + k * 256) * 8);
#pragma unroll
    for (int k = 0; k < kDropGroups; ++k) {
        const int64_t g = g0 + k * 256;
        uint64_t f[4];
        if (g < full) {
            unpack8x2(v[k], f);
            drop8(f, rng((uint64_t)g), thr, fac2);
            st_stream(y + g * 8, pack8x2(f));
        } else if (g * 8 < count) {                        // the last, partial group
            const int m = (int)(count - g * 8);
            float s[8];
            for (int e = 0; e < 8; ++e) s[e] = e < m ? __bfloat162float(x[g * 8 + e]) : 0.f;
            for (int e = 0; e < 4; ++e) f[e] = pack2f(s[2 * e], s[2 * e + 1]);
            drop8(f, rng((uint64_t)g), thr, fac2);
            for (int e = 0; e < 4; ++e) unpack2f(f[e], s[2 * e], s[2 * e + 1]);
            for (int e = 0; e < m; ++e) y[g * 8 + e] = __float2bfloat16_rn(s[e]);
        }
    }
}

// ---- host side -----------------------------------------------------------------------------------------------------
// Warps a row and vectors a lane for C channels.  Forward: 4 vectors a lane keep a warp's loads wide.  Backward: 2, since
// its three tensors and the column sums of 4 would take 180 registers a thread and leave one block on an SM.
struct RowPlan { int vpt, wpr, threads, teams; };
static RowPlan plan_row(int C, bool bwd) {
    const int nv = C / 8;
    RowPlan p;
    p.vpt = nv <= 32 ? 1 : (nv <= 64 || (bwd && nv <= 1024)) ? 2 : 4;
    p.wpr = 1;
    while (p.wpr * 32 * p.vpt < nv) p.wpr *= 2;
    p.threads = p.wpr * 32 > kBlockThreads ? p.wpr * 32 : kBlockThreads;
    p.teams = p.threads / (p.wpr * 32);
    return p;
}

#define MHCL_ROW_CASE(V, W, ...) if (p.vpt == V && p.wpr == W) { constexpr int VPT = V, WPR = W; __VA_ARGS__; }

static DropArgs drop_args(float p, const uint64_t* rng) {
    DropArgs d;
    d.threshold = (uint32_t)drop_threshold(p);
    d.factor = drop_factor((int)d.threshold);
    d.rng = p > 0.f ? rng : nullptr;
    return d;
}

int block_parts(int64_t T, int C, int sm_count) {
    const RowPlan p = plan_row(C, true);
    const int64_t need = (T + p.teams - 1) / p.teams, cap = (int64_t)sm_count * (512 / p.threads);
    return (int)(need < cap ? need : cap);
}

void launch_block_fwd(const mhclite_ctx* c, int64_t T, const void* x, const void* gate, const float* w, const float* scale,
                      float eps, float p_drop, const uint64_t* rng, void* out, float* rstd, cudaStream_t s) {
    const RowPlan p = plan_row(c->C, false);
    const unsigned grid = (unsigned)((T + p.teams - 1) / p.teams);
    const DropArgs da = drop_args(p_drop, rng);
    c->launches += 1;
#define MHCL_FWD(V, W)                                                                                                  \
    MHCL_ROW_CASE(V, W, {                                                                                               \
        auto k = gate ? (da.rng ? block_fwd_k<VPT, WPR, true, true> : block_fwd_k<VPT, WPR, true, false>)               \
                      : (da.rng ? block_fwd_k<VPT, WPR, false, true> : block_fwd_k<VPT, WPR, false, false>);            \
        k<<<grid, p.threads, 0, s>>>(T, c->C, (const uint4*)x, (const uint4*)gate, (const float4*)w, scale, eps, da,    \
                                     (uint4*)out, rstd);                                                                \
    })
    MHCL_FWD(1, 1) MHCL_FWD(2, 1) MHCL_FWD(4, 1) MHCL_FWD(4, 2) MHCL_FWD(4, 4) MHCL_FWD(4, 8) MHCL_FWD(4, 16)
#undef MHCL_FWD
}

void launch_block_bwd(const mhclite_ctx* c, int64_t T, const void* x, const void* gate, const float* w, const float* scale,
                      const float* rstd, float p_drop, const uint64_t* rng, const void* dy, void* dx, void* dgate, float* dw,
                      float* dscale, int accumulate, float* dw_part, double* ds_part, cudaStream_t s) {
    const RowPlan p = plan_row(c->C, true);
    const int parts = block_parts(T, c->C, c->sm_count);
    const size_t smem = (size_t)p.teams * c->C * sizeof(float);
    const DropArgs da = drop_args(p_drop, rng);
    c->launches += 2;
#define MHCL_BWD(V, W)                                                                                                  \
    MHCL_ROW_CASE(V, W, {                                                                                               \
        auto k = gate ? (da.rng ? block_bwd_k<VPT, WPR, true, true> : block_bwd_k<VPT, WPR, true, false>)               \
                      : (da.rng ? block_bwd_k<VPT, WPR, false, true> : block_bwd_k<VPT, WPR, false, false>);            \
        if (smem > 48 * 1024) cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);          \
        k<<<parts, p.threads, smem, s>>>(T, c->C, (const uint4*)x, (const uint4*)gate, (const float4*)w, scale, rstd, da, \
                                         (const uint4*)dy, (uint4*)dx, (uint4*)dgate, dw_part, dscale ? ds_part : nullptr); \
    })
    MHCL_BWD(1, 1) MHCL_BWD(2, 1) MHCL_BWD(2, 2) MHCL_BWD(2, 4) MHCL_BWD(2, 8) MHCL_BWD(2, 16) MHCL_BWD(4, 16)
#undef MHCL_BWD
    colsum_k<<<(c->C + 31) / 32, 256, 0, s>>>(c->C, parts, dw_part, ds_part, dw, dscale, accumulate);
}

void launch_dropout(const mhclite_ctx* c, int64_t count, const void* x, float p, const uint64_t* rng, void* y, cudaStream_t s) {
    const int64_t groups = (count + 7) / 8, per = 256 * kDropGroups;
    DropArgs da = drop_args(p, rng);
    da.rng = rng;                                          // read for p = 0 too (everything stays)
    c->launches += 1;
    dropout_k<<<(unsigned)((groups + per - 1) / per), 256, 0, s>>>(count, (const __nv_bfloat16*)x, da, (__nv_bfloat16*)y);
}

}  // namespace mhcl
