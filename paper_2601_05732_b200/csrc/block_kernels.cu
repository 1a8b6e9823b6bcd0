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

__device__ __forceinline__ float sigmoidf(float a) { return __fdividef(1.f, 1.f + __expf(-a)); }

struct DropArgs {
    const uint64_t* rng;      // device (seed, offset); null: no dropout
    uint32_t threshold;
    float factor;
};

template <int VPT, int WPR, bool GATE, bool DROP>
__global__ void __launch_bounds__(WPR * 32 > kBlockThreads ? WPR * 32 : kBlockThreads)
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
    float ss = 0.f;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        float f[8];
        unpack8(xv[k], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(f[e], f[e], ss);
    }
    ss = team_sum<WPR>(ss, red, slot);
    const float r = rsqrtf(ss / (float)C + eps);
    if (lt == 0) rstd[t] = r;
    const float s = scale ? __ldg(scale) : 1.f;
    uint64_t seed = 0, offset = 0;
    if (DROP) { seed = __ldg((const unsigned long long*)da.rng); offset = __ldg((const unsigned long long*)da.rng + 1); }
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int v = lt + k * WPR * 32;
        if (v >= nv) continue;
        float f[8], g[8];
        unpack8(xv[k], f);
        if (GATE) unpack8(gv[k], g);
        const float4 w0 = __ldg(w + 2 * v), w1 = __ldg(w + 2 * v + 1);
        const float wf[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            f[e] = f[e] * r * wf[e];
            if (GATE) f[e] *= sigmoidf(g[e]);
        }
        if (DROP) drop8(f, (uint64_t)(t * nv + v), seed, offset, da.threshold, da.factor);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= s;
        st_stream(out + t * nv + v, pack8(f));
    }
}

// With z = drop'(dy) s, oh = o r, e = z sigmoid(a) w:
//   do = r (e - oh mean(e oh)),  da = z oh w sig (1 - sig),  dw = sum_t z sig oh,  ds = sum dy drop(sig oh w).
// The scale's sum runs over all T C elements and may cancel: it is added up in 64 bits from the rows on.
template <int VPT, int WPR, bool GATE, bool DROP>
__global__ void __launch_bounds__(WPR * 32 > kBlockThreads ? WPR * 32 : kBlockThreads)
block_bwd_k(int64_t T, int C, const uint4* __restrict__ x, const uint4* __restrict__ gate, const float4* __restrict__ w,
            const float* __restrict__ scale, const float* __restrict__ rstd, DropArgs da, const uint4* __restrict__ dy,
            uint4* __restrict__ dx, uint4* __restrict__ dgate, float* __restrict__ dw_part, double* __restrict__ ds_part) {
    extern __shared__ float sm[];                          // [teams][C] column sums
    __shared__ float red[2 * 16];
    __shared__ double dred[16];
    const int nv = C >> 3, lt = threadIdx.x % (WPR * 32), teams = blockDim.x / (WPR * 32), team = threadIdx.x / (WPR * 32);
    int slot = 0;
    const float s = scale ? __ldg(scale) : 1.f;
    uint64_t seed = 0, offset = 0;
    if (DROP) { seed = __ldg((const unsigned long long*)da.rng); offset = __ldg((const unsigned long long*)da.rng + 1); }
    float acc[VPT][8];
#pragma unroll
    for (int k = 0; k < VPT; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[k][e] = 0.f;
    double dsum = 0.0;
    for (int64_t t = (int64_t)blockIdx.x * teams + team; t < T; t += (int64_t)gridDim.x * teams) {
        uint4 xv[VPT], gv[VPT], yv[VPT];
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            const int v = lt + k * WPR * 32;
            xv[k] = yv[k] = gv[k] = make_uint4(0, 0, 0, 0);
            if (v < nv) {
                xv[k] = ld_stream(x + t * nv + v);
                yv[k] = ld_stream(dy + t * nv + v);
                if (GATE) gv[k] = ld_stream(gate + t * nv + v);
            }
        }
        const float r = __ldg(rstd + t);
        float ds = 0.f;
        float z[VPT][8];                                   // drop'(dy) s sig
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            const int v = lt + k * WPR * 32;
            if (v >= nv) continue;
            float f[8], g[8];
            unpack8(xv[k], f);
            unpack8(yv[k], z[k]);
            if (GATE) unpack8(gv[k], g);
            if (DROP) drop8(z[k], (uint64_t)(t * nv + v), seed, offset, da.threshold, da.factor);
            const float4 w0 = __ldg(w + 2 * v), w1 = __ldg(w + 2 * v + 1);
            const float wf[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
            float da8[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float oh = f[e] * r;
                if (GATE) {
                    const float sg = sigmoidf(g[e]);
                    z[k][e] *= sg;
                    da8[e] = z[k][e] * s * oh * wf[e] * (1.f - sg);
                }
                const float c = z[k][e] * oh;              // without s: the factor of dw and ds
                acc[k][e] = fmaf(c, s, acc[k][e]);
                ds = fmaf(c, wf[e], ds);
            }
            if (GATE) st_stream(dgate + t * nv + v, pack8(da8));
        }
        float m = team_sum<WPR>(ds, red, slot);                // sum_c of e oh / s, and the row's part of ds
        if (lt == 0) dsum += (double)m;
        m *= s / (float)C;
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            const int v = lt + k * WPR * 32;
            if (v >= nv) continue;
            float f[8];
            unpack8(xv[k], f);
            const float4 w0 = __ldg(w + 2 * v), w1 = __ldg(w + 2 * v + 1);
            const float wf[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = r * (z[k][e] * s * wf[e] - f[e] * r * m);
            st_stream(dx + t * nv + v, pack8(f));
        }
    }
    // column sums of the block: the teams' rows through shared memory, in a fixed order
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int v = lt + k * WPR * 32;
        if (v < nv)
#pragma unroll
            for (int e = 0; e < 8; ++e) sm[team * C + v * 8 + e] = acc[k][e];
    }
    if (lt == 0) dred[team] = dsum;
    __syncthreads();
    for (int c = threadIdx.x; c < C; c += blockDim.x) {
        float a = 0.f;
        for (int i = 0; i < teams; ++i) a += sm[i * C + c];
        dw_part[(int64_t)blockIdx.x * C + c] = a;
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

__global__ void __launch_bounds__(256) dropout_k(int64_t count, const __nv_bfloat16* __restrict__ x, DropArgs da,
                                                 __nv_bfloat16* __restrict__ y) {
    const uint64_t seed = __ldg((const unsigned long long*)da.rng), offset = __ldg((const unsigned long long*)da.rng + 1);
    const int64_t full = count >> 3;
    for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g * 8 < count; g += (int64_t)gridDim.x * 256) {
        float f[8];
        if (g < full) {
            unpack8(ld_stream(x + g * 8), f);
            drop8(f, (uint64_t)g, seed, offset, da.threshold, da.factor);
            st_stream(y + g * 8, pack8(f));
        } else {                                           // the last, partial group
            const int m = (int)(count - g * 8);
            for (int e = 0; e < 8; ++e) f[e] = e < m ? __bfloat162float(x[g * 8 + e]) : 0.f;
            drop8(f, (uint64_t)g, seed, offset, da.threshold, da.factor);
            for (int e = 0; e < m; ++e) y[g * 8 + e] = __float2bfloat16_rn(f[e]);
        }
    }
}

// ---- host side -----------------------------------------------------------------------------------------------------
// Warps a row and vectors a lane for C channels: 4 vectors a lane keep a warp's loads wide and few rows' worth of
// registers; short rows take fewer.
struct RowPlan { int vpt, wpr; };
static RowPlan plan_row(int C) {
    const int nv = C / 8;
    RowPlan p;
    p.vpt = nv <= 32 ? 1 : nv <= 64 ? 2 : 4;
    p.wpr = 1;
    while (p.wpr * 32 * p.vpt < nv) p.wpr *= 2;
    return p;
}

#define MHCL_ROW_DISPATCH(p, ...)                                                        \
    if ((p).vpt == 1) { constexpr int VPT = 1, WPR = 1; __VA_ARGS__; }                   \
    else if ((p).vpt == 2) { constexpr int VPT = 2, WPR = 1; __VA_ARGS__; }              \
    else if ((p).wpr == 1) { constexpr int VPT = 4, WPR = 1; __VA_ARGS__; }              \
    else if ((p).wpr == 2) { constexpr int VPT = 4, WPR = 2; __VA_ARGS__; }              \
    else if ((p).wpr == 4) { constexpr int VPT = 4, WPR = 4; __VA_ARGS__; }              \
    else if ((p).wpr == 8) { constexpr int VPT = 4, WPR = 8; __VA_ARGS__; }              \
    else { constexpr int VPT = 4, WPR = 16; __VA_ARGS__; }

static DropArgs drop_args(float p, const uint64_t* rng) {
    DropArgs d;
    d.threshold = (uint32_t)drop_threshold(p);
    d.factor = drop_factor((int)d.threshold);
    d.rng = p > 0.f ? rng : nullptr;
    return d;
}

int block_parts(int64_t T, int C, int sm_count) {
    const RowPlan p = plan_row(C);
    const int threads = p.wpr * 32 > kBlockThreads ? p.wpr * 32 : kBlockThreads, teams = threads / (p.wpr * 32);
    const int64_t need = (T + teams - 1) / teams, cap = (int64_t)sm_count * (512 / threads);
    return (int)(need < cap ? need : cap);
}

void launch_block_fwd(const mhclite_ctx* c, int64_t T, const void* x, const void* gate, const float* w, const float* scale,
                      float eps, float p_drop, const uint64_t* rng, void* out, float* rstd, cudaStream_t s) {
    const RowPlan p = plan_row(c->C);
    const int threads = p.wpr * 32 > kBlockThreads ? p.wpr * 32 : kBlockThreads, teams = threads / (p.wpr * 32);
    const unsigned grid = (unsigned)((T + teams - 1) / teams);
    const DropArgs da = drop_args(p_drop, rng);
    c->launches += 1;
    MHCL_ROW_DISPATCH(p, {
        auto k = gate ? (da.rng ? block_fwd_k<VPT, WPR, true, true> : block_fwd_k<VPT, WPR, true, false>)
                      : (da.rng ? block_fwd_k<VPT, WPR, false, true> : block_fwd_k<VPT, WPR, false, false>);
        k<<<grid, threads, 0, s>>>(T, c->C, (const uint4*)x, (const uint4*)gate, (const float4*)w, scale, eps, da, (uint4*)out, rstd);
    })
}

void launch_block_bwd(const mhclite_ctx* c, int64_t T, const void* x, const void* gate, const float* w, const float* scale,
                      const float* rstd, float p_drop, const uint64_t* rng, const void* dy, void* dx, void* dgate, float* dw,
                      float* dscale, int accumulate, float* dw_part, double* ds_part, cudaStream_t s) {
    const RowPlan p = plan_row(c->C);
    const int threads = p.wpr * 32 > kBlockThreads ? p.wpr * 32 : kBlockThreads, teams = threads / (p.wpr * 32);
    const int parts = block_parts(T, c->C, c->sm_count);
    const size_t smem = (size_t)teams * c->C * sizeof(float);
    const DropArgs da = drop_args(p_drop, rng);
    c->launches += 2;
    MHCL_ROW_DISPATCH(p, {
        auto k = gate ? (da.rng ? block_bwd_k<VPT, WPR, true, true> : block_bwd_k<VPT, WPR, true, false>)
                      : (da.rng ? block_bwd_k<VPT, WPR, false, true> : block_bwd_k<VPT, WPR, false, false>);
        if (smem > 48 * 1024) cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        k<<<parts, threads, smem, s>>>(T, c->C, (const uint4*)x, (const uint4*)gate, (const float4*)w, scale, rstd, da,
                                       (const uint4*)dy, (uint4*)dx, (uint4*)dgate, dw_part, dscale ? ds_part : nullptr);
    })
    colsum_k<<<(c->C + 31) / 32, 256, 0, s>>>(c->C, parts, dw_part, ds_part, dw, dscale, accumulate);
}

void launch_dropout(const mhclite_ctx* c, int64_t count, const void* x, float p, const uint64_t* rng, void* y, cudaStream_t s) {
    const int64_t need = ((count + 7) / 8 + 255) / 256, cap = (int64_t)c->sm_count * 8 * 4;
    DropArgs da = drop_args(p, rng);
    da.rng = rng;                                          // read for p = 0 too (everything stays)
    c->launches += 1;
    dropout_k<<<(unsigned)(need < cap ? need : cap), 256, 0, s>>>(count, (const __nv_bfloat16*)x, da, (__nv_bfloat16*)y);
}

}  // namespace mhcl
