// Distillation from a teacher's top logits, on the tiles of the cross entropy (included by ce_kernels.cu):
//   x[t,v] = (logit_scale / temperature) <h_t, W_v>,  lse_t = log sum_v exp x[t,v],  logp[t,k] = x[t,id_k] - lse_t,
//   p[t,:] = softmax(z[t,:] / temperature) over the present entries,  loss_t = sum_k p_k (log p_k - logp_k),
//   dx[t,v] = dloss_t (exp(x[t,v] - lse_t) - sum_{k: id_k = v} p_k).
// An entry is present where its id is one of the table's; z = -inf makes its weight 0.  A row whose entries are all absent
// or of weight 0 is left out before the products, as a row without a target is.
#pragma once

namespace mhcl {

constexpr int kDsPer = kDistillMaxK / 32;                  // entries of a row that a lane holds

// A row's entries over the lanes of a warp: entry i * 32 + lane in place i.
struct DsRow {
    int id[kDsPer];             // -1 where absent
    float z[kDsPer];
    bool live;                  // some entry has weight (or is NaN)
};
template <typename Z> __device__ __forceinline__ float ds_float(Z v);
template <> __device__ __forceinline__ float ds_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float ds_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename Z>
__device__ __forceinline__ DsRow ds_load(int64_t t, int K, int64_t V, const int64_t* ids, const Z* z, int* status) {
    DsRow r;
    bool any = false;
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < kDsPer; ++i) {
        r.id[i] = -1;
        r.z[i] = -INFINITY;
        const int k = i * 32 + lane;
        if (k < K) {
            const int64_t id = ids[t * K + k];
            if (id >= 0 && id < V) {
                r.id[i] = (int)id;
                r.z[i] = ds_float(z[t * K + k]);
                any = any || r.z[i] != -INFINITY;
            } else if (id >= V && status) {
                report_index(status, MHCLITE_OP_LINEAR_DISTILL, t, id);
            }
        }
    }
    r.live = __any_sync(0xffffffffu, any);
    return r;
}
// z becomes the logarithm of the entry's weight; -inf where there is none.
__device__ __forceinline__ void ds_weights(DsRow& r, float inv_tau) {
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int i = 0; i < kDsPer; ++i) top = fmaxf(top, r.z[i]);
    top = warp_max(top);
    if (top == -INFINITY) top = 0.f;
#pragma unroll
    for (int i = 0; i < kDsPer; ++i) {
        r.z[i] = (r.z[i] - top) * inv_tau;
        sum += expf(r.z[i]);
    }
    const float b = logf(warp_sum(sum));
#pragma unroll
    for (int i = 0; i < kDsPer; ++i) r.z[i] -= b;
}

// Which rows have a teacher: target 0 or -1 for ce_rows_k; logp of the others is cleared.
template <typename Z>
__global__ void __launch_bounds__(256) ds_live_k(int64_t T, int K, int64_t V, const int64_t* ids, const Z* z, int64_t* target, float* logp,
                                                 int* status) {
    pdl_wait();
    pdl_launch();
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (t >= T) return;
    const DsRow r = ds_load(t, K, V, ids, z, status);
    if (lane == 0) target[t] = r.live ? 0 : -1;
    if (logp && !r.live)
        for (int k = lane; k < K; k += 32) logp[t * K + k] = 0.f;
}

// <h_t, W_id> of every present entry: a warp an entry.
__global__ void __launch_bounds__(256) ds_dot_k(int64_t entries, int K, int64_t V, int C, const int64_t* ids, const uint4* h, const uint4* W,
                                                float* dots) {
    pdl_wait();
    pdl_launch();
    const int lane = threadIdx.x & 31, nv = C >> 3;
    const int64_t warps = (int64_t)gridDim.x * 8;
    for (int64_t e = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); e < entries; e += warps) {
        const int64_t id = ids[e], t = e / K;
        if (id < 0 || id >= V) continue;
        float sum = 0.f;
        for (int v = lane; v < nv; v += 32) {
            float a[8], b[8];
            unpack8(ld_dep(h + t * nv + v), a);
            unpack8(ld_dep(W + id * nv + v), b);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(a[i], b[i], sum);
        }
        sum = warp_sum(sum);
        if (lane == 0) dots[e] = sum;
    }
}

// Joins the (maximum, sum) pairs of 32 rows a block as ce_join_k does, then a warp a row forms loss, lse and logp.  live and
// rows are null where every row is in the pairs (a handful of tokens).
template <typename Z>
__global__ void __launch_bounds__(1024) ds_join_k(int64_t T, int K, int64_t V, const int* live, const int* rows, int n_parts, int pitch,
                                                  const float2* part, const float* dots, const int64_t* ids, const Z* z, float k2,
                                                  float inv_tau, float* loss, float* lse, float* logp, int* status) {
    __shared__ float2 red[32][33];
    __shared__ float2 joined[32];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = blockIdx.x * 32 + lane, n = live ? *live : (int)T;
    if (blockIdx.x * 32 >= n) return;
    float m = -INFINITY, s = 0.f;
    if (r < n) {
#pragma unroll 8
        for (int k = warp; k < n_parts; k += 32) {
            const float2 p = part[(int64_t)k * pitch + r];
            const float top = fmaxf(m, p.x), base = top == -INFINITY ? 0.f : top;
            s = s * ex2(m - base) + p.y * ex2(p.x - base);
            m = top;
        }
    }
    red[warp][lane] = make_float2(m, s);
    __syncthreads();
    {                                                                   // lane: a range of tiles, warp: a row
        const float2 p = red[lane][warp];
        const float top = warp_max(p.x), base = top == -INFINITY ? 0.f : top;
        const float sum = warp_sum(p.y * ex2(p.x - base));
        if (lane == 0) joined[warp] = make_float2(top, sum);
    }
    __syncwarp();
    const int row = blockIdx.x * 32 + warp;
    if (row >= n) return;
    const int64_t t = rows ? rows[row] : row;
    DsRow e = ds_load(t, K, V, ids, z, rows ? nullptr : status);
    const float top = joined[warp].x, base = top == -INFINITY ? 0.f : top, b = log2f(joined[warp].y);
    ds_weights(e, inv_tau);
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < kDsPer; ++i) {
        const int k = i * 32 + lane;
        if (k >= K) continue;
        // x - lse as a difference to the row's largest logit, so that a likely id keeps its digits
        const float q = e.live && e.id[i] >= 0 ? (fmaf(dots[t * K + k], k2, -base) - b) * kLn2 : 0.f;
        logp[t * K + k] = q;
        if (e.live && e.z[i] != -INFINITY) l += expf(e.z[i]) * (e.z[i] - q);
    }
    l = warp_sum(l);
    if (lane == 0) {
        lse[t] = e.live ? (top + b) * kLn2 : 0.f;
        loss[t] = l;
    }
}

// Entries of G that the teacher has a share in, over what the product's epilogue wrote there: a warp a row.  An id that occurs
// twice has the sum of its weights, and both of its entries write the same.
template <typename Z>
__global__ void __launch_bounds__(256) ds_fix_k(int K, int64_t V, const int* live, const int* rows, int v0, int vn, const int64_t* ids,
                                                const Z* z, float inv_tau, const float* logp, const float* dloss, const uint32_t* ref, int refs,
                                                __nv_bfloat16* G, int64_t pitch) {
    pdl_wait();
    pdl_launch();
    const int lane = threadIdx.x & 31, n = *live;
    const int row = blockIdx.x * 8 + (threadIdx.x >> 5);
    const float top = ce_ref(ref, refs);
    if (row >= n) return;
    const int64_t t = rows[row];
    DsRow e = ds_load(t, K, V, ids, z, nullptr);
    ds_weights(e, inv_tau);
    float p[kDsPer], sum[kDsPer];
#pragma unroll
    for (int i = 0; i < kDsPer; ++i) { p[i] = expf(e.z[i]); sum[i] = 0.f; }
#pragma unroll
    for (int j = 0; j < kDsPer; ++j) {
        if (j * 32 >= K) break;
        for (int l = 0; l < 32; ++l) {
            const int id = __shfl_sync(0xffffffffu, e.id[j], l);
            const float w = __shfl_sync(0xffffffffu, p[j], l);
#pragma unroll
            for (int i = 0; i < kDsPer; ++i)
                if (id == e.id[i]) sum[i] += w;
        }
    }
    const float f = dloss[t] / top;
#pragma unroll
    for (int i = 0; i < kDsPer; ++i) {
        const int at = e.id[i] - v0;
        if (e.id[i] >= 0 && at >= 0 && at < vn) G[row * pitch + at] = __float2bfloat16_rn((expf(logp[t * K + i * 32 + lane]) - sum[i]) * f);
    }
}

// ---- host side -------------------------------------------------------------------------------------------------------
struct DsPlan { CePlan ce; int64_t* target; float* dots; size_t bytes; };
static DsPlan plan_ds(int64_t T, int64_t V, int K, int C, int grad, void* base) {
    DsPlan p;
    char* b = (char*)base;
    p.ce = plan_ce(T, V, C, grad, base);
    size_t off = ce_scratch_bytes(T, V, C, grad);
    off = (off + 255) & ~(size_t)255;
    auto take = [&](size_t n) { char* at = b + off; off += (n + 255) & ~(size_t)255; return at; };
    p.target = (int64_t*)take((size_t)T * 8);
    p.dots = grad ? nullptr : (float*)take((size_t)T * K * 4);
    p.bytes = off;
    return p;
}
size_t distill_scratch_bytes(int64_t T, int64_t V, int K, int C, int grad) { return plan_ds(T, V, K, C, grad, nullptr).bytes; }

template <typename Z>
static void launch_ds_live(const mhclite_ctx* c, int64_t T, int64_t V, int K, const int64_t* ids, const Z* z, int64_t* target, float* logp,
                           int* status, cudaStream_t s) {
    c->launches += 1;
    launch_after(ds_live_k<Z>, dim3((unsigned)((T + 7) / 8)), dim3(256), 0, s, T, K, V, ids, z, target, logp, status);
}

template <typename Z>
static bool ds_fwd(const mhclite_ctx* c, int64_t T, int64_t V, int K, const void* h, const void* W, const int64_t* ids, const Z* z, float scale,
                   float inv_tau, float* loss, float* lse, float* logp, void* scratch, cudaStream_t s) {
    const DsPlan p = plan_ds(T, V, K, c->C, 0, scratch);
    const int64_t entries = T * K, blocks = (entries + 7) / 8, most = (int64_t)c->sm_count * 32;
    const float k2 = scale * kLog2e;
    c->launches += 2;
    launch_after(ds_dot_k, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, s, entries, K, V, c->C, ids, (const uint4*)h,
                 (const uint4*)W, p.dots);
    const SmallPlan q = plan_small(T, c->C);
    if (q.stages) {
        const int grid = launch_ce_small(c, q, T, V, h, W, nullptr, scale, (float2*)scratch, nullptr, s);
        launch_after(ds_join_k<Z>, dim3(1), dim3(1024), 0, s, T, K, V, nullptr, nullptr, grid, kSmTokens, (const float2*)scratch, p.dots, ids, z,
                     k2, inv_tau, loss, lse, logp, c->op_status);
        return true;
    }
    launch_ds_live(c, T, V, K, ids, z, p.target, logp, c->op_status, s);
    if (!launch_ce_stats(c, p.ce, T, V, h, W, p.target, nullptr, scale, loss, lse, s)) return false;
    launch_after(ds_join_k<Z>, dim3((unsigned)((T + 31) / 32)), dim3(1024), 0, s, T, K, V, p.ce.live, p.ce.rows, 2 * p.ce.n_tiles, p.ce.Tpad,
                 p.ce.part, p.dots, ids, z, k2, inv_tau, loss, lse, logp, c->op_status);
    return true;
}
bool launch_linear_distill_fwd(const mhclite_ctx* c, int64_t T, int64_t V, int K, const void* h, const void* W, const int64_t* ids,
                               const void* z, int z_f32, float scale, float inv_tau, float* loss, float* lse, float* logp, void* scratch,
                               cudaStream_t s) {
    return z_f32 ? ds_fwd(c, T, V, K, h, W, ids, (const float*)z, scale, inv_tau, loss, lse, logp, scratch, s)
                 : ds_fwd(c, T, V, K, h, W, ids, (const __nv_bfloat16*)z, scale, inv_tau, loss, lse, logp, scratch, s);
}

template <typename Z>
static bool ds_bwd(const mhclite_ctx* c, int64_t T, int64_t V, int K, const void* h, const void* W, const int64_t* ids, const Z* z, float scale,
                   float inv_tau, const float* lse, const float* logp, const float* dloss, void* dh, void* dW, void* scratch, cudaStream_t s) {
    const DsPlan p = plan_ds(T, V, K, c->C, 1, scratch);
    launch_ds_live(c, T, V, K, ids, z, p.target, nullptr, c->op_status, s);
    return launch_ce_grads(c, p.ce, T, V, h, W, p.target, nullptr, scale, lse, dloss, dh, dW, s, [&](int v0, int vn) {
        c->launches += 1;
        launch_after(ds_fix_k<Z>, dim3((unsigned)((T + 7) / 8)), dim3(256), 0, s, K, V, p.ce.live, p.ce.rows, v0, vn, ids, z, inv_tau, logp, dloss,
                     p.ce.ref, p.ce.row_blocks, p.ce.G, p.ce.piece);
    });
}
bool launch_linear_distill_bwd(const mhclite_ctx* c, int64_t T, int64_t V, int K, const void* h, const void* W, const int64_t* ids,
                               const void* z, int z_f32, float scale, float inv_tau, const float* lse, const float* logp, const float* dloss,
                               void* dh, void* dW, void* scratch, cudaStream_t s) {
    return z_f32 ? ds_bwd(c, T, V, K, h, W, ids, (const float*)z, scale, inv_tau, lse, logp, dloss, dh, dW, scratch, s)
                 : ds_bwd(c, T, V, K, h, W, ids, (const __nv_bfloat16*)z, scale, inv_tau, lse, logp, dloss, dh, dW, scratch, s);
}

}  // namespace mhcl
