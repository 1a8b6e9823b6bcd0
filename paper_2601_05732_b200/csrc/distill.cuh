// Distillation from a teacher's top logits, on the tiles of the cross entropy (included by ce_kernels.cu):
//   x[t,v] = (logit_scale / temperature) <h_t, W_v>,  lse_t = log sum_v exp x[t,v],  logp[t,k] = x[t,id_k] - lse_t,
//   p[t,:] = softmax(z[t,:] / temperature) over the present entries,  loss_t = sum_k p_k (log p_k - logp_k),
//   dx[t,v] = dloss_t (exp(x[t,v] - lse_t) - sum_{k: id_k = v} p_k).
// An entry is present where its id is one of the table's; z = -inf makes its weight 0.  A row whose entries are all absent
// or of weight 0 is left out before the products, as a row without a target is.
//
// Forward: ds_sort_k sorts each row's entries by id; the product's epilogue (CE_PICK) picks their logits from the tiles on the way,
// where a dot product each would read T K C values again (4099 x 1536, 256 entries: 3.2 GB through L2, 925 us for the call
// against 550); ds_join_k forms the loss.  Backward: the epilogue (CE_PATCH) writes the bracket at the entries, formed in
// fp32 from the forward's logp, over what the tile has there, before the bf16 tile goes out.
// What bounds it: the tensor cores, and behind them the power cap, as the cross entropy (16384 x 2048 x 50257, 64 entries, loss and
// gradients 10.2 ms, the cross entropy 10.25); the small kernels
// around the product take 45 us for 4099 rows of 256 entries.
#pragma once

#include <type_traits>

namespace mhcl {

// A row's entries over the lanes of a warp, PER (1, 2, 4 or 8) each: entry i * 32 + lane in place i.
template <int PER>
struct DsRow {
    int id[PER];                // -1 where absent
    float z[PER];
    bool live;                  // some entry has weight (or is NaN)
};
template <int PER>
__device__ __forceinline__ DsRow<PER> ds_load(int64_t t, int K, int64_t V, const int64_t* ids, const void* z, int z_f32, int* status) {
    DsRow<PER> r;
    const int lane = threadIdx.x & 31;
    int64_t id[PER];
    float v[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {                                     // all loads before the first use
        const int k = i * 32 + lane;
        id[i] = k < K ? ids[t * K + k] : -1;
        v[i] = k >= K ? 0.f : z_f32 ? ((const float*)z)[t * K + k] : __bfloat162float(((const __nv_bfloat16*)z)[t * K + k]);
    }
    bool any = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const bool in = id[i] >= 0 && id[i] < V;
        r.id[i] = in ? (int)id[i] : -1;
        r.z[i] = in ? v[i] : -INFINITY;
        any = any || r.z[i] != -INFINITY;
        if (id[i] >= V && status) report_index(status, MHCLITE_OP_LINEAR_DISTILL, t, id[i]);
    }
    r.live = __any_sync(0xffffffffu, any);
    return r;
}
// z becomes the logarithm of the entry's weight; -inf where there is none.
template <int PER>
__device__ __forceinline__ void ds_weights(DsRow<PER>& r, float inv_tau) {
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) top = fmaxf(top, r.z[i]);
    top = warp_max(top);
    if (top == -INFINITY) top = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        r.z[i] = (r.z[i] - top) * inv_tau;
        sum += expf(r.z[i]);
    }
    const float b = logf(warp_sum(sum));
#pragma unroll
    for (int i = 0; i < PER; ++i) r.z[i] -= b;
}

// A warp's 32 PER keys by rising value, key lane * PER + i in place i of a lane: Batcher's bitonic network, exchanges between
// lanes where the distance reaches beyond one.
template <int PER, typename KEY>
__device__ __forceinline__ void ds_sort(KEY (&key)[PER]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int size = 2; size <= 32 * PER; size *= 2)
#pragma unroll
        for (int apart = size / 2; apart > 0; apart /= 2) {
            if (apart >= PER) {
                const int other = apart / PER;
                // within ascending runs the lower lane keeps the smaller key
                const bool small = ((lane & other) == 0) == ((lane * PER & size) == 0);
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const KEY y = __shfl_xor_sync(0xffffffffu, key[i], other);
                    key[i] = (y < key[i]) == small ? y : key[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    if (i & apart) continue;
                    const bool up = size < PER ? (i & size) == 0 : (lane * PER & size) == 0;
                    const KEY x = key[i], y = key[i | apart];
                    const bool swap = (y < x) == up;
                    key[i] = swap ? y : x;
                    key[i | apart] = swap ? x : y;
                }
            }
        }
}

// A row's entries by rising id, absent ones last, for the tiles' epilogues: each one's place in its 128 columns (`cols`), and which
// is the first from every 128 columns on (`first`), so that an epilogue needs no search.  With them, for the forward's join, their
// numbers in the caller's order (`order`) and the logarithms of their weights (`weights`, +inf where absent), for the backward
// what the bracket is there, exp(logp) - the id's weights (`weights` too).  A warp a row.  Rows with a teacher get 0 in
// `target`, which ce_rows_k lists them by, others -1 and, in the forward, logp 0.
// KEY holds id and number: 32 bits do for vocabularies below 2^23 (256 entries of 4099 rows: 24 -> 20 us).
template <int PER, bool GRAD, typename KEY>
__global__ void __launch_bounds__(256) ds_sort_k(int64_t T, int K, int64_t V, const int64_t* ids, const void* z, int z_f32, float inv_tau,
                                                 const float* logp_in, int entries, uint8_t* cols, uint8_t* order, float* weights,
                                                 uint16_t* first, int blocks, int64_t* target, float* logp, int* status) {
    constexpr int NUMBER = sizeof(KEY) == 4 ? 8 : 32;                   // bits of the number, below the id
    constexpr KEY ABSENT = sizeof(KEY) == 4 ? 0x7FFFFF : 0x7FFFFFFF;
    auto id_of = [](KEY k) { return (k >> NUMBER) == ABSENT ? 0x7FFFFFFF : (int)(k >> NUMBER); };
    auto number_of = [](KEY k) { return (int)(k & (((KEY)1 << NUMBER) - 1)); };
    auto place = [](int at) { return at + (at >> 3); };                 // lanes PER apart meet different banks
    __shared__ int id_s[8][36 * PER];
    __shared__ float p_s[8][32 * PER], w_s[GRAD ? 8 : 1][GRAD ? 32 * PER : 1];
    pdl_wait();
    pdl_launch();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, ws = GRAD ? warp : 0;
    const int64_t t = (int64_t)blockIdx.x * 8 + warp;
    if (t >= T) return;
    DsRow<PER> r = ds_load<PER>(t, K, V, ids, z, z_f32, status);
    if (lane == 0) target[t] = r.live ? 0 : -1;
    if (!r.live) {
        if (!GRAD)
            for (int k = lane; k < K; k += 32) logp[t * K + k] = 0.f;
        return;
    }
    KEY key[PER];
    ds_weights(r, inv_tau);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int k = i * 32 + lane;
        key[i] = (r.id[i] < 0 ? ABSENT : (KEY)r.id[i]) << NUMBER | (KEY)k;       // as numbered where ids are equal
        p_s[warp][k] = GRAD ? expf(r.z[i]) : r.id[i] < 0 ? INFINITY : r.z[i];
    }
    ds_sort(key);
    bool twice = false;
    const int before = __shfl_up_sync(0xffffffffu, id_of(key[PER - 1]), 1);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int id = id_of(key[i]), prior = i ? id_of(key[i ? i - 1 : 0]) : lane ? before : -1;
        id_s[warp][place(lane * PER + i)] = id;
        twice = twice || (id == prior && id != 0x7FFFFFFF);
    }
    __syncwarp();
    if (GRAD) {
#pragma unroll
        for (int i = 0; i < PER; ++i) w_s[ws][lane * PER + i] = p_s[warp][number_of(key[i])];
        __syncwarp();
        if (__any_sync(0xffffffffu, twice)) {                           // an id's entries, which lie side by side, all get their sum
            for (int i = 0; i < PER; ++i) {
                const int at = lane * PER + i, id = id_s[warp][place(at)];
                if (id == 0x7FFFFFFF) continue;
                int from = at;
                while (from > 0 && id_s[warp][place(from - 1)] == id) --from;
                float sum = 0.f;
                for (; from < 32 * PER && id_s[warp][place(from)] == id; ++from) sum += w_s[ws][from];
                p_s[warp][at] = sum;
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < PER; ++i) w_s[ws][lane * PER + i] = p_s[warp][lane * PER + i];
        }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int at = lane * PER + i, id = id_of(key[i]), k = number_of(key[i]);
        if (at >= K) continue;
        cols[t * entries + at] = (uint8_t)(id & 127);
        if (GRAD) {
            weights[t * entries + at] = id != 0x7FFFFFFF ? expf(logp_in[t * K + k]) - w_s[ws][at] : 0.f;
        } else {
            weights[t * entries + at] = p_s[warp][k];
            order[t * entries + at] = (uint8_t)k;
        }
    }
#pragma unroll 4
    for (int b = lane; b <= blocks; b += 32) {
        int at = 0;
#pragma unroll
        for (int step = 16 * PER; step > 0; step /= 2)                  // how many entries lie below the block
            if (id_s[warp][place(at + step - 1)] < b * 128) at += step;
        at += id_s[warp][place(at)] < b * 128;
        first[t * (blocks + 1) + b] = (uint16_t)at;
    }
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

// Joins the (maximum, sum) pairs of 8 rows a block, 32 ranges of tiles side by side, then a warp a row forms loss, lse and logp:
// of the listed rows with their entries as ds_sort_k left them (LISTED), or of all rows with the entries as they came (a handful
// of tokens, with ds_dot_k's products).
template <int PER, bool LISTED>
__global__ void __launch_bounds__(256, 4) ds_join_k(int64_t T, int K, int64_t V, const int* live, const int* rows, int n_parts, int pitch,
                                                 const float2* part, const float* dots, int entries, const uint8_t* order, const float* weights,
                                                 const int64_t* ids, const void* z, int z_f32, float k2, float inv_tau, float* loss, float* lse,
                                                 float* logp, int* status) {
    __shared__ float2 red[32][9];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = LISTED ? *live : (int)T;
    if (blockIdx.x * 8 >= n) return;
    const int r = blockIdx.x * 8 + (lane & 7), range = warp * 4 + (lane >> 3), row = blockIdx.x * 8 + warp;
    DsRow<PER> e;                                                       // z: log weights
    float x[PER];
    int k[PER];
    int64_t t = 0;
    if (row < n) {                                                      // its loads run beside those of the pairs
        t = LISTED ? rows[row] : row;
        if (!LISTED) e = ds_load<PER>(t, K, V, ids, z, z_f32, status);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int at = i * 32 + lane;
            k[i] = at;
            if (LISTED) {
                k[i] = at < K ? order[t * entries + at] : K;
                e.z[i] = at < K ? weights[t * entries + at] : INFINITY;
                e.id[i] = e.z[i] == INFINITY ? -1 : 0;
                x[i] = at < K ? dots[t * entries + at] : 0.f;
            } else {
                x[i] = e.id[i] >= 0 ? dots[t * entries + at] : 0.f;
            }
        }
    }
    float m = -INFINITY, s = 0.f;
    if (r < n) {
#pragma unroll 8
        for (int i = range; i < n_parts; i += 32) {
            const float2 p = part[(int64_t)i * pitch + r];
            const float top = fmaxf(m, p.x), base = top == -INFINITY ? 0.f : top;
            s = s * ex2(m - base) + p.y * ex2(p.x - base);
            m = top;
        }
    }
    red[range][lane & 7] = make_float2(m, s);
    __syncthreads();
    if (row >= n) return;
    const float2 p = red[lane][warp];                                   // lane: a range of tiles, warp: a row
    const float top = warp_max(p.x), base = top == -INFINITY ? 0.f : top;
    const float b = log2f(warp_sum(p.y * ex2(p.x - base)));
    if (!LISTED) ds_weights(e, inv_tau);
    const bool alive = LISTED || e.live;
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (k[i] >= K) continue;
        // x - lse as a difference to the row's largest logit, so that a likely id keeps its digits
        const bool in = alive && e.id[i] >= 0;
        const float q = in ? (fmaf(x[i], k2, -base) - b) * kLn2 : 0.f;
        logp[t * K + k[i]] = q;
        if (in && e.z[i] != -INFINITY) l += expf(e.z[i]) * (e.z[i] - q);
    }
    l = warp_sum(l);
    if (lane == 0) {
        lse[t] = alive ? (top + b) * kLn2 : 0.f;
        loss[t] = l;
    }
}

// ---- host side -------------------------------------------------------------------------------------------------------
struct DsPlan { CePlan ce; int64_t* target; float *dots, *weights; uint8_t *cols, *order; uint16_t* first; int blocks, entries; size_t bytes; };
static DsPlan plan_ds(int64_t T, int64_t V, int K, int C, int grad, void* base) {
    DsPlan p;
    char* b = (char*)base;
    p.ce = plan_ce(T, V, C, grad, base);
    size_t off = (ce_scratch_bytes(T, V, C, grad) + 255) & ~(size_t)255;
    auto take = [&](size_t n) { char* at = b + off; off += (n + 255) & ~(size_t)255; return at; };
    p.target = (int64_t*)take((size_t)T * 8);
    p.entries = (K + 7) / 8 * 8;
    p.weights = (float*)take((size_t)T * p.entries * 4);
    p.cols = (uint8_t*)take((size_t)T * p.entries);
    p.dots = (float*)take(grad ? 0 : (size_t)T * p.entries * 4);
    p.order = (uint8_t*)take(grad ? 0 : (size_t)T * p.entries);
    p.blocks = 2 * p.ce.n_tiles;
    p.first = (uint16_t*)take((size_t)T * (p.blocks + 1) * 2);
    p.bytes = off;
    return p;
}
size_t distill_scratch_bytes(int64_t T, int64_t V, int K, int C, int grad) { return plan_ds(T, V, K, C, grad, nullptr).bytes; }

// Calls f with the entries a lane holds, as a compile-time number.
template <typename F>
static auto ds_per(int K, F f) {
    return K <= 32 ? f(std::integral_constant<int, 1>()) : K <= 64 ? f(std::integral_constant<int, 2>())
           : K <= 128 ? f(std::integral_constant<int, 4>()) : f(std::integral_constant<int, 8>());
}
template <bool GRAD>
static void launch_ds_sort(const mhclite_ctx* c, const DsPlan& p, int64_t T, int64_t V, int K, const int64_t* ids, const void* z, int z_f32,
                           float inv_tau, const float* logp_in, float* logp, cudaStream_t s) {
    c->launches += 1;
    ds_per(K, [&](auto per) {
        constexpr int PER = decltype(per)::value;
        launch_after(V < (1 << 23) ? ds_sort_k<PER, GRAD, uint32_t> : ds_sort_k<PER, GRAD, unsigned long long>, dim3((unsigned)((T + 7) / 8)), dim3(256), 0, s, T, K, V, ids, z, z_f32, inv_tau, logp_in,
                     p.entries, p.cols, p.order, p.weights, p.first, p.blocks, p.target, logp, c->op_status);
    });
}

bool launch_linear_distill_fwd(const mhclite_ctx* c, int64_t T, int64_t V, int K, const void* h, const void* W, const int64_t* ids,
                               const void* z, int z_f32, float scale, float inv_tau, float* loss, float* lse, float* logp, void* scratch,
                               cudaStream_t s) {
    const DsPlan p = plan_ds(T, V, K, c->C, 0, scratch);
    const SmallPlan q = plan_small(T, c->C);
    const float k2 = scale * kLog2e;
    const dim3 grid((unsigned)((T + 7) / 8)), block(256);
    if (q.stages) {
        const int64_t entries = T * K;
        const float2* part = (const float2*)scratch;
        c->launches += 1;
        launch_after(ds_dot_k, dim3((unsigned)((entries + 7) / 8)), block, 0, s, entries, K, V, c->C, ids, (const uint4*)h, (const uint4*)W, p.dots);
        const int parts = launch_ce_small<false>(c, q, T, V, h, W, nullptr, scale, (float2*)scratch, nullptr, s);
        ds_per(K, [&](auto per) {
            launch_after(ds_join_k<decltype(per)::value, false>, grid, block, 0, s, T, K, V, nullptr, nullptr, parts, kSmTokens, part, p.dots, K, nullptr,
                         nullptr, ids, z, z_f32, k2, inv_tau, loss, lse, logp, c->op_status);
        });
        return true;
    }
    launch_ds_sort<false>(c, p, T, V, K, ids, z, z_f32, inv_tau, nullptr, logp, s);
    CeArgs a = {};
    a.cols = p.cols; a.values = p.dots; a.from = p.first; a.entries = p.entries; a.blocks = p.blocks;
    if (!launch_ce_stats<CE_PICK>(c, p.ce, a, T, V, h, W, p.target, scale, loss, lse, s)) return false;
    ds_per(K, [&](auto per) {
        launch_after(ds_join_k<decltype(per)::value, true>, grid, block, 0, s, T, K, V, p.ce.live, p.ce.rows, 2 * p.ce.n_tiles, p.ce.Tpad, p.ce.part, p.dots,
                     p.entries, p.order, p.weights, nullptr, nullptr, 0, k2, inv_tau, loss, lse, logp, nullptr);
    });
    return true;
}

bool launch_linear_distill_bwd(const mhclite_ctx* c, int64_t T, int64_t V, int K, const void* h, const void* W, const int64_t* ids,
                               const void* z, int z_f32, float scale, float inv_tau, const float* lse, const float* logp, const float* dloss,
                               void* dh, void* dW, void* scratch, cudaStream_t s) {
    const DsPlan p = plan_ds(T, V, K, c->C, 1, scratch);
    launch_ds_sort<true>(c, p, T, V, K, ids, z, z_f32, inv_tau, logp, nullptr, s);
    CeArgs a = {};
    a.cols = p.cols; a.values = p.weights; a.from = p.first; a.entries = p.entries; a.blocks = p.blocks;
    return launch_ce_grads<CE_PATCH>(c, p.ce, a, T, V, h, W, p.target, scale, lse, dloss, dh, dW, s);
}

}  // namespace mhcl
