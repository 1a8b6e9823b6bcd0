// The lookup that fills the residual streams and its gradient:
//   x0[t,j,:] = bf16(scale E[id_t,:])  for every stream j,
//   dE[v,:] (+)= scale sum_{t: id_t = v} sum_j g[t,j,:].
//
// The forward is bound by the n rows it writes a token.  The gradient is bound by the n rows it reads a token and the
// table it writes; its sums must not depend on the order in which blocks run, so the tokens are sorted first (stable:
// tokens of one id stay in ascending order; embed_rank_k for up to 6144 tokens, embed_sort_k beyond, embed_few_k without a sort for up to 192), then embed_grad_k
// walks the sorted list in chunks, one warp a chunk and 256 channels, and keeps the running sum of the current id in fp32
// registers.  An id whose tokens span several chunks leaves one partial row a chunk, which embed_join_k adds up in order: a
// token as frequent as the commonest word does not serialise.  Rows that no token meets are zeroed by further blocks of
// embed_grad_k, so each row of dE is written once.  The three launches overlap their starts (programmatic launch).
#include "common.cuh"
#include "kernels.h"

namespace mhcl {

template <bool F32>
__global__ void __launch_bounds__(256) embed_fwd_k(int64_t T, int64_t V, int C, int n, int tpt, const int64_t* ids,
                                                   const void* E, float scale, uint4* x0,
                                                   int* status) {
    pdl_wait();
    pdl_launch();
    const int nv = C >> 3, per = 256 / tpt, lt = threadIdx.x % tpt;
    const int64_t t = (int64_t)blockIdx.x * per + threadIdx.x / tpt;
    if (t >= T) return;
    const int64_t id = ids[t];
    const bool ok = id >= 0 && id < V;
    if (!ok && lt == 0) report_index(status, MHCLITE_OP_EMBED, t, id);
    uint4* row = x0 + t * n * nv;
    for (int v = lt; v < nv; v += tpt) {
        float f[8];
        if (!ok) {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = 0.f;
        } else if (F32) {
            const float4* p = (const float4*)E + (id * nv + v) * 2;
            const float4 a = ld_dep(p), b = ld_dep(p + 1);
            f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
        } else {
            unpack8(ld_dep((const uint4*)E + id * nv + v), f);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= scale;
        if (!ok)
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = 0.f;
        const uint4 o = pack8(f);
        for (int j = 0; j < n; ++j) st_stream(row + j * nv + v, o);
    }
}

// ---- stable sort of the tokens by id ---------------------------------------------------------------------------------
// Few tokens: every block holds all keys in shared memory and ranks 32 tokens at a time by counting the keys below theirs
// (T^2 comparisons, spread over all SMs), which needs no exchange between blocks.  The whole gradient, 3 streams of 1536
// channels and 1000 rows: 2048 tokens 21 us (29 with the cluster's sort), 4096 27.5 (34), 8192 39 (38).
constexpr int kRankMax = 6144;
__device__ __forceinline__ uint32_t embed_key(int64_t id, int64_t i, int64_t V, bool say, int* status) {
    const bool ok = id >= 0 && id < V;
    if (!ok && say) report_index(status, MHCLITE_OP_EMBED_BWD, i, id);
    return ok ? (uint32_t)id : (uint32_t)V;                    // tokens without a row go last
}
__global__ void __launch_bounds__(256) embed_rank_k(int T, int64_t V, const int64_t* ids, uint2* list,
                                                    int* status) {
    __shared__ __align__(16) uint32_t key[kRankMax];
    __shared__ int below[8][32];
    pdl_wait();
    pdl_launch();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, quads = (T + 3) / 4;
    for (int i0 = tid; i0 < quads * 4; i0 += 256 * 8) {        // eight loads in flight
        int64_t id[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) id[k] = i0 + k * 256 < T ? ld_dep(ids + i0 + k * 256) : 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int i = i0 + k * 256;
            if (i >= quads * 4) break;
            key[i] = i < T ? embed_key(id[k], i, V, blockIdx.x == 0, status) : 0xFFFFFFFFu;
        }
    }
    __syncthreads();
    for (int b = blockIdx.x * 32; b < T; b += gridDim.x * 32) {
        // a lane takes one token, a warp an eighth of the keys
        const int i = b + lane;
        const uint32_t mine = i < T ? key[i] : 0;
        const int per = (quads + 7) / 8, q0 = warp * per, q1 = q0 + per < quads ? q0 + per : quads;
        int n = 0;
        // keys of earlier tokens count when equal too: below mine + 1 before this block of 32 tokens, below mine behind it
        auto count = [&](int qa, int qb, uint32_t limit) {
#pragma unroll 8
            for (int q = qa; q < qb; ++q) {
                const uint4 k = *reinterpret_cast<const uint4*>(key + 4 * q);
                if (k.x < limit) ++n;
                if (k.y < limit) ++n;
                if (k.z < limit) ++n;
                if (k.w < limit) ++n;
            }
        };
        const int qb = b / 4, qe = qb + 8;
        count(q0, min(q1, qb), mine + 1);
        for (int j = max(4 * q0, 4 * qb); j < min(4 * q1, 4 * qe); ++j) n += key[j] < mine + (j < i ? 1 : 0) ? 1 : 0;
        count(max(q0, qe), q1, mine);
        below[warp][lane] = n;
        __syncthreads();
        if (warp == 0 && i < T) {
            int rank = 0;
#pragma unroll
            for (int w = 0; w < 8; ++w) rank += below[w][lane];
            list[rank] = make_uint2(mine, (uint32_t)i);
        }
        __syncthreads();
    }
}

// More tokens: one cluster of up to 16 blocks sorts, least significant digit first, 9 bits a pass (two passes for tables
// below 2^18 rows): a warp owns a contiguous range of the list and counts its digits in shared memory, the blocks exchange
// their totals through distributed shared memory, and each warp then walks its range again and places the tokens.  A range
// is read eight vectors of 32 entries at a time, so that a pass costs a few memory latencies, which are what bounds it; a
// launch a pass would cost more than the pass.
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kSortBits = 9, kSortBins = 1 << kSortBits, kSortAhead = 8, kSortMaxBlocks = 16;
constexpr int kSortSmem = kSortWarps * kSortBins * 4;

__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t ld_peer(const uint32_t* p, uint32_t rank) {   // 32 bits of another block's shared memory
    uint32_t a = (uint32_t)__cvta_generic_to_shared(p), b, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(b) : "r"(a), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(b) : "memory");
    return v;
}

// The lanes of `live` whose digit equals this lane's, by one vote a bit: a match instruction visits the distinct values one
// after the other and took most of the sort's time (65536 tokens of 100000 rows: 59 us, now 27).
__device__ __forceinline__ uint32_t same_digit(uint32_t live, uint32_t d) {
    uint32_t m = live;
#pragma unroll
    for (int i = 0; i < kSortBits; ++i) {
        const uint32_t set = (uint32_t)((int32_t)(d << (31 - i)) >> 31);       // all ones where the bit is set
        m &= ~(__ballot_sync(live, set) ^ set);
    }
    return m;
}

__global__ void __launch_bounds__(kSortThreads) embed_sort_k(int T, int64_t V, int passes, const int64_t* ids,
                                                             uint2* buf0, uint2* buf1, int* status) {
    extern __shared__ uint32_t cnt[];                          // [warp][bin]
    __shared__ uint32_t tot[kSortBins], off[kSortBins], wsum[kSortBins / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int me = (int)cluster_rank(), nb = (int)cluster_size();
    const int warps = nb * kSortWarps, per = ((T - 1) / warps / 32 + 1) * 32;                  // entries a warp, a multiple of 32
    const int64_t begin = (int64_t)(me * kSortWarps + warp) * per;
    const int i0 = begin < T ? (int)begin : T, i1 = T - i0 < per ? T : i0 + per;
    uint32_t* mine = cnt + warp * kSortBins;
    pdl_wait();
    pdl_launch();
    uint2 *src = buf0, *dst = buf1;
    for (int p = 0; p < passes; ++p) {
        const int shift = p * kSortBits;
        for (int i = tid; i < kSortWarps * kSortBins / 4; i += kSortThreads) reinterpret_cast<uint4*>(cnt)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        for (int b = i0; b < i1; b += 32 * kSortAhead) {
            uint32_t key[kSortAhead];
#pragma unroll
            for (int k = 0; k < kSortAhead; ++k) {
                const int i = b + k * 32 + lane;
                if (i < i1) key[k] = p == 0 ? embed_key(ld_dep(ids + i), i, V, true, status) : ld_dep_l2(src + i).x;
            }
#pragma unroll
            for (int k = 0; k < kSortAhead; ++k) {
                const int i = b + k * 32 + lane;
                if (i < i1) {
                    if (p == 0) src[i] = make_uint2(key[k], (uint32_t)i);
                    atomicAdd(mine + ((key[k] >> shift) & (kSortBins - 1)), 1u);
                }
            }
        }
        __syncthreads();
        if (tid < kSortBins) {                                 // the warps' counts become offsets within the block
            uint32_t run = 0;
#pragma unroll 16
            for (int w = 0; w < kSortWarps; ++w) { const uint32_t c = cnt[w * kSortBins + tid]; cnt[w * kSortBins + tid] = run; run += c; }
            tot[tid] = run;
        }
        cluster_sync_all();
        uint32_t before = 0, all = 0, inc = 0;
        if (tid < kSortBins) {
            for (int r0 = 0; r0 < nb; r0 += 8) {
                uint32_t c[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) c[r] = r0 + r < nb ? ld_peer(&tot[tid], r0 + r) : 0;
#pragma unroll
                for (int r = 0; r < 8; ++r) { if (r0 + r < me) before += c[r]; all += c[r]; }
            }
            inc = all;                                         // inclusive scan over the digits
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const uint32_t u = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += u; }
            if (lane == 31) wsum[warp] = inc;
        }
        __syncthreads();
        if (tid < kSortBins) {
            uint32_t add = 0;
#pragma unroll
            for (int w = 0; w < kSortBins / 32; ++w) add += w < warp ? wsum[w] : 0;
            off[tid] = inc - all + before + add;
        }
        __syncthreads();
        for (int b = i0; b < i1; b += 32 * kSortAhead) {
            uint2 kv[kSortAhead];
#pragma unroll
            for (int k = 0; k < kSortAhead; ++k)
                if (b + k * 32 + lane < i1) kv[k] = ld_dep_l2(src + b + k * 32 + lane);
#pragma unroll
            for (int k = 0; k < kSortAhead; ++k) {
                if (b + k * 32 >= i1) break;
                const bool in = b + k * 32 + lane < i1;
                const uint32_t live = __ballot_sync(0xffffffffu, in);
                if (in) {
                    const uint32_t d = (kv[k].x >> shift) & (kSortBins - 1), peers = same_digit(live, d);
                    const uint32_t rank = __popc(peers & ((1u << lane) - 1u)), base = mine[d];
                    __syncwarp(live);
                    if (rank == 0) mine[d] = base + __popc(peers);
                    __stcg(dst + off[d] + base + rank, kv[k]);
                }
                __syncwarp();
            }
        }
        uint2* h = src; src = dst; dst = h;
        cluster_sync_all();
    }
}

// ---- sums over the sorted list ---------------------------------------------------------------------------------------
// The cluster's sort leaves most SMs and all of HBM idle for some 20 us: the table's last rows, up to 96 MB of them, are
// cleared meanwhile, met or not (rare words stand there in the tables of text).  This launch starts once the sort has begun
// and by then has seen the stream's earlier work done; it ends after the sort, so that what follows may wait for it alone.
constexpr int64_t kEarlyZero = (int64_t)96 << 20;         // 65536 x 1024, 100000 rows: 176 us without, 172 with 64 MB, 170
__global__ void __launch_bounds__(256) embed_zero_k(float4* to, int64_t n) {
    pdl_launch();
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) __stcs(to + i, zero);
    pdl_wait();
}

constexpr int kZeroRows = 64;          // rows a block looks over for those that no token meets

// Warp (chunk, slice) adds up `R` list entries for channels [256 slice, 256 slice + 256), 8 a lane.
template <int N_>
__global__ void __launch_bounds__(256) embed_grad_k(int64_t T, int64_t V, int64_t to_zero, int C, int R, int64_t sum_blocks, int slices,
                                                    const uint2* list,
                                                    const uint4* g, float scale, float* dE,
                                                    float* own, float* cont, int accumulate) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nv = C >> 3;
    pdl_wait();
    pdl_launch();
    if (blockIdx.x >= sum_blocks) {                            // rows that no token meets
        __shared__ uint32_t met[kZeroRows / 32];
        __shared__ int64_t range[2];
        const int64_t v0 = (int64_t)(blockIdx.x - sum_blocks) * kZeroRows, v1 = v0 + kZeroRows < to_zero ? v0 + kZeroRows : to_zero;
        if (threadIdx.x < kZeroRows / 32) met[threadIdx.x] = 0;
        if (warp < 2) {                                        // the entries of these rows: a warp finds each end
            const int64_t bound = warp == 0 ? v0 : v1;
            int64_t lo = -1, hi = T;                           // the first entry not below `bound` lies in (lo, hi]
            while (hi - lo > 1) {
                const int64_t step = (hi - lo + 31) / 32, probe = lo + 1 + lane * step;
                const int n = __popc(__ballot_sync(0xffffffffu, (probe < hi) & (ld_dep(&list[probe < hi ? probe : 0].x) < bound)));
                const int64_t end = lo + 1 + n * step;
                if (n > 0) lo += 1 + (n - 1) * step;
                hi = end < hi ? end : hi;
                if (n == 0) break;
            }
            if (lane == 0) range[warp] = hi;
        }
        __syncthreads();
        if (threadIdx.x < kZeroRows) {                         // a thread a row: is it among them?
            const int64_t v = v0 + threadIdx.x, end = range[1];        // (rows behind v1 are not looked at again)
            int64_t lo = range[0], hi = end;
            while (lo < hi) {
                const int64_t mid = (lo + hi) >> 1;
                if (ld_dep(&list[mid].x) < v) lo = mid + 1; else hi = mid;
            }
            if (lo < end && ld_dep(&list[lo].x) == v) atomicOr(&met[threadIdx.x >> 5], 1u << lane);
        }
        __syncthreads();
        const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int64_t v = v0 + warp; v < v1; v += 8) {
            if (met[(v - v0) >> 5] >> ((v - v0) & 31) & 1u) continue;
            float4* row = (float4*)(dE + v * C);
            for (int c = lane; c < C / 4; c += 32) __stcs(row + c, zero);
        }
        return;
    }
    const int64_t unit = (int64_t)blockIdx.x * 8 + warp;
    const int64_t chunk = unit / slices;
    const int v = (int)(unit % slices) * 32 + lane;            // this lane's 16-byte vector of a row
    const int64_t p0 = chunk * R;
    if (p0 >= T) return;
    const int cnt = (int)(T - p0 < R ? T - p0 : R);
    const uint2 mine = lane < cnt ? ld_dep(list + p0 + lane) : make_uint2(0xFFFFFFFFu, 0);
    const uint32_t prev = p0 > 0 ? ld_dep(&list[p0 - 1].x) : 0xFFFFFFFFu;
    const uint32_t next = p0 + cnt < T ? ld_dep(&list[p0 + cnt].x) : 0xFFFFFFFFu;
    const bool act = v < nv;
    float acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    constexpr int U = 16 / N_ > 4 ? 4 : 16 / N_;               // tokens whose rows are in flight together
    for (int i = 0; i < cnt; i += U) {
        uint4 d[U][N_];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const uint32_t t = __shfl_sync(0xffffffffu, mine.y, (i + k) & 31);
            if (act && i + k < cnt) {
#pragma unroll
                for (int j = 0; j < N_; ++j) d[k][j] = ld_dep_stream(g + ((int64_t)t * N_ + j) * nv + v);
            }
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (i + k >= cnt) break;
            const uint32_t key = __shfl_sync(0xffffffffu, mine.x, i + k);
            const uint32_t after = i + k + 1 < cnt ? __shfl_sync(0xffffffffu, mine.x, (i + k + 1) & 31) : next;
            if (act) {
#pragma unroll
                for (int j = 0; j < N_; ++j) {
                    float f[8];
                    unpack8(d[k][j], f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[e] += f[e];
                }
            }
            const bool last = i + k + 1 == cnt;
            if (key != after || last) {
                const uint32_t first_key = __shfl_sync(0xffffffffu, mine.x, 0);
                if (act && key < V) {
                    const bool began_before = key == first_key && prev == key;
                    float* to = began_before ? cont + chunk * C : (last && after == key) ? own + chunk * C : nullptr;
                    if (to) {
                        float4* o = (float4*)(to + v * 8);
                        o[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
                        o[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
                    } else {
                        float4* o = (float4*)(dE + (int64_t)key * C + v * 8);
                        float4 a = accumulate ? o[0] : make_float4(0.f, 0.f, 0.f, 0.f), b = accumulate ? o[1] : a;
                        a.x += scale * acc[0]; a.y += scale * acc[1]; a.z += scale * acc[2]; a.w += scale * acc[3];
                        b.x += scale * acc[4]; b.y += scale * acc[5]; b.z += scale * acc[6]; b.w += scale * acc[7];
                        o[0] = a; o[1] = b;
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] = 0.f;
            }
        }
    }
}

// The ids that span chunks: the warp of the chunk in which such an id begins adds up its partial rows; ids of more than
// kJoinAlone parts are shared out among the block's warps, a range of the parts each, joined in order.
constexpr int kJoinAlone = 16;
__device__ __forceinline__ void add4(float4& a, const float4& x) { a.x += x.x; a.y += x.y; a.z += x.z; a.w += x.w; }
__device__ __forceinline__ void join_sum(const float* part, int64_t c0, int64_t c1, int C, int v, float4& a, float4& b) {
#pragma unroll 4
    for (int64_t c = c0; c < c1; ++c) {
        const float4* q = (const float4*)(part + c * C + v * 8);
        add4(a, ld_dep(q));
        add4(b, ld_dep(q + 1));
    }
}
__device__ __forceinline__ void join_store(float* dE, uint32_t key, int C, int v, float scale, int accumulate, const float4& a, const float4& b) {
    float4* o = (float4*)(dE + (int64_t)key * C + v * 8);
    float4 s0 = accumulate ? o[0] : make_float4(0.f, 0.f, 0.f, 0.f), s1 = accumulate ? o[1] : s0;
    s0.x += scale * a.x; s0.y += scale * a.y; s0.z += scale * a.z; s0.w += scale * a.w;
    s1.x += scale * b.x; s1.y += scale * b.y; s1.z += scale * b.z; s1.w += scale * b.w;
    o[0] = s0; o[1] = s1;
}
__global__ void __launch_bounds__(256) embed_join_k(int64_t T, int64_t V, int C, int R, const uint2* list,
                                                    const float* own, const float* cont, float scale,
                                                    float* dE, int accumulate) {
    __shared__ float4 red[8][32][2];
    __shared__ int64_t first_s[8], end_s[8];
    __shared__ uint32_t key_s[8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nv = C >> 3;
    const int64_t chunk = (int64_t)blockIdx.x * 8 + warp, p0 = chunk * R, p1 = p0 + R;
    const int v = blockIdx.y * 32 + lane;
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    pdl_wait();
    if (lane == 0) end_s[warp] = 0;
    if (p1 < T) {
        const int64_t at[4] = {p1 - 1, p1, p0, p0 > 0 ? p0 - 1 : p0};                // one load for the four
        const uint32_t mine = ld_dep(&list[at[lane & 3]].x);
        const uint32_t key = __shfl_sync(0xffffffffu, mine, 0), next = __shfl_sync(0xffffffffu, mine, 1);
        const uint32_t head = __shfl_sync(0xffffffffu, mine, 2), prev = __shfl_sync(0xffffffffu, mine, 3);
        const bool began_before = p0 > 0 && head == key && prev == key;
        if (key < V && next == key && !began_before) {
            // chunks of this id in a row, mostly few: one look at the next 32, and a search only where all are
            const int64_t head_at = p1 + (int64_t)lane * R;
            const uint32_t same = __ballot_sync(0xffffffffu, (head_at < T) & (ld_dep(&list[head_at < T ? head_at : p1].x) == key));
            const int run = same == 0xffffffffu ? 32 : __ffs(~same) - 1;
            int64_t lo = p1 + (int64_t)(run - 1) * R, hi = run < 32 ? lo + 1 : T;     // the last entry known to be of the id
            while (hi - lo > 1) {
                const int64_t step = (hi - lo + 31) / 32, probe = lo + lane * step;
                const uint32_t same = __ballot_sync(0xffffffffu, (probe < hi) & (ld_dep(&list[probe < hi ? probe : lo].x) == key));
                const int n = __popc(same);                    // probes 0 .. n-1 are of the id (probe 0 is)
                const int64_t l = lo + (int64_t)(n - 1) * step;
                hi = l + step < hi ? l + step : hi;
                lo = l;
            }
            const int64_t c1 = lo / R + 1;                     // chunks chunk + 1 .. c1 - 1 hold the rest
            if (c1 - chunk - 1 <= kJoinAlone) {
                if (v < nv) {
                    float4 a = zero, b = zero;
                    join_sum(own, chunk, chunk + 1, C, v, a, b);
                    join_sum(cont, chunk + 1, c1, C, v, a, b);
                    join_store(dE, key, C, v, scale, accumulate, a, b);
                }
            } else if (lane == 0) {
                first_s[warp] = chunk; end_s[warp] = c1; key_s[warp] = key;
            }
        }
    }
    __syncthreads();
    for (int j = 0; j < 8; ++j) {
        const int64_t c1 = end_s[j], c0 = first_s[j] + 1;
        if (c1 == 0) continue;
        const int64_t per = (c1 - c0 + 7) / 8, a0 = c0 + warp * per, a1 = a0 + per < c1 ? a0 + per : c1;
        float4 a = zero, b = zero;
        if (v < nv) join_sum(cont, a0, a1, C, v, a, b);
        red[warp][lane][0] = a;
        red[warp][lane][1] = b;
        __syncthreads();
        if (warp == 0 && v < nv) {
            a = b = zero;
            join_sum(own, c0 - 1, c0, C, v, a, b);
            for (int w = 0; w < 8; ++w) { add4(a, red[w][lane][0]); add4(b, red[w][lane][1]); }
            join_store(dE, key_s[j], C, v, scale, accumulate, a, b);
        }
        __syncthreads();
    }
}

// ---- a handful of tokens ---------------------------------------------------------------------------------------------
// Up to 192 tokens: every block sees all keys at once, so nothing is sorted and one launch does it all.  The block of an
// id's first token and of 256 channels adds up the id's tokens, an eighth of the list a warp in ascending order, then the
// warps in order; further blocks clear the rows that no token meets.  3 streams of 1536 channels, 1000 rows: 64
// tokens 11 us, with the sort and its two further launches 14; 200 tokens 13.0 and 14.2, 512 tokens 16.5 and 15.6.
constexpr int kFewTokens = 192;
template <int N_>
__global__ void __launch_bounds__(256) embed_few_k(int T, int64_t V, int C, int64_t sum_blocks, int slices, const int64_t* ids,
                                                   const uint4* g, float scale, float* dE, int accumulate,
                                                   int* status) {
    __shared__ uint32_t key[kFewTokens];
    __shared__ uint32_t met[kZeroRows / 32];
    __shared__ float4 red[8][32][2];
    pdl_wait();
    pdl_launch();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nv = C >> 3;
    for (int i = tid; i < T; i += 256) key[i] = embed_key(ld_dep(ids + i), i, V, blockIdx.x == 0, status);
    if (tid < kZeroRows / 32) met[tid] = 0;
    __syncthreads();
    if (blockIdx.x >= sum_blocks) {
        const int64_t v0 = (int64_t)(blockIdx.x - sum_blocks) * kZeroRows, v1 = v0 + kZeroRows < V ? v0 + kZeroRows : V;
        for (int i = tid; i < T; i += 256)
            if (key[i] >= v0 && key[i] < v1) atomicOr(&met[(key[i] - v0) >> 5], 1u << ((key[i] - v0) & 31));
        __syncthreads();
        const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int64_t v = v0 + warp; v < v1; v += 8) {
            if (met[(v - v0) >> 5] >> ((v - v0) & 31) & 1u) continue;
            float4* row = (float4*)(dE + v * C);
            for (int c = lane; c < C / 4; c += 32) __stcs(row + c, zero);
        }
        return;
    }
    const int i = (int)(blockIdx.x / slices), v = (int)(blockIdx.x - (int64_t)i * slices) * 32 + lane;
    const uint32_t k = key[i];
    bool earlier = false;
    for (int j = tid; j < i; j += 256) earlier |= key[j] == k;
    if (__syncthreads_or(earlier || k >= V)) return;           // another block has the id's first token, or it has no row
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int per = ((T + 7) / 8 + 31) / 32 * 32;              // tokens a warp
    constexpr int U = 16 / N_ > 4 ? 4 : 16 / N_;
    for (int b = warp * per; b < T && b < (warp + 1) * per; b += 32) {
        uint32_t same = __ballot_sync(0xffffffffu, b + lane < T && key[min(b + lane, T - 1)] == k);
        while (same) {
            uint4 d[U][N_];
            int n = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (same) {
                    const int t = b + __ffs(same) - 1;
                    same &= same - 1;
                    ++n;
                    if (v < nv) {
#pragma unroll
                        for (int j = 0; j < N_; ++j) d[u][j] = ld_dep_stream(g + ((int64_t)t * N_ + j) * nv + v);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u >= n || v >= nv) break;
#pragma unroll
                for (int j = 0; j < N_; ++j) {
                    float f[8];
                    unpack8(d[u][j], f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[e] += f[e];
                }
            }
        }
    }
    red[warp][lane][0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    red[warp][lane][1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
    __syncthreads();
    if (warp != 0 || v >= nv) return;
    float4 a = red[0][lane][0], c = red[0][lane][1];
#pragma unroll
    for (int w = 1; w < 8; ++w) { add4(a, red[w][lane][0]); add4(c, red[w][lane][1]); }
    join_store(dE, k, C, v, scale, accumulate, a, c);
}

// ---- host side -------------------------------------------------------------------------------------------------------
void launch_embed_fwd(const mhclite_ctx* c, int64_t T, int64_t V, const int64_t* ids, const void* E, int table_f32, float scale,
                      void* x0, cudaStream_t s) {
    int tpt = 32;                                              // threads a token
    while (tpt < 256 && tpt * 8 < c->C) tpt *= 2;
    const unsigned grid = (unsigned)((T + 256 / tpt - 1) / (256 / tpt));
    c->launches += 1;
    auto k = table_f32 ? embed_fwd_k<true> : embed_fwd_k<false>;
    launch_after(k, dim3(grid), dim3(256), 0, s, T, V, c->C, c->n, tpt, ids, E, scale, (uint4*)x0, c->op_status);
}

// List entries a warp adds up: 32 where that leaves enough warps to fill the GPU (a B200's 148 SMs: the number also gives the
// scratch's size, which callers ask for without a context), fewer for short lists.
static int embed_chunk(int64_t T, int C) {
    const int64_t slices = (C / 8 + 31) / 32;
    int R = 32;
    while (R > 4 && (T + R - 1) / R * slices < 148 * 24) R /= 2;
    return R;
}

struct EmbedScratch { uint2 *buf0, *buf1; float *own, *cont; size_t bytes; };
static EmbedScratch plan_embed(int64_t T, int C, void* base) {
    EmbedScratch p;
    char* b = (char*)base;
    size_t off = 0;
    const int64_t chunks = (T + embed_chunk(T, C) - 1) / embed_chunk(T, C);
    auto take = [&](size_t n) { char* at = b + off; off += (n + 255) & ~(size_t)255; return at; };
    p.buf0 = (uint2*)take((size_t)T * 8);
    p.buf1 = (uint2*)take((size_t)T * 8);
    p.own = (float*)take((size_t)chunks * C * 4);
    p.cont = (float*)take((size_t)chunks * C * 4);
    p.bytes = off;
    return p;
}
size_t embed_scratch_bytes(int64_t T, int C) { return T <= kFewTokens ? 0 : plan_embed(T, C, nullptr).bytes; }

cudaError_t launch_embed_bwd(const mhclite_ctx* c, int64_t T, int64_t V, const int64_t* ids, const void* g, float scale, float* dE,
                             int accumulate, void* scratch, cudaStream_t s) {
    const int slices = (c->C / 8 + 31) / 32;
    cudaError_t e = cudaSuccess;
    if (T <= kFewTokens) {
        const int64_t sum_blocks = T * slices;
        const int64_t zero_blocks = accumulate ? 0 : (V + kZeroRows - 1) / kZeroRows;
        c->launches += 1;
        MHCL_DISPATCH_N(c->n, e = launch_after(embed_few_k<N_>, dim3((unsigned)(sum_blocks + zero_blocks)), dim3(256), 0, s, (int)T, V, c->C,
                                               sum_blocks, slices, ids, (const uint4*)g, scale, dE, accumulate, c->op_status))
        return e;
    }
    const EmbedScratch p = plan_embed(T, c->C, scratch);
    c->launches += 2;
    int64_t to_zero = accumulate ? 0 : V;                      // the table's first rows, left to embed_grad_k
    const uint2* list = p.buf0;
    if (T <= kRankMax) {
        const int blocks = (int)((T + 31) / 32);
        e = launch_after(embed_rank_k, dim3(blocks < c->sm_count * 2 ? blocks : c->sm_count * 2), dim3(256), 0, s, (int)T, V, ids, p.buf0,
                         c->op_status);
        if (e != cudaSuccess) return e;
    } else {
        int bits = 1;
        while ((V >> bits) != 0) ++bits;                       // keys run to V
        const int passes = (bits + kSortBits - 1) / kSortBits;
        int nb = kSortMaxBlocks;                               // blocks of the cluster, with at least 64 tokens a warp
        while (nb > 1 && T <= (int64_t)(nb / 2) * kSortWarps * 64) nb /= 2;
        static SmemOnce once;
        smem_limit(once, embed_sort_k, c->device, kSortSmem);
        cudaFuncSetAttribute(embed_sort_k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        for (;; nb /= 2) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(nb);
            cfg.blockDim = dim3(kSortThreads);
            cfg.dynamicSmemBytes = kSortSmem;
            cfg.stream = s;
            cudaLaunchAttribute at[2];
            at[0].id = cudaLaunchAttributeClusterDimension;
            at[0].val.clusterDim.x = nb; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
            at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
            at[1].val.programmaticStreamSerializationAllowed = 1;
            cfg.attrs = at;
            cfg.numAttrs = 2;
            e = cudaLaunchKernelEx(&cfg, embed_sort_k, (int)T, V, passes, ids, p.buf0, p.buf1, c->op_status);
            if (e == cudaSuccess) break;
            if (nb <= 8) return e;                             // clusters beyond 8 blocks need not exist on every device
            cudaGetLastError();
        }
        if (passes & 1) list = p.buf1;
        const int64_t early = accumulate ? 0 : (kEarlyZero / (c->C * 4) < V ? kEarlyZero / (c->C * 4) : V);
        if (early * c->C * 4 >= kEarlyZero / 4) {              // worth a launch
            to_zero = V - early;
            c->launches += 1;
            e = launch_after(embed_zero_k, dim3(c->sm_count * 4), dim3(256), 0, s, (float4*)(dE + to_zero * c->C), early * c->C / 4);
            if (e != cudaSuccess) return e;
        }
    }
    const int R = embed_chunk(T, c->C);
    const int64_t chunks = (T + R - 1) / R, sum_blocks = (chunks * slices + 7) / 8;
    const int64_t zero_blocks = (to_zero + kZeroRows - 1) / kZeroRows;
    MHCL_DISPATCH_N(c->n, e = launch_after(embed_grad_k<N_>, dim3((unsigned)(sum_blocks + zero_blocks)), dim3(256), 0, s, T, V, to_zero, c->C, R,
                                           sum_blocks, slices, list, (const uint4*)g, scale, dE, p.own, p.cont, accumulate))
    if (e != cudaSuccess) return e;
    if (chunks < 2) return cudaSuccess;                        // no id can span chunks
    c->launches += 1;
    return launch_after(embed_join_k, dim3((unsigned)((chunks + 7) / 8), (unsigned)slices), dim3(256), 0, s, T, V, c->C, R, list, p.own,
                        p.cont, scale, dE, accumulate);
}

}  // namespace mhcl
