// Softmax cross entropy of h W^T over a large vocabulary, without the logits in memory:
//   l[t,v] = scale <h_t, W_v>,  lse_t = log sum_v exp l[t,v],  loss_t = lse_t - l[t,target_t],
//   G[t,v] = scale dloss_t (exp(l[t,v] - lse_t) - [v = target_t]),  dh = G W,  dW = G^T h.
//
// Forward: one tcgen05 matrix product whose epilogue reduces each tile of logits, still in tensor memory, to (maximum, sum)
// pairs of 128 columns of a row; ce_join_k joins a row's pairs.  Backward: the vocabulary in pieces.  A piece's logits are
// computed again (2 T V C operations more, against T V values written, and read back twice), turned into G in bf16, and G
// enters the two products.  Kept in 16 bits as they are, the logits would move exp(l - lse) by percents; kept as differences to
// a row's maximum they would serve, but only in a call that has dloss before the loss, and in chunks of tokens that each add to
// all of dW: not built.  A piece holds all tokens, so its rows of dW are complete at once; dh adds up over the pieces in fp32.
//
// Rows without a target (padding, prompts) are left out before the products: ce_rows_k lists the others and copies their
// h side by side, so such rows cost nothing, and what they hold (NaN included) reaches neither loss nor gradients.
//
// What bounds it: the tensor cores, and behind them the power cap.  16384 x 2048 x 50257 on one B200: the forward's product
// takes 1.94 ms alone (1.74 PFLOP/s, 94 % of the tensor cycles) and 2.34 ms in a long run at 985 W (1.44 PFLOP/s), where
// each instruction of the other warps counts: the waits sleep in hardware and the usual-case epilogues run on packed pairs.
//
// Tiles: 256 x 256 a pair of CTAs (tcgen05 cta_group::2: each CTA stages 128 rows of A and 128 columns of B, and holds 128
// rows of the accumulator), K in steps of 64 (one 128-byte swizzle row of bf16) through a ring of TMA stages, accumulators
// double buffered in tensor memory so that the epilogue of one tile overlaps the products of the next.
#include "common.cuh"
#include "kernels.h"
#include "mma.cuh"
#include "tc.cuh"

namespace mhcl {

constexpr int kCeM = 256, kCeN = 256, kCeK = 64;       // tile of a pair
constexpr int kCeHalf = 128;                           // rows of A, columns of B and accumulator rows of one CTA
constexpr int kCeStages = 6;                           // at most: the modes that write bf16 tiles give one up for staging
constexpr int kCeABytes = kCeHalf * kCeK * 2, kCeStage = 2 * kCeABytes;
constexpr int kCeEpiWarps = 8;                         // two per tensor-memory quadrant: columns 0..127 and 128..255
constexpr int kCeThreads = 64 + 32 * kCeEpiWarps;      // warp 0: TMA, warp 1: MMA, the others: epilogue
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

enum CeMode { CE_STATS = 0, CE_GRAD = 1, CE_DH = 2, CE_DW = 3 };

struct CeArgs {
    const int* live;            // number of rows with a target
    const int* rows;            // [live] their token indices
    int64_t V;
    int C;
    int v0, vn;                 // the piece: rows v0 .. v0 + vn of W (vn a multiple of 256 except for the last piece)
    int m_tiles, n_tiles;       // at most; m_tiles of the row-wise modes is cut to `live` on the device
    int group;                  // row tiles whose column tiles follow each other (ce_tile)
    int a_box;                  // rows of A that a copy brings in (128; fewer for a handful of tokens)
    int splits;                 // CE_DH: ranges of the vocabulary that are added up apart
    float scale;
    // CE_STATS
    float2* part;               // [2 n_tiles][Tpad] (maximum, sum) in base 2 of 128 columns each
    float* tlogit;              // [Tpad] <h_t, W_target>, before the scale
    const int64_t* target;
    int Tpad;
    // CE_GRAD
    const float* lse;
    const float* dloss;
    const uint32_t* ref;        // [refs] bits of the largest finite |dloss| of each block of ce_rows_k
    int refs;
    __nv_bfloat16* G;           // [Tpad][pitch]
    int64_t pitch;
    // CE_DH
    float* dh_acc;              // [splits][Tpad][C] sums over the pieces so far
    __nv_bfloat16* dh;          // [T][C]
    int wide;                   // every run of 16 channels of dh begins on a 32-byte boundary
    int first, last;
    // CE_DW
    __nv_bfloat16* dW;          // [V][C]
    int* status;
};

// The modes whose epilogue writes bf16 tiles send them through shared memory, 64 columns of a warp's 32 rows at a time, so
// that a store covers whole 128-byte lines: a thread a row writes 32 bytes here and there, which held dW of few tokens (all
// epilogue) at 2.7 TB/s.
constexpr int kCeStagePitch = 144;                     // bytes a row: 128 and 16, so that neither side meets a bank twice
__host__ __device__ constexpr bool ce_staged(int mode) { return mode == CE_GRAD || mode == CE_DW; }
__host__ __device__ constexpr int ce_stages(int mode) { return ce_staged(mode) ? kCeStages - 1 : kCeStages; }
__host__ __device__ constexpr int ce_smem(int mode) {
    return ce_stages(mode) * kCeStage + (ce_staged(mode) ? kCeEpiWarps * 32 * kCeStagePitch : 0) + 256 + 1024;
}

struct CeCtl {
    uint64_t full[kCeStages], empty[kCeStages], acc_full[2], acc_empty[2];
    uint32_t tmem_base;
    int abort[3];
};

// Relative error 2^-22, two units in the last place of fp32: far below the rounding of G, and a sum of such terms in lse comes
// out no further off than any one of them.
__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// lse and loss of a row from the largest logit `top` in base 2, the sum s of 2^(l - top) and the target's product x: the loss
// is the difference log s - (l - top), formed before either is added to a logit in size, so that a target as likely as 1 does
// not lose its digits.  l - top comes unrounded (fused) as it does in s; at one common rounding error the two cancel.
__device__ __forceinline__ void lse_and_loss(float top, float s, float x, float k2, float& lse, float& loss) {
    const float b = log2f(s), d = (b - fmaf(x, k2, top == -INFINITY ? 0.f : -top)) * kLn2;
    lse = (top + b) * kLn2;
    loss = d < 0.f ? 0.f : d;                  // by the last bits of s
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ uint64_t ex2_pair(uint64_t x) {
    float a, b;
    unpack2f(x, a, b);
    return pack2f(ex2(a), ex2(b));
}

// The bracket of a row is kept as (p - [v = target]) dloss / ref in bf16, with ref the largest |dloss|; the products'
// epilogues multiply by scale ref in fp32.  Equal dloss (a mean over the tokens) then cost no rounding, where 1 / T rounded
// to bf16 would put one common error of up to 2^-9 on every gradient.
__device__ __forceinline__ float ce_ref(const uint32_t* ref, int refs) {          // by a whole warp
    uint32_t top = 0;
    for (int i = threadIdx.x & 31; i < refs; i += 32) top = max(top, ref[i]);
    top = __reduce_max_sync(0xffffffffu, top);
    return top > 0 ? __uint_as_float(top) : 1.f;
}

// 32 bytes to global memory in one instruction (a full sector a thread); p has to be 32-byte aligned, which callers' tensors
// need not be.
__device__ __forceinline__ void st32(void* p, const uint4& a, const uint4& b) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x),
                 "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
}

// ---- pairs of CTAs -----------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cta_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t leader_addr(uint32_t a) {            // the same shared-memory offset in CTA 0 of the pair
    uint32_t b;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(b) : "r"(a));
    return b;
}
__device__ __forceinline__ void pair_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Into this CTA's shared memory; the bytes count on a barrier of the pair's leader.
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void tc_mma_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, {%5, %5, %5, %5, %5, %5, %5, %5}, p;\n\t}"
                 ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(0u) : "memory");
}
// Arrives on the barrier at this offset in both CTAs when the MMAs issued so far are done.
__device__ __forceinline__ void tc_commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// A wait on a barrier that gives up after some four seconds, or when another role of the CTA has.  The hint lets the
// hardware keep the warp asleep meanwhile.
__device__ __forceinline__ bool ce_wait(uint32_t bar, uint32_t parity, volatile int* abort, int where, int index) {
    uint64_t t0 = 0, t;
    for (uint32_t i = 0;; ++i) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(bar), "r"(parity), "r"(1000000u) : "memory");
        if (ok) return true;
        if (abort[0]) return false;
        if ((i & 63) == 63) {
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
            if (t0 == 0) t0 = t;
            if (t - t0 > 4000000000ull) break;
        }
    }
    if (abort[0] == 0) { abort[1] = where; abort[2] = index; }
    abort[0] = 1;
    return false;
}
// Arrives on a barrier of the pair's leader.  It orders tensor-memory reads alone (after tcgen05.fence), so it asks for no
// release at cluster scope: that would wait for the warp's stores to global memory.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// Tile order: groups of row tiles, column tiles inside a group, so that the CTAs of a wave share operands in L2.
__device__ __forceinline__ void ce_tile(int i, int group, int mt, int nt, int& m, int& n) {
    const int per = group * nt, g = i / per, r = i - g * per, gm = min(group, mt - g * group);
    n = r / gm;
    m = g * group + (r - n * gm);
}

template <int MODE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kCeThreads, 1)
ce_gemm_k(const __grid_constant__ CUtensorMap tma, const __grid_constant__ CUtensorMap tmb, const CeArgs a) {
    constexpr bool A_MN = MODE == CE_DW, B_MN = MODE == CE_DH || MODE == CE_DW;
    constexpr int STAGES = ce_stages(MODE);
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    CeCtl* ctl = reinterpret_cast<CeCtl*>(smem + STAGES * kCeStage);
    static_assert(sizeof(CeCtl) <= 256, "control block");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = cta_rank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    volatile int* abort = ctl->abort;
    pdl_wait();
    pdl_launch();
    const int live = *a.live;
    const int mt = MODE == CE_DW ? a.m_tiles : (live + kCeM - 1) / kCeM, nt = a.n_tiles, per = mt * nt;
    const int splits = MODE == CE_DH ? a.splits : 1, tiles = per * splits;
    const int ksize = MODE == CE_DW ? live : MODE == CE_DH ? a.vn : a.C;
    const int ksteps = (ksize + kCeK - 1) / kCeK;

    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(smem_u32(&ctl->full[s]), 1); mbar_init(smem_u32(&ctl->empty[s]), 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(smem_u32(&ctl->acc_full[s]), 1); mbar_init(smem_u32(&ctl->acc_empty[s]), 2 * kCeEpiWarps); }
        abort[0] = abort[1] = abort[2] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {                                      // both CTAs of the pair take part
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    pair_sync();
    tc_fence_after();
    const uint32_t tmem = ctl->tmem_base;

    if (warp == 0) {
        if (lane == 0) {
            int it = 0;
            bool ok = true;
            for (int i = pair; i < tiles && ok; i += pairs) {
                const int split = MODE == CE_DH ? i / per : 0;
                int m, n;
                ce_tile(i - split * per, a.group, mt, nt, m, n);
                const int am = m * kCeM + (int)rank * kCeHalf, bn = n * kCeN + (int)rank * kCeHalf;
                // rows behind the list are not copied: what their half of the accumulator then holds is not read
                const int a_bytes = A_MN ? kCeABytes : a.a_box * 128;
                const bool a_second = A_MN || m * kCeM + kCeHalf < live;
                const int k1 = (int)((int64_t)ksteps * (split + 1) / splits);
                for (int k = (int)((int64_t)ksteps * split / splits); k < k1; ++k, ++it) {
                    const int s = it % STAGES;
                    ok = ce_wait(smem_u32(&ctl->empty[s]), ((it / STAGES) & 1) ^ 1, abort, 1, it);
                    if (!ok) break;
                    const uint32_t own = smem_u32(&ctl->full[s]), full = leader_addr(own);
                    const uint32_t sa = smem_u32(smem + s * kCeStage), sb = sa + kCeABytes;
                    if (rank == 0) mbar_expect_tx(own, 2 * kCeABytes + (a_second ? 2 : 1) * a_bytes);      // of both CTAs
                    if (A_MN) {
                        for (int b = 0; b < kCeHalf / 64; ++b) tma_load_2d_pair(sa + b * 8192, &tma, full, am + b * 64, k * kCeK);
                    } else if (rank == 0 || a_second) {
                        tma_load_2d_pair(sa, &tma, full, k * kCeK, am);
                    }
                    if (B_MN) {
                        for (int b = 0; b < kCeHalf / 64; ++b)
                            tma_load_2d_pair(sb + b * 8192, &tmb, full, bn + b * 64, (MODE == CE_DH ? a.v0 : 0) + k * kCeK);
                    } else {
                        tma_load_2d_pair(sb, &tmb, full, k * kCeK, a.v0 + bn);
                    }
                }
            }
            // the last products release their stages on both CTAs' barriers: neither CTA leaves before they have
            for (int d = 0; d < STAGES && ok; ++d, ++it)
                if (it >= STAGES) ok = ce_wait(smem_u32(&ctl->empty[it % STAGES]), ((it / STAGES) & 1) ^ 1, abort, 5, it);
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            constexpr uint32_t idesc = umma_idesc_mn(kCeM, kCeN, A_MN, B_MN);
            int it = 0, j = 0;
            bool ok = true;
            for (int i = pair; i < tiles && ok; i += pairs, ++j) {
                const int buf = j & 1;
                ok = ce_wait(smem_u32(&ctl->acc_empty[buf]), ((j >> 1) & 1) ^ 1, abort, 2, j);
                if (!ok) break;
                tc_fence_after();
                const int split = MODE == CE_DH ? i / per : 0;
                const int k0 = (int)((int64_t)ksteps * split / splits), k1 = (int)((int64_t)ksteps * (split + 1) / splits);
                for (int k = k0; k < k1; ++k, ++it) {
                    const int s = it % STAGES;
                    ok = ce_wait(smem_u32(&ctl->full[s]), (it / STAGES) & 1, abort, 3, it);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t sa = smem_u32(smem + s * kCeStage), sb = sa + kCeABytes;
#pragma unroll
                    for (int kk = 0; kk < kCeK / 16; ++kk) {
                        const uint64_t ad = A_MN ? smem_desc(sa + kk * 2048, 8192, 1024, 2) : smem_desc(sa + kk * 32, 16, 1024, 2);
                        const uint64_t bd = B_MN ? smem_desc(sb + kk * 2048, 8192, 1024, 2) : smem_desc(sb + kk * 32, 16, 1024, 2);
                        tc_mma_pair(tmem + buf * kCeN, ad, bd, idesc, (k > k0 || kk > 0) ? 1u : 0u);
                    }
                    tc_commit_pair(smem_u32(&ctl->empty[s]));
                }
                if (ok) tc_commit_pair(smem_u32(&ctl->acc_full[buf]));
            }
        }
    } else {
        const int quad = warp & 3, half = (warp - 2) >> 2, row = (int)rank * kCeHalf + quad * 32 + lane;
        const float ref = MODE == CE_STATS ? 1.f : ce_ref(a.ref, a.refs);
        const uint32_t staging = smem_u32(smem + STAGES * kCeStage + 256) + (warp - 2) * (32 * kCeStagePitch);
        bool ok = true;
        int j = 0;
        for (int i = pair; i < tiles && ok; i += pairs, ++j) {
            const int buf = j & 1;
            ok = ce_wait(smem_u32(&ctl->acc_full[buf]), (j >> 1) & 1, abort, 4, j);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            const int split = MODE == CE_DH ? i / per : 0;
            int m, n;
            ce_tile(i - split * per, a.group, mt, nt, m, n);
            const int r = m * kCeM + row;                       // row of the list, or of the piece (CE_DW)
            const int n0 = n * kCeN + half * kCeHalf;           // this warp's 128 columns
            const uint32_t acc = tmem + ((uint32_t)(quad * 32) << 16) + buf * kCeN + half * kCeHalf;
            // once the tile has been read from tensor memory, before what was read is written out
            auto hand_back = [&] {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(leader_addr(smem_u32(&ctl->acc_empty[buf])));
            };
            if (MODE == CE_STATS || MODE == CE_GRAD) {
                const bool in = r < live;
                const int t = in ? a.rows[r] : 0;
                const int tgt = in ? (int)(a.target[t] - a.v0) - n0 : -1;            // the target's column among them
                const int cols = (int)(a.V - a.v0) - n0;                             // of the vocabulary (the rest is padding)
                const float k2 = a.scale * kLog2e;
                if (MODE == CE_STATS) {
                    float mx = -INFINITY, sum = 0.f;
#pragma unroll 1
                    for (int c0 = 0; c0 < kCeHalf; c0 += 32) {
                        if (c0 >= cols) break;
                        float v[32];
                        tc_ld32(acc + c0, v);
                        if (__any_sync(0xffffffffu, tgt >= c0 && tgt < c0 + 32)) {
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (tgt == c0 + e) a.tlogit[r] = v[e];
                            __syncwarp();
                        }
                        if (k2 > 0.f && c0 + 32 <= cols) {             // the usual case, in as few instructions as it takes
                            float t0 = v[0], t1 = v[1];
#pragma unroll
                            for (int e = 2; e < 30; e += 4) { t0 = max3(t0, v[e], v[e + 1]); t1 = max3(t1, v[e + 2], v[e + 3]); }
                            const float top = fmaxf(mx, max3(fmaxf(t0, t1), v[30], v[31]) * k2), base = top == -INFINITY ? 0.f : top;
                            const uint64_t kk = pack2f(k2, k2), bb = pack2f(-base, -base);
                            uint64_t s0 = 0, s1 = 0;
#pragma unroll
                            for (int e = 0; e < 32; e += 4) {
                                s0 = add2(s0, ex2_pair(fma2(pack2f(v[e], v[e + 1]), kk, bb)));
                                s1 = add2(s1, ex2_pair(fma2(pack2f(v[e + 2], v[e + 3]), kk, bb)));
                            }
                            float x, y;
                            unpack2f(add2(s0, s1), x, y);
                            sum = sum * ex2(mx - base) + (x + y);
                            mx = top;
                            continue;
                        }
                        float top = mx;
#pragma unroll
                        for (int e = 0; e < 32; ++e) top = fmaxf(top, c0 + e < cols ? v[e] * k2 : -INFINITY);
                        const float base = top == -INFINITY ? 0.f : top;
                        sum *= ex2(mx - base);
#pragma unroll
                        for (int e = 0; e < 32; ++e) sum += c0 + e < cols ? ex2(fmaf(v[e], k2, -base)) : 0.f;
                        mx = top;
                    }
                    hand_back();
                    if (in) a.part[(int64_t)(2 * n + half) * a.Tpad + r] = make_float2(mx, sum);
                } else {
                    const float lse2 = in ? a.lse[t] * kLog2e : 0.f, f = in ? a.dloss[t] / ref : 0.f;
                    __nv_bfloat16* out = a.G + (int64_t)(r - lane) * a.pitch + n0;
#pragma unroll 1
                    for (int c0 = 0; c0 < kCeHalf; c0 += 64) {
#pragma unroll
                        for (int h = 0; h < 64; h += 32) {
                            float v[32];
                            tc_ld32(acc + c0 + h, v);
                            // the usual case: every row and column counts, and no row's target is among the columns
                            if (__all_sync(0xffffffffu, in && c0 + h + 32 <= cols && (tgt < c0 + h || tgt >= c0 + h + 32))) {
                                const uint64_t kk = pack2f(k2, k2), ll = pack2f(-lse2, -lse2), ff = pack2f(f, f);
#pragma unroll
                                for (int e = 0; e < 32; e += 8) {
                                    uint64_t p[4];
#pragma unroll
                                    for (int i2 = 0; i2 < 4; ++i2)
                                        p[i2] = mul2(ex2_pair(fma2(pack2f(v[e + 2 * i2], v[e + 2 * i2 + 1]), kk, ll)), ff);
                                    sts128(staging + lane * kCeStagePitch + (h + e) * 2, pack8x2(p));
                                }
                                continue;
                            }
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                v[e] = ex2(fmaf(v[e], k2, -lse2));
                                if (tgt == c0 + h + e) v[e] -= 1.f;
                                v[e] = (in && c0 + h + e < cols) ? v[e] * f : 0.f;
                            }
#pragma unroll
                            for (int e = 0; e < 32; e += 8) sts128(staging + lane * kCeStagePitch + (h + e) * 2, pack8(v + e));
                        }
                        if (c0 + 64 == kCeHalf) hand_back();
                        __syncwarp();
#pragma unroll
                        for (int i8 = 0; i8 < 8; ++i8) {
                            const int rr = i8 * 4 + (lane >> 3), cc = (lane & 7) * 8;
                            *reinterpret_cast<uint4*>(out + (int64_t)rr * a.pitch + c0 + cc) = lds128(staging + rr * kCeStagePitch + cc * 2);
                        }
                        __syncwarp();
                    }
                }
            } else if (MODE == CE_DW) {
                const float f = ksteps == 0 ? 0.f : a.scale * ref;          // no row has a target: nothing was accumulated
                __nv_bfloat16* out = a.dW + (int64_t)(a.v0 + r - lane) * a.C + n0;
                const int rows_in = a.vn - (r - lane);                      // of this warp's 32
#pragma unroll 1
                for (int c0 = 0; c0 < kCeHalf; c0 += 64) {
#pragma unroll
                    for (int h = 0; h < 64; h += 32) {
                        float v[32];
                        tc_ld32(acc + c0 + h, v);
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = ksteps == 0 ? 0.f : v[e] * f;
#pragma unroll
                        for (int e = 0; e < 32; e += 8) sts128(staging + lane * kCeStagePitch + (h + e) * 2, pack8(v + e));
                    }
                    if (c0 + 64 == kCeHalf) hand_back();
                    __syncwarp();
#pragma unroll
                    for (int i8 = 0; i8 < 8; ++i8) {
                        const int rr = i8 * 4 + (lane >> 3), cc = (lane & 7) * 8;
                        if (rr < rows_in && n0 + c0 + cc < a.C)
                            *reinterpret_cast<uint4*>(out + (int64_t)rr * a.C + c0 + cc) = lds128(staging + rr * kCeStagePitch + cc * 2);
                    }
                    __syncwarp();
                }
            } else {
                const bool in = r < live;
                const int64_t orow = in ? a.rows[r] : 0;
                const float f = a.scale * ref;
                // a short last piece may have fewer K steps than ranges
                const bool empty = (int64_t)ksteps * split / splits == (int64_t)ksteps * (split + 1) / splits;
#pragma unroll 1
                for (int c0 = 0; c0 < kCeHalf; c0 += 32) {
                    float v[32];
                    __syncwarp();                                       // rows behind the list skip the stores below
                    tc_ld32(acc + c0, v);
                    if (c0 + 32 == kCeHalf) hand_back();
                    const int c = n0 + c0;
                    if (!in) continue;
                    if (empty) {                                        // nothing was accumulated
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = 0.f;
                    }
                    if (splits > 1 || !a.first || !a.last) {
                        float* p = a.dh_acc + ((int64_t)split * a.Tpad + r) * a.C + c;
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            if (c + e >= a.C) continue;
                            if (!a.first) {
                                const float4 x = *(const float4*)(p + e), y = *(const float4*)(p + e + 4);
                                v[e] += x.x; v[e + 1] += x.y; v[e + 2] += x.z; v[e + 3] += x.w;
                                v[e + 4] += y.x; v[e + 5] += y.y; v[e + 6] += y.z; v[e + 7] += y.w;
                            }
                            if (splits > 1 || !a.last) st32(p + e, *(const uint4*)(v + e), *(const uint4*)(v + e + 4));
                        }
                        if (splits > 1 || !a.last) continue;
                    }
                    __nv_bfloat16* out = a.dh + orow * a.C + c;
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] *= f;
#pragma unroll
                    for (int e = 0; e < 32; e += 16) {
                        if (a.wide && c + e + 16 <= a.C) {              // whole sectors
                            st32(out + e, pack8(v + e), pack8(v + e + 8));
                        } else {
                            if (c + e < a.C) *reinterpret_cast<uint4*>(out + e) = pack8(v + e);
                            if (c + e + 8 < a.C) *reinterpret_cast<uint4*>(out + e + 8) = pack8(v + e + 8);
                        }
                    }
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (ctl->abort[0]) {
        for (int i = 0; i < 64; ++i) __nanosleep(2000);        // copies in flight land before the memory is given up
        if (tid == 0) report_wait(a.status, MHCLITE_OP_LINEAR_CE + 100 * MODE, ctl->abort[1], (int)blockIdx.x, ctl->abort[2]);
    }
    __syncthreads();
    pair_sync();                                               // the other CTA's products may read this one's memory until here
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// ---- rows with a target ----------------------------------------------------------------------------------------------
// Block b handles `per` tokens: counts the targets before them, numbers its own rows, copies their h side by side, and
// clears the outputs of the rows without a target (loss and lse, or dh).  In the backward it also leaves the largest finite
// |dloss| of its rows (as bits), and the last block pads the list's h with zero rows to the next multiple of 64, the K step
// of G^T h.
__global__ void __launch_bounds__(1024) ce_rows_k(int64_t T, int64_t V, int C, int64_t per, int Tpad, const int64_t* target,
                                                  const uint4* h, uint4* hl, int* rows,
                                                  int* live, float* loss, float* lse,
                                                  uint4* dh, const float* dloss, uint32_t* ref,
                                                  int* status) {
    __shared__ int wcnt[32], base_s;
    pdl_wait();
    pdl_launch();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nv = C >> 3;
    const int64_t t0 = blockIdx.x * per, t1 = t0 + per < T ? t0 + per : T;
    int mine = 0;
    for (int64_t t = tid; t < t0; t += 1024) { const int64_t y = target[t]; mine += y >= 0 && y < V; }
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (lane == 0) wcnt[warp] = mine;
    __syncthreads();
    if (warp == 0) {
        const int v = __reduce_add_sync(0xffffffffu, wcnt[lane]);
        if (lane == 0) base_s = v;
    }
    __syncthreads();
    int base = base_s;
    uint32_t top = 0;
    for (int64_t b = t0; b < t1; b += 32) {                     // every warp numbers all of the block's rows: no exchange
        const int64_t t = b + lane;
        const int64_t y = t < t1 ? target[t] : -1;
        const bool ok = y >= 0 && y < V;
        const uint32_t m = __ballot_sync(0xffffffffu, ok);
        if (warp == 0 && t < t1) {
            if (ok) {
                rows[base + __popc(m & ((1u << lane) - 1u))] = (int)t;
                if (dloss) {
                    const uint32_t d = __float_as_uint(dloss[t]) & 0x7FFFFFFFu;
                    if (d < 0x7F800000u && d > top) top = d;
                }
            } else {
                if (loss) { loss[t] = 0.f; lse[t] = 0.f; }
                if (y >= V) report_index(status, MHCLITE_OP_LINEAR_CE, t, y);
            }
        }
        for (int i = warp; i < 32 && b + i < t1; i += 32) {     // a warp a row
            if (m >> i & 1u) {
                uint4* to = hl + (int64_t)(base + __popc(m & ((1u << i) - 1u))) * nv;
                const uint4* from = h + (b + i) * nv;
                for (int v = lane; v < nv; v += 32) to[v] = ld_dep_stream(from + v);
            } else if (dh) {
                for (int v = lane; v < nv; v += 32) dh[(b + i) * nv + v] = make_uint4(0, 0, 0, 0);
            }
        }
        base += __popc(m);
    }
    if (dloss && warp == 0) {
        top = __reduce_max_sync(0xffffffffu, top);
        if (lane == 0) ref[blockIdx.x] = top;
    }
    if (t1 == T) {
        if (tid == 0) *live = base;
        const int pad = dloss ? min(Tpad, (base + kCeK - 1) / kCeK * kCeK) : base;
        for (int64_t i = tid; i < (int64_t)(pad - base) * nv; i += 1024) hl[(int64_t)base * nv + i] = make_uint4(0, 0, 0, 0);
    }
}

// Joins the (maximum, sum) pairs of a row: 32 rows a block, 32 ranges of tiles side by side.
__global__ void __launch_bounds__(1024) ce_join_k(const int* live, const int* rows, int n_parts, int Tpad,
                                                  const float2* part, const float* tlogit,
                                                  float k2, float* loss, float* lse) {
    __shared__ float2 red[32][32];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = blockIdx.x * 32 + lane, n = *live;
    if (blockIdx.x * 32 >= n) return;
    float m = -INFINITY, s = 0.f;
    if (r < n) {
#pragma unroll 8
        for (int k = warp; k < n_parts; k += 32) {
            const float2 p = part[(int64_t)k * Tpad + r];
            const float top = fmaxf(m, p.x), base = top == -INFINITY ? 0.f : top;
            s = s * ex2(m - base) + p.y * ex2(p.x - base);
            m = top;
        }
    }
    red[warp][lane] = make_float2(m, s);
    __syncthreads();
    if (warp != 0 || r >= n) return;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 32; ++w) top = fmaxf(top, red[w][lane].x);
    const float base = top == -INFINITY ? 0.f : top;
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 32; ++w) s += red[w][lane].y * ex2(red[w][lane].x - base);
    const int t = rows[r];
    float l, x;
    lse_and_loss(top, s, tlogit[r], k2, l, x);
    lse[t] = l;
    loss[t] = x;
}

// dh of the rows whose vocabulary was added up in several ranges: the ranges in order, eight channels a thread.
__global__ void __launch_bounds__(256) ce_dh_join_k(const int* live, const int* rows, int C, int Tpad, int splits,
                                                    const float* acc, const uint32_t* ref, int refs, float scale,
                                                    __nv_bfloat16* dh) {
    pdl_wait();
    const int nv = C >> 3, n = *live;
    const float f = scale * ce_ref(ref, refs);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)n * nv; i += (int64_t)gridDim.x * 256) {
        const int r = (int)(i / nv), c = (int)(i - (int64_t)r * nv) * 8;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int s = 0; s < splits; ++s) {
            const float4* p = (const float4*)(acc + ((int64_t)s * Tpad + r) * C + c);
            const float4 x = ld_dep(p), y = ld_dep(p + 1);
            v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
            v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= f;
        *reinterpret_cast<uint4*>(dh + (int64_t)rows[r] * C + c) = pack8(v);
    }
}

// ---- a handful of tokens ---------------------------------------------------------------------------------------------
// Forward for up to 32 tokens: the weights are read once and everything else is small, so the kernel is a stream over W.
// The 256-row tiles above leave it waiting: ten microseconds to start and drain, and whole rounds of tiles.  Here a CTA
// takes 16 (32, 64 for short rows) rows of W at a time (m16n8k16 with the rows of W as M and the tokens as N) and its 16
// warps share the channels.  A lane takes 16 bytes of a row and uses them as the operands of two products: the sum over k
// does not mind the order, as long as h is taken in the same one.  So each lane copies (cp.async) just the bytes that it
// will multiply, STAGES - 1 steps of 32 KB a CTA ahead, and nothing about W is exchanged or waited for between warps.  h
// stays in shared memory; the warps' partial logits meet there, and a thread keeps the running (maximum, sum) of one (row
// slot, token) over the CTA's rows.
// One token, 2048 channels, 50257 words: 43 us, against 62 with the tiles, 51 with one step ahead in registers and 61
// with bulk copies of a row piece each, of which the copy engine starts too few.
constexpr int kSmWarps = 16, kSmThreads = kSmWarps * 32, kSmTokens = 32;

// WK (4, 8 or 16) warps share the channels of a row, 64 of them each a step; WR = 16 / WK groups of 16 rows a unit; NB
// blocks of 8 tokens.
template <int NB, int STAGES>
__global__ void __launch_bounds__(kSmThreads, 1)
ce_small_k(int T, int64_t V, int C, int wk_log, const uint4* h, const uint4* W,
           const int64_t* target, float scale, float2* part, float* tlogit) {
    extern __shared__ __align__(16) unsigned char sm_raw[];
    pdl_wait();
    pdl_launch();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
    const int WK = 1 << wk_log, WR = kSmWarps >> wk_log, wk = warp & (WK - 1), wr = warp >> wk_log;
    const int KB = 64 * WK, blocks = (C + KB - 1) / KB, nv = C >> 3, rows = 16 * WR;
    const int hpitch = blocks * KB * 2 + 64;                               // 64 more: rows of h meet different banks
    const uint32_t ring = smem_u32(sm_raw) + tid * 16;                     // [STAGES][4][thread] of 16 bytes
    unsigned char* hs = sm_raw + STAGES * 4 * kSmThreads * 16;             // [8 NB][hpitch]
    float* red = reinterpret_cast<float*>(hs + 8 * NB * hpitch);           // [2][16 warps][NB][4][32]
    const int64_t units = (V + rows - 1) / rows;
    const int steps = (int)((units - blockIdx.x + gridDim.x - 1) / gridDim.x) * blocks;

    auto fetch = [&](int st) {                                             // 2 chunks of 32 channels of rows g and g + 8
        if (st < steps) {
            const int64_t unit = blockIdx.x + (int64_t)(st / blocks) * gridDim.x;
            int64_t r0 = unit * rows + wr * 16 + g, r1 = r0 + 8;           // rows behind the table are read twice, not joined
            if (r0 >= V) r0 = V - 1;
            if (r1 >= V) r1 = V - 1;
            const int v = ((st % blocks) * KB + wk * 64) / 8 + t4;
            const uint32_t to = ring + (st % STAGES) * (4 * kSmThreads * 16);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const bool in = v + c * 4 < nv;
                const int at = in ? v + c * 4 : 0;
                cp_async16(to + (2 * c) * (kSmThreads * 16), W + r0 * nv + at, in ? 16 : 0);
                cp_async16(to + (2 * c + 1) * (kSmThreads * 16), W + r1 * nv + at, in ? 16 : 0);
            }
        }
        cp_async_commit();
    };
#pragma unroll
    for (int st = 0; st < STAGES - 1; ++st) fetch(st);
    for (int i = tid; i < 8 * NB * (hpitch / 16); i += kSmThreads) {
        const int r = i / (hpitch / 16), v = i - r * (hpitch / 16);
        *reinterpret_cast<uint4*>(hs + r * hpitch + v * 16) = (r < T && v < nv) ? ld_dep(h + (int64_t)r * nv + v) : make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
    constexpr int kElems = 128 * NB;                                       // logits of a group: 16 rows x 8 NB tokens
    const int elems = kElems * WR;                                         // at most 512 NB: NB of them a thread
    float mx[NB], sum[NB], acc[NB][4];
#pragma unroll
    for (int i = 0; i < NB; ++i) { mx[i] = -INFINITY; sum[i] = 0.f; }
    for (int st = 0; st < steps; ++st) {
        const int b = st % blocks, u = st / blocks;
        if (b == 0)
#pragma unroll
            for (int i = 0; i < NB; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
        cp_async_wait<STAGES - 2>();
        fetch(st + STAGES - 1);                                            // into the slot of step st - 1
        const uint32_t wp = ring + (st % STAGES) * (4 * kSmThreads * 16);
        const uint32_t hp = smem_u32(hs) + g * hpitch + (b * KB + wk * 64) * 2 + t4 * 16;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const uint4 lo = lds128(wp + (2 * c) * (kSmThreads * 16)), hi = lds128(wp + (2 * c + 1) * (kSmThreads * 16));
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const uint4 x = lds128(hp + i * 8 * hpitch + c * 64);
                mma_bf16(acc[i], {lo.x, hi.x, lo.y, hi.y}, x.x, x.y);
                mma_bf16(acc[i], {lo.z, hi.z, lo.w, hi.w}, x.z, x.w);
            }
        }
        if (b + 1 < blocks) continue;
        float* mine = red + ((u & 1) * kSmWarps + warp) * kElems;
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) mine[(i * 4 + e) * 32 + lane] = acc[i][e];
        __syncthreads();
        const int64_t unit = blockIdx.x + (int64_t)u * gridDim.x;
        const float k2 = scale * kLog2e;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int x = tid + j * kSmThreads;
            if (x >= elems) break;
            const int er = x / kElems, y = x - er * kElems, l = y & 31, e = (y >> 5) & 3, i = y >> 7;
            const float* p = red + ((u & 1) * kSmWarps + er * WK) * kElems + y;
            float v = 0.f;
#pragma unroll 4
            for (int w = 0; w < WK; ++w) v += p[w * kElems];
            const int64_t row = unit * rows + er * 16 + (l >> 2) + (e >> 1) * 8;
            const int tok = i * 8 + (l & 3) * 2 + (e & 1);
            if (row >= V) continue;
            if (tok < T && row == target[tok]) tlogit[tok] = v;
            const float top = fmaxf(mx[j], v * k2), base = top == -INFINITY ? 0.f : top;
            sum[j] = sum[j] * ex2(mx[j] - base) + ex2(fmaf(v, k2, -base));
            mx[j] = top;
        }
    }
    __syncthreads();
    float2* fin = reinterpret_cast<float2*>(red);                      // [elems]
#pragma unroll
    for (int j = 0; j < NB; ++j)
        if (tid + j * kSmThreads < elems) fin[tid + j * kSmThreads] = make_float2(mx[j], sum[j]);
    __syncthreads();
    if (tid < 8 * NB && tid < T) {                                     // a token's 16 WR row slots
        const int i = tid >> 3, l3 = (tid & 7) >> 1, e0 = tid & 1;
        float m = -INFINITY, t = 0.f;
        for (int k = 0; k < rows; ++k) {
            const int er = k >> 4, l = (k & 7) * 4 + l3, e = e0 + ((k >> 3) & 1) * 2;
            const float2 p = fin[er * kElems + (i * 4 + e) * 32 + l];
            const float top = fmaxf(m, p.x), base = top == -INFINITY ? 0.f : top;
            t = t * ex2(m - base) + p.y * ex2(p.x - base);
            m = top;
        }
        part[blockIdx.x * kSmTokens + tid] = make_float2(m, t);
    }
}
// Joins the CTAs' pairs: a lane a token, the warps' shares of the CTAs side by side.
__global__ void __launch_bounds__(512) ce_small_join_k(int T, int64_t V, int parts, const float2* part, const float* tlogit,
                                                       const int64_t* target, float k2, float* loss, float* lse,
                                                       int* status) {
    __shared__ float2 red[16][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float m = -INFINITY, s = 0.f;
    pdl_wait();                                                // launched beside ce_small_k: its results from here on
    if (lane < T) {
#pragma unroll 10
        for (int k = warp; k < parts; k += 16) {
            const float2 p = part[k * kSmTokens + lane];
            const float top = fmaxf(m, p.x), base = top == -INFINITY ? 0.f : top;
            s = s * ex2(m - base) + p.y * ex2(p.x - base);
            m = top;
        }
    }
    red[warp][lane] = make_float2(m, s);
    __syncthreads();
    if (warp != 0 || lane >= T) return;
    const int64_t y = target[lane];
    float l = 0.f, x = 0.f;
    if (y >= 0 && y < V) {
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 16; ++w) top = fmaxf(top, red[w][lane].x);
        const float base = top == -INFINITY ? 0.f : top;
        s = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w) s += red[w][lane].y * ex2(red[w][lane].x - base);
        lse_and_loss(top, s, tlogit[lane], k2, l, x);
    } else if (y >= V) {
        report_index(status, MHCLITE_OP_LINEAR_CE, lane, y);
    }
    lse[lane] = l;
    loss[lane] = x;
}

// ---- host side -------------------------------------------------------------------------------------------------------
constexpr int kCeRowBlocks = 296;
struct CePlan {
    int Tpad, n_tiles, a_box;
    int pieces; int64_t piece;             // vocabulary rows a piece, a multiple of 256
    int splits;                            // ranges of a piece's vocabulary in the product dh = G W
    int64_t rows_per; int row_blocks;      // tokens a block of ce_rows_k, and its blocks
    int *live, *rows;
    uint32_t* ref;
    __nv_bfloat16* hl;
    float2* part; float* tlogit;
    __nv_bfloat16* G; float* dh_acc;
    size_t bytes;
};
// Rounds that `tiles` tiles take on the pairs of CTAs (a B200's 74: the plan gives the scratch's size, which callers ask for
// without a context, so it does not look at the device).
constexpr int kCePairs = 74;
static int64_t ce_rounds(int64_t tiles) { return (tiles + kCePairs - 1) / kCePairs; }

// Pieces of the vocabulary in the backward.  G of a piece takes at most about 384 MB; below that, the width whose products
// leave the fewest pairs of CTAs idle in their last rounds, in steps of K over all pieces (16384 tokens, 2048 channels,
// 50257 words: five pieces of 45 tiles, 3 % more rounds than tiles would fill).
static void ce_pieces(CePlan& p, int64_t V, int C) {
    const int64_t mt = p.Tpad / kCeM, ct = (C + kCeN - 1) / kCeN, nt = p.n_tiles;
    int64_t most = ((int64_t)192 << 20) / p.Tpad / kCeN;
    if (most < 1) most = 1;
    if (most > nt) most = nt;
    int64_t best = most, best_cost = INT64_MAX;
    for (int64_t w = most; w > 0 && w * 2 >= most; w -= 1 + most / 128) {
        int64_t cost = 0;
        for (int64_t v = 0; v < nt; v += w) {
            const int64_t n = nt - v < w ? nt - v : w;
            cost += ce_rounds(mt * n) * ((C + 63) / 64) + ce_rounds(n * ct) * (p.Tpad / 64) + ce_rounds(mt * ct) * n * 4 + 48;
        }
        if (cost < best_cost) { best_cost = cost; best = w; }
    }
    p.piece = best * kCeN;
    p.pieces = (int)((V + p.piece - 1) / p.piece);
    // dh has few tiles where tokens are few: its K is then split.  A split costs a pass over its partial sums, about a
    // step of K for every 40 KB an SM pair moves.
    p.splits = 1;
    best_cost = INT64_MAX;
    const int64_t ks = p.piece / kCeK;
    for (int s = 1; s <= 64 && s * 4 <= ks; ++s) {
        const int64_t cost = ce_rounds(mt * ct * s) * ((ks + s - 1) / s + 4) + (s > 1 ? 8 + s * (mt * ct * 2 * kCeM * kCeN * 4 / kCePairs / 40000) : 0);
        if (cost < best_cost) { best_cost = cost; p.splits = s; }
    }
}
static CePlan plan_ce(int64_t T, int64_t V, int C, int grad, void* base) {
    CePlan p;
    char* b = (char*)base;
    size_t off = 0;
    auto take = [&](size_t n) { char* at = b + off; off += (n + 255) & ~(size_t)255; return at; };
    p.Tpad = (int)round_up64(T > 0 ? T : 1, kCeM);
    p.n_tiles = (int)((V + kCeN - 1) / kCeN);
    p.a_box = T < kCeHalf ? (int)round_up64(T > 0 ? T : 1, 8) : kCeHalf;
    p.live = (int*)take(256);
    p.ref = (uint32_t*)take(kCeRowBlocks * 4);
    p.rows_per = 32;
    while ((T + p.rows_per - 1) / p.rows_per > kCeRowBlocks) p.rows_per += 32;
    p.row_blocks = (int)((T + p.rows_per - 1) / p.rows_per);
    p.rows = (int*)take((size_t)p.Tpad * 4);
    p.hl = (__nv_bfloat16*)take((size_t)p.Tpad * C * 2);
    p.part = nullptr; p.tlogit = nullptr; p.G = nullptr; p.dh_acc = nullptr;
    p.pieces = 1; p.piece = 0; p.splits = 1;
    if (!grad) {
        p.part = (float2*)take((size_t)p.n_tiles * 2 * p.Tpad * 8);
        p.tlogit = (float*)take((size_t)p.Tpad * 4);
    } else {
        ce_pieces(p, V, C);
        p.G = (__nv_bfloat16*)take((size_t)p.Tpad * p.piece * 2);
        p.dh_acc = (float*)take(p.pieces > 1 || p.splits > 1 ? (size_t)p.splits * p.Tpad * C * 4 : 0);
    }
    p.bytes = off;
    return p;
}
// (the few-token forward keeps a pair and a logit for each of 32 tokens and up to 256 SMs)
size_t ce_scratch_bytes(int64_t T, int64_t V, int C, int grad) {
    const size_t n = plan_ce(T, V, C, grad, nullptr).bytes, few = (256 + 1) * kSmTokens * 8;
    return n > few ? n : few;
}

static void launch_ce_rows(const mhclite_ctx* c, const CePlan& p, int64_t T, int64_t V, const int64_t* target, const void* h,
                           float* loss, float* lse, void* dh, const float* dloss, cudaStream_t s) {
    c->launches += 1;
    launch_after(ce_rows_k, dim3(p.row_blocks), dim3(1024), 0, s, T, V, c->C, p.rows_per, p.Tpad, target, (const uint4*)h, (uint4*)p.hl, p.rows,
                 p.live, loss, lse, (uint4*)dh, dloss, p.ref, c->op_status);
}

template <int MODE>
static void launch_ce_gemm(const mhclite_ctx* c, const CUtensorMap& ma, const CUtensorMap& mb, CeArgs a, cudaStream_t s) {
    constexpr int smem = ce_smem(MODE);
    const int64_t tiles = (int64_t)a.m_tiles * a.n_tiles * (MODE == CE_DH ? a.splits : 1);
    static SmemOnce once;
    smem_limit(once, ce_gemm_k<MODE>, c->device, smem);
    c->launches += 1;
    // Few column tiles: a group takes them all in one wave, and its rows of A are read from HBM once.  Many: the group's rows
    // of A (32 tiles of 2048 channels: 34 MB) stay in L2 while B streams past.  Loss and gradients of 16384 x 2048 x 50257 in a
    // long run: 10.05 ms, with groups of 16 10.14, of 8 10.31, of 64 10.43.  At 512 channels all take 3.07 ms; at 4096, where
    // 32 tiles are 67 MB (32000 words), groups of 16 would take 13.0 ms and these take 13.9.
    a.group = a.n_tiles <= 9 ? kCePairs / a.n_tiles : 32;
    const int64_t pairs = tiles < c->sm_count / 2 ? tiles : c->sm_count / 2;
    launch_after(ce_gemm_k<MODE>, dim3((unsigned)(2 * pairs)), dim3(kCeThreads), smem, s, ma, mb, a);
}

// Tensor maps: a K-major operand is copied in boxes of 64 k x `rows` rows, an MN-major one in boxes of 64 x 64 k.
static bool map_k(CUtensorMap* m, const void* p, int64_t rows, int64_t k, int64_t pitch, int box_rows) {
    return make_tensor_map_2d(m, p, (uint64_t)k, (uint64_t)rows, (uint64_t)pitch, kCeK, (uint32_t)box_rows, 128);
}
static bool map_mn(CUtensorMap* m, const void* p, int64_t k, int64_t mn, int64_t pitch) {
    return make_tensor_map_2d(m, p, (uint64_t)mn, (uint64_t)k, (uint64_t)pitch, 64, kCeK, 128);
}

// Shape of ce_small_k; stages = 0 where it does not apply: more than 32 tokens, or rows of h so long that fewer than three
// stages of W fit beside them.
struct SmallPlan { int wk_log, nb, stages, smem; };
static SmallPlan plan_small(int64_t T, int C) {
    SmallPlan p = {2, T <= 8 ? 1 : T <= 16 ? 2 : 4, 0, 0};
    if (T > kSmTokens) return p;
    while ((64 << p.wk_log) < C && (1 << p.wk_log) < kSmWarps) ++p.wk_log;
    const int64_t fixed = 8 * p.nb * (round_up64(C, 64 << p.wk_log) * 2 + 64) + 2 * kSmWarps * 128 * p.nb * 4, stage = 4 * kSmThreads * 16;
    const int64_t fit = (226 * 1024 - fixed) / stage;
    p.stages = fixed > 226 * 1024 || fit < 3 ? 0 : fit >= 5 ? 5 : 3;
    p.smem = (int)(fixed + p.stages * stage);
    return p;
}

bool launch_linear_ce_fwd(const mhclite_ctx* c, int64_t T, int64_t V, const void* h, const void* W, const int64_t* target, float scale,
                          float* loss, float* lse, void* scratch, cudaStream_t s) {
    const SmallPlan q = plan_small(T, c->C);
    if (q.stages) {
        float2* part = (float2*)scratch;                       // [CTAs][32], then the targets' logits
        float* tlogit = (float*)(part + (size_t)c->sm_count * kSmTokens);
        const int64_t units = (V + (256 >> q.wk_log) - 1) / (256 >> q.wk_log);
        const int grid = (int)(units < c->sm_count ? units : c->sm_count);
        auto k = q.stages == 5 ? (q.nb == 1 ? ce_small_k<1, 5> : q.nb == 2 ? ce_small_k<2, 5> : ce_small_k<4, 5>)
                               : (q.nb == 1 ? ce_small_k<1, 3> : q.nb == 2 ? ce_small_k<2, 3> : ce_small_k<4, 3>);
        static SmemOnce once[3][2];
        smem_limit(once[q.nb >> 1][q.stages == 5], k, c->device, 226 * 1024);
        c->launches += 2;
        launch_after(k, dim3(grid), dim3(kSmThreads), q.smem, s, (int)T, V, c->C, q.wk_log, (const uint4*)h, (const uint4*)W, target, scale, part, tlogit);
        launch_after(ce_small_join_k, dim3(1), dim3(512), 0, s, (int)T, V, grid, part, tlogit, target, scale * kLog2e, loss, lse, c->op_status);
        return true;
    }
    const CePlan p = plan_ce(T, V, c->C, 0, scratch);
    CUtensorMap mh, mw;
    if (!map_k(&mh, p.hl, p.Tpad, c->C, c->C, p.a_box) || !map_k(&mw, W, V, c->C, c->C, kCeHalf)) return false;
    launch_ce_rows(c, p, T, V, target, h, loss, lse, nullptr, nullptr, s);
    CeArgs a = {};
    a.live = p.live; a.rows = p.rows; a.V = V; a.C = c->C; a.v0 = 0; a.vn = (int)V;
    a.m_tiles = p.Tpad / kCeM; a.n_tiles = p.n_tiles; a.scale = scale;
    a.a_box = p.a_box; a.part = p.part; a.tlogit = p.tlogit; a.target = target; a.Tpad = p.Tpad; a.status = c->op_status;
    launch_ce_gemm<CE_STATS>(c, mh, mw, a, s);
    c->launches += 1;
    launch_after(ce_join_k, dim3((unsigned)((T + 31) / 32)), dim3(1024), 0, s, p.live, p.rows, 2 * p.n_tiles, p.Tpad, p.part, p.tlogit, scale * kLog2e, loss, lse);
    return true;
}

bool launch_linear_ce_bwd(const mhclite_ctx* c, int64_t T, int64_t V, const void* h, const void* W, const int64_t* target, float scale,
                          const float* lse, const float* dloss, void* dh, void* dW, void* scratch, cudaStream_t s) {
    const CePlan p = plan_ce(T, V, c->C, 1, scratch);
    const int C = c->C;
    CUtensorMap mh, mw, mg, mwn, mgt, mhn;
    if (!map_k(&mh, p.hl, p.Tpad, C, C, p.a_box) || !map_k(&mw, W, V, C, C, kCeHalf) || !map_k(&mg, p.G, p.Tpad, p.piece, p.piece, p.a_box) ||
        !map_mn(&mwn, W, V, C, C) || !map_mn(&mgt, p.G, p.Tpad, p.piece, p.piece) || !map_mn(&mhn, p.hl, p.Tpad, C, C))
        return false;
    launch_ce_rows(c, p, T, V, target, h, nullptr, nullptr, dh, dloss, s);
    CeArgs a = {};
    a.live = p.live; a.rows = p.rows; a.V = V; a.C = C; a.scale = scale; a.target = target; a.Tpad = p.Tpad;
    a.lse = lse; a.dloss = dloss; a.G = p.G; a.pitch = p.piece; a.dh_acc = p.dh_acc; a.dh = (__nv_bfloat16*)dh;
    a.wide = C % 16 == 0 && ((uintptr_t)dh & 31) == 0;
    a.dW = (__nv_bfloat16*)dW; a.ref = p.ref; a.refs = p.row_blocks; a.a_box = p.a_box; a.splits = p.splits; a.status = c->op_status;
    for (int i = 0; i < p.pieces; ++i) {
        a.v0 = (int)(i * p.piece);
        a.vn = (int)(V - a.v0 < p.piece ? V - a.v0 : p.piece);
        a.first = i == 0; a.last = i + 1 == p.pieces;
        a.m_tiles = p.Tpad / kCeM; a.n_tiles = (a.vn + kCeN - 1) / kCeN;
        launch_ce_gemm<CE_GRAD>(c, mh, mw, a, s);
        a.m_tiles = (a.vn + kCeM - 1) / kCeM; a.n_tiles = (C + kCeN - 1) / kCeN;
        launch_ce_gemm<CE_DW>(c, mgt, mhn, a, s);
        a.m_tiles = p.Tpad / kCeM;
        launch_ce_gemm<CE_DH>(c, mg, mwn, a, s);
    }
    if (p.splits > 1) {
        const int64_t blocks = (T * (C / 8) + 255) / 256, most = (int64_t)c->sm_count * 16;
        c->launches += 1;
        launch_after(ce_dh_join_k, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, s, p.live, p.rows, C, p.Tpad, p.splits,
                     p.dh_acc, p.ref, p.row_blocks, scale, (__nv_bfloat16*)dh);
    }
    return true;
}

}  // namespace mhcl
