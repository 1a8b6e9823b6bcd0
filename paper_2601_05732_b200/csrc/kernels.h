// Launchers of the library's kernels (host side). Each enqueues on the given stream and returns.
#pragma once
#include "common.cuh"

namespace mhcl {

// stream_kernels.cu
void launch_premix_fwd(const mhclite_ctx* c, int64_t T, const void* x, const float* H_pre, void* u, cudaStream_t s);
void launch_postres_fwd(const mhclite_ctx* c, int64_t T, const void* x, const void* y, const float* H_res,
                        const float* H_post, void* x_next, cudaStream_t s);
void launch_postres_bwd(const mhclite_ctx* c, int64_t T, const void* x, const void* y, const float* H_res,
                        const float* H_post, const void* g, void* dy, float* dH_res, float* dH_post, void* dx,
                        int acc, cudaStream_t s);
void launch_premix_bwd(const mhclite_ctx* c, int64_t T, const void* x, const float* H_pre, const void* du,
                       float* dH_pre, void* dx, int acc, cudaStream_t s);
void launch_tail_mix(const mhclite_ctx* c, int64_t T, const void* x, const void* g, const void* du, const float* H_res,
                     const float* H_pre, float* dH_pre, void* dx, cudaStream_t s);
void launch_ds_gap(const mhclite_ctx* c, int64_t T, const float* H_res, float* l1, float* cdev, cudaStream_t s);
void launch_ds_gap_stats(const mhclite_ctx* c, int64_t T, const float* H_res, float* stats, cudaStream_t s);
void launch_log_inv_nu_hist(const mhclite_ctx* c, int64_t T, const float* X, int bins, float lo, float hi,
                            unsigned long long* hist, cudaStream_t s);
void launch_depth_product(const mhclite_ctx* c, int64_t T, const float* H_res, float* P, int first, cudaStream_t s);
void launch_relative_range(const mhclite_ctx* c, int64_t T, const float* X, float* nu, cudaStream_t s);

// proj_kernels.cu : RMSNorm statistics + the skinny projection and its gradient
// proj_mma.cu: W' = diag(gain) W packed as bf16 hi/lo MMA fragments; qpart[s][t][c] = partial x W' of K slice s,
// ssq[s][t] = partial sum of squares (the activation kernels add the slices and apply rstd)
void launch_pack_w(const mhclite_ctx* c, const ProjPlan& p, int N, const float* W, const float* gain, void* Wp,
                   cudaStream_t s);
void launch_proj_fwd_mma(const mhclite_ctx* c, int64_t T, const ProjPlan& p, const void* x, const void* Wp,
                         float* qpart, float* ssq, cudaStream_t s);
// dx[t,m] (+)= sum_c e[t,c] gain[m] W[m,c] - x[t,m] kappa[t]   (e = rstd*alpha*dz)
void launch_proj_bwd_dx(const mhclite_ctx* c, int64_t T, int N, int Npad, const void* x, const float* W,
                        const float* gain, const float* e, const float* kappa, void* dx, int acc, cudaStream_t s);
// G[m,c] = sum_t x[t,m] e[t,c];  dW (+)= gain (.) G ;  dgain[m] (+)= sum_c W[m,c] G[m,c]
void launch_proj_bwd_dw(const mhclite_ctx* c, int64_t T, int N, int Npad, const void* x, const float* W,
                        const float* gain, const float* e, float* G, float* dW, float* dgain, int acc,
                        cudaStream_t s);

// proj_tc.cu : the same projection on tcgen05 / TMA / tensor memory (up to 256 columns); tail_tc.cu : the
// backward of wide projections (n = 5) on tcgen05
bool tensor_maps_available();
bool launch_tail_g_tc(const mhclite_ctx* c, int64_t T, const TailPlan& p, const void* x, const void* ehi,
                      const void* elo, float* Gpart, int* status, cudaStream_t s);
size_t tail_wb_bytes(int n, int C, int Kp);
bool launch_tail_dx_tc(const mhclite_ctx* c, int64_t T, int N, const TailPlan& p, const void* x, const void* g,
                       const void* du, const void* ehi, const float* kappa, const float* H_res, const float* H_pre,
                       const float* W, const float* gain, void* Wb, void* dx, int acc_dx, int* status, cudaStream_t s);
// tail_ftc.cu : narrow projections, dx and the G partials [f_splits][nC][Kp] in one tcgen05 kernel
void plan_tail_ftc(int n, int C, int64_t T, int sm_count, TailPlan* p);
bool launch_tail_ftc_prep(const mhclite_ctx* c, int N, const TailPlan& p, const float* W, const float* gain, void* Wf,
                          float* zero_db, float* zero_dalpha, cudaStream_t s);
bool launch_tail_ftc(const mhclite_ctx* c, int64_t T, int N, const TailPlan& p, const void* x, const void* g,
                     const void* du, const void* ehi, const void* elo, const float* kappa, const float* H_res,
                     const float* H_pre, const float* W, const float* gain, void* Wf, bool wf_packed, void* dx,
                     int acc_dx, float* Gpart, int* status, cudaStream_t s);
// db[N], dalpha[3] (+)= the nparts per-block partials alone (for a backward that does not end in launch_tail_finish)
void launch_dpart_sum(const mhclite_ctx* c, int N, const float* dpart, int nparts, float* db, float* dalpha, int acc_params,
                      cudaStream_t s);
// dpart (null: none): nparts per-block partials of db / dalpha, added up into db[N], dalpha[3] by the same launch
void launch_tail_finish(const mhclite_ctx* c, int N, int Kp, int splits, const float* W, const float* gain,
                        const float* Gpart, float* dW, float* dgain, int acc_params, cudaStream_t s,
                        const float* dpart = nullptr, int nparts = 0, float* db = nullptr, float* dalpha = nullptr);
bool proj_tc_supported(int n, int C, int N);
int proj_tc_nq(int N);
void launch_pack_wt(const mhclite_ctx* c, const ProjPlan& p, int N, const float* W, const float* gain, void* Wt,
                    cudaStream_t s);
bool launch_proj_fwd_tc(const mhclite_ctx* c, int64_t T, int N, const ProjPlan& p, const void* x, const void* Wt,
                        float* qpart, float* ssq, int* status, cudaStream_t s);

// postres_proj.cu : the merge of one layer fused with the RMSNorm statistics and projection of the next
bool postres_proj_supported(int n, int C, int N);
bool launch_postres_proj(const mhclite_ctx* c, int64_t T, int N, const ProjPlan& pp, const void* x, const void* y,
                         const float* H_res, const float* H_post, void* x_next, const void* Wt, float* qpart, float* ssq,
                         int* status, cudaStream_t s);

// act_kernels.cu : per-token activations, H_res assembly and their gradients
void launch_lite_act_fwd(const mhclite_ctx* c, int64_t T, const ProjPlan& pp, const float* qpart, const float* ssq,
                         float eps, const float* b, const float* alpha, float* H_res, float* H_pre, float* H_post,
                         float* a_saved, float* p_saved, float* rstd, cudaStream_t s);
void launch_lite_act_bwd(const mhclite_ctx* c, int64_t T, int Npad, const float* a, const float* p, const float* rstd,
                         const float* alpha, const float* H_pre, const float* H_post, const float* dH_res,
                         const float* dH_pre, const float* dH_post, float* e, void* ehi, void* elo, int Kp,
                         float* kappa, float* db, float* dalpha, cudaStream_t s);
// mappings + pre-mix in one kernel; dH_pre + activation backward in one kernel (the fused call sequences)
void launch_lite_act_premix(const mhclite_ctx* c, int64_t T, const ProjPlan& pp, const float* qpart, const float* ssq,
                            float eps, const float* b, const float* alpha, float* H_res, float* H_pre, float* H_post,
                            float* a_saved, float* p_saved, float* rstd, const void* x, void* u, cudaStream_t s,
                            float* u_rstd = nullptr, float eps_u = 0.f);
// u_rstd[t] = (mean_c u[t,c]^2 + eps)^-1/2 of a stored u [T][C] (bf16), one warp per token
void launch_row_rstd(const mhclite_ctx* c, int64_t T, const void* u, float eps, float* u_rstd, cudaStream_t s);
int launch_lite_tailpre(const mhclite_ctx* c, int64_t T, const void* x, const void* du, const float* a, const float* p,
                        const float* rstd, const float* alpha, const float* H_pre, const float* H_post,
                        const float* dH_res, const float* dH_post, float* dH_pre_ws, float* e, int Npad, void* ehi,
                        void* elo, int Kp, float* kappa, float* db, float* dalpha, cudaStream_t s);
// the SK path's counterparts of the two fused kernels above
void launch_sk_act_premix(const mhclite_ctx* c, int64_t T, int iters, const ProjPlan& pp, const float* qpart,
                          const float* ssq, float eps, const float* b, const float* alpha, float* H_res, float* H_pre,
                          float* H_post, float* p_saved, float* rstd, const void* x, void* u, cudaStream_t s);
int launch_sk_tailpre(const mhclite_ctx* c, int64_t T, int iters, const void* x, const void* du, const float* p,
                      const float* b, const float* rstd, const float* alpha, const float* H_pre, const float* H_post,
                      const float* dH_res, const float* dH_post, float* e, int Npad, void* ehi, void* elo, int Kp,
                      float* kappa, float* db, float* dalpha, cudaStream_t s);
void launch_sk_act_fwd(const mhclite_ctx* c, int64_t T, int iters, const ProjPlan& pp, const float* qpart,
                       const float* ssq, float eps, const float* b, const float* alpha, float* H_res, float* H_pre,
                       float* H_post, float* p_saved, float* rstd, cudaStream_t s);
void launch_sk_act_bwd(const mhclite_ctx* c, int64_t T, int Npad, int iters, const float* p, const float* b,
                       const float* rstd, const float* alpha, const float* H_pre, const float* H_post,
                       const float* dH_res, const float* dH_pre, const float* dH_post, float* e, void* ehi, void* elo,
                       int Kp, float* kappa, float* db, float* dalpha, cudaStream_t s);

// tail_mma.cu : tensor-core projection / RMSNorm backward, optionally fused with the rest of dx (g != NULL)
void launch_tail_mma(const mhclite_ctx* c, int64_t T, int N, const TailPlan& p, const void* x, const void* g,
                     const void* du, const void* ehi, const void* elo, const float* kappa, const float* H_res,
                     const float* H_pre, const float* W, const float* gain, void* dx, int acc_dx, float* Gpart,
                     float* dW, float* dgain, int acc_params, cudaStream_t s);

// Launches a kernel that may begin while the one before it on the stream still runs (programmatic dependent launch): it
// waits for that kernel's results itself (pdl_wait), before its first access to global memory.  (embed_zero_k alone writes
// before it waits: what it clears is free from the moment its predecessor has begun, see there.)
template <typename... P, typename... A>
inline cudaError_t launch_after(void (*k)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k, static_cast<P>(args)...);
}
// The same for a grid of clusters of `size` blocks.
template <typename... P, typename... A>
inline cudaError_t launch_cluster_after(void (*k)(P...), dim3 grid, dim3 block, int size, size_t smem, cudaStream_t s, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)size; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k, static_cast<P>(args)...);
}
#ifdef __CUDACC__
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Loads of such a kernel.  Its life begins while its predecessor may still write what it is going to read, so the read-only
// path, whose promise is that nobody writes the data while the kernel lives, is not open to it: neither __ldg, nor ld.global.nc,
// nor a const __restrict__ pointer, behind which the compiler may choose either and lift it over pdl_wait.  Its pointers are
// plain ones and its loads ordinary ones, which pdl_wait holds back.
template <typename T>
__device__ __forceinline__ T ld_dep(const T* p) { return *p; }
// what other blocks of the same kernel wrote: from L2
__device__ __forceinline__ uint2 ld_dep_l2(const uint2* p) {
    uint2 r;
    asm volatile("ld.global.cg.v2.b32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(p) : "memory");
    return r;
}
// activations, touched once
__device__ __forceinline__ uint4 ld_dep_stream(const void* p) {
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}
#endif

// Raises a kernel's limit of dynamic shared memory once a device (the call costs more than the launch's other set-up).
struct SmemOnce { unsigned long long done = 0; };
template <typename K>
inline void smem_limit(SmemOnce& once, K k, int device, int bytes) {
    const unsigned long long bit = 1ull << (device & 63);
    if (__atomic_load_n(&once.done, __ATOMIC_RELAXED) & bit) return;
    cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    __atomic_fetch_or(&once.done, bit, __ATOMIC_RELAXED);
}

// block_kernels.cu : the norms around a sublayer, with gate, scale and dropout, and dropout alone
constexpr int kMaxRowC = 16384;               // channels of a row that a team of warps holds in registers
int block_parts(int64_t T, int C, int sm_count, bool gate);
void launch_block_fwd(const mhclite_ctx* c, int64_t T, const void* x, const void* gate, const float* w, const float* scale,
                      float eps, float p_drop, const uint64_t* rng, void* out, float* rstd, cudaStream_t s);
// dw_part [block_parts][C], ds_part [block_parts] (used when dscale is given)
void launch_block_bwd(const mhclite_ctx* c, int64_t T, const void* x, const void* gate, const float* w, const float* scale,
                      const float* rstd, float p_drop, const uint64_t* rng, const void* dy, void* dx, void* dgate, float* dw,
                      float* dscale, int accumulate, float* dw_part, double* ds_part, cudaStream_t s);
void launch_dropout(const mhclite_ctx* c, int64_t count, const void* x, float p, const uint64_t* rng, void* y, cudaStream_t s);

// embed_kernels.cu : token rows into the residual streams, and the table's gradient
void launch_embed_fwd(const mhclite_ctx* c, int64_t T, int64_t V, const int64_t* ids, const void* E, int table_f32, float scale,
                      void* x0, cudaStream_t s);
size_t embed_scratch_bytes(int64_t T, int C);
cudaError_t launch_embed_bwd(const mhclite_ctx* c, int64_t T, int64_t V, const int64_t* ids, const void* g, float scale, float* dE,
                             int accumulate, void* scratch, cudaStream_t s);

// ce_kernels.cu : cross entropy of h W^T without the logits in memory; false when the tensor maps could not be built
size_t ce_scratch_bytes(int64_t T, int64_t V, int C, int grad);
bool launch_linear_ce_fwd(const mhclite_ctx* c, int64_t T, int64_t V, const void* h, const void* W, const int64_t* target, float scale,
                          float* loss, float* lse, void* scratch, cudaStream_t s);
bool launch_linear_ce_bwd(const mhclite_ctx* c, int64_t T, int64_t V, const void* h, const void* W, const int64_t* target, float scale,
                          const float* lse, const float* dloss, void* dh, void* dW, void* scratch, cudaStream_t s);
// distill.cuh : distillation from a teacher's top logits on the same tiles; scale includes 1 / temperature
constexpr int kDistillMaxK = 256;             // a teacher's entries a row
size_t distill_scratch_bytes(int64_t T, int64_t V, int K, int C, int grad);
bool launch_linear_distill_fwd(const mhclite_ctx* c, int64_t T, int64_t V, int K, const void* h, const void* W, const int64_t* ids,
                               const void* z, int z_f32, float scale, float inv_tau, float* loss, float* lse, float* logp, void* scratch,
                               cudaStream_t s);
bool launch_linear_distill_bwd(const mhclite_ctx* c, int64_t T, int64_t V, int K, const void* h, const void* W, const int64_t* ids,
                               const void* z, int z_f32, float scale, float inv_tau, const float* lse, const float* logp, const float* dloss,
                               void* dh, void* dW, void* scratch, cudaStream_t s);
// seq_losses.cuh : losses of whole sequences from the losses of their tokens, with their gradients (dnll null: without)
size_t seq_scratch_bytes(int64_t T, int64_t S);
void launch_policy_loss(const mhclite_ctx* c, int64_t T, int64_t S, const float* nll, const float* nll_old, const float* nll_ref,
                        const int64_t* target, const int64_t* starts, const float* adv, int token_adv, double clip_low, double clip_high,
                        double kl_weight, int mean, const float* dloss, float* loss, float* stats, float* dnll, void* scratch, cudaStream_t s);
void launch_preference_loss(const mhclite_ctx* c, int64_t T, int64_t P, const float* nll, const float* nll_ref, const int64_t* target,
                            const int64_t* starts, double beta, double margin, double smoothing, int mean, const float* dloss, float* loss,
                            float* reward, float* dnll, void* scratch, cudaStream_t s);

}  // namespace mhcl
