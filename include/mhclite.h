/*
 * mhclite.h -- C ABI of the mHC-lite residual-mixing library for NVIDIA B200 (sm_100a).
 *
 * The library computes, for every token independently, the dynamic residual
 * mixing step of a Hyper-Connections layer with n residual streams of C channels:
 *
 *     x_{l+1} = H_res x_l + H_post^T f(H_pre x_l)                        (paper Eq. (1))
 *
 * with the mHC-lite mappings (paper Eq. (4), (5)):
 *
 *     x' = RMSNorm(flatten(x_l))                        flatten is stream-major, m = j*C + c
 *     z  = alpha (.) (x' W) + b                         columns [res (n!) | pre (n) | post (n)]
 *     H_pre = sigmoid(z_pre), H_post = 2 sigmoid(z_post), a = softmax(z_res)
 *     H_res = sum_k a_k P_k                             P_k[i][sigma_k(i)] = 1, sigma in lexicographic order
 *
 * and, as a comparison path, the mHC mapping of paper Eq. (2),
 * H_res = SK(exp(mat(z_res))) with `iters` Sinkhorn-Knopp iterations (one
 * iteration = normalise all columns, then all rows).  The sublayer f is the
 * caller's: the forward is split in "before f" (coeffs, premix) and "after f"
 * (postres); the backward in "before f's backward" (postres_bwd) and "after"
 * (premix_bwd, coeffs_bwd, or the fused tail).
 *
 * Conventions for every entry point
 *   - Pointers are DEVICE pointers on the context's device unless the name ends
 *     in _host.  The caller owns every buffer, including the workspace; the
 *     library allocates no device memory.  All pointers must be 16-byte aligned.
 *   - bf16 tensors are raw 16-bit patterns (mhclite_bf16); fp32 tensors are float.
 *   - Layouts are dense row-major: x [T][n][C], y/u/du/dy [T][C], H_res [T][n][n]
 *     (row i = output stream), H_pre/H_post [T][n], W [n*C][N], N = n!+2n
 *     (n*n+2n for the SK path).
 *   - Calls are asynchronous on `stream` (a cudaStream_t passed as void*; NULL is
 *     the default stream) and never synchronise the device.  Calls that use the
 *     workspace (coeffs_fwd, coeffs_bwd, the fused calls, the SK calls) must not
 *     overlap on the GPU with another call on the same context.
 *   - No output buffer may alias an input buffer of the same call (the kernels read activations through the
 *     read-only data path and by TMA, and write whole tiles): in-place use such as x_next == x, dx == g or
 *     dx == x is refused with MHCLITE_ERR_BAD_ARG where it can be told from the pointers, and undefined for
 *     partial overlaps.  The one read-modify-write is dx with accumulate_dx != 0.
 *   - Return value: MHCLITE_OK (0) or a negative mhclite_status.  Nothing is
 *     launched when arguments are rejected.  T == 0 is a valid no-op.
 *   - Arithmetic: bf16 in, fp32 accumulate, bf16 (activations) or fp32
 *     (coefficients, parameter gradients) out.
 */
#ifndef MHCLITE_H_
#define MHCLITE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define MHCLITE_API __attribute__((visibility("default")))
#else
#define MHCLITE_API
#endif

typedef uint16_t mhclite_bf16;
typedef struct mhclite_ctx mhclite_ctx;

typedef enum mhclite_status {
    MHCLITE_OK = 0,
    MHCLITE_ERR_BAD_ARG = -1,      /* n not in [2,5], C % 8 != 0, T < 0, null / misaligned pointer, ... */
    MHCLITE_ERR_CUDA = -2,         /* a CUDA runtime call or launch failed; see mhclite_last_error */
    MHCLITE_ERR_WORKSPACE = -3,    /* workspace missing or smaller than mhclite_workspace_bytes */
    MHCLITE_ERR_TIMEOUT = -4,      /* a bounded device-side wait gave up (status word, never a trap) */
    MHCLITE_ERR_INDEX = -5         /* a token index outside the table was met (status words, see mhclite_set_status_words) */
} mhclite_status;

/* ---- context -------------------------------------------------------------------------------- */

/* Creates a context for n streams (2..5) of C channels (multiple of 8) on CUDA device `device`,
 * and uploads the permutation tables to that device's constant memory.  *out is written on success. */
MHCLITE_API int mhclite_create(mhclite_ctx** out, int n, int C, int device);
MHCLITE_API int mhclite_destroy(mhclite_ctx* ctx);

/* Human-readable name of a status code (static string). */
MHCLITE_API const char* mhclite_status_string(int status);
/* Text of the last error recorded on this context (valid until the next call on it). */
MHCLITE_API const char* mhclite_last_error(const mhclite_ctx* ctx);

/* Permutation table of paper Theorem 3.1 / Section 3.2: sigma_host[k*n + i] = sigma_k(i), the n!
 * permutations of (0..n-1) in lexicographic order, k = 0 the identity.  Host buffer of n!*n bytes. */
MHCLITE_API int mhclite_perm_table(int n, uint8_t* sigma_host);
/* The same table read back from the device's constant memory (what the warp-per-token kernels index; the
 * thread-per-token kernels for n <= 4 use a compile-time copy generated by the same successor rule). */
MHCLITE_API int mhclite_perm_table_device(mhclite_ctx* ctx, uint8_t* sigma_host);

/* Scratch the workspace-using calls need for up to T tokens (kind: 0 = mHC-lite, 1 = SK path). */
MHCLITE_API size_t mhclite_workspace_bytes(int n, int C, int64_t T, int kind);
/* Attaches caller-owned device scratch (256-byte aligned).  It must stay valid until replaced. */
MHCLITE_API int mhclite_set_workspace(mhclite_ctx* ctx, void* workspace, size_t bytes);

/* Paper Section 5 ("larger n"): restricts the convex combination of Eq. (5) to a SUBSET of K of the n!
 * permutation matrices; H_res stays exactly doubly stochastic and the projection narrows to N = K + 2n columns.
 *   table: DEVICE buffer of K*n bytes, caller-owned, table[k*n + i] = sigma_k(i); it must stay valid and
 *          unchanged while attached.  Rows must be distinct permutations of (0..n-1), 1 <= K <= n!
 *          (MHCLITE_ERR_BAD_ARG otherwise).  The call reads the table back once to check it (synchronous).
 *   K = 0 or table = NULL detaches the subset (all n! permutations again).
 * With a subset attached every mHC-lite entry point of the context takes W [nC, K+2n], b [K+2n],
 * a_saved [T, K], p_saved [T, K+2n] and dW / db of those sizes; the workspace is sized by
 * mhclite_workspace_bytes_subset.  The SK comparison path is not affected. */
MHCLITE_API int mhclite_set_perm_subset(mhclite_ctx* ctx, int K, const uint8_t* table);
MHCLITE_API size_t mhclite_workspace_bytes_subset(int n, int C, int64_t T, int K);

/* ---- forward -------------------------------------------------------------------------------- */

/* Paper Eq. (4), (5): the mappings of every token.
 *   in : x [T,n,C] bf16, W [nC,N] f32, b [N] f32, alpha [3] f32 = (res, pre, post), gain [nC] f32
 *        (RMSNorm weight), eps (RMSNorm epsilon, host scalar)
 *   out: H_res [T,n,n], H_pre [T,n], H_post [T,n] f32;
 *        saved for the backward: a_saved [T,n!] (softmax weights), p_saved [T,N] (x' W before alpha
 *        and bias), rstd [T] (1/sqrt(mean(x^2)+eps)).  */
MHCLITE_API int mhclite_coeffs_fwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x,
                       const float* W, const float* b, const float* alpha, const float* gain, float eps,
                       float* H_res, float* H_pre, float* H_post,
                       float* a_saved, float* p_saved, float* rstd, void* stream);

/* Paper Eq. (1), inner term: u[t,c] = sum_j H_pre[t,j] x[t,j,c].  u [T,C] bf16. */
MHCLITE_API int mhclite_premix_fwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x, const float* H_pre,
                       mhclite_bf16* u, void* stream);

/* Paper Eq. (1): x_next[t,i,c] = sum_j H_res[t,i,j] x[t,j,c] + H_post[t,i] y[t,c].  x_next [T,n,C] bf16. */
MHCLITE_API int mhclite_postres_fwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x, const mhclite_bf16* y,
                        const float* H_res, const float* H_post, mhclite_bf16* x_next, void* stream);

/* coeffs_fwd followed by premix_fwd with x read once (same results as the two calls). */
MHCLITE_API int mhclite_pre_fwd_fused(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x,
                          const float* W, const float* b, const float* alpha, const float* gain, float eps,
                          float* H_res, float* H_pre, float* H_post,
                          float* a_saved, float* p_saved, float* rstd, mhclite_bf16* u, void* stream);
/* The same, and the row statistic of the RMSNorm that usually opens the sublayer f of paper Eq. (1):
 *   u_rstd[t] = (mean_c u[t,c]^2 + eps_u)^-1/2   over the stored (bf16-rounded) u,   u_rstd [T] fp32,
 * produced by the pre-mix kernel while it writes u, so that the caller's normalisation of u is a row scale (which a
 * GEMM can apply to its operand or in its epilogue) and costs no pass over u.  u itself is written un-normalised:
 * du of the backward calls stays the gradient with respect to it.  For n = 5 and for contexts with a permutation subset a
 * separate kernel computes the statistic from u.  The paper has no counterpart (its sublayers normalise on their own). */
MHCLITE_API int mhclite_pre_fwd_fused_ustat(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x,
                          const float* W, const float* b, const float* alpha, const float* gain, float eps,
                          float* H_res, float* H_pre, float* H_post,
                          float* a_saved, float* p_saved, float* rstd, mhclite_bf16* u,
                          float* u_rstd, float eps_u, void* stream);

/* Layers back to back (the paper's models stack 6, 12 or 24 of them, Section 4): the merge of layer l, paper Eq. (1),
 * fused with what layer l+1 does first with its result, the RMSNorm statistics and the projection of Eq. (4):
 *   x_next[t,i,c] = sum_j H_res[t,i,j] x[t,j,c] + H_post[t,i] y[t,c]              (as mhclite_postres_fwd)
 *   and, left in the context's workspace, sum_m x_next[t,m]^2 and x_next[t,:] (diag(gain_next) W_next)
 * so that x_next is not read again for the next layer's projection.  W_next [nC,N], gain_next [nC] are layer
 * l+1's.  The next call on the context must be mhclite_pre_fwd_resume with x = x_next and the same T; any other
 * workspace-using call in between discards the partials.  x_next must not alias x. */
MHCLITE_API int mhclite_postres_fwd_next_proj(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x, const mhclite_bf16* y,
                        const float* H_res, const float* H_post, mhclite_bf16* x_next,
                        const float* W_next, const float* gain_next, void* stream);
/* The rest of mhclite_pre_fwd_fused for the layer whose projection mhclite_postres_fwd_next_proj has left in the
 * workspace: the mappings of Eq. (4), (5) and the pre-mix of Eq. (1).  Same outputs as mhclite_pre_fwd_fused(x, W_next,
 * b, alpha, gain_next, ...).  MHCLITE_ERR_BAD_ARG when no partials of this x and T are pending. */
MHCLITE_API int mhclite_pre_fwd_resume(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x,
                        const float* b, const float* alpha, float eps,
                        float* H_res, float* H_pre, float* H_post,
                        float* a_saved, float* p_saved, float* rstd, mhclite_bf16* u, void* stream);

/* ---- backward (exact gradient of Eq. (1), (4), (5)) ------------------------------------------ */

/* Gradient of postres_fwd given g = dL/dx_next [T,n,C] bf16:
 *   dy[t,c]      = sum_i H_post[t,i] g[t,i,c]                        [T,C] bf16
 *   dH_post[t,i] = <g[t,i,:], y[t,:]>, dH_res[t,i,j] = <g[t,i,:], x[t,j,:]>     f32
 *   dx[t,j,c]   (+)= sum_i H_res[t,i,j] g[t,i,c]    (skipped when dx is NULL; added to dx when
 *                                                    accumulate_dx != 0, else stored)           */
MHCLITE_API int mhclite_postres_bwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x, const mhclite_bf16* y,
                        const float* H_res, const float* H_post, const mhclite_bf16* g,
                        mhclite_bf16* dy, float* dH_res, float* dH_post,
                        mhclite_bf16* dx, int accumulate_dx, void* stream);

/* Gradient of premix_fwd given du = dL/du [T,C] bf16:
 *   dH_pre[t,j] = <du[t,:], x[t,j,:]>;  dx[t,j,c] (+)= H_pre[t,j] du[t,c]  (dx may be NULL). */
MHCLITE_API int mhclite_premix_bwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x, const float* H_pre,
                       const mhclite_bf16* du, float* dH_pre,
                       mhclite_bf16* dx, int accumulate_dx, void* stream);

/* Gradient of coeffs_fwd: from (dH_res, dH_pre, dH_post) back through the permutation sum, softmax,
 * sigmoids, the affine maps and RMSNorm.
 *   dx [T,n,C] bf16 (+)= dL/dx through the mappings;  dW [nC,N], db [N], dalpha [3], dgain [nC] f32,
 *   summed over the T tokens (added to the buffers when accumulate_params != 0, else stored). */
MHCLITE_API int mhclite_coeffs_bwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x,
                       const float* W, const float* alpha, const float* gain, float eps,
                       const float* a_saved, const float* p_saved, const float* rstd,
                       const float* H_pre, const float* H_post,
                       const float* dH_res, const float* dH_pre, const float* dH_post,
                       mhclite_bf16* dx, int accumulate_dx,
                       float* dW, float* db, float* dalpha, float* dgain, int accumulate_params,
                       void* stream);

/* Allocation-free variant of mhclite_coeffs_bwd (the paper has no counterpart: this is a property of
 * the library, not of the method).  It is for callers that cannot hand the library a workspace because
 * they cannot allocate device memory where the call is made: code running inside an allocator or
 * memory-pool callback, a process with a memory budget fixed at start-up, a plug-in that only ever
 * sees its inputs and outputs.  Same arguments as mhclite_coeffs_bwd and the same results up to the rounding
 * of that call's tensor-core path (this one keeps the operands of the projection backward in fp32), but the scratch is
 * a fixed array of mhclite_static_scratch_bytes() bytes inside the library's device image (every GPU
 * that loads the library holds it until the process exits) and no workspace needs to be attached.
 *   - The call needs about 4 * (T * Np + T + n * C * Np) bytes of it, Np = n!+2n rounded up to 8;
 *     problem sizes that need more than the array holds are rejected with MHCLITE_ERR_WORKSPACE
 *     and nothing is launched.
 *   - The call allocates and frees nothing.  The first call on each device looks up the array's
 *     device address (a synchronous, one-time set-up): make that first call before any stream capture.
 *   - All calls on a device share the one array and it keeps the previous call's contents; each call
 *     rewrites or clears every part it reads, so back-to-back calls on one stream are fine, but two
 *     calls that overlap on the GPU (different streams, different contexts) race on it. */
MHCLITE_API size_t mhclite_static_scratch_bytes(void);
MHCLITE_API int mhclite_coeffs_bwd_static(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x,
                       const float* W, const float* alpha, const float* gain, float eps,
                       const float* a_saved, const float* p_saved, const float* rstd,
                       const float* H_pre, const float* H_post,
                       const float* dH_res, const float* dH_pre, const float* dH_post,
                       mhclite_bf16* dx, int accumulate_dx,
                       float* dW, float* db, float* dalpha, float* dgain, int accumulate_params,
                       void* stream);

/* premix_bwd + coeffs_bwd + the H_res^T g term of postres_bwd, writing the complete dx once:
 *   dx[t,j,c] = sum_i H_res[t,i,j] g[t,i,c] + H_pre[t,j] du[t,c] + (gradient through the mappings).
 * dH_res and dH_post come from a preceding mhclite_postres_bwd call made with dx = NULL.
 * Reproducibility: for n <= 4 with C a multiple of 64 (no permutation subset attached) db, dalpha and dx are the
 * same bit for bit from run to run (db / dalpha are added up from per-block partials in a fixed order); dW and dgain
 * agree to fp32 rounding (the accumulation order inside the tensor-core kernel follows the arrival of the data).
 * On the other shapes db and dalpha are accumulated with atomics. */
MHCLITE_API int mhclite_tail_bwd_fused(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x,
                           const float* W, const float* alpha, const float* gain, float eps,
                           const float* a_saved, const float* p_saved, const float* rstd,
                           const float* H_res, const float* H_pre, const float* H_post,
                           const mhclite_bf16* g, const mhclite_bf16* du,
                           const float* dH_res, const float* dH_post,
                           mhclite_bf16* dx,
                           float* dW, float* db, float* dalpha, float* dgain, int accumulate_params,
                           void* stream);

/* ---- mHC comparison path (paper Eq. (2)): H_res = SK_iters(exp(mat(z_res))) ------------------ */

/* W_sk [nC, n*n+2n], b_sk [n*n+2n], columns [res (row-major n x n) | pre | post].  iters in [1,64]
 * (the paper's mHC uses 20).  The largest residual logit is subtracted before exp. */
MHCLITE_API int mhc_sk20_coeffs_fwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x,
                        const float* W_sk, const float* b_sk, const float* alpha, const float* gain,
                        float eps, int iters,
                        float* H_res, float* H_pre, float* H_post, float* p_saved, float* rstd,
                        void* stream);
/* mhc_sk20_coeffs_fwd followed by mhclite_premix_fwd in one kernel after the projection (paper Eq. (2), then the
 * inner term of Eq. (1)): the SK path's counterpart of mhclite_pre_fwd_fused, same results as the two calls. */
MHCLITE_API int mhc_sk20_pre_fwd_fused(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x,
                        const float* W_sk, const float* b_sk, const float* alpha, const float* gain,
                        float eps, int iters,
                        float* H_res, float* H_pre, float* H_post, float* p_saved, float* rstd,
                        mhclite_bf16* u, void* stream);
/* Gradient of mhc_sk20_coeffs_fwd; the SK iterates are recomputed from p_saved, not stored. */
MHCLITE_API int mhc_sk20_coeffs_bwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x,
                        const float* W_sk, const float* b_sk, const float* alpha, const float* gain,
                        float eps, int iters,
                        const float* p_saved, const float* rstd, const float* H_pre, const float* H_post,
                        const float* dH_res, const float* dH_pre, const float* dH_post,
                        mhclite_bf16* dx, int accumulate_dx,
                        float* dW, float* db, float* dalpha, float* dgain, int accumulate_params,
                        void* stream);

/* The SK path's counterpart of mhclite_tail_bwd_fused: dH_pre, the SK activation backward and the
 * projection backward, with dx = H_res^T g + H_pre du + (gradient through the mappings) written once.
 * dH_res and dH_post come from mhclite_postres_bwd called with dx = NULL (the streaming calls
 * premix_* / postres_* take coefficients, so they serve both paths). */
MHCLITE_API int mhc_sk20_tail_bwd_fused(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* x,
                        const float* W_sk, const float* b_sk, const float* alpha, const float* gain,
                        float eps, int iters,
                        const float* p_saved, const float* rstd,
                        const float* H_res, const float* H_pre, const float* H_post,
                        const mhclite_bf16* g, const mhclite_bf16* du,
                        const float* dH_res, const float* dH_post,
                        mhclite_bf16* dx,
                        float* dW, float* db, float* dalpha, float* dgain, int accumulate_params,
                        void* stream);

/* ---- doubly-stochastic diagnostics (paper Section 3.1 footnote) -------------------------------- */

/* Per token: l1_err[t] = ||H 1 - 1||_1 + ||H^T 1 - 1||_1 and colsum_dev[t] = max_j |sum_i H[i][j] - 1|
 * of H = H_res[t] (either output may be NULL). */
MHCLITE_API int mhclite_ds_gap(mhclite_ctx* ctx, int64_t T, const float* H_res, float* l1_err, float* colsum_dev,
                   void* stream);

/* The same gap as population statistics over all T tokens in one pass (the procedure behind the column-sum plots of
 * the paper's Section 3.1 / Fig. 3): stats [4] f32 (device) = { max_t l1_err, sum_t l1_err, max_t colsum_dev,
 * sum_t colsum_dev }; divide the sums by T for the means.  The sums are added in an unspecified order. */
MHCLITE_API int mhclite_ds_gap_stats(mhclite_ctx* ctx, int64_t T, const float* H_res, float* stats, void* stream);

/* Histogram over the tokens of log10(1/nu), nu the relative range of paper Eq. (3) of X[t] (the procedure behind
 * the paper's Fig. 4): `bins` equal bins on [lo, hi), values outside clamped to the first / last bin; hist is a
 * DEVICE array of bins + 1 64-bit counters, hist[bins] counting the matrices without a positive entry. */
MHCLITE_API int mhclite_log_inv_nu_histogram(mhclite_ctx* ctx, int64_t T, const float* X, int bins, float lo, float hi,
                                 unsigned long long* hist, void* stream);

/* Product of the residual mappings over depth (paper Section 3.1: prod_l H_res_l must stay doubly stochastic
 * for the signal to keep its norm across layers).  Per token: P[t] <- H_res[t] P[t], later layers multiplying
 * on the left as x_{l+1} = H_l x_l composes; with first != 0, P[t] <- H_res[t].  P is [T][n][n] fp32, updated
 * in place, and must not alias H_res.  Its gap is read with mhclite_ds_gap(P). */
MHCLITE_API int mhclite_depth_product(mhclite_ctx* ctx, int64_t T, const float* H_res, float* P, int first,
                                      void* stream);

/* Relative range of paper Eq. (3), per token: nu[t] = (smallest positive entry) / (largest entry) of the
 * n x n matrix X[t] (0 when no entry is positive); 1/nu bounds the Sinkhorn-Knopp iteration count. */
MHCLITE_API int mhclite_relative_range(mhclite_ctx* ctx, int64_t T, const float* X, float* nu, void* stream);

/* ---- around the stack: lookup, block norms, dropout, loss -------------------------------------------
 *
 * What a model adds to a stack of mixing layers: the token rows that fill x_0, the norms that enclose a sublayer f, and
 * the loss of the last hidden rows.  (Paper Section 4 trains such models; it takes these parts as given.)
 *   - C and n are the context's, C at most 16384 for the block calls.
 *   - Calls that need scratch take it as an argument (device, 256-byte aligned, at least the stated bytes, no contents
 *     to keep between calls; NULL where 0 bytes are stated), not from the attached workspace: calls with scratch of their
 *     own may overlap on the GPU, and each captured graph keeps its own.
 *   - Token ids and targets are int64 (8-byte aligned); other pointers 16-byte aligned.
 *   - T == 0 launches no kernel, but parameter gradients that are not accumulated are then set to zero.
 *   - Results are the same bit for bit from run to run. */

/* Attaches 8 device ints (caller-owned; NULL detaches) in which the calls below record the first token index outside its
 * table and the first wait that gave up; mhclite_device_status reports them, the wait before the index, until the words are
 * attached again.  The words, and the attached workspace's, are cleared by this call, which waits for all work queued on the
 * device before and for the clearing (not while a stream is being captured).  They must stay valid as long as calls made,
 * or captured into a graph, while they were attached can run. */
MHCLITE_API int mhclite_set_status_words(mhclite_ctx* ctx, int32_t* words);
typedef enum mhclite_op {          /* the operator named in such a report */
    MHCLITE_OP_EMBED = 20,
    MHCLITE_OP_EMBED_BWD = 21,
    MHCLITE_OP_LINEAR_CE = 22
} mhclite_op;

/* x0[t,j,:] = bf16(scale * E[ids[t],:]) for each of the n streams j.  E [V,C], fp32 when table_f32 != 0, else bf16;
 * x0 [T,n,C] bf16.  A token whose id is outside [0, V) gets zero rows and is reported (MHCLITE_ERR_INDEX). */
MHCLITE_API int mhclite_embed_fwd(mhclite_ctx* ctx, int64_t T, int64_t V, const int64_t* ids, const void* E, int table_f32,
                        float scale, mhclite_bf16* x0, void* stream);
/* Gradient of embed_fwd from g = dL/dx0 [T,n,C] bf16:
 *   dE[v,:] (+)= scale * sum over {t: ids[t] = v} and the streams of g[t,j,:]      [V,C] f32
 * added to dE when accumulate != 0 (rows of other tokens stay untouched), else stored (their rows are zeroed).
 * Tokens outside [0, V) are left out and reported. */
MHCLITE_API size_t mhclite_embed_scratch_bytes(int C, int64_t T, int64_t V);
MHCLITE_API int mhclite_embed_bwd(mhclite_ctx* ctx, int64_t T, int64_t V, const int64_t* ids, const mhclite_bf16* g, float scale,
                        float* dE, int accumulate, void* scratch, size_t scratch_bytes, void* stream);

/* The norm that opens a sublayer: v[t,c] = u[t,c] rstd[t] w[c], rstd[t] = (mean_c u[t,c]^2 + eps)^-1/2.
 * u, v [T,C] bf16; w [C], rstd [T] f32 (saved for the backward). */
MHCLITE_API int mhclite_block_in_fwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* u, const float* w, float eps,
                        mhclite_bf16* v, float* rstd, void* stream);
/* du [T,C] bf16 and dw [C] f32 (added when accumulate_params != 0) from dv [T,C] bf16. */
MHCLITE_API size_t mhclite_block_scratch_bytes(int C, int64_t T);
MHCLITE_API int mhclite_block_in_bwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* u, const float* w, const float* rstd,
                        const mhclite_bf16* dv, mhclite_bf16* du, float* dw, int accumulate_params,
                        void* scratch, size_t scratch_bytes, void* stream);

/* What closes a sublayer, its output o [T,C] bf16 normalised, gated, dropped out and scaled before the merge:
 *   y[t,c] = s drop(sigmoid(gate[t,c]) o[t,c] rstd[t] w[c])
 * gate [T,C] bf16 or NULL (no gate), s = *scale (f32, device) or 1 for NULL, drop as in mhclite_dropout with the element
 * index t C + c (p_drop = 0: none, rng may be NULL).  rstd as in block_in_fwd. */
MHCLITE_API int mhclite_block_out_fwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* o, const mhclite_bf16* gate, const float* w,
                        const float* scale, float eps, float p_drop, const uint64_t* rng, mhclite_bf16* y, float* rstd,
                        void* stream);
/* Its gradient from dy [T,C] bf16: d_o, dgate [T,C] bf16 (dgate is given if and only if gate is), dw [C], dscale [1] f32
 * (dscale may be NULL; both added when accumulate_params != 0).  rng must hold the values of the forward call. */
MHCLITE_API int mhclite_block_out_bwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* o, const mhclite_bf16* gate, const float* w,
                        const float* scale, const float* rstd, float p_drop, const uint64_t* rng, const mhclite_bf16* dy,
                        mhclite_bf16* d_o, mhclite_bf16* dgate, float* dw, float* dscale, int accumulate_params,
                        void* scratch, size_t scratch_bytes, void* stream);

/* y[i] = x[i] / (1 - p) where element i stays, 0 where it is dropped, for any count of bf16 elements; the same call on dy
 * is the gradient.  The mask is not stored: element i stays when its 16 bits of Philox4x32-10 (key: the seed; counter: the
 * 64-bit group i / 8, then the 64-bit offset; half-word i % 8 of the four output words, low halves first) are at least
 * round(65536 p), and p counts as rounded to that multiple of 2^-16.  0 <= p < 1 - 2^-17.
 *   rng [2] device: (seed, offset), read when the kernel runs, so that a captured graph draws new masks when the caller
 *   changes the offset between replays.  Dropped elements are 0 whatever x holds. */
MHCLITE_API int mhclite_dropout(mhclite_ctx* ctx, int64_t count, const mhclite_bf16* x, float p, const uint64_t* rng,
                        mhclite_bf16* y, void* stream);

/* Softmax cross entropy of the logits l[t,v] = logit_scale <h[t,:], W[v,:]>, which are never stored:
 *   lse[t] = log sum_v exp l[t,v],   loss[t] = lse[t] - l[t,target[t]]        [T] f32
 * h [T,C], W [V,C] bf16.  Rows with a negative target have none: loss and lse are 0, h is not used.  A target of V or
 * more counts as none and is reported.  T V < 2^46. */
MHCLITE_API size_t mhclite_linear_ce_scratch_bytes(int C, int64_t T, int64_t V, int backward);
MHCLITE_API int mhclite_linear_ce_fwd(mhclite_ctx* ctx, int64_t T, int64_t V, const mhclite_bf16* h, const mhclite_bf16* W,
                        const int64_t* target, float logit_scale, float* loss, float* lse,
                        void* scratch, size_t scratch_bytes, void* stream);
/* Gradient from dloss [T] f32 (dL/dloss; the reduction over tokens is the caller's) and the forward's lse:
 *   dh[t,:] = dloss[t] logit_scale (sum_v softmax(l)[t,v] W[v,:] - W[target[t],:])    [T,C] bf16, 0 without a target
 *   dW[v,:] = sum_t dloss[t] logit_scale (softmax(l)[t,v] - [v = target[t]]) h[t,:]   [V,C] bf16 (overwritten)
 * The bracket enters the products rounded to bf16; sums are fp32. */
MHCLITE_API int mhclite_linear_ce_bwd(mhclite_ctx* ctx, int64_t T, int64_t V, const mhclite_bf16* h, const mhclite_bf16* W,
                        const int64_t* target, float logit_scale, const float* lse, const float* dloss,
                        mhclite_bf16* dh, mhclite_bf16* dW, void* scratch, size_t scratch_bytes, void* stream);

/* ---- whole step from host buffers -------------------------------------------------------------- */

/* Bytes of device staging mhclite_step_host needs for T tokens. */
MHCLITE_API size_t mhclite_step_host_bytes(int n, int C, int64_t T);

/* One forward + backward pass of the layer (paper Eq. (1), (4), (5) and their gradient) with the
 * activations in HOST memory and the sublayer's results supplied: copies x, y, g = dL/dx_next and
 * du = dL/du host->device into `staging`, runs pre_fwd_fused, postres_fwd, postres_bwd and
 * tail_bwd_fused, and copies u, x_next, dy, dx device->host.  Parameters and their gradients stay on
 * the device.  The tokens are processed in up to eight chunks so that the copies in, the kernels and the
 * copies out of successive chunks overlap (two copy streams owned by the context, made on the first call
 * and tied to `stream` by events: the call stays ordered on `stream`); the parameter gradients of the chunks
 * add up.  Host buffers should be page-locked for the copies to be asynchronous; results are valid once
 * `stream` has been synchronised.  `staging` is caller-owned device scratch (256-byte aligned) of
 * at least mhclite_step_host_bytes; the context's workspace must be attached as well. */
MHCLITE_API int mhclite_step_host(mhclite_ctx* ctx, int64_t T,
                      const mhclite_bf16* x_host, const mhclite_bf16* y_host,
                      const mhclite_bf16* g_host, const mhclite_bf16* du_host,
                      const float* W, const float* b, const float* alpha, const float* gain, float eps,
                      mhclite_bf16* u_host, mhclite_bf16* x_next_host,
                      mhclite_bf16* dy_host, mhclite_bf16* dx_host,
                      float* dW, float* db, float* dalpha, float* dgain, int accumulate_params,
                      void* staging, size_t staging_bytes, void* stream);

/* Per-kernel device time, for roofline accounting.  With timing on, the library records a pair of CUDA
 * events on the call's stream around each launch of the kernels below (a few microseconds of overhead
 * per launch: switch it off for throughput runs).  mhclite_kernel_time_ms returns the duration of the
 * most recent launch of that kernel; the caller must have synchronised the stream since.  A kernel that
 * the problem size routes around (the fallbacks replace some of them) has no time: MHCLITE_ERR_BAD_ARG. */
typedef enum mhclite_kernel {
    MHCLITE_KERNEL_PROJ_FWD = 0,     /* tensor-core projection + sum of squares        reads x            */
    MHCLITE_KERNEL_ACT_PREMIX = 1,   /* mappings + pre-mix                              reads x, writes u  */
    MHCLITE_KERNEL_POSTRES_FWD = 2,  /* merge                                           reads x, y; writes x_next */
    MHCLITE_KERNEL_POSTRES_BWD = 3,  /* merge backward                                  reads g, x, y; writes dy  */
    MHCLITE_KERNEL_TAIL_PRE = 4,     /* dH_pre + activation backward                    reads x, du        */
    MHCLITE_KERNEL_TAIL_DX = 5,      /* projection backward + dx (+ dW): tail_ftc_k (n <= 4, C % 64 == 0),
                                        tail_dx_tc_k (n = 5), tail_mma_k otherwise   reads x, g, du; writes dx */
    MHCLITE_KERNEL_COUNT = 6
} mhclite_kernel;
MHCLITE_API int mhclite_set_kernel_timing(mhclite_ctx* ctx, int on);
MHCLITE_API int mhclite_kernel_time_ms(mhclite_ctx* ctx, int kernel, float* ms);

/* Synchronous check of the device status word: kernels that wait on hardware barriers do so with a bound
 * and, instead of hanging, record MHCLITE_ERR_TIMEOUT there and return.  Waits for all work queued on the
 * device, whatever its stream, then copies the words to the host; returns MHCLITE_OK or the recorded status. */
MHCLITE_API int mhclite_device_status(mhclite_ctx* ctx);

/* Number of kernels this context has launched since it was created (for accounting; host counter). */
MHCLITE_API int64_t mhclite_kernel_launches(const mhclite_ctx* ctx);

#ifdef __cplusplus
}
#endif
#endif /* MHCLITE_H_ */
