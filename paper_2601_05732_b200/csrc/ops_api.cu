// C ABI of the operators around the stack: argument checks, scratch planning and kernel sequencing.
#include <math.h>

#include "api_checks.cuh"
#include "common.cuh"
#include "kernels.h"
#include "philox.cuh"

using namespace mhcl;

#define MHCL_PTR8(ctx, p)                                                                           \
    do {                                                                                            \
        if (!(p)) return fail(ctx, MHCLITE_ERR_BAD_ARG, "null pointer: %s", #p);                    \
        if ((uintptr_t)(p) & 7) return fail(ctx, MHCLITE_ERR_BAD_ARG, "pointer not 8-byte aligned: %s", #p); \
    } while (0)

static int check_scratch(mhclite_ctx* ctx, const void* scratch, size_t given, size_t need) {
    if (need == 0) return MHCLITE_OK;
    if (!scratch || given < need)
        return fail(ctx, MHCLITE_ERR_WORKSPACE, "scratch of %zu bytes needed, %zu given", need, scratch ? given : (size_t)0);
    if ((uintptr_t)scratch & 255) return fail(ctx, MHCLITE_ERR_BAD_ARG, "scratch not 256-byte aligned");
    return MHCLITE_OK;
}
constexpr int64_t kMaxTokens = ((int64_t)1 << 31) - 256;      // T and V stay below it
static int check_table(mhclite_ctx* ctx, int64_t T, int64_t V) {
    if (V < 1 || V >= kMaxTokens) return fail(ctx, MHCLITE_ERR_BAD_ARG, "V must be in [1, 2^31 - 256)");
    if (T >= kMaxTokens) return fail(ctx, MHCLITE_ERR_BAD_ARG, "T must be below 2^31 - 256");
    return MHCLITE_OK;
}
static int check_drop(mhclite_ctx* ctx, float p, const uint64_t* rng) {
    if (!(p >= 0.f && p < 1.f) || drop_threshold(p) > 65535) return fail(ctx, MHCLITE_ERR_BAD_ARG, "p must be in [0, 1 - 2^-17)");
    if (p > 0.f) MHCL_PTR8(ctx, rng);
    return MHCLITE_OK;
}
static int check_row(mhclite_ctx* ctx) {
    if (ctx->C > kMaxRowC) return fail(ctx, MHCLITE_ERR_BAD_ARG, "C above %d channels", kMaxRowC);
    return MHCLITE_OK;
}

// Partial rows of the block gradients: their number depends on the SMs, so the scratch is sized for the most there can be.
struct BlockScratch { float* dw; double* ds; size_t bytes; };
static BlockScratch plan_block(int C, int64_t T, int sm_count, void* base) {
    BlockScratch b;
    const int gated = block_parts(T, C, sm_count, true), plain = block_parts(T, C, sm_count, false);
    const size_t parts = (size_t)(gated > plain ? gated : plain), dw = (parts * C * 4 + 255) & ~(size_t)255;
    b.dw = (float*)base;
    b.ds = (double*)((char*)base + dw);
    b.bytes = parts <= 1 ? 0 : dw + ((parts * 8 + 255) & ~(size_t)255);      // one block writes the sums itself
    return b;
}

extern "C" {

int mhclite_embed_fwd(mhclite_ctx* ctx, int64_t T, int64_t V, const int64_t* ids, const void* E, int table_f32, float scale,
                      mhclite_bf16* x0, void* stream) {
    MHCL_REQUIRE_CTX(ctx); MHCL_REQUIRE_T(ctx, T);
    int rc = check_table(ctx, T, V);
    if (rc) return rc;
    if (T == 0) return MHCLITE_OK;
    MHCL_PTR8(ctx, ids); MHCL_PTR(ctx, E); MHCL_PTR(ctx, x0);
    MHCL_NO_ALIAS(ctx, x0, E); MHCL_NO_ALIAS(ctx, x0, ids);
    MHCL_DEVICE(ctx);
    launch_embed_fwd(ctx, T, V, ids, E, table_f32, scale, x0, (cudaStream_t)stream);
    MHCL_LAUNCH_CHECK(ctx, "embed_fwd");
    return MHCLITE_OK;
}

size_t mhclite_embed_scratch_bytes(int C, int64_t T, int64_t V) {
    if (C <= 0 || C % 8 || T < 0 || V < 1 || T >= kMaxTokens || V >= kMaxTokens) return 0;
    return embed_scratch_bytes(T, C);
}

int mhclite_embed_bwd(mhclite_ctx* ctx, int64_t T, int64_t V, const int64_t* ids, const mhclite_bf16* g, float scale, float* dE,
                      int accumulate, void* scratch, size_t scratch_bytes, void* stream) {
    MHCL_REQUIRE_CTX(ctx); MHCL_REQUIRE_T(ctx, T);
    int rc = check_table(ctx, T, V);
    if (rc) return rc;
    MHCL_PTR(ctx, dE);
    if (T == 0) {
        if (accumulate) return MHCLITE_OK;
        MHCL_DEVICE(ctx);
        return check_cuda(ctx, cudaMemsetAsync(dE, 0, (size_t)V * ctx->C * 4, (cudaStream_t)stream), "zero dE");
    }
    MHCL_PTR8(ctx, ids); MHCL_PTR(ctx, g);
    MHCL_NO_ALIAS(ctx, dE, g); MHCL_NO_ALIAS(ctx, dE, ids);
    if ((rc = check_scratch(ctx, scratch, scratch_bytes, embed_scratch_bytes(T, ctx->C)))) return rc;
    MHCL_DEVICE(ctx);
    return check_cuda(ctx, launch_embed_bwd(ctx, T, V, ids, g, scale, dE, accumulate, scratch, (cudaStream_t)stream), "embed_bwd");
}

int mhclite_block_in_fwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* u, const float* w, float eps, mhclite_bf16* v, float* rstd,
                         void* stream) {
    return mhclite_block_out_fwd(ctx, T, u, nullptr, w, nullptr, eps, 0.f, nullptr, v, rstd, stream);
}

int mhclite_block_out_fwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* o, const mhclite_bf16* gate, const float* w,
                          const float* scale, float eps, float p_drop, const uint64_t* rng, mhclite_bf16* y, float* rstd, void* stream) {
    MHCL_REQUIRE_CTX(ctx); MHCL_REQUIRE_T(ctx, T);
    int rc = check_row(ctx);
    if (rc) return rc;
    if (!(eps >= 0.f)) return fail(ctx, MHCLITE_ERR_BAD_ARG, "eps must be >= 0");
    if ((rc = check_drop(ctx, p_drop, rng))) return rc;
    if (T == 0) return MHCLITE_OK;
    MHCL_PTR(ctx, o); MHCL_OPT_PTR(ctx, gate); MHCL_PTR(ctx, w); MHCL_PTR(ctx, y); MHCL_PTR(ctx, rstd);
    if ((uintptr_t)scale & 3) return fail(ctx, MHCLITE_ERR_BAD_ARG, "pointer not 4-byte aligned: scale");
    MHCL_NO_ALIAS(ctx, y, o); MHCL_NO_ALIAS(ctx, y, gate);
    MHCL_DEVICE(ctx);
    launch_block_fwd(ctx, T, o, gate, w, scale, eps, p_drop, rng, y, rstd, (cudaStream_t)stream);
    MHCL_LAUNCH_CHECK(ctx, "block_fwd");
    return MHCLITE_OK;
}

size_t mhclite_block_scratch_bytes(int C, int64_t T) {
    if (C <= 0 || C % 8 || C > kMaxRowC || T < 0) return 0;
    return plan_block(C, T, 160, nullptr).bytes;          // as many SMs as an sm_100a device has, or more
}

int mhclite_block_in_bwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* u, const float* w, const float* rstd, const mhclite_bf16* dv,
                         mhclite_bf16* du, float* dw, int accumulate_params, void* scratch, size_t scratch_bytes, void* stream) {
    return mhclite_block_out_bwd(ctx, T, u, nullptr, w, nullptr, rstd, 0.f, nullptr, dv, du, nullptr, dw, nullptr, accumulate_params,
                                 scratch, scratch_bytes, stream);
}

int mhclite_block_out_bwd(mhclite_ctx* ctx, int64_t T, const mhclite_bf16* o, const mhclite_bf16* gate, const float* w,
                          const float* scale, const float* rstd, float p_drop, const uint64_t* rng, const mhclite_bf16* dy,
                          mhclite_bf16* d_o, mhclite_bf16* dgate, float* dw, float* dscale, int accumulate_params,
                          void* scratch, size_t scratch_bytes, void* stream) {
    MHCL_REQUIRE_CTX(ctx); MHCL_REQUIRE_T(ctx, T);
    int rc = check_row(ctx);
    if (rc) return rc;
    if ((rc = check_drop(ctx, p_drop, rng))) return rc;
    MHCL_PTR(ctx, dw);
    if (((uintptr_t)scale | (uintptr_t)dscale) & 3) return fail(ctx, MHCLITE_ERR_BAD_ARG, "pointer not 4-byte aligned: scale or dscale");
    if (T == 0) {
        if (accumulate_params) return MHCLITE_OK;
        MHCL_DEVICE(ctx);
        cudaError_t e = cudaMemsetAsync(dw, 0, (size_t)ctx->C * 4, (cudaStream_t)stream);
        if (e == cudaSuccess && dscale) e = cudaMemsetAsync(dscale, 0, 4, (cudaStream_t)stream);
        return check_cuda(ctx, e, "zero dw");
    }
    MHCL_PTR(ctx, o); MHCL_OPT_PTR(ctx, gate); MHCL_PTR(ctx, w); MHCL_PTR(ctx, rstd); MHCL_PTR(ctx, dy); MHCL_PTR(ctx, d_o);
    MHCL_OPT_PTR(ctx, dgate);
    if (!gate != !dgate) return fail(ctx, MHCLITE_ERR_BAD_ARG, "dgate is given if and only if gate is");
    MHCL_NO_ALIAS(ctx, d_o, o); MHCL_NO_ALIAS(ctx, d_o, dy); MHCL_NO_ALIAS(ctx, d_o, gate);
    if (gate) { MHCL_NO_ALIAS(ctx, dgate, o); MHCL_NO_ALIAS(ctx, dgate, dy); MHCL_NO_ALIAS(ctx, dgate, gate); MHCL_NO_ALIAS(ctx, dgate, d_o); }
    if ((rc = check_scratch(ctx, scratch, scratch_bytes, plan_block(ctx->C, T, ctx->sm_count, nullptr).bytes))) return rc;
    const BlockScratch b = plan_block(ctx->C, T, ctx->sm_count, scratch);
    MHCL_DEVICE(ctx);
    launch_block_bwd(ctx, T, o, gate, w, scale, rstd, p_drop, rng, dy, d_o, dgate, dw, dscale, accumulate_params, b.dw, b.ds,
                     (cudaStream_t)stream);
    MHCL_LAUNCH_CHECK(ctx, "block_bwd");
    return MHCLITE_OK;
}

int mhclite_dropout(mhclite_ctx* ctx, int64_t count, const mhclite_bf16* x, float p, const uint64_t* rng, mhclite_bf16* y, void* stream) {
    MHCL_REQUIRE_CTX(ctx);
    if (count < 0) return fail(ctx, MHCLITE_ERR_BAD_ARG, "count < 0");
    int rc = check_drop(ctx, p, rng);
    if (rc) return rc;
    if (count == 0) return MHCLITE_OK;
    MHCL_PTR(ctx, x); MHCL_PTR(ctx, y); MHCL_PTR8(ctx, rng);
    MHCL_NO_ALIAS(ctx, y, x);
    MHCL_DEVICE(ctx);
    launch_dropout(ctx, count, x, p, rng, y, (cudaStream_t)stream);
    MHCL_LAUNCH_CHECK(ctx, "dropout");
    return MHCLITE_OK;
}

constexpr int64_t kMaxLogits = (int64_t)1 << 46;               // T V stays below it

size_t mhclite_linear_ce_scratch_bytes(int C, int64_t T, int64_t V, int backward) {
    if (C <= 0 || C % 8 || T < 0 || V < 1 || T >= kMaxTokens || V >= kMaxTokens || (T > 0 && V >= kMaxLogits / T)) return 0;
    return ce_scratch_bytes(T, V, C, backward);
}

static int check_ce(mhclite_ctx* ctx, int64_t T, int64_t V, float logit_scale) {
    int rc = check_table(ctx, T, V);
    if (rc) return rc;
    if (T > 0 && V >= kMaxLogits / T) return fail(ctx, MHCLITE_ERR_BAD_ARG, "T V must be below 2^46");
    if (!(logit_scale - logit_scale == 0.f)) return fail(ctx, MHCLITE_ERR_BAD_ARG, "logit_scale must be finite");
    if (!tensor_maps_available()) return fail(ctx, MHCLITE_ERR_CUDA, "the driver has no tensor-map encoder");
    return MHCLITE_OK;
}

int mhclite_linear_ce_fwd(mhclite_ctx* ctx, int64_t T, int64_t V, const mhclite_bf16* h, const mhclite_bf16* W, const int64_t* target,
                          float logit_scale, float* loss, float* lse, void* scratch, size_t scratch_bytes, void* stream) {
    MHCL_REQUIRE_CTX(ctx); MHCL_REQUIRE_T(ctx, T);
    int rc = check_ce(ctx, T, V, logit_scale);
    if (rc) return rc;
    if (T == 0) return MHCLITE_OK;
    MHCL_PTR(ctx, h); MHCL_PTR(ctx, W); MHCL_PTR8(ctx, target); MHCL_PTR(ctx, loss); MHCL_PTR(ctx, lse);
    MHCL_NO_ALIAS(ctx, loss, lse);
    if ((rc = check_scratch(ctx, scratch, scratch_bytes, ce_scratch_bytes(T, V, ctx->C, 0)))) return rc;
    MHCL_DEVICE(ctx);
    if (!launch_linear_ce_fwd(ctx, T, V, h, W, target, logit_scale, loss, lse, scratch, (cudaStream_t)stream))
        return fail(ctx, MHCLITE_ERR_CUDA, "linear_ce_fwd: building a tensor map failed");
    MHCL_LAUNCH_CHECK(ctx, "linear_ce_fwd");
    return MHCLITE_OK;
}

int mhclite_linear_ce_bwd(mhclite_ctx* ctx, int64_t T, int64_t V, const mhclite_bf16* h, const mhclite_bf16* W, const int64_t* target,
                          float logit_scale, const float* lse, const float* dloss, mhclite_bf16* dh, mhclite_bf16* dW, void* scratch,
                          size_t scratch_bytes, void* stream) {
    MHCL_REQUIRE_CTX(ctx); MHCL_REQUIRE_T(ctx, T);
    int rc = check_ce(ctx, T, V, logit_scale);
    if (rc) return rc;
    MHCL_PTR(ctx, dW);
    if (T == 0) {
        MHCL_DEVICE(ctx);
        return check_cuda(ctx, cudaMemsetAsync(dW, 0, (size_t)V * ctx->C * 2, (cudaStream_t)stream), "zero dW");
    }
    MHCL_PTR(ctx, h); MHCL_PTR(ctx, W); MHCL_PTR8(ctx, target); MHCL_PTR(ctx, lse); MHCL_PTR(ctx, dloss); MHCL_PTR(ctx, dh);
    MHCL_NO_ALIAS(ctx, dh, h); MHCL_NO_ALIAS(ctx, dh, W); MHCL_NO_ALIAS(ctx, dW, h); MHCL_NO_ALIAS(ctx, dW, W); MHCL_NO_ALIAS(ctx, dh, dW);
    if ((rc = check_scratch(ctx, scratch, scratch_bytes, ce_scratch_bytes(T, V, ctx->C, 1)))) return rc;
    MHCL_DEVICE(ctx);
    if (!launch_linear_ce_bwd(ctx, T, V, h, W, target, logit_scale, lse, dloss, dh, dW, scratch, (cudaStream_t)stream))
        return fail(ctx, MHCLITE_ERR_CUDA, "linear_ce_bwd: building a tensor map failed");
    MHCL_LAUNCH_CHECK(ctx, "linear_ce_bwd");
    return MHCLITE_OK;
}

size_t mhclite_linear_distill_scratch_bytes(int C, int64_t T, int64_t V, int K, int backward) {
    if (mhclite_linear_ce_scratch_bytes(C, T, V, backward) == 0 || K < 1 || K > kDistillMaxK) return 0;
    return distill_scratch_bytes(T, V, K, C, backward);
}

// The student's scale with the temperature in it, in `scale`.
static int check_distill(mhclite_ctx* ctx, int64_t T, int64_t V, int K, float logit_scale, float temperature, float* scale) {
    if (K < 1 || K > kDistillMaxK) return fail(ctx, MHCLITE_ERR_BAD_ARG, "K must be in [1, %d]", kDistillMaxK);
    const float inv = 1.f / temperature;
    if (!(temperature > 0.f && inv > 0.f && inv - inv == 0.f)) return fail(ctx, MHCLITE_ERR_BAD_ARG, "temperature must be positive, it and its reciprocal finite");
    *scale = (float)((double)logit_scale / temperature);
    return check_ce(ctx, T, V, *scale);
}

int mhclite_linear_distill_fwd(mhclite_ctx* ctx, int64_t T, int64_t V, int K, const mhclite_bf16* h, const mhclite_bf16* W, const int64_t* ids,
                               const void* teacher, int teacher_f32, float logit_scale, float temperature, float* loss, float* lse,
                               float* logp, void* scratch, size_t scratch_bytes, void* stream) {
    MHCL_REQUIRE_CTX(ctx); MHCL_REQUIRE_T(ctx, T);
    float scale;
    int rc = check_distill(ctx, T, V, K, logit_scale, temperature, &scale);
    if (rc) return rc;
    if (T == 0) return MHCLITE_OK;
    MHCL_PTR(ctx, h); MHCL_PTR(ctx, W); MHCL_PTR8(ctx, ids); MHCL_PTR(ctx, teacher); MHCL_PTR(ctx, loss); MHCL_PTR(ctx, lse);
    MHCL_PTR(ctx, logp);
    MHCL_NO_ALIAS(ctx, loss, lse); MHCL_NO_ALIAS(ctx, loss, logp); MHCL_NO_ALIAS(ctx, lse, logp); MHCL_NO_ALIAS(ctx, logp, teacher);
    MHCL_NO_ALIAS(ctx, loss, teacher); MHCL_NO_ALIAS(ctx, lse, teacher);
    if ((rc = check_scratch(ctx, scratch, scratch_bytes, distill_scratch_bytes(T, V, K, ctx->C, 0)))) return rc;
    MHCL_DEVICE(ctx);
    if (!launch_linear_distill_fwd(ctx, T, V, K, h, W, ids, teacher, teacher_f32, scale, 1.f / temperature, loss, lse, logp, scratch,
                                   (cudaStream_t)stream))
        return fail(ctx, MHCLITE_ERR_CUDA, "linear_distill_fwd: building a tensor map failed");
    MHCL_LAUNCH_CHECK(ctx, "linear_distill_fwd");
    return MHCLITE_OK;
}

int mhclite_linear_distill_bwd(mhclite_ctx* ctx, int64_t T, int64_t V, int K, const mhclite_bf16* h, const mhclite_bf16* W, const int64_t* ids,
                               const void* teacher, int teacher_f32, float logit_scale, float temperature, const float* lse,
                               const float* logp, const float* dloss, mhclite_bf16* dh, mhclite_bf16* dW, void* scratch,
                               size_t scratch_bytes, void* stream) {
    MHCL_REQUIRE_CTX(ctx); MHCL_REQUIRE_T(ctx, T);
    float scale;
    int rc = check_distill(ctx, T, V, K, logit_scale, temperature, &scale);
    if (rc) return rc;
    MHCL_PTR(ctx, dW);
    if (T == 0) {
        MHCL_DEVICE(ctx);
        return check_cuda(ctx, cudaMemsetAsync(dW, 0, (size_t)V * ctx->C * 2, (cudaStream_t)stream), "zero dW");
    }
    MHCL_PTR(ctx, h); MHCL_PTR(ctx, W); MHCL_PTR8(ctx, ids); MHCL_PTR(ctx, teacher); MHCL_PTR(ctx, lse); MHCL_PTR(ctx, logp);
    MHCL_PTR(ctx, dloss); MHCL_PTR(ctx, dh);
    MHCL_NO_ALIAS(ctx, dh, h); MHCL_NO_ALIAS(ctx, dh, W); MHCL_NO_ALIAS(ctx, dW, h); MHCL_NO_ALIAS(ctx, dW, W); MHCL_NO_ALIAS(ctx, dh, dW);
    if ((rc = check_scratch(ctx, scratch, scratch_bytes, distill_scratch_bytes(T, V, K, ctx->C, 1)))) return rc;
    MHCL_DEVICE(ctx);
    if (!launch_linear_distill_bwd(ctx, T, V, K, h, W, ids, teacher, teacher_f32, scale, 1.f / temperature, lse, logp, dloss, dh, dW, scratch,
                                   (cudaStream_t)stream))
        return fail(ctx, MHCLITE_ERR_CUDA, "linear_distill_bwd: building a tensor map failed");
    MHCL_LAUNCH_CHECK(ctx, "linear_distill_bwd");
    return MHCLITE_OK;
}

constexpr int64_t kMaxSequences = (int64_t)1 << 30;            // their number stays below it

size_t mhclite_policy_scratch_bytes(int64_t T, int64_t S) {
    if (T < 0 || T >= kMaxTokens || S < 0 || S >= kMaxSequences) return 0;
    return seq_scratch_bytes(T, S);
}
size_t mhclite_preference_scratch_bytes(int64_t T, int64_t P) { return P < 0 || P >= kMaxSequences / 2 ? 0 : mhclite_policy_scratch_bytes(T, 2 * P); }

// What both losses check beside their own arguments.
static int check_sequences(mhclite_ctx* ctx, int64_t T, int64_t S, const float* nll, const int64_t* target, const int64_t* starts,
                           const float* dloss, const float* loss, const float* table, const float* dnll) {
    if (T >= kMaxTokens) return fail(ctx, MHCLITE_ERR_BAD_ARG, "T must be below 2^31 - 256");
    if (S < 0 || S >= kMaxSequences) return fail(ctx, MHCLITE_ERR_BAD_ARG, "the number of sequences must be in [0, 2^30)");
    if (S > 0) {
        MHCL_PTR8(ctx, starts); MHCL_PTR(ctx, loss); MHCL_PTR(ctx, table);
        MHCL_NO_ALIAS(ctx, loss, table); MHCL_NO_ALIAS(ctx, loss, dloss); MHCL_NO_ALIAS(ctx, table, dloss);
        if (T > 0) {
            MHCL_PTR(ctx, nll); MHCL_PTR8(ctx, target);
            MHCL_NO_ALIAS(ctx, loss, nll); MHCL_NO_ALIAS(ctx, table, nll);
        }
    }
    if (T > 0 && S > 0 && !dloss != !dnll) return fail(ctx, MHCLITE_ERR_BAD_ARG, "dloss and dnll are given both or neither");
    MHCL_OPT_PTR(ctx, dloss); MHCL_OPT_PTR(ctx, dnll);
    if (dnll) {
        MHCL_NO_ALIAS(ctx, dnll, nll); MHCL_NO_ALIAS(ctx, dnll, dloss); MHCL_NO_ALIAS(ctx, dnll, loss); MHCL_NO_ALIAS(ctx, dnll, table);
    }
    return MHCLITE_OK;
}
// Without a sequence the gradient is 0.
static int no_sequences(mhclite_ctx* ctx, int64_t T, float* dnll, void* stream) {
    if (T == 0 || !dnll) return MHCLITE_OK;
    MHCL_DEVICE(ctx);
    return check_cuda(ctx, cudaMemsetAsync(dnll, 0, (size_t)T * 4, (cudaStream_t)stream), "zero dnll");
}

int mhclite_policy_loss(mhclite_ctx* ctx, int64_t T, int64_t S, const float* nll, const float* nll_old, const float* nll_ref,
                        const int64_t* target, const int64_t* starts, const float* adv, int token_adv, double clip_low, double clip_high,
                        double kl_weight, int mean, const float* dloss, float* loss, float* stats, float* dnll, void* scratch,
                        size_t scratch_bytes, void* stream) {
    MHCL_REQUIRE_CTX(ctx); MHCL_REQUIRE_T(ctx, T);
    if (!(clip_low >= 0 && clip_low <= 1)) return fail(ctx, MHCLITE_ERR_BAD_ARG, "clip_low must be in [0, 1]");
    if (!(clip_high >= 0)) return fail(ctx, MHCLITE_ERR_BAD_ARG, "clip_high must be >= 0");
    if (!(fabs(kl_weight) <= 3e38)) return fail(ctx, MHCLITE_ERR_BAD_ARG, "kl_weight must be finite");
    int rc = check_sequences(ctx, T, S, nll, target, starts, dloss, loss, stats, dnll);
    if (rc) return rc;
    if (S == 0) return no_sequences(ctx, T, dnll, stream);
    if (T > 0) {
        MHCL_PTR(ctx, nll_old); MHCL_OPT_PTR(ctx, nll_ref); MHCL_PTR(ctx, adv);
        MHCL_NO_ALIAS(ctx, loss, adv); MHCL_NO_ALIAS(ctx, stats, adv);
        MHCL_NO_ALIAS(ctx, loss, nll_old); MHCL_NO_ALIAS(ctx, stats, nll_old);
        if (nll_ref) { MHCL_NO_ALIAS(ctx, loss, nll_ref); MHCL_NO_ALIAS(ctx, stats, nll_ref); }
        if (dnll) { MHCL_NO_ALIAS(ctx, dnll, nll_old); MHCL_NO_ALIAS(ctx, dnll, nll_ref); MHCL_NO_ALIAS(ctx, dnll, adv); }
    }
    if ((rc = check_scratch(ctx, scratch, scratch_bytes, seq_scratch_bytes(T, S)))) return rc;
    MHCL_DEVICE(ctx);
    launch_policy_loss(ctx, T, S, nll, nll_old, nll_ref, target, starts, adv, token_adv, clip_low, clip_high, kl_weight, mean, dloss, loss, stats,
                       T > 0 ? dnll : nullptr, scratch, (cudaStream_t)stream);
    MHCL_LAUNCH_CHECK(ctx, "policy_loss");
    return MHCLITE_OK;
}

int mhclite_preference_loss(mhclite_ctx* ctx, int64_t T, int64_t P, const float* nll, const float* nll_ref, const int64_t* target,
                            const int64_t* starts, double beta, double margin, double smoothing, int mean, const float* dloss, float* loss,
                            float* reward, float* dnll, void* scratch, size_t scratch_bytes, void* stream) {
    MHCL_REQUIRE_CTX(ctx); MHCL_REQUIRE_T(ctx, T);
    if (!(fabs(beta) <= 3e38) || !(fabs(margin) <= 3e38)) return fail(ctx, MHCLITE_ERR_BAD_ARG, "beta and margin must be finite");
    if (!(smoothing >= 0 && smoothing <= 1)) return fail(ctx, MHCLITE_ERR_BAD_ARG, "smoothing must be in [0, 1]");
    if (P < 0 || P >= kMaxSequences / 2) return fail(ctx, MHCLITE_ERR_BAD_ARG, "the number of pairs must be in [0, 2^29)");
    int rc = check_sequences(ctx, T, 2 * P, nll, target, starts, dloss, loss, reward, dnll);
    if (rc) return rc;
    if (P == 0) return no_sequences(ctx, T, dnll, stream);
    if (T > 0) {
        MHCL_OPT_PTR(ctx, nll_ref);
        if (nll_ref) { MHCL_NO_ALIAS(ctx, loss, nll_ref); MHCL_NO_ALIAS(ctx, reward, nll_ref); }
        if (dnll) MHCL_NO_ALIAS(ctx, dnll, nll_ref);
    }
    if ((rc = check_scratch(ctx, scratch, scratch_bytes, seq_scratch_bytes(T, 2 * P)))) return rc;
    MHCL_DEVICE(ctx);
    launch_preference_loss(ctx, T, P, nll, nll_ref, target, starts, beta, margin, smoothing, mean, dloss, loss, reward, T > 0 ? dnll : nullptr,
                           scratch, (cudaStream_t)stream);
    MHCL_LAUNCH_CHECK(ctx, "preference_loss");
    return MHCLITE_OK;
}

}  // extern "C"
