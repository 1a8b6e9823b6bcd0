// Argument checks and the device guard that the C entry points share.
#pragma once
#include "common.cuh"

namespace mhcl {

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Makes the context's device current for the duration of a call.
struct DeviceGuard {
    int prev = -1;
    bool switched = false;
    cudaError_t err = cudaSuccess;
    explicit DeviceGuard(int dev) {
        err = cudaGetDevice(&prev);
        if (err == cudaSuccess && prev != dev) { err = cudaSetDevice(dev); switched = (err == cudaSuccess); }
    }
    ~DeviceGuard() { if (switched) cudaSetDevice(prev); }
};

}  // namespace mhcl

#define MHCL_REQUIRE_CTX(ctx)  do { if (!(ctx)) return MHCLITE_ERR_BAD_ARG; (ctx)->err[0] = 0; } while (0)
#define MHCL_REQUIRE_T(ctx, T) do { if ((T) < 0) return fail(ctx, MHCLITE_ERR_BAD_ARG, "T < 0"); } while (0)
#define MHCL_PTR(ctx, p)                                                                            \
    do {                                                                                            \
        if (!(p)) return fail(ctx, MHCLITE_ERR_BAD_ARG, "null pointer: %s", #p);                    \
        if (!aligned16(p)) return fail(ctx, MHCLITE_ERR_BAD_ARG, "pointer not 16-byte aligned: %s", #p); \
    } while (0)
#define MHCL_OPT_PTR(ctx, p)                                                                        \
    do {                                                                                            \
        if ((p) && !aligned16(p)) return fail(ctx, MHCLITE_ERR_BAD_ARG, "pointer not 16-byte aligned: %s", #p); \
    } while (0)
// An output that aliases an input is refused: the kernels read activations through the read-only path and by TMA.
#define MHCL_NO_ALIAS(ctx, out, in)                                                                 \
    do {                                                                                            \
        if ((const void*)(out) == (const void*)(in))                                                \
            return fail(ctx, MHCLITE_ERR_BAD_ARG, "%s must not alias %s", #out, #in);               \
    } while (0)
#define MHCL_DEVICE(ctx)                                                                            \
    DeviceGuard guard_((ctx)->device);                                                              \
    if (guard_.err != cudaSuccess) return check_cuda(ctx, guard_.err, "cudaSetDevice")
#define MHCL_LAUNCH_CHECK(ctx, what) do { int rc_ = check_cuda(ctx, cudaGetLastError(), what); if (rc_) return rc_; } while (0)
