// Host-side helpers of the C entry points: the current device for the duration of a call, the error a failed runtime
// call leaves in the context, and the checks of alignment and overlap.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "sama_internal.h"

namespace sama {

struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
        if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
    }
    ~DeviceGuard() {
        int cur = -1;
        if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
    }
};

inline int cuda_fail(sama_ctx* ctx, cudaError_t e) {
    if (ctx) ctx->last_cuda_error = (int)e;
    return SAMA_ERR_CUDA;
}
#define SAMA_CUDA(ctx, expr)                                   \
    do {                                                       \
        cudaError_t e__ = (expr);                              \
        if (e__ != cudaSuccess) return cuda_fail((ctx), e__);  \
    } while (0)

// For calls that set up an operator on first use: running out of memory there is what running out of it for the workspace is.
inline int setup_fail(sama_ctx* ctx, cudaError_t e) {
    cuda_fail(ctx, e);
    if (e != cudaErrorMemoryAllocation) return SAMA_ERR_CUDA;
    cudaGetLastError();   // (not an error that the next call should find)
    return SAMA_ERR_NOMEM;
}
#define SAMA_SETUP(ctx, expr)                                   \
    do {                                                        \
        cudaError_t e__ = (expr);                               \
        if (e__ != cudaSuccess) return setup_fail((ctx), e__);  \
    } while (0)

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// true if [a, a+na) and [b, b+nb) share a byte
inline bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
    if (!a || !b || na == 0 || nb == 0) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}

}  // namespace sama
