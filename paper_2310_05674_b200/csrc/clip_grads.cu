// Global gradient norm over many tensors, and clipping.
//
//   norm = sqrt( sum over tensors i and elements j of g_ij^2 ),   c = min(1, max_norm / norm),   out_ij = c g_ij
//
// Bound by memory traffic.  The tensors' addresses, lengths and types travel in the kernel's parameters (no copy, no
// plan on the device), and each block takes an equal, contiguous share of the elements of all tensors together, cut
// into chunks that never cross a tensor.  Squares are summed in double: a square of any fp32 or bf16 value neither
// overflows nor vanishes there, and the partial sums of the blocks are added in a fixed order.
#include <cmath>

#include "num_types.h"
#include "sama_internal.h"

namespace sama {

namespace {

constexpr int kClipThreads = 256;
constexpr int kGroup = 8;  // elements per thread and access: 16 bytes of a 16-bit type, 32 of fp32

struct ClipEntry {
    const void* in;
    void* out;
    int64_t n;
    int32_t first_chunk;
    uint8_t dtype, out_dtype, in_vec, out_vec;  // *_vec: the address is 16-byte aligned
};
template <int CAP>
struct ClipArgs {
    int n_entries, n_chunks, chunk;   // chunk: elements, a multiple of kGroup * kClipThreads
    int n_partials, partial0;         // all launches' block partials, and where this launch's begin
    int last;                         // this launch adds them up
    float max_norm;
    double* partials;
    ClipState* state;
    float* norm_out;
    DeviceScalars* sc;
    ClipEntry e[CAP];
};

__device__ __forceinline__ double clip_warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
    return v;
}
// Sum over the block in a fixed order; valid in thread 0.
__device__ __forceinline__ double clip_block_sum(double v, double* smem) {
    v = clip_warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
    __syncthreads();
    double t = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < kClipThreads / 32; ++w) t += smem[w];
    return t;
}

// The last entry whose first chunk is <= c.
template <int CAP>
__device__ __forceinline__ int entry_of(const ClipArgs<CAP>& a, int c) {
    int lo = 0, hi = a.n_entries - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.e[mid].first_chunk <= c) lo = mid; else hi = mid - 1;
    }
    return lo;
}

template <typename T>
__device__ __forceinline__ double chunk_sumsq(const T* __restrict__ p, int n, bool vec) {
    constexpr int U = 4;
    double acc[2] = {0.0, 0.0};
    if (vec) {
        const int groups = n / kGroup;
        for (int i = threadIdx.x; i < groups; i += U * kClipThreads) {
            float v[U][kGroup];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i + u * kClipThreads < groups) {
                    load_n<T, kGroup, true>(p + (int64_t)(i + u * kClipThreads) * kGroup, v[u]);
                } else {
#pragma unroll
                    for (int j = 0; j < kGroup; ++j) v[u][j] = 0.f;
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < kGroup; ++j) acc[j & 1] = fma((double)v[u][j], (double)v[u][j], acc[j & 1]);
        }
    }
    // the rest, or a tensor at an odd address: neighbouring threads take neighbouring elements
    const int done = vec ? n / kGroup * kGroup : 0;
    for (int i = done + threadIdx.x; i < n; i += kGroup * kClipThreads) {
        float v[kGroup];
#pragma unroll
        for (int u = 0; u < kGroup; ++u) v[u] = i + u * kClipThreads < n ? to_float(p[i + u * kClipThreads]) : 0.f;
#pragma unroll
        for (int u = 0; u < kGroup; ++u) acc[u & 1] = fma((double)v[u], (double)v[u], acc[u & 1]);
    }
    return acc[0] + acc[1];
}

// The factor.  Below 2^-100 it may leave fp32's normal range (a limit of 1e-30 on a norm of 1e38), where only double
// still holds it.  0 marks a norm that is not finite: zeros are written whatever the gradients are.
struct Factor {
    float f;
    double d;
    bool in_double;
    __device__ explicit Factor(double c) : f((float)c), d(c), in_double(c < 7.888609052210118e-31 && c != 0.0) {}
    __device__ __forceinline__ float operator()(float x) const {
        if (in_double) return (float)((double)x * d);
        return f == 0.f ? 0.f : x * f;
    }
};

template <int N>
__device__ __forceinline__ void store_as(int dtype, void* q, int64_t at, const float* v) {
    if (dtype == SAMA_F32) store_n<float, N>(static_cast<float*>(q) + at, v);
    else if (dtype == SAMA_BF16) store_n<__nv_bfloat16, N>(static_cast<__nv_bfloat16*>(q) + at, v);
    else store_n<__half, N>(static_cast<__half*>(q) + at, v);
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const ClipEntry& e, int64_t at, int n, const Factor& by) {
    constexpr int U = 4;
    const T* p = static_cast<const T*>(e.in) + at;
    void* const q = e.out;
    const int to = e.out_dtype;
    const int groups = e.in_vec && e.out_vec ? n / kGroup : 0;
    for (int i = threadIdx.x; i < groups; i += U * kClipThreads) {
        float v[U][kGroup];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * kClipThreads < groups) load_n<T, kGroup>(p + (int64_t)(i + u * kClipThreads) * kGroup, v[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * kClipThreads < groups) {
#pragma unroll
                for (int j = 0; j < kGroup; ++j) v[u][j] = by(v[u][j]);
                store_as<kGroup>(to, q, at + (int64_t)(i + u * kClipThreads) * kGroup, v[u]);
            }
    }
    for (int i = groups * kGroup + threadIdx.x; i < n; i += kGroup * kClipThreads) {
        float v[kGroup];
#pragma unroll
        for (int u = 0; u < kGroup; ++u)
            if (i + u * kClipThreads < n) v[u] = to_float(p[i + u * kClipThreads]);
#pragma unroll
        for (int u = 0; u < kGroup; ++u)
            if (i + u * kClipThreads < n) {
                v[u] = by(v[u]);
                store_as<1>(to, q, at + i + u * kClipThreads, v + u);
            }
    }
}

template <int CAP>
__global__ void __launch_bounds__(kClipThreads)
grad_norm_kernel(const __grid_constant__ ClipArgs<CAP> a) {
    __shared__ double smem[kClipThreads / 32];
    __shared__ bool is_last;
    pdl_trigger();
    pdl_wait();
    const int c0 = (int)((int64_t)a.n_chunks * blockIdx.x / gridDim.x);
    const int c1 = (int)((int64_t)a.n_chunks * (blockIdx.x + 1) / gridDim.x);
    double acc = 0.0;
    if (c0 < c1) {
        int k = entry_of(a, c0);
        for (int c = c0; c < c1; ++c) {
            while (k + 1 < a.n_entries && a.e[k + 1].first_chunk <= c) ++k;
            const ClipEntry& e = a.e[k];
            const int64_t at = (int64_t)(c - e.first_chunk) * a.chunk;
            const int n = (int)min((int64_t)a.chunk, e.n - at);
            if (e.dtype == SAMA_F32) acc += chunk_sumsq(static_cast<const float*>(e.in) + at, n, e.in_vec);
            else if (e.dtype == SAMA_BF16) acc += chunk_sumsq(static_cast<const __nv_bfloat16*>(e.in) + at, n, e.in_vec);
            else acc += chunk_sumsq(static_cast<const __half*>(e.in) + at, n, e.in_vec);
        }
    }
    const double total = clip_block_sum(acc, smem);
    if (threadIdx.x == 0) {
        a.partials[a.partial0 + blockIdx.x] = total;
        __threadfence();
        is_last = atomicAdd(&a.sc->counter, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!is_last) return;
    __threadfence();
    double v = 0.0;
    if (a.last)
        for (int i = threadIdx.x; i < a.n_partials; i += kClipThreads) v += __ldcg(a.partials + i);
    const double sum = clip_block_sum(v, smem);
    if (threadIdx.x == 0) {
        a.sc->counter = 0u;
        if (a.last) {
            const double norm = sqrt(sum);
            double c = 1.0;
            if (!isfinite(norm)) {
                c = 0.0;
                atomicOr(&a.sc->status, (int)SAMA_DEV_NONFINITE_GRAD);
            } else if (norm > (double)a.max_norm) {
                c = (double)a.max_norm / norm;
            }
            a.state->factor = c;
            if (a.norm_out) *a.norm_out = (float)norm;
        }
    }
}

template <int CAP>
__global__ void __launch_bounds__(kClipThreads)
grad_scale_kernel(const __grid_constant__ ClipArgs<CAP> a) {
    pdl_trigger();
    pdl_wait();
    const Factor by(a.state->factor);
    const int c0 = (int)((int64_t)a.n_chunks * blockIdx.x / gridDim.x);
    const int c1 = (int)((int64_t)a.n_chunks * (blockIdx.x + 1) / gridDim.x);
    if (c0 >= c1) return;
    int k = entry_of(a, c0);
    for (int c = c0; c < c1; ++c) {
        while (k + 1 < a.n_entries && a.e[k + 1].first_chunk <= c) ++k;
        const ClipEntry& e = a.e[k];
        if (!e.out || (e.out == e.in && by.f == 1.f)) continue;  // nothing to write
        const int64_t at = (int64_t)(c - e.first_chunk) * a.chunk;
        const int n = (int)min((int64_t)a.chunk, e.n - at);
        if (e.dtype == SAMA_F32) chunk_scale<float>(e, at, n, by);
        else if (e.dtype == SAMA_BF16) chunk_scale<__nv_bfloat16>(e, at, n, by);
        else chunk_scale<__half>(e, at, n, by);
    }
}

// One launch's worth of tensors.
constexpr int kCapSmall = 112, kCapLarge = 960;  // 3.6 KB and 31 KB of parameters

template <int CAP>
void fill(ClipArgs<CAP>& a, const sama_tensor_t* t, int first, int count, int chunk) {
    int64_t chunks = 0;
    a.n_entries = 0;
    for (int i = first; i < first + count; ++i) {
        if (t[i].n == 0) continue;
        ClipEntry& e = a.e[a.n_entries++];
        e.in = t[i].in;
        e.out = t[i].out;
        e.n = t[i].n;
        e.first_chunk = (int32_t)chunks;
        e.dtype = (uint8_t)t[i].dtype;
        e.out_dtype = (uint8_t)t[i].out_dtype;
        e.in_vec = (reinterpret_cast<uintptr_t>(t[i].in) & 15u) == 0;
        e.out_vec = (reinterpret_cast<uintptr_t>(t[i].out) & 15u) == 0;
        chunks += (t[i].n + chunk - 1) / chunk;
    }
    a.n_chunks = (int)chunks;
    a.chunk = chunk;
}

template <int CAP>
cudaError_t run_clip(sama_ctx* ctx, const sama_tensor_t* t, int n, int64_t total, bool any_out, float max_norm,
                     float* norm_out, ClipState* state, cudaStream_t st) {
    const int launches = n > 0 ? (n + CAP - 1) / CAP : 1;
    const int64_t lanes = (int64_t)kClipThreads * kGroup;
    // at most 2^31 chunks; enough of them for every block to get a share, few enough for a block's bookkeeping
    int64_t chunk = total / ((int64_t)ctx->sm_count * 4 * 8) / lanes * lanes;
    if (chunk < lanes) chunk = lanes;
    if (chunk > 16 * lanes) chunk = 16 * lanes;
    int grid = ctx->sm_count * 4;
    if (grid > kMaxPartials / launches) grid = kMaxPartials / launches;
    ClipArgs<CAP> a;
    a.n_partials = launches * grid;
    a.max_norm = max_norm;
    a.partials = ctx->partials;
    a.state = state;
    a.norm_out = norm_out;
    a.sc = ctx->scalars;
    for (int pass = 0; pass < (any_out ? 2 : 1); ++pass)
        for (int l = 0; l < launches; ++l) {
            fill(a, t, l * CAP, n - l * CAP < CAP ? n - l * CAP : CAP, (int)chunk);
            a.partial0 = l * grid;
            a.last = l == launches - 1;
            KernelScope scope(ctx, SAMA_K_CLIP, -1, st);
            const cudaError_t e = pass == 0 ? launch_dependent(grad_norm_kernel<CAP>, dim3(grid), dim3(kClipThreads), 0, st, a)
                                            : launch_dependent(grad_scale_kernel<CAP>, dim3(grid), dim3(kClipThreads), 0, st, a);
            if (e != cudaSuccess) return e;
        }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_clip_grads(sama_ctx* ctx, const sama_tensor_t* t, int n, float max_norm, float* norm_out,
                              cudaStream_t st) {
    int64_t total = 0;
    bool any_out = false;
    for (int i = 0; i < n; ++i) {
        total += t[i].n;
        any_out = any_out || (t[i].out && t[i].n > 0);
    }
    ClipState* state = &ctx->scalars->clip;
    if (n <= kCapSmall) return run_clip<kCapSmall>(ctx, t, n, total, any_out, max_norm, norm_out, state, st);
    return run_clip<kCapLarge>(ctx, t, n, total, any_out, max_norm, norm_out, state, st);
}

}  // namespace sama
