// Global gradient norm over many tensors, and clipping.
//
//   norm = sqrt( sum over tensors i and elements j of g_ij^2 ),   c = min(1, max_norm / norm),   out_ij = c g_ij
//
// Bound by memory traffic.  The tensors' addresses, lengths and types travel in the kernel's parameters (no copy, no
// plan on the device), and each block takes an equal, contiguous share of the elements of all tensors together, cut
// into chunks that never cross a tensor.  Squares are summed in double: a square of any fp32 or bf16 value neither
// overflows nor vanishes there, and the partial sums of the blocks are added in a fixed order.  (The conversion
// instruction to double runs at four values per cycle and SM, a third of what bf16 gradients arrive at; integer
// operations put the bits of a normal fp32 value where a double has them, see sum_group.)
//
// Two launches, norm and scaling; the second goes through each block's share backwards, in up to eight blocks, so that what the
// first read last comes out of L2 and the stores of one block do not wait for another's loads.  110 M bf16 elements into
// the flat fp32 vector (221 MB read twice, 440 MB written) 149 us, 355 M fp32 elements (1.42 GB read twice, 1.42 GB
// written) 670 us, 6.4 TB/s.
//
// Up to 2^19 elements in at most 112 tensors, where launches are all that counts, one cluster of 16 CTAs does both, a warp
// at a time to a chunk, so that a hundred small tensors are nearly as quick as one.  Measured against the two launches:
// 203,530 elements in 4 tensors 6.3 us (11), 500,000 in 4 8.6 (13) and in 100 10.8 (14); beyond, 1,040,000 in 4 13.3 (13.0)
// and in 100 17 (14).  With more tensors than 112, finding a warp's tensor in 31 KB of cold parameters eats the gain
// (370 tensors, 300,000 elements: 14.1 against 13.9).  (Its 1024 threads have 64 registers each and spill 24 bytes; the two
// kernels of the other way spill nothing.)
#include <cmath>
#include <type_traits>

#include "num_types.h"
#include "sama_internal.h"

namespace sama {

namespace {

constexpr int kClipThreads = 256;
constexpr int kLane = 16;              // bytes per thread and access
constexpr int kChunkUnit = 8 * 1024;   // chunks are multiples of this many elements: aligned shares for every type
constexpr int kCapSmall = 112, kCapLarge = 960;  // tensors of one launch: 3.6 KB and 31 KB of parameters
constexpr int kFewElements = 1 << 19, kFewCtas = 16, kFewThreads = 1024, kFewWarps = kFewCtas * kFewThreads / 32;
constexpr int kFewChunk = 512;   // a round of a warp's loads

struct ClipEntry {
    const void* in;
    void* out;
    int64_t n;
    int32_t first_chunk;
    uint8_t dtype, out_dtype, in_vec, out_vec;  // *_vec: the address is 16-byte aligned
};
template <int CAP>
struct ClipArgs {
    int n_entries, n_chunks, chunk;   // chunk: elements, a multiple of kChunkUnit
    int n_partials, partial0;         // all launches' block partials, and where this launch's begin
    int last;                         // this launch adds them up
    int parts;                        // scaling blocks per share
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
template <int THREADS>
__device__ __forceinline__ double clip_block_sum(double v, double* smem) {
    v = clip_warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
    __syncthreads();
    double t = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < THREADS / 32; ++w) t += smem[w];
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

// A normal fp32 value's magnitude as a double: exponent re-biased, mantissa moved.  Zero and subnormal values come out
// below 2^-126, infinities and NaN at 2^128 and above, where no finite value's does.
__device__ __forceinline__ double magnitude(uint32_t bits) {
    return __hiloint2double((int)(((bits & 0x7fffffffu) >> 3) + 0x38000000u), (int)(bits << 29));
}
// Adds the squares of 16 bytes of values to acc, and their bits (without the sign) to any.
template <typename T>
__device__ __forceinline__ void sum_group(const uint4& x, double* acc, uint32_t& any) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) {
            const double m = magnitude(w[j]);
            acc[j & 1] = fma(m, m, acc[j & 1]);
            any |= w[j] & 0x7fffffffu;
        } else if constexpr (std::is_same<T, __half>::value) {
            const float2 f = unpack2<T>(w[j]);   // (a subnormal fp16 value is a normal fp32 one)
            const double m0 = magnitude(__float_as_uint(f.x)), m1 = magnitude(__float_as_uint(f.y));
            acc[0] = fma(m0, m0, acc[0]);
            acc[1] = fma(m1, m1, acc[1]);
            any |= w[j] & 0x7fff7fffu;
        } else {
            // the low mantissa bits of a bf16 value are zero, so the double's low word is
            const double m0 = __hiloint2double((int)(((w[j] & 0x7fffu) << 13) + 0x38000000u), 0);
            const double m1 = __hiloint2double((int)(((w[j] & 0x7fff0000u) >> 3) + 0x38000000u), 0);
            acc[0] = fma(m0, m0, acc[0]);
            acc[1] = fma(m1, m1, acc[1]);
            any |= w[j] & 0x7fff7fffu;
        }
    }
}

// This thread's share of a chunk: sum of squares of n elements, THREADS threads, neighbouring threads on neighbouring
// 16 bytes (or elements, where the tensor starts at an odd address).  (Ordinary loads, not the read-only path: the one-cluster
// kernel may write the same tensor afterwards.)
template <typename T, int THREADS>
__device__ __forceinline__ double chunk_sumsq(const T* p, int n, bool vec, int tid) {
    constexpr int PER = kLane / sizeof(T), U = 4;
    double sum = 0.0;
    const int groups = vec ? n / PER : 0;
    if (vec) {
        double acc[2] = {0.0, 0.0};
        uint32_t any = 0;
        const uint4* q = reinterpret_cast<const uint4*>(p);
#pragma unroll 1
        for (int i = tid; i < groups; i += U * THREADS) {
            uint4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = i + u * THREADS < groups ? q[i + u * THREADS] : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int u = 0; u < U; ++u) sum_group<T>(v[u], acc, any);
        }
        sum = acc[0] + acc[1];
        // Values that are not finite (2^256 and above: at least 2^254 in a share), or so small that what zeros and
        // subnormals add could count (below 2^-245 in a share): once more with the converting instruction.  A share of
        // zeros is 0.
        if (any == 0) {
            sum = 0.0;
        } else if (!(sum < 2.894802230932905e76) || sum < 6.525304467998525e-55) {
            sum = 0.0;
#pragma unroll 1
            for (int i = tid; i < groups; i += THREADS)
#pragma unroll 1
                for (int j = 0; j < PER; ++j) {
                    const double x = (double)to_float(p[(int64_t)i * PER + j]);
                    sum = fma(x, x, sum);
                }
        }
    }
    constexpr int W = 8;
#pragma unroll 1
    for (int i = groups * PER + tid; i < n; i += W * THREADS) {
        float v[W];
#pragma unroll
        for (int u = 0; u < W; ++u) v[u] = i + u * THREADS < n ? to_float(p[i + u * THREADS]) : 0.f;
#pragma unroll
        for (int u = 0; u < W; ++u) sum = fma((double)v[u], (double)v[u], sum);
    }
    return sum;
}
template <int THREADS>
__device__ __forceinline__ double entry_sumsq(const ClipEntry& e, int64_t at, int n, int tid) {
    if (e.dtype == SAMA_F32) return chunk_sumsq<float, THREADS>(static_cast<const float*>(e.in) + at, n, e.in_vec, tid);
    if (e.dtype == SAMA_BF16) return chunk_sumsq<__nv_bfloat16, THREADS>(static_cast<const __nv_bfloat16*>(e.in) + at, n, e.in_vec, tid);
    return chunk_sumsq<__half, THREADS>(static_cast<const __half*>(e.in) + at, n, e.in_vec, tid);
}

// min(1, max_norm / norm), or 0 and the status bit for a norm that is not finite.
__device__ __forceinline__ double clip_factor(double sum, float max_norm, float* norm_out, int32_t* status) {
    const double norm = sqrt(sum);
    if (norm_out) *norm_out = (float)norm;
    if (!isfinite(norm)) {
        atomicOr(status, (int)SAMA_DEV_NONFINITE_GRAD);
        return 0.0;
    }
    return norm > (double)max_norm ? (double)max_norm / norm : 1.0;
}

// The factor.  Below 2^-100 it may leave fp32's normal range (a limit of 1e-30 on a norm of 1e38), where only double
// still holds it; 0 marks a norm that is not finite, for which zeros are written whatever the gradients are.  Neither
// is worth a fast path; `plain` is every other case.
struct Factor {
    float f;
    double d;
    bool plain;
    __device__ explicit Factor(double c) : f((float)c), d(c), plain(c >= 7.888609052210118e-31) {}
    __device__ __forceinline__ float slow(float x) const { return d == 0.0 ? 0.f : (float)((double)x * d); }
};

// Four or eight consecutive values, 8 or 16 bytes: loads and stores that are both contiguous over a warp.
template <typename T, int N>
__device__ __forceinline__ void get_few(const T* p, float* v) {
    if constexpr (sizeof(T) == 2 && N == 4) {
        const uint2 x = __ldcs(reinterpret_cast<const uint2*>(p));
        const float2 a = unpack2<T>(x.x), b = unpack2<T>(x.y);
        v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
    } else {
        load_n<T, N>(p, v);
    }
}
template <typename T, int N>
__device__ __forceinline__ void put_few(T* p, const float* v) {
    if constexpr (sizeof(T) == 2 && N == 4) __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3])));
    else store_n<T, N, true>(p, v);
}
template <typename T, typename TO, int THREADS>
__device__ __forceinline__ void chunk_scale(const T* p, TO* q, int n, bool vec, Factor by, int tid) {
    constexpr int PER = sizeof(T) == 2 && sizeof(TO) == 2 ? 8 : 4, U = 32 / PER;
    if (!by.plain) {
#pragma unroll 1
        for (int i = tid; i < n; i += THREADS) q[i] = from_float<TO>(by.slow(to_float(p[i])));
        return;
    }
    const float f = by.f;
    const int groups = vec ? n / PER : 0;
    // (whole rounds without conditions, then what is left: conditions on every access cost hundreds of spilled bytes)
    auto round = [&](auto count, int i) {
        constexpr int R = decltype(count)::value;
        float x[R][PER];
#pragma unroll
        for (int u = 0; u < R; ++u) get_few<T, PER>(p + (int64_t)(i + u * THREADS) * PER, x[u]);
#pragma unroll
        for (int u = 0; u < R; ++u) {
#pragma unroll
            for (int j = 0; j < PER; ++j) x[u][j] *= f;
            put_few<TO, PER>(q + (int64_t)(i + u * THREADS) * PER, x[u]);
        }
    };
    int i = tid;
#pragma unroll 1
    for (; i + (U - 1) * THREADS < groups; i += U * THREADS) round(std::integral_constant<int, U>(), i);
#pragma unroll 1
    for (; i + 3 * THREADS < groups; i += 4 * THREADS) round(std::integral_constant<int, 4>(), i);
#pragma unroll 1
    for (; i < groups; i += THREADS) round(std::integral_constant<int, 1>(), i);
    constexpr int W = 8;
    i = groups * PER + tid;
#pragma unroll 1
    for (; i + (W - 1) * THREADS < n; i += W * THREADS) {
        float v[W];
#pragma unroll
        for (int u = 0; u < W; ++u) v[u] = to_float(p[i + u * THREADS]);
#pragma unroll
        for (int u = 0; u < W; ++u) q[i + u * THREADS] = from_float<TO>(v[u] * f);
    }
#pragma unroll 1
    for (; i < n; i += THREADS) q[i] = from_float<TO>(to_float(p[i]) * f);
}
template <typename T, int THREADS>
__device__ __forceinline__ void scale_from(const ClipEntry& e, int64_t at, int n, const Factor& by, int tid) {
    const T* p = static_cast<const T*>(e.in) + at;
    const bool vec = e.in_vec && e.out_vec;
    if (e.out_dtype == SAMA_F32) chunk_scale<T, float, THREADS>(p, static_cast<float*>(e.out) + at, n, vec, by, tid);
    else if (e.out_dtype == SAMA_BF16) chunk_scale<T, __nv_bfloat16, THREADS>(p, static_cast<__nv_bfloat16*>(e.out) + at, n, vec, by, tid);
    else chunk_scale<T, __half, THREADS>(p, static_cast<__half*>(e.out) + at, n, vec, by, tid);
}
template <int THREADS>
__device__ __forceinline__ void entry_scale(const ClipEntry& e, int64_t at, int n, const Factor& by, int tid) {
    if (!e.out || (e.out == e.in && by.f == 1.f)) return;   // nothing to write
    if (e.dtype == SAMA_F32) scale_from<float, THREADS>(e, at, n, by, tid);
    else if (e.dtype == SAMA_BF16) scale_from<__nv_bfloat16, THREADS>(e, at, n, by, tid);
    else scale_from<__half, THREADS>(e, at, n, by, tid);
}

template <int CAP>
__global__ void __launch_bounds__(kClipThreads, 4)
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
            acc += entry_sumsq<kClipThreads>(e, at, (int)min((int64_t)a.chunk, e.n - at), threadIdx.x);
        }
    }
    const double total = clip_block_sum<kClipThreads>(acc, smem);
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
    const double sum = clip_block_sum<kClipThreads>(v, smem);
    if (threadIdx.x == 0) {
        a.sc->counter = 0u;
        if (a.last) a.state->factor = clip_factor(sum, a.max_norm, a.norm_out, &a.sc->status);
    }
}

template <int CAP>
__global__ void __launch_bounds__(kClipThreads, 4)
grad_scale_kernel(const __grid_constant__ ClipArgs<CAP> a) {
    pdl_trigger();
    pdl_wait();
    const Factor by(a.state->factor);
    // a.parts blocks for each of the norm's, the last parts of all shares first: those are in L2
    const int shares = gridDim.x / a.parts, share = blockIdx.x % shares, part = a.parts - 1 - blockIdx.x / shares;
    const int first = (int)((int64_t)a.n_chunks * share / shares), n = (int)((int64_t)a.n_chunks * (share + 1) / shares) - first;
    const int c0 = first + (int)((int64_t)n * part / a.parts), c1 = first + (int)((int64_t)n * (part + 1) / a.parts);
    if (c0 >= c1) return;
    int k = entry_of(a, c1 - 1);
    for (int c = c1 - 1; c >= c0; --c) {
        while (a.e[k].first_chunk > c) --k;
        const ClipEntry& e = a.e[k];
        const int64_t at = (int64_t)(c - e.first_chunk) * a.chunk;
        entry_scale<kClipThreads>(e, at, (int)min((int64_t)a.chunk, e.n - at), by, threadIdx.x);
    }
}

// Both in one cluster of kFewCtas CTAs, whose warps take chunks in turn: hundreds of small tensors are as quick as one.
__global__ void __launch_bounds__(kFewThreads)
grad_clip_few_kernel(const __grid_constant__ ClipArgs<kCapSmall> a) {
    __shared__ double smem[kFewThreads / 32], total, factor;
    pdl_trigger();
    pdl_wait();
    const uint32_t rank = blockIdx.x;
    const int lane = threadIdx.x & 31, first = (int)rank + kFewCtas * (int)(threadIdx.x >> 5);
    double acc = 0.0;
    for (int c = first; c < a.n_chunks; c += kFewWarps) {
        const ClipEntry& e = a.e[entry_of(a, c)];
        const int64_t at = (int64_t)(c - e.first_chunk) * a.chunk;
        acc += entry_sumsq<32>(e, at, (int)min((int64_t)a.chunk, e.n - at), lane);
    }
    const double mine = clip_block_sum<kFewThreads>(acc, smem);
    if (threadIdx.x == 0) total = mine;
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (threadIdx.x < 32) {
        double v = 0.0;
        if (threadIdx.x < kFewCtas) {
            uint32_t addr;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"((uint32_t)__cvta_generic_to_shared(&total)), "r"(threadIdx.x));
            asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(addr) : "memory");
        }
        v = clip_warp_sum(v);
        if (threadIdx.x == 0) {
            factor = clip_factor(v, a.max_norm, rank == 0 ? a.norm_out : nullptr, &a.sc->status);
        }
    }
    // no CTA leaves before all have read its total
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    const Factor by(factor);
    for (int c = first; c < a.n_chunks; c += kFewWarps) {
        const ClipEntry& e = a.e[entry_of(a, c)];
        const int64_t at = (int64_t)(c - e.first_chunk) * a.chunk;
        entry_scale<32>(e, at, (int)min((int64_t)a.chunk, e.n - at), by, lane);
    }
}

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
    // enough chunks for every block to get an even share, few enough for a block's bookkeeping
    int64_t chunk = total / ((int64_t)ctx->sm_count * 4 * 8) / kChunkUnit * kChunkUnit;
    if (chunk < kChunkUnit) chunk = kChunkUnit;
    if (chunk > 4 * kChunkUnit) chunk = 4 * kChunkUnit;
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
            // A block per chunk of a share, up to eight.  With 1, 2, 4, 8 and 16: 355 M fp32 elements 704, 699, 676, 670, 665 us,
            // 110 M bf16 elements into fp32 158, 155, 149, 147, 146; 8 M fp32 elements, which have one or two chunks per share,
            // 17.6, 17.9, 18.4, 20.2, 25.2.
            a.parts = a.n_chunks / grid;
            a.parts = a.parts < 1 ? 1 : a.parts > 8 ? 8 : a.parts;
            KernelScope scope(ctx, SAMA_K_CLIP, -1, st);
            const cudaError_t e = pass == 0 ? launch_dependent(grad_norm_kernel<CAP>, dim3(grid), dim3(kClipThreads), 0, st, a)
                                            : launch_dependent(grad_scale_kernel<CAP>, dim3(grid * a.parts), dim3(kClipThreads), 0, st, a);
            if (e != cudaSuccess) return e;
        }
    return cudaSuccess;
}

cudaError_t run_few(sama_ctx* ctx, const sama_tensor_t* t, int n, int64_t total, float max_norm, float* norm_out, cudaStream_t st) {
    ClipArgs<kCapSmall> a;
    // an equal share for every warp, in whole rounds of its loads
    fill(a, t, 0, n, total <= kFewWarps * kFewChunk ? kFewChunk : (int)((total + kFewWarps * kFewChunk - 1) / (kFewWarps * kFewChunk)) * kFewChunk);
    a.max_norm = max_norm;
    a.norm_out = norm_out;
    a.sc = ctx->scalars;
    if (!ctx->clip_ready) {
        const cudaError_t e = cudaFuncSetAttribute(grad_clip_few_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        ctx->clip_ready = 1;
    }
    KernelScope scope(ctx, SAMA_K_CLIP, -1, st);
    return launch_clustered(kFewCtas, grad_clip_few_kernel, dim3(kFewCtas), dim3(kFewThreads), 0, st, a);
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
    if (total <= kFewElements && n <= kCapSmall) return run_few(ctx, t, n, total, max_norm, norm_out, st);
    if (n <= kCapSmall) return run_clip<kCapSmall>(ctx, t, n, total, any_out, max_norm, norm_out, state, st);
    return run_clip<kCapLarge>(ctx, t, n, total, any_out, max_norm, norm_out, state, st);
}

}  // namespace sama
