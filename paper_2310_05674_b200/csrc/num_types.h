// The element types of the text-model operators (sama_dtype): conversion to and from fp32, and 16-byte groups.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "sama.h"

namespace sama {

inline size_t dtype_size(int dtype) { return dtype == SAMA_F32 ? 4 : 2; }
inline bool dtype_valid(int dtype) { return dtype == SAMA_F32 || dtype == SAMA_BF16 || dtype == SAMA_F16; }

#ifdef __CUDACC__
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
// Rounds to nearest, ties to even.
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// Two adjacent values in one 32-bit register, the first in the low half.
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t v);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t v) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t v) {
    return __half22float2(*reinterpret_cast<const __half2*>(&v));
}

// N consecutive values as fp32 (N = 1, or a multiple of 16 bytes).  KEEP: data that will be read again.  (Ordinary loads:
// kernels start while the launch before them may still be writing what they will read, which is no case for the read-only path.)
template <typename T, int N, bool KEEP = false>
__device__ __forceinline__ void load_n(const T* p, float* v) {
    if constexpr (N == 1) {
        v[0] = to_float(*p);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const float4* q = reinterpret_cast<const float4*>(p) + i;
            const float4 x = KEEP ? *q : __ldcs(q);
            v[4 * i] = x.x; v[4 * i + 1] = x.y; v[4 * i + 2] = x.z; v[4 * i + 3] = x.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            const uint4* q = reinterpret_cast<const uint4*>(p) + i;
            const uint4 x = KEEP ? *q : __ldcs(q);
            const uint32_t r[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 f = unpack2<T>(r[j]);
                v[8 * i + 2 * j] = f.x;
                v[8 * i + 2 * j + 1] = f.y;
            }
        }
    }
}
// PASS: data that should not displace what is in L2.
template <typename T, int N, bool PASS = false>
__device__ __forceinline__ void store_n(T* p, const float* v) {
    if constexpr (N == 1) {
        *p = from_float<T>(v[0]);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const float4 x = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            float4* q = reinterpret_cast<float4*>(p) + i;
            if (PASS) __stcs(q, x); else *q = x;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            const uint4 x = make_uint4(pack2<T>(v[8 * i], v[8 * i + 1]), pack2<T>(v[8 * i + 2], v[8 * i + 3]),
                                       pack2<T>(v[8 * i + 4], v[8 * i + 5]), pack2<T>(v[8 * i + 6], v[8 * i + 7]));
            uint4* q = reinterpret_cast<uint4*>(p) + i;
            if (PASS) __stcs(q, x); else *q = x;
        }
    }
}
#endif

}  // namespace sama
