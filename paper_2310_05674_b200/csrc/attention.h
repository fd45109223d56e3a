// What the attention kernels share: the packed texts, how a block finds its own, what a query sees, and the scores.
#pragma once
#include <type_traits>

#include "attention_sizes.h"
#include "num_types.h"
#include "sama_internal.h"
#include "tc_ptx.h"

namespace sama {

constexpr int kAttnRows = 128;   // rows of a score tile: the lanes of tensor memory

struct AttnShape {
    const int32_t *q_starts, *k_starts, *prefix;
    const float* slopes;
    int32_t* status;
    int n_texts, n_q, n_k, heads, kv_heads, group, dim, causal;   // group: heads per key head
    float scale, cap;
};

struct AttnOperands {
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    int dtype;
};
// attention_fwd.cu, attention_bwd.cu
cudaError_t launch_attention(sama_ctx* ctx, const AttnShape& a, const AttnOperands& op, void* out, float* lse, cudaStream_t st);
size_t attention_grad_workspace(const AttnShape& a);
cudaError_t launch_attention_grad(sama_ctx* ctx, const AttnShape& a, const AttnOperands& op, const void* out, const float* lse,
                                  const void* dout, void* dq, void* dk, void* dv, void* ws, cudaStream_t st);


struct PagedShape {
    const int32_t *page_table, *lengths;
    const float* slopes;
    int32_t* status;
    int64_t n_pages, page_stride;
    int n_seqs, max_pages, page_size, heads, kv_heads, group, dim;
    float scale, cap;
};
// attention_paged.cu
size_t paged_workspace(const sama_ctx* ctx);
cudaError_t launch_paged(sama_ctx* ctx, const PagedShape& a, int dtype, const void* q, const void* k_new, const void* v_new,
                         void* k_cache, void* v_cache, void* out, void* ws, cudaStream_t st);

enum AttnCap { kNoCap, kCap, kWideCap };
inline AttnCap attn_cap(float cap) { return cap <= 0.f ? kNoCap : cap <= 64.f ? kCap : kWideCap; }

#ifdef __CUDACC__

__device__ __forceinline__ int attn_start(const int32_t* starts, int i, int n) { return min(max(starts[i], 0), n); }

// Tiles of TILE rows are counted so that a text's first is number starts[t] / TILE + t: texts leave gaps of at most one
// tile, there are n / TILE + n_texts numbers in all, and a block finds the text of its number by search, without a pass
// over the texts before it.  All lanes of a warp probe at a time.  Returns the text, or -1; `tile`: number within it.
template <int TILE>
__device__ __forceinline__ int attn_find(const int32_t* starts, int n_texts, int n, int slot, int* tile) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = n_texts, first = 0;
    do {
        const int step = (hi - lo + 31) / 32, t = lo + lane * step;
        const int at = t < hi ? attn_start(starts, t, n) / TILE + t : 0x7fffffff;
        const uint32_t before = __ballot_sync(0xffffffffu, at <= slot);
        if (!(before & 1u)) return -1;   // (before the first text; or starts that fall)
        const int last = 31 - __clz(before);
        first = __shfl_sync(0xffffffffu, at, last);
        lo += last * step;
        hi = min(hi, lo + step);
    } while (hi - lo > 1);
    *tile = slot - first;
    return lo;
}
// Starts that fall or lie outside are clamped, here and wherever they are used, and reported.
__device__ __forceinline__ AttnText attn_text(const AttnShape& a, int t) {
    AttnText x;
    x.q0 = attn_start(a.q_starts, t, a.n_q);
    x.lq = max(attn_start(a.q_starts, t + 1, a.n_q) - x.q0, 0);
    x.k0 = attn_start(a.k_starts, t, a.n_k);
    x.lk = max(attn_start(a.k_starts, t + 1, a.n_k) - x.k0, 0);
    x.prefix = a.prefix ? min(max(a.prefix[t], 0), x.lk) : 0;
    return x;
}
__device__ __forceinline__ void attn_check_starts(const AttnShape& a) {
    bool bad = false;
    for (int i = threadIdx.x; i <= a.n_texts; i += blockDim.x) {
        const int q = a.q_starts[i], k = a.k_starts[i];
        bad |= q < 0 || q > a.n_q || k < 0 || k > a.n_k || (i > 0 && (a.q_starts[i - 1] > q || a.k_starts[i - 1] > k));
    }
    if (bad) atomicOr(a.status, (int)SAMA_DEV_BAD_INDEX);
}

// Two fp32 operations in one instruction: the scores' arithmetic takes most of the issue slots.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// tanh(z) = 1 - 2 / (1 + exp 2z) has an absolute error of two units in the last place of 1 (the hardware's own approximation
// 2^-11, a hundredth of a weight at a cap of 30), which is a relative one of 2.5e-7 beyond 0.75.  Below, tanh is a polynomial,
// z p(z^2) with p of degree 4 through tanh(z) / z at the Chebyshev points of [0, 0.75^2]: 7e-7 of tanh(z).  The first takes two of
// the three results of the special-function unit per score (16 a cycle and SM), so it is left out where all scores of a
// warp's tile are within 0.75 caps (and, in the backward pass, seen).  Elsewhere it serves for all of them up to a cap of 64, where its error
// is 1e-5 of a weight at most; with larger caps (kernels of their own) each score has the form that is good for it.
__device__ __forceinline__ float attn_tanh(float z) { return fmaf(-2.f, fast_rcp(1.f + fast_exp2(2.f * kLog2e * z)), 1.f); }
constexpr float kTanhNear = 0.75f;
enum { kNear, kFar, kAny };
struct AttnTanh {   // times `factor`, of `scale` times its argument
    float k[5], scale, factor;
    __device__ __forceinline__ AttnTanh(float scale, float factor) : scale(scale), factor(factor) {
        const float c[5] = {0.999999404f, -0.333281934f, 0.132584617f, -0.0500416085f, 0.0129166516f}, s2 = scale * scale;
        float f = factor * scale;
#pragma unroll
        for (int i = 0; i < 5; ++i) { k[i] = c[i] * f; f *= s2; }
    }
    __device__ __forceinline__ bool is_near(float x) const { return fabsf(x) * scale <= kTanhNear; }
    __device__ __forceinline__ float2 near(float2 x) const {
        const float2 u = mul2(x, x);
        return mul2(x, fma2(fma2(fma2(fma2(both(k[4]), u, both(k[3])), u, both(k[2])), u, both(k[1])), u, both(k[0])));
    }
    // FORM: kNear, kFar, kAny
    template <int FORM> __device__ __forceinline__ float2 of(float2 x) const { return FORM == kNear ? near(x) : FORM == kFar ? far(x) : any(x); }
    __device__ __forceinline__ float2 far(float2 x) const { return make_float2(factor * attn_tanh(x.x * scale), factor * attn_tanh(x.y * scale)); }
    __device__ __forceinline__ float2 any(float2 x) const {
        const float2 y = near(x), z = far(x);
        return make_float2(is_near(x.x) ? y.x : z.x, is_near(x.y) ? y.y : z.y);
    }
};
// The largest of N values, in eight chains: one would wait for each result before the next.
template <int N, typename F>
__device__ __forceinline__ float attn_max(F&& value) {
    float m[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) m[i] = value(i);
#pragma unroll
    for (int k = 8; k < N; k += 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = fmaxf(m[i], value(k + i));
    return fmaxf(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), fmaxf(fmaxf(m[4], m[5]), fmaxf(m[6], m[7])));
}

// One lane of the warp, the same each time.
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}

// D (fp32) += A B^T with A, 128 rows of 16-bit values two to a column, in tensor memory.
__device__ __forceinline__ void umma16_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// As make_desc, for a tile whose rows run along the contraction (MN-major): 64 values of N per row of 128 bytes, 8 rows to
// a swizzle block, the next 64 values of N `rows` rows further on.
__device__ __forceinline__ uint64_t attn_desc_mn(uint32_t saddr, int rows) {
    return (uint64_t)((saddr & 0x3FFFF) >> 4) | ((uint64_t)((rows * 128) >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// 32 accumulator columns of this warp's 32 rows; tmem_wait_ld has to follow.
__device__ __forceinline__ void tmem_ld32_nowait(uint32_t taddr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 16 columns of this warp's 32 rows, to tensor memory; tmem_wait_st has to follow.
__device__ __forceinline__ void tmem_st16_nowait(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr));
}
// 32 lanes' rows of a tile in shared memory, 16 bytes at a time: a lane writes its own row (`mine`, in the tile) from column
// `col`, 8 values.  Swizzled: the lanes of a warp write to different banks, here and where whole rows are read.
template <int D>
__device__ __forceinline__ uint32_t attn_chunk(uint32_t tile, int row, int chunk) { return tile + (uint32_t)row * (D * 2) + (uint32_t)((chunk ^ (row & 7)) << 4); }
template <typename T, int D>
__device__ __forceinline__ void attn_stage(uint32_t tile, int mine, int col, const float* v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(attn_chunk<D>(tile, mine, col / 8)), "r"(pack2<T>(v[0], v[1])),
                 "r"(pack2<T>(v[2], v[3])), "r"(pack2<T>(v[4], v[5])), "r"(pack2<T>(v[6], v[7])) : "memory");
}
// The tile's first `rows` rows go to memory, rows `ld` elements apart, by warps of which this is `warp`: a row's columns by
// lanes next to one another.  (With each lane storing its own row, 2 KB from the next, the stores of an encoder's dK and dV
// took 3500 of a CTA's 28,000 cycles.)
template <typename T, int D, int WARPS>
__device__ __forceinline__ void attn_unstage(uint32_t tile, int rows, int dim, T* to, int64_t ld, int warp) {
    constexpr int LANES = D / 8, AT_ONCE = 32 / LANES, EACH = kAttnRows / WARPS;
    const int chunk = (int)(threadIdx.x & 31) % LANES, r0 = warp * EACH + (int)(threadIdx.x & 31) / LANES;
#pragma unroll
    for (int i = 0; i < EACH; i += AT_ONCE) {
        const int r = r0 + i;
        uint4 v;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(attn_chunk<D>(tile, r, chunk)) : "memory");
        if (r < rows && 8 * chunk < dim) *reinterpret_cast<uint4*>(to + r * ld + 8 * chunk) = v;
    }
}
// Rows [from, rows) of a tile of COLS 64-column blocks become zeros: rows of another text, whose values must not meet
// weights of 0 in a product.
// Shared out among `warps` warps, of which this is `warp`.
template <int COLS>
__device__ __forceinline__ void attn_zero_rows(uint32_t tile, int from, int rows, int warp, int warps) {
    const int n = (rows - from) * 8;   // 16-byte chunks of a block
    for (int i = 32 * warp + (threadIdx.x & 31); i < n * COLS; i += 32 * warps) {
        const int block = i / n, at = i - block * n;
        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + (uint32_t)(block * rows + from) * 128u + 16u * at), "r"(0) : "memory");
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
}

#endif  // __CUDACC__

// Tensor map of [n][heads][dim] with rows `stride` elements apart: boxes of `rows` rows of one head's 64 columns.
inline bool attn_map(CUtensorMap* map, const void* p, int dtype, int dim, int heads, int64_t n, int64_t stride, int rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)n};
    const cuuint64_t strides[2] = {(cuuint64_t)dim * 2, (cuuint64_t)stride * 2};
    const cuuint32_t box[3] = {64, 1, (cuuint32_t)rows}, step[3] = {1, 1, 1};
    return fn(map, dtype == SAMA_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(p),
              dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace sama
