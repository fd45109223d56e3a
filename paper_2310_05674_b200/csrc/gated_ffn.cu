// Gated feed-forward block and its backward pass on the 5th-generation tensor cores, bf16 or fp16 operands, fp32 sums.
//
//   G = X Wg^T,  U = X Wu^T,  H = a(G) * U,  Y = H Wd^T
//   dH = dY Wd,  dG = dH * U * a'(G),  dU = dH * a(G)
//   dX = dG Wg + dU Wu,  dWg = dG^T X,  dWu = dU^T X,  dWd = dY^T H
//
// Five launches of one persistent kernel template, two forward and three backward:
//   gate-up   both projections of a tile of X in one pass: the tile of the right operand is half rows of Wg and half the
//             same rows of Wu, so one accumulator holds G and U of the same features side by side and the epilogue forms
//             H from registers.  G and U are stored only if a backward pass will want them.
//   down      Y = H Wd^T
//   d-hidden  dH = dY Wd, whose epilogue reads G and U and leaves dG, dU and H (formed again rather than kept)
//   d-input   dX as one product over the concatenated contraction (dG, dU) x (Wg, Wu)
//   d-weights the three weight gradients as one launch over the tiles of all three
// H, dG and dU are rounded to the operands' type between launches, as any operand of a 16-bit product has to be, and so are
// G and U where they are kept for the backward pass; every sum stays in fp32 until its one rounding on the way out.  The
// forward pass forms H from the unrounded sums, the backward pass forms it again from the rounded G and U: a last place of
// H against writing and reading another matrix of that size.  In fp16, what exceeds 65504 in any of them is infinite.
//
// Up to 16 tokens go another way, see ffn_few_kernel.
//
// Operands are read as they lie in memory: where the contraction runs along a matrix's rows, the tile is loaded and
// described to the tensor core "MN-major" instead of being transposed by a pass of its own.
//
// Roles of the 10 warps: warp 0 copies (TMA, 128-byte swizzle, 32 KB stages), warp 1 issues products, warps 2..9 read
// finished accumulators and bring them out through shared memory while the next tile is multiplied (two accumulators in
// tensor memory).  A CTA pair works on a 256 x 256 tile with cta_group::2 products; shapes with too few of those take
// 128 x 128 tiles on single CTAs, or share a tile's contraction.  Every wait is bounded: one that expires raises
// SAMA_DEV_TIMEOUT, stops the CTA's work, lets its copies land and exits.
//
// What bounds it (us on one B200, bf16): long contractions the tensor cores and the power limit (2048 tokens, 2048 x 5504,
// forward and backward 316, 1310 TFLOP/s; 4096 tokens, 4096 x 8192 1650 to 1950, by the card's temperature); short ones
// reading tensor memory, 64 bytes per cycle and SM, 2000 cycles for a pair's tile (64 tokens, 4096 x 8192: the weight
// gradients, 201 MB, 54); few tokens the weights' way from memory and the start and end of two launches (45 tokens, 4096 x
// 8192: 49, of which the weights' 201 MB at copy speed are 31); small models the launches (1024 tokens, 1024 x 2736: 89) and
// the host (128 tokens, 256 x 688: 29 on the device in a graph; the host takes 17 for its five launches and 25 tensor maps).
#include <type_traits>

#include "num_types.h"
#include "sama_internal.h"
#include "tc_ptx.h"

namespace sama {

namespace {

constexpr int BM = 128;         // rows of a CTA's share of the output tile
constexpr int BK = 64;          // contraction per stage: one 128-byte row of 16-bit values
constexpr int OPERAND = BM * BK * 2;              // bytes of either operand's share of a stage
constexpr int STAGE = 2 * OPERAND;
constexpr int EPI = 8;          // epilogue warps
constexpr int THREADS = 64 + 32 * EPI;

enum Mode { GATE_UP, PLAIN, D_HIDDEN };

// How a launch follows the one before it.  d-input and d-weights need d-hidden, not each other: d-input lets d-weights
// start once its own wait is over, and d-weights, which then finds d-hidden complete, waits for d-input at its very end
// only, so that whatever follows still finds both complete.  Its CTAs fill the SMs that d-input leaves or never used
// (2048 tokens, 2048 x 5504, forward and backward: 317 us against 322 one after the other).
enum Link { AFTER, LEADS, BESIDE };

// Staging of one epilogue warp: 32 rows of 64 columns, in 16 bits, or (d-hidden) in fp32.  Rows of 64 columns because the
// load and store units take a cycle per 128-byte line: with steps of 16 columns the d-hidden epilogue of a pair's tile
// was 25 % slower, although twice as many warps shared it.
//
// Units: a CTA pair on a 256 x 256 tile, a CTA on a 128 x 128 tile, or a cluster of 2, 4 or 8 CTAs on one 128 x 128 tile
// whose contraction they share.  The latter exchange sums through distributed shared memory: a warp's 32 x 64 block of
// the tile goes to the CTA that finishes it, which receives 64 KB in all and stages its output in the same place.
enum Unit { SINGLE, PAIRED, SHARED };
__host__ __device__ constexpr int staging_of(int mode, int unit) { return unit == SHARED || mode == D_HIDDEN ? 8192 : 4096; }
__host__ __device__ constexpr int stages_of(int mode, int unit) { return unit == SHARED || mode == D_HIDDEN ? 5 : 6; }
__host__ __device__ constexpr int smem_of(int mode, int unit) {
    return stages_of(mode, unit) * STAGE + EPI * staging_of(mode, unit) + 256 + 1024;
}


struct Problem {
    CUtensorMap a[2], b[2];     // [1]: the second part of the contraction, or (gate-up) the second right operand
    CUtensorMap o[3];           // outputs that can be written in aligned 16-byte groups
    int M, N;                   // rows and columns of the output (gate-up: features)
    int num_kb, kb_first;       // k-blocks, and how many of them the first maps cover
    int tiles_m, tiles_n, item0;
    void* out[3];
    const void* in[2];          // d-hidden: G and U, rows of whole aligned 16-byte groups
    int64_t ldo[3], ldi[2];
    int cols[3];                // columns of out[i] that may be written
    int vec_out;                // bit i: out[i] can be written in aligned 16-byte groups
};
template <int G>
struct alignas(64) Params {
    Problem p[G];
    // Tiles in the order of the work: `whole` of them, then the others in `split` parts of their contraction each.
    int n_items, whole, split, group_m, act;
    int link;
    float4* parts;      // sums of split tiles: [split tile][part][CTA of the tile][epilogue warp][64 columns / 4][32 rows]
    int* arrived;       // [split tile][CTA of the tile][epilogue warp]: parts stored, zero between launches
    int32_t* status;
};

// ---------------------------------------------------------------- PTX for 16-bit products

// D (fp32) += A B^T, 16 of the contraction per instruction.
__device__ __forceinline__ void umma16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma16_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// Instruction descriptor: fp32 accumulator (bit 4), operand type (bits 7 and 10: 0 fp16, 1 bf16; both the same),
// operands stored MN-major (bits 15, 16), N / 8 (bit 17), M / 16 (bit 24).
__host__ __device__ constexpr uint32_t idesc16(bool bf16, bool a_mn, bool b_mn, int m, int n) {
    return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
// Shared-memory descriptor of an MN-major tile with the 128-byte swizzle: rows of the contraction are 64 consecutive
// elements of M (or N), 128 bytes; 8 rows make a swizzle block of 1024 bytes (the stride offset); the next 64 elements
// of M lie BK rows further on (the leading offset).
__device__ __forceinline__ uint64_t make_desc_mn(uint32_t saddr) {
    return (uint64_t)((saddr & 0x3FFFF) >> 4) | ((uint64_t)((BK * 128) >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
// Into this CTA's shared memory, counted on the leader's barrier.
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, uint32_t leader_bar, int x, int y) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(map), "r"(leader_bar), "r"(x), "r"(y) : "memory");
}

// A block of rows from shared memory; what lies beyond the matrix is not written.
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int x, int y) {
    asm volatile(
        "cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];\n\tcp.async.bulk.commit_group;"
        ::"l"(map), "r"(src), "r"(x), "r"(y) : "memory");
}
// This thread's stores have read shared memory, or (ALL) have been made.
template <bool ALL>
__device__ __forceinline__ void tma_store_wait() {
    if (ALL) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    else asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}

// 16 accumulator columns of this warp's 32 rows, from and to tensor memory.
__device__ __forceinline__ void tmem_ld16_nowait(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float* v) {
    uint32_t r[16];
    tmem_ld16_nowait(taddr, r);
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_ld16x2(uint32_t a0, uint32_t a1, float* v0, float* v1) {
    uint32_t r0[16], r1[16];
    tmem_ld16_nowait(a0, r0);
    tmem_ld16_nowait(a1, r1);
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) { v0[i] = __uint_as_float(r0[i]); v1[i] = __uint_as_float(r1[i]); }
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float* v) {
    uint32_t r[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(v[i]);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr));
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// ---------------------------------------------------------------- activations

// 2^x and 1 / x to two units in the last place; results below the normal range are 0.
__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float fast_rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.44269504f;

// a(x), and with GRAD its derivative.
template <int ACT, bool GRAD>
__device__ __forceinline__ float2 activate(float x) {
    if constexpr (ACT == SAMA_ACT_SILU) {
        const float s = fast_rcp(1.f + fast_exp2(-kLog2e * x));   // the power overflows to infinity for x < -88: s = 0, as it should
        return make_float2(x * s, GRAD ? s * fmaf(x, 1.f - s, 1.f) : 0.f);
    } else if constexpr (ACT == SAMA_ACT_RELU) {
        return make_float2(x > 0.f ? x : (x != x ? x : 0.f), x > 0.f ? 1.f : 0.f);
    } else if constexpr (ACT == SAMA_ACT_GELU) {
        // The normal distribution function by Abramowitz and Stegun 7.1.26, absolute error 7.5e-8, whose exponential is
        // the density's: p(-|x|) = poly(t) exp(-x^2 / 2) / 2 with t = 1 / (1 + 0.3275911 |x| / sqrt 2).
        const float e = fast_exp2(-0.5f * kLog2e * x * x);
        const float t = fast_rcp(fmaf(0.3275911f * 0.70710678f, fabsf(x), 1.f));
        float q = fmaf(1.061405429f, t, -1.453152027f);
        q = fmaf(q, t, 1.421413741f);
        q = fmaf(q, t, -0.284496736f);
        q = fmaf(q, t, 0.254829592f);
        q *= 0.5f * t * e;
        const float p = x > 0.f ? 1.f - q : q;
        return make_float2(x * p, GRAD ? fmaf(x * 0.39894228f, e, p) : 0.f);
    } else {
        // 0.5 (1 + tanh z) = 1 / (1 + exp(-2 z))
        const float z2 = 1.59576912f * x * fmaf(0.044715f * x, x, 1.f);
        const float p = fast_rcp(1.f + fast_exp2(-kLog2e * z2));
        // (the slope of z is bounded: where x^2 overflows, p (1 - p) is 0 and so is their product)
        return make_float2(x * p, GRAD ? fmaf(x * p * (1.f - p), 1.59576912f * fminf(fmaf(0.134145f * x, x, 1.f), 1e30f), p) : 0.f);
    }
}

// Runs fn with the activation as a constant, so that the choice is made once and not per element.
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& fn) {
    if (act == SAMA_ACT_SILU) fn(std::integral_constant<int, SAMA_ACT_SILU>());
    else if (act == SAMA_ACT_GELU) fn(std::integral_constant<int, SAMA_ACT_GELU>());
    else if (act == SAMA_ACT_GELU_TANH) fn(std::integral_constant<int, SAMA_ACT_GELU_TANH>());
    else fn(std::integral_constant<int, SAMA_ACT_RELU>());
}

// ---------------------------------------------------------------- stores

// Writes a block of 32 rows x CU columns that a warp holds as packed pairs, one row per lane, in whole row segments:
// through `stg` with 16-byte chunks permuted by row, so that neither side has bank conflicts.  Rows of aligned 16-byte
// groups are fetched from there by the copy engine (the permutation is its 128- or 64-byte swizzle).
template <typename T, int CU>
__device__ __forceinline__ void store_rows(uint4* stg, const uint32_t* packed, const CUtensorMap* map, T* dst, int64_t ld,
                                           int row0, int rows, int col0, int cols, bool vec, int lane) {
    constexpr int LPR = CU / 8;  // 16-byte chunks of a row
    auto at = [](int r, int c) { return r * LPR + (c ^ (LPR == 8 ? (r & 7) : ((r >> 1) & 3))); };
    static_assert(CU == 64 || CU == 32, "rows of 128 or 64 bytes");
    if (lane == 0) tma_store_wait<false>();
    __syncwarp();
#pragma unroll
    for (int c = 0; c < LPR; ++c)
        stg[at(lane, c)] = make_uint4(packed[4 * c], packed[4 * c + 1], packed[4 * c + 2], packed[4 * c + 3]);
    if (vec) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (vec) {
        if (lane == 0 && rows > 0 && col0 < cols) tma_store_2d(map, smem_u32(stg), col0, row0);
    } else {
        // rows that start anywhere: neighbouring lanes take neighbouring elements
        // Four values per lane, stored as two words that start on a 4-byte boundary: in a row that starts between two
        // words they begin one value further on, and the second takes its last value from the next lane.
        constexpr int LANES = CU / 4, ROWS = 32 / LANES;   // of a row, at a time
        const int k = lane % LANES;
        const uint2* s = reinterpret_cast<const uint2*>(stg);
#pragma unroll 2
        for (int r = lane / LANES; r < 32; r += ROWS) {
            const uint2 v = s[at(r, k >> 1) * 2 + (k & 1)];
            const uint32_t next = __shfl_down_sync(0xffffffffu, v.x, 1);
            if (r >= rows) continue;
            uint16_t* d = reinterpret_cast<uint16_t*>(dst) + (int64_t)(row0 + r) * ld + col0;
            const int left = cols - col0 - 4 * k;            // values from this lane's first on
            const bool odd = (reinterpret_cast<uintptr_t>(d) & 2u) != 0;
            d += 4 * k;
            if (left >= 5 || (left == 4 && !odd)) {
                if (!odd) {
                    reinterpret_cast<uint32_t*>(d)[0] = v.x;
                    reinterpret_cast<uint32_t*>(d)[1] = v.y;
                } else {
                    if (k == 0) d[0] = (uint16_t)v.x;
                    *reinterpret_cast<uint32_t*>(d + 1) = __funnelshift_r(v.x, v.y, 16);
                    if (k + 1 < LANES) *reinterpret_cast<uint32_t*>(d + 3) = __funnelshift_r(v.y, next, 16);
                    else d[3] = (uint16_t)(v.y >> 16);
                }
            } else {
                const uint32_t w[2] = {v.x, v.y};
                for (int j = odd && k > 0 ? 1 : 0; j < min(left, 4); ++j) d[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
            }
        }
    }
}

// Eight consecutive values of a row, zeros beyond `cols`.
template <typename T>
__device__ __forceinline__ uint4 load8(const T* p, int col, int cols, bool vec) {
    if (vec) return *reinterpret_cast<const uint4*>(p + col);
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p) + col;
    uint32_t r[4];
    if (col + 8 <= cols) {
        if ((reinterpret_cast<uintptr_t>(q) & 2u) == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) r[j] = reinterpret_cast<const uint32_t*>(q)[j];
        } else {   // the words around a value at an odd place, within the eight
            uint32_t w[5];
            w[0] = (uint32_t)*q << 16;
#pragma unroll
            for (int j = 0; j < 3; ++j) w[j + 1] = reinterpret_cast<const uint32_t*>(q + 1)[j];
            w[4] = q[7];
#pragma unroll
            for (int j = 0; j < 4; ++j) r[j] = __funnelshift_r(w[j], w[j + 1], 16);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t lo = col + 2 * j < cols ? q[2 * j] : 0, hi = col + 2 * j + 1 < cols ? q[2 * j + 1] : 0;
            r[j] = lo | (hi << 16);
        }
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// x / y for x >= 0, y > 0 and a quotient below 2^20: that of floats is off by one at most.  (Every role makes two per tile.)
__device__ __forceinline__ int quotient(int x, int y) {
    const int q = (int)((float)x * fast_rcp((float)y)), r = x - q * y;
    return r < 0 ? q - 1 : r >= y ? q + 1 : q;
}

// ---------------------------------------------------------------- the kernel

template <typename T, int MODE, int UNIT, bool A_MN, bool B_MN, int G>
__global__ void __launch_bounds__(THREADS, 1)
ffn_kernel(const __grid_constant__ Params<G> P) {
    constexpr bool PAIR = UNIT == PAIRED;
    constexpr int STAGES = stages_of(MODE, UNIT), STAGING = staging_of(MODE, UNIT);
    constexpr int BN = PAIR ? 256 : 128;                // accumulator columns
    constexpr int TN = MODE == GATE_UP ? BN / 2 : BN;   // output columns (features) of a tile
    constexpr int TM = PAIR ? 2 * BM : BM;
    constexpr uint32_t IDESC = idesc16(std::is_same<T, __nv_bfloat16>::value, A_MN, B_MN, TM, BN);
    constexpr uint32_t TMEM_COLS = 2 * BN;

    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;       // swizzled tiles need 1024-byte alignment
    const uint32_t staging = base + STAGES * STAGE;
    const uint32_t bars = staging + EPI * STAGING;
    auto full_bar = [&](int s) { return bars + 8u * s; };
    auto empty_bar = [&](int s) { return bars + 8u * (STAGES + s); };
    auto acc_full_bar = [&](int b) { return bars + 8u * (2 * STAGES + b); };
    auto acc_empty_bar = [&](int b) { return bars + 8u * (2 * STAGES + 2 + b); };
    const uint32_t tmem_slot = bars + 8u * (2 * STAGES + 4);
    volatile uint32_t* tmem_ptr_slot = reinterpret_cast<volatile uint32_t*>(smem_raw + (tmem_slot - raw));
    volatile uint32_t* abort_flag = tmem_ptr_slot + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
    const int unit = (int)blockIdx.x / (PAIR ? 2 : 1), n_units = (int)gridDim.x / (PAIR ? 2 : 1);

    // Work item -> problem, tile and range of k-blocks.  Tiles that run together cover group_m row tiles of a few column
    // tiles, so that one wave's operands come out of L2.
    struct Work { int tm, tn, kb0, kb1, part, split_tile; };   // split_tile < 0: a whole tile
    auto locate = [&](int item, Work& w) -> const Problem& {
        const int over = item - P.whole;
        int tile = item;
        w.split_tile = -1;
        if (over >= 0) {
            w.split_tile = quotient(over, P.split);
            w.part = over - w.split_tile * P.split;
            tile = P.whole + w.split_tile;
        }
        int g = 0;
#pragma unroll
        for (int i = 1; i < G; ++i)
            if (tile >= P.p[i].item0) g = i;
        const Problem& q = P.p[g];
        w.kb0 = 0;
        w.kb1 = q.num_kb;
        if (over >= 0) {
            w.kb0 = quotient(q.num_kb * w.part, P.split);
            w.kb1 = quotient(q.num_kb * (w.part + 1), P.split);
        }
        const int t = tile - q.item0, per_group = P.group_m * q.tiles_n, group = quotient(t, per_group), rem = t - group * per_group;
        const int first = group * P.group_m, size = min(P.group_m, q.tiles_m - first);
        w.tn = quotient(rem, size);
        w.tm = first + rem - w.tn * size;
        return q;
    };

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full_bar(b), 1);
            mbar_init(acc_empty_bar(b), EPI * (PAIR ? 2 : 1));
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        if (PAIR) tmem_alloc_pair(tmem_slot, TMEM_COLS); else tmem_alloc(tmem_slot, TMEM_COLS);
    }
    tc_fence_before();
    __syncthreads();
    if (UNIT != SINGLE) cluster_sync();  // the other CTAs run, and their barriers exist, before anything reaches them
    tc_fence_after();
    const uint32_t tmem_base = *tmem_ptr_slot;
    if (P.link == AFTER) pdl_trigger();
    if (P.link != BESIDE) pdl_wait();
    if (P.link != AFTER) pdl_trigger();

    auto raise_timeout = [&]() {
        *abort_flag = 1;
        atomicOr(P.status, (int)SAMA_DEV_TIMEOUT);
    };

    if (warp == 0) {
        // ---------------------------------------------------------- copies
        if (lane == 0) {
            int issued = 0, s = 0;
            uint32_t empty_parity = 1;
            bool ok = true;
            for (int item = unit; ok && item < P.n_items; item += n_units) {
                Work w;
                const Problem& q = locate(item, w);
                const int m0 = w.tm * TM + (int)rank * BM;
                const int n0 = w.tn * TN + (PAIR && MODE != GATE_UP ? (int)rank * BM : 0);
                for (int kb = w.kb0; kb < w.kb1; ++kb) {
                    if (issued >= STAGES && !mbar_wait(empty_bar(s), empty_parity, abort_flag)) { raise_timeout(); ok = false; break; }
                    const uint32_t sa = base + s * STAGE, sb = sa + OPERAND;
                    const int part = MODE != GATE_UP && kb >= q.kb_first;
                    const int k0 = (kb - (part ? q.kb_first : 0)) * BK;
                    const CUtensorMap* ma = &q.a[part];
                    const CUtensorMap* mb = &q.b[MODE == GATE_UP ? (PAIR ? (int)rank : 0) : part];
                    const uint32_t bar = PAIR ? (full_bar(s) & kPeerBitMask) : full_bar(s);
                    if (!PAIR || rank == 0) mbar_expect_tx(full_bar(s), STAGE * (PAIR ? 2 : 1));
                    auto load = [&](uint32_t dst, const CUtensorMap* map, int x, int y) {
                        if (PAIR) tma_load_2d_pair(dst, map, bar, x, y); else tma_load_2d(dst, map, bar, x, y);
                    };
                    if (A_MN) {
                        load(sa, ma, m0, k0);
                        load(sa + OPERAND / 2, ma, m0 + 64, k0);
                    } else {
                        load(sa, ma, k0, m0);
                    }
                    if (B_MN) {
                        load(sb, mb, n0, k0);
                        load(sb + OPERAND / 2, mb, n0 + 64, k0);
                    } else if (MODE == GATE_UP && !PAIR) {
                        load(sb, &q.b[0], k0, n0);
                        load(sb + OPERAND / 2, &q.b[1], k0, n0);
                    } else {
                        load(sb, mb, k0, n0);
                    }
                    ++issued;
                    if (++s == STAGES) { s = 0; empty_parity ^= 1u; }
                }
            }
            if (*abort_flag && rank == 0) {
                // let the copies already issued land before the CTA's shared memory goes away
                for (int i = (issued > STAGES ? issued - STAGES : 0); i < issued; ++i) mbar_wait(full_bar(i % STAGES), (i / STAGES) & 1);
            }
        }
        if (UNIT == SHARED) {
            __syncwarp();
            cluster_sync();
        }
    } else if (warp == 1) {
        // ---------------------------------------------------------- products (the leader's, for a pair)
        if (lane == 0 && rank == 0) {
            int s = 0, t = 0;  // t counts tiles: accumulator t & 1
            uint32_t full_parity = 0;
            bool ok = true;
            for (int item = unit; ok && item < P.n_items; item += n_units, ++t) {
                Work w;
                locate(item, w);
                const int buf = t & 1;
                if (t >= 2 && !mbar_wait(acc_empty_bar(buf), ((t >> 1) - 1) & 1, abort_flag)) { raise_timeout(); break; }
                tc_fence_after();
                const uint32_t acc = tmem_base + (uint32_t)buf * BN;
                for (int kb = w.kb0; kb < w.kb1; ++kb) {
                    if (!mbar_wait(full_bar(s), full_parity, abort_flag)) { raise_timeout(); ok = false; break; }
                    tc_fence_after();
                    const uint32_t sa = base + s * STAGE, sb = sa + OPERAND;
                    const uint64_t da = A_MN ? make_desc_mn(sa) : make_desc(sa), db = B_MN ? make_desc_mn(sb) : make_desc(sb);
#pragma unroll
                    for (int k = 0; k < BK / 16; ++k) {
                        // 16 of the contraction: 32 bytes along a K-major row, 16 rows of 128 bytes of an MN-major tile
                        const uint64_t ka = (uint64_t)((A_MN ? k * 2048 : k * 32) >> 4), kbo = (uint64_t)((B_MN ? k * 2048 : k * 32) >> 4);
                        if (PAIR) umma16_pair(acc, da + ka, db + kbo, IDESC, kb > w.kb0 || k > 0);
                        else umma16(acc, da + ka, db + kbo, IDESC, kb > w.kb0 || k > 0);
                    }
                    if (PAIR) umma_commit_pair(empty_bar(s)); else umma_commit(empty_bar(s));
                    if (++s == STAGES) { s = 0; full_parity ^= 1u; }
                }
                if (!ok) break;
                if (PAIR) umma_commit_pair(acc_full_bar(buf)); else umma_commit(acc_full_bar(buf));
            }
        }
        if (UNIT == SHARED) {
            __syncwarp();
            cluster_sync();
        }
    } else {
        // ---------------------------------------------------------- epilogue
        const int quarter = warp & 3;               // a warp may only touch TMEM lanes [32 quarter, 32 quarter + 32)
        const int share = (warp - 2) >> 2;          // which CPW of the accumulator's columns (gate-up: half of G, half of U)
        constexpr int CPW = BN / (EPI / 4), STEPS = CPW / 16;
        const uint32_t lane_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
        uint4* stg = reinterpret_cast<uint4*>(smem_raw + (staging - raw) + (warp - 2) * STAGING);
        const int my_tiles = unit < P.n_items ? (P.n_items - unit + n_units - 1) / n_units : 0;
        bool ok = true;
        int t = 0;
        for (int item = unit; item < P.n_items; item += n_units, ++t) {
            Work w;
            const Problem& q = locate(item, w);
            const int tn = w.tn;
            const int buf = t & 1;
            const int row0 = w.tm * TM + (int)rank * BM + quarter * 32;
            const int rows = min(32, q.M - row0);   // may be negative: nothing to store
            const uint32_t acc = lane_addr + (uint32_t)buf * BN;
            // d-hidden: a lane handles eight columns of rows lane / 8 + 4 i.  It has G and U of four rows at a time in
            // registers; those of the first four are on their way while the tile is still being multiplied.
            const int c8 = lane & 7, r0 = lane >> 3;
            uint4 vg[4], vu[4];
            auto load_gu = [&](int i0, int col) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = r0 + 4 * (i0 + i);
                    vg[i] = vu[i] = make_uint4(0, 0, 0, 0);
                    if (r < rows && col < q.N) {
                        vg[i] = *reinterpret_cast<const uint4*>(static_cast<const T*>(q.in[0]) + (row0 + r) * q.ldi[0] + col);
                        vu[i] = *reinterpret_cast<const uint4*>(static_cast<const T*>(q.in[1]) + (row0 + r) * q.ldi[1] + col);
                    }
                }
            };
            const int dh_col = tn * TN + share * CPW + 8 * c8;
            if (MODE == D_HIDDEN) load_gu(0, dh_col);
            if (lane == 0) {
                // the tile is complete when its barrier flips, or never if another role gave up
                const long long t0 = clock64();
                while (!mbar_try(acc_full_bar(buf), (t >> 1) & 1)) {
                    if (*abort_flag) { ok = false; break; }
                    if (clock64() - t0 > 2 * kWaitCycles) { raise_timeout(); ok = false; break; }
                }
            }
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (!ok) {
                if (UNIT == SHARED) cluster_sync();   // the other CTAs wait for this one there
                break;
            }
            tc_fence_after();
            // Hands the accumulator back.  (Not for the last two tiles: nobody waits for them, and no arrival may be
            // on its way to the other CTA when that one exits.)
            auto release = [&]() {
                tc_fence_before();
                __syncwarp();
                if (lane == 0 && t + 2 < my_tiles) {
                    if (PAIR) mbar_arrive_cluster(acc_empty_bar(buf) & kPeerBitMask); else mbar_arrive(acc_empty_bar(buf));
                }
            };
            // gate-up: half of the steps are columns of G, the others the same columns of U
            auto column = [&](int step) {
                return MODE == GATE_UP ? (step / (STEPS / 2)) * TN + share * (CPW / 2) + step % (STEPS / 2) * 16 : share * CPW + step * 16;
            };
            if constexpr (UNIT == SHARED) {
                // Block (quarter, share) of the tile goes to one CTA of the cluster, part by part; its warp there adds the
                // parts in their order, puts the sums back into tensor memory and goes on with them.
                const int block = quarter * 2 + share, per_cta = EPI / P.split;
                const uint32_t owner = (uint32_t)(block / per_cta);
                const uint32_t place = staging + (uint32_t)(block % per_cta) * P.split * 8192u + (uint32_t)lane * 16u;
                const uint32_t there = map_to_rank(place + (uint32_t)w.part * 8192u, owner);
#pragma unroll 1
                for (int st = 0; st < STEPS; ++st) {
                    float v[16];
                    tmem_ld16(acc + column(st), v);
#pragma unroll
                    for (int k = 0; k < 4; ++k) st_cluster_f4(there + (uint32_t)(st * 4 + k) * 512u, v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
                }
                cluster_sync();
                if (owner != (uint32_t)w.part) break;   // (one tile per cluster)
                const float4* parts = reinterpret_cast<const float4*>(smem_raw + (place - raw));
#pragma unroll 1
                for (int st = 0; st < STEPS; ++st) {
                    float sum[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[j] = 0.f;
#pragma unroll 2
                    for (int p = 0; p < P.split; ++p)
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float4 x = parts[p * 512 + (st * 4 + k) * 32];
                            sum[4 * k] += x.x; sum[4 * k + 1] += x.y; sum[4 * k + 2] += x.z; sum[4 * k + 3] += x.w;
                        }
                    tmem_st16(acc + column(st), sum);
                }
                // from here on the block's own place, which only this warp reads, is its staging area
                stg = reinterpret_cast<uint4*>(smem_raw + (place - raw) - lane * 16);
            }
            // A tile whose contraction is split: every part's warps leave their sums in the workspace; the one that finds
            // all others there adds them up in the order of the parts (its own among them), puts the result back into
            // tensor memory and goes on with it.
            if (UNIT != SHARED && w.split_tile >= 0) {
                constexpr int CTAS = PAIR ? 2 : 1, SLAB = STEPS * 4 * 32;
                const int64_t stride = (int64_t)CTAS * EPI * SLAB;
                float4* base = P.parts + (((int64_t)w.split_tile * P.split * CTAS + rank) * EPI + (warp - 2)) * SLAB + lane;
#pragma unroll 1
                for (int st = 0; st < STEPS; ++st) {
                    float v[16];
                    tmem_ld16(acc + column(st), v);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        __stcg(base + w.part * stride + (st * 4 + k) * 32, make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]));
                }
                __threadfence();
                __syncwarp();
                int* counter = P.arrived + (w.split_tile * CTAS + (int)rank) * EPI + (warp - 2);
                int before = 0;
                if (lane == 0) before = atomicAdd(counter, 1);
                before = __shfl_sync(0xffffffffu, before, 0);
                if (before != P.split - 1) {
                    release();
                    continue;
                }
                if (lane == 0) *counter = 0;
                __threadfence();
#pragma unroll 1
                for (int st = 0; st < STEPS; ++st) {
                    // up to four parts' values on their way at a time
                    float sum[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[j] = 0.f;
                    for (int p0 = 0; p0 < P.split; p0 += 4) {
                        float4 x[4][4];
#pragma unroll
                        for (int p = 0; p < 4; ++p)
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                x[p][k] = p0 + p < P.split ? __ldcg(base + (p0 + p) * stride + (st * 4 + k) * 32) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                        for (int p = 0; p < 4; ++p)
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                sum[4 * k] += x[p][k].x; sum[4 * k + 1] += x[p][k].y; sum[4 * k + 2] += x[p][k].z; sum[4 * k + 3] += x[p][k].w;
                            }
                    }
                    tmem_st16(acc + column(st), sum);
                }
            }
            if constexpr (MODE == GATE_UP) {
                constexpr int CU = CPW / 2;         // features per warp: 64 or 32
                uint32_t pg[CU / 2], pu[CU / 2], ph[CU / 2];
                with_act(P.act, [&](auto kind) {
#pragma unroll
                    for (int st = 0; st < STEPS / 2; ++st) {
                        float g[16], u[16];
                        tmem_ld16x2(acc + column(st), acc + column(st + STEPS / 2), g, u);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            pg[8 * st + j] = pack2<T>(g[2 * j], g[2 * j + 1]);
                            pu[8 * st + j] = pack2<T>(u[2 * j], u[2 * j + 1]);
                            ph[8 * st + j] = pack2<T>(activate<decltype(kind)::value, false>(g[2 * j]).x * u[2 * j],
                                                      activate<decltype(kind)::value, false>(g[2 * j + 1]).x * u[2 * j + 1]);
                        }
                    }
                });
                release();
                const int col0 = tn * TN + share * CU;
                if (q.out[0]) {
                    store_rows<T, CU>(stg, pg, &q.o[0], static_cast<T*>(q.out[0]), q.ldo[0], row0, rows, col0, q.cols[0], q.vec_out & 1, lane);
                    store_rows<T, CU>(stg, pu, &q.o[1], static_cast<T*>(q.out[1]), q.ldo[1], row0, rows, col0, q.cols[1], q.vec_out & 2, lane);
                }
                store_rows<T, CU>(stg, ph, &q.o[2], static_cast<T*>(q.out[2]), q.ldo[2], row0, rows, col0, q.cols[2], q.vec_out & 4, lane);
            } else if constexpr (MODE == PLAIN) {
#pragma unroll 1
                for (int c = 0; c < CPW; c += 64) {
                    uint32_t packed[32];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float v[32];
                        tmem_ld32(acc + share * CPW + c + 32 * i, v);
#pragma unroll
                        for (int j = 0; j < 16; ++j) packed[16 * i + j] = pack2<T>(v[2 * j], v[2 * j + 1]);
                    }
                    if (c + 64 == CPW) release();
                    store_rows<T, 64>(stg, packed, &q.o[0], static_cast<T*>(q.out[0]), q.ldo[0], row0, rows, tn * TN + share * CPW + c,
                                      q.cols[0], q.vec_out & 1, lane);
                }
            } else {
                // The block goes through shared memory in fp32, so that G and U are read, and dG, dU and H written, in
                // row segments of 128 bytes.
                float4* sf = reinterpret_cast<float4*>(stg);   // 32 rows of sixteen 16-byte chunks, permuted by row
                auto at = [](int r, int c) { return r * 16 + (c ^ (r & 7)); };
#pragma unroll 1
                for (int c = 0; c < CPW; c += 64) {
                    const int col = dh_col + c;
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float v[32];
                        tmem_ld32(acc + share * CPW + c + 32 * i, v);
#pragma unroll
                        for (int k = 0; k < 8; ++k) sf[at(lane, 8 * i + k)] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
                    }
                    if (c + 64 == CPW) release();
                    __syncwarp();
                    // (not unrolled: code that runs once per tile is fetched once per tile)
#pragma unroll 1
                    for (int h = 0; h < 2; ++h) {
                        const uint4 cg[4] = {vg[0], vg[1], vg[2], vg[3]}, cu[4] = {vu[0], vu[1], vu[2], vu[3]};
                        if (h == 0) load_gu(4, col);
                        else if (c + 64 < CPW) load_gu(0, col + 64);
                        with_act(P.act, [&](auto kind) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int r = r0 + 4 * (4 * h + i);
                                if (r >= rows || col >= q.cols[0]) continue;
                                const float4 d0 = sf[at(r, 2 * c8)], d1 = sf[at(r, 2 * c8 + 1)];
                                const float dh[8] = {d0.x, d0.y, d0.z, d0.w, d1.x, d1.y, d1.z, d1.w};
                                const uint32_t wg[4] = {cg[i].x, cg[i].y, cg[i].z, cg[i].w}, wu[4] = {cu[i].x, cu[i].y, cu[i].z, cu[i].w};
                                uint32_t og[4], ou[4], oh[4];
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    const float2 g = unpack2<T>(wg[j]), u = unpack2<T>(wu[j]);
                                    const float2 a0 = activate<decltype(kind)::value, true>(g.x), a1 = activate<decltype(kind)::value, true>(g.y);
                                    og[j] = pack2<T>(dh[2 * j] * u.x * a0.y, dh[2 * j + 1] * u.y * a1.y);
                                    ou[j] = pack2<T>(dh[2 * j] * a0.x, dh[2 * j + 1] * a1.x);
                                    oh[j] = pack2<T>(a0.x * u.x, a1.x * u.y);
                                }
                                const int64_t to = (int64_t)(row0 + r) * q.ldo[0] + col;   // all three have the same layout
                                *reinterpret_cast<uint4*>(static_cast<T*>(q.out[0]) + to) = make_uint4(og[0], og[1], og[2], og[3]);
                                *reinterpret_cast<uint4*>(static_cast<T*>(q.out[1]) + to) = make_uint4(ou[0], ou[1], ou[2], ou[3]);
                                *reinterpret_cast<uint4*>(static_cast<T*>(q.out[2]) + to) = make_uint4(oh[0], oh[1], oh[2], oh[3]);
                            }
                        });
                    }
                }
            }
        }
    }
    tma_store_wait<true>();   // (of threads that have made any)
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_relaxed();  // the leader's products use the other CTA's shared and tensor memory
    if (warp == 1) {
        tc_fence_after();
        if (PAIR) tmem_dealloc_pair(tmem_base, TMEM_COLS); else tmem_dealloc(tmem_base, TMEM_COLS);
    }
    if (P.link == BESIDE) pdl_wait();
}

// ---------------------------------------------------------------- few tokens

// Up to 16 tokens (a decode step): the products are bound by reading the weights once, 6 d f bytes, and a 128-row tile
// would leave the tensor core mostly zeros to multiply and two thirds of the machine idle on Y = H Wd^T.  Here a block
// takes 8 features (8 rows of Wg and of Wu, or of Wd) and its 8 warps share the contraction, so there are f / 8 and d / 8
// blocks; weights go from memory straight to the registers of m16n8k16 products, 16 bytes per load.  (A thread's 8
// consecutive k are used as the k-indices that the instruction wants from it; the tokens' operand is read with the same
// permutation, so the sum is over the same products.)  The warps' partial sums are added in a fixed order.
// 1 token, 4096 x 8192: 37 us for 201 MB, 5.5 TB/s.  The limit: at 16 tokens this and the tiles take the same 48 us at 4096
// x 8192, and 9 against 14 at 512 x 1376; at 17, with twice the products here, 91 against 48 and 20 against 18 (1024 x 2736).
constexpr int kFewTokens = 16, kFewWarps = 8;

struct FewArgs {
    const void* x;        // [M][K], ld
    const void* w[2];     // [N][K]
    void* out[3];         // gate-up: G, U (or null) and H; down: Y
    int64_t ldx, ldo[3];
    int M, N, K, act;
};

// (The read-only path: no launch of the block writes weights, and whatever wrote them has ended when gate-up goes on.)
__device__ __forceinline__ uint4 load_weights(const void* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
template <typename T>
__device__ __forceinline__ void mma16816(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// VEC: rows of x and w are 16-byte aligned (K is then a multiple of 8).  WIDE: more than 8 tokens.
template <typename T, bool GATE, bool VEC, bool WIDE>
__global__ void __launch_bounds__(32 * kFewWarps, 32 / kFewWarps)
ffn_few_kernel(const __grid_constant__ FewArgs a) {
    constexpr int NT = GATE ? 2 : 1, U = 8 / NT;   // eight weight loads in flight per thread
    __shared__ float red[kFewWarps][NT][kFewTokens][8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int n0 = blockIdx.x * 8;
    // Steps of 32 of the contraction.  Gate-up: a warp takes a contiguous eighth of them.  Down: they are dealt out in runs
    // of U, so that what the warps read at a time is contiguous.  (Each the faster way for its kernel, 1 token, 4096 x
    // 8192: gate-up 25 us against 27 in runs, down 14 us against 16 in eighths.)
    const int steps = (a.K + 31) / 32, mine = (steps + U * kFewWarps - 1) / (U * kFewWarps) * U;
    auto step_of = [&](int i) { return GATE ? warp * mine + i : (i / U * kFewWarps + warp) * U + i % U; };
    // rows beyond the matrix: some row that exists, its results are not stored
    const T* w[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) w[j] = static_cast<const T*>(a.w[j]) + (int64_t)min(n0 + g, a.N - 1) * a.K;
    const T* x0 = static_cast<const T*>(a.x) + (int64_t)min(g, a.M - 1) * a.ldx;
    const T* x1 = static_cast<const T*>(a.x) + (int64_t)min(g + 8, a.M - 1) * a.ldx;
    float acc[NT][4] = {};
    uint4 v[U][NT];
    auto fetch_step = [&](uint4 (&r)[NT], int i) {
        const int k = step_of(i) * 32 + 8 * t;
#pragma unroll
        for (int j = 0; j < NT; ++j)
            r[j] = i >= mine || k >= a.K ? make_uint4(0, 0, 0, 0) : (VEC ? load_weights(w[j] + k) : load8(w[j], k, a.K, false));
    };
    auto fetch = [&]() {
#pragma unroll
        for (int u = 0; u < U; ++u) fetch_step(v[u], u);
    };
    if (GATE) {
        // The dependent launch may read its weights before this kernel has ended, so it must not start before whatever
        // wrote them has: wait first.
        pdl_wait();
        pdl_trigger();
        fetch();
    } else {
        fetch();   // the weights were there before the gate-up kernel started; H was not
        pdl_trigger();
        pdl_wait();
    }
    for (int i = 0; i < mine; i += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = step_of(i + u) * 32 + 8 * t;
            const bool in = k < a.K;
            const uint4 zero = make_uint4(0, 0, 0, 0);
            const uint4 p = in ? load8(x0, k, a.K, VEC) : zero, q = WIDE && in ? load8(x1, k, a.K, VEC) : zero;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                mma16816<T>(acc[j], p.x, q.x, p.y, q.y, v[u][j].x, v[u][j].y);
                mma16816<T>(acc[j], p.z, q.z, p.w, q.w, v[u][j].z, v[u][j].w);
            }
            fetch_step(v[u], i + u + U);
        }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        *reinterpret_cast<float2*>(&red[warp][j][g][2 * t]) = make_float2(acc[j][0], acc[j][1]);
        if (WIDE) *reinterpret_cast<float2*>(&red[warp][j][g + 8][2 * t]) = make_float2(acc[j][2], acc[j][3]);
    }
    __syncthreads();
    const int m = threadIdx.x >> 3, f = threadIdx.x & 7;
    static_assert(32 * kFewWarps >= 8 * kFewTokens, "a thread per output");
    if (m >= a.M || n0 + f >= a.N) return;
    float sum[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        sum[j] = 0.f;
#pragma unroll
        for (int i = 0; i < kFewWarps; ++i) sum[j] += red[i][j][m][f];
    }
    auto put = [&](int i, float val) { static_cast<T*>(a.out[i])[m * a.ldo[i] + n0 + f] = from_float<T>(val); };
    if (GATE) {
        if (a.out[0]) {
            put(0, sum[0]);
            put(1, sum[NT - 1]);
        }
        with_act(a.act, [&](auto kind) { put(2, activate<decltype(kind)::value, false>(sum[0]).x * sum[NT - 1]); });
    } else {
        put(0, sum[0]);
    }
}

// Rows of `cols` values at any address -> rows of `ld` (a multiple of 8) at an aligned one: what TMA can read.  All
// matrices of a call in one launch, weights too, in every call of more than 16 tokens and every backward pass.  Memory-bound where it counts (21 tokens, 3148 x 7198: 272 MB read and written, 54 us).
struct AlignJobs {
    static constexpr int kMost = 7;
    const void* src[kMost];
    void* dst[kMost];
    int64_t first[kMost + 1];   // 16-byte groups of the matrices before
    uintptr_t end[kMost];       // where src ends
    int cols[kMost], ld[kMost];
    int n;
};
template <typename T>
__global__ void __launch_bounds__(256)
align_rows_kernel(const __grid_constant__ AlignJobs a) {
    pdl_trigger();
    pdl_wait();
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < a.first[a.n]; i += (int64_t)gridDim.x * blockDim.x) {
        int k = 0;
        while (i >= a.first[k + 1]) ++k;
        const int groups = a.ld[k] / 8;
        const int64_t at = i - a.first[k];
        const int64_t r = at >> 32 ? at / groups : (int64_t)((uint32_t)at / (uint32_t)groups);   // (the wide division costs 100 instructions)
        const int c = (int)(at - r * groups) * 8;
        const T* row = static_cast<const T*>(a.src[k]) + r * a.cols[k];
        const uintptr_t from = reinterpret_cast<uintptr_t>(row + c), block = from & ~(uintptr_t)15;
        uint4 v;
        if (c + 8 <= a.cols[k] && block >= reinterpret_cast<uintptr_t>(a.src[k]) && block + 32 <= a.end[k]) {
            // eight values out of the two aligned 16-byte blocks they lie in, both within the matrix
            const uint4 x = reinterpret_cast<const uint4*>(block)[0], y = reinterpret_cast<const uint4*>(block)[1];
            uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
            const int shift = (int)(from & 15) >> 1;   // in values
            if (shift & 4)
#pragma unroll
                for (int j = 0; j < 6; ++j) w[j] = w[j + 2];
            if (shift & 2)
#pragma unroll
                for (int j = 0; j < 5; ++j) w[j] = w[j + 1];
            if (shift & 1)
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = __funnelshift_r(w[j], w[j + 1], 16);
            v = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            v = load8(row, c, a.cols[k], false);
        }
        *reinterpret_cast<uint4*>(static_cast<T*>(a.dst[k]) + r * a.ld[k] + c) = v;
    }
}

// ---------------------------------------------------------------- host side

inline int up8(int x) { return (x + 7) & ~7; }
inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
inline bool vec_rows(const void* p, int ld) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld % 8 == 0; }

// A matrix of 16-bit values as TMA reads it.
struct Matrix {
    const void* p;
    int64_t rows;
    int cols, ld;
};

// Box of box_cols x box_rows; columns and rows beyond the matrix read as zero.
bool make_map2(CUtensorMap* map, const Matrix& m, int dtype, int box_cols, int box_rows) {   // rows of 128 or 64 bytes
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)m.cols, (cuuint64_t)m.rows};
    cuuint64_t strides[1] = {(cuuint64_t)m.ld * 2};
    cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, estr[2] = {1, 1};
    return fn(map, dtype == SAMA_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
              const_cast<void*>(m.p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// The tile of 128 rows (or columns, MN-major) that one CTA stages.
bool operand_map(CUtensorMap* map, const Matrix& m, int dtype, bool mn_major, int rows = BM) {
    return mn_major ? make_map2(map, m, dtype, 64, BK) : make_map2(map, m, dtype, BK, rows);
}

inline int blocks_of(int64_t x, int b) { return (int)((x + b - 1) / b); }

// How a launch's tiles are worked on.
struct TilePlan {
    Unit unit;
    int whole, split;
};
constexpr int kMaxSplitTiles = 256, kMaxSplitParts = 512;   // of 128 x 128 values per CTA; twice as many per CTA of a pair

template <typename T, int MODE, int UNIT, bool A_MN, bool B_MN, int G>
cudaError_t launch_ffn(sama_ctx* ctx, Params<G>& P, int kind, const TilePlan& plan, cudaStream_t st) {
    constexpr bool PAIR = UNIT == PAIRED;
    auto* kernel = ffn_kernel<T, MODE, UNIT, A_MN, B_MN, G>;
    const uint32_t bit = 1u << (6 * kind + 2 * UNIT + (std::is_same<T, __half>::value ? 1 : 0));
    if (!(ctx->ffn_ready & bit)) {  // once per context: the opt-in to this much shared memory
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_of(MODE, UNIT));
        if (e != cudaSuccess) return e;
        ctx->ffn_ready |= bit;
    }
    const int tm = PAIR ? 2 * BM : BM, tn = (PAIR ? 256 : 128) / (MODE == GATE_UP ? 2 : 1);
    int tiles = 0;
    for (int g = 0; g < G; ++g) {
        Problem& q = P.p[g];
        q.tiles_m = blocks_of(q.M, tm);
        q.tiles_n = blocks_of(q.N, tn);
        q.item0 = tiles;
        tiles += q.tiles_m * q.tiles_n;
    }
    P.whole = plan.whole;
    P.split = plan.split;
    P.n_items = plan.split > 1 ? plan.whole + (tiles - plan.whole) * plan.split : tiles;
    P.parts = reinterpret_cast<float4*>(ctx->ffn_parts);
    P.arrived = ctx->ffn_arrived;
    P.group_m = 8;
    P.status = &ctx->scalars->status;
    const int max_units = PAIR ? ctx->ffn_pair_units : ctx->sm_count, items = P.n_items;
    const int units = UNIT == SHARED || items < max_units ? items : max_units;   // (shared: one tile per cluster)
    ctx->ffn_path[kind] = 16 * plan.split + (PAIR ? SAMA_FFN_PAIRS : UNIT == SHARED ? SAMA_FFN_CLUSTERS : SAMA_FFN_SINGLE);
    KernelScope scope(ctx, SAMA_K_FFN, kind, st);
    return launch_clustered(PAIR ? 2 : UNIT == SHARED ? plan.split : 1, kernel, dim3(units * (PAIR ? 2 : 1)), dim3(THREADS),
                            (size_t)smem_of(MODE, UNIT), st, P);
}

// Once per context: how many CTA pairs and clusters of the kernel can be resident, and the workspace of split tiles.
cudaError_t prepare_ffn(sama_ctx* ctx) {
    if (ctx->ffn_pair_units > 0) return cudaSuccess;
    auto* kernel = ffn_kernel<__nv_bfloat16, PLAIN, PAIRED, false, false, 1>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_of(PLAIN, PAIRED));
    if (e != cudaSuccess) return e;
    auto* sharing = ffn_kernel<__nv_bfloat16, PLAIN, SHARED, false, false, 1>;
    e = cudaFuncSetAttribute(sharing, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_of(PLAIN, SHARED));
    if (e != cudaSuccess) return e;
    auto resident = [&](auto* k, int size, int smem, int* clusters) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(ctx->sm_count / size * size);
        cfg.blockDim = dim3(THREADS);
        cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = size;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        return cudaOccupancyMaxActiveClusters(clusters, k, &cfg);
    };
    int clusters = 0;
    if ((e = resident(kernel, 2, smem_of(PLAIN, PAIRED), &clusters)) != cudaSuccess) return e;
    if (clusters < 1) return cudaErrorLaunchOutOfResources;
    for (int i = 0; i < 3; ++i)
        if ((e = resident(sharing, 2 << i, smem_of(PLAIN, SHARED), &ctx->ffn_clusters[i])) != cudaSuccess) return e;
    const size_t counters = sizeof(int) * kMaxSplitTiles * 2 * EPI;
    if (!ctx->ffn_parts && (e = cudaMalloc(&ctx->ffn_parts, sizeof(float) * kMaxSplitParts * BM * 128)) != cudaSuccess) return e;
    if (!ctx->ffn_arrived && (e = cudaMalloc(&ctx->ffn_arrived, counters)) != cudaSuccess) return e;
    if ((e = cudaMemset(ctx->ffn_arrived, 0, counters)) != cudaSuccess || (e = cudaDeviceSynchronize()) != cudaSuccess) return e;
    ctx->ffn_pair_units = clusters < ctx->sm_count / 2 ? clusters : ctx->sm_count / 2;
    return cudaSuccess;
}

// The fastest plan by estimate.  A launch's time is its rounds of tiles, each the longer of multiplying it and storing the
// one before.  A last round that would leave half of the pairs without a tile splits the contraction of its tiles instead,
// which costs an exchange through L2; tiles too few for one round of CTAs are shared by clusters.
// (`tail`: a last round may be split while the others are not.)
TilePlan plan_tiles(const sama_ctx* ctx, const Problem* p, int n, Mode mode, bool tail = true) {
    TilePlan best = {SINGLE, 1 << 30, 1};
    double best_cost = -1.0;
    for (int u = SINGLE; u <= SHARED; ++u) {
        const bool pair = u == PAIRED;
        const int tm = pair ? 256 : 128, tn = (pair ? 256 : 128) / (mode == GATE_UP ? 2 : 1), units = pair ? ctx->ffn_pair_units : ctx->sm_count;
        // microseconds, measured with a contraction of 64 (storing) and of 4096 (multiplying); a tile stores while the next
        // one multiplies
        const double t_exchange = pair ? 9.0 : 3.0;
        const double t_store = mode == GATE_UP ? (pair ? 5.6 : 3.0) : mode == PLAIN ? (pair ? 3.5 : 2.0) : (pair ? 12.5 : 6.0);
        int64_t tiles = 0;
        int least_kb = 1 << 30, most_kb = 0;
        for (int i = 0; i < n; ++i) {
            if (p[i].M == 0) continue;
            tiles += (int64_t)blocks_of(p[i].M, tm) * blocks_of(p[i].N, tn);
            least_kb = p[i].num_kb < least_kb ? p[i].num_kb : least_kb;
            most_kb = p[i].num_kb > most_kb ? p[i].num_kb : most_kb;
        }
        const int64_t rounds = tiles / units, rest = tiles - rounds * units;
        for (int split = u == SHARED ? 2 : 1; split <= 8; split = u == SHARED ? 2 * split : split + 1) {
            if (u == SINGLE && split > 1) break;
            if (split > 1 && (rest == 0 || rest * split > units || least_kb < 2 * split)) break;
            if (pair && split > 1 && (rest > kMaxSplitTiles || rest * split * 4 > kMaxSplitParts || (rounds > 0 && !tail))) break;
            if (u == SHARED && (rounds > 0 || tiles > ctx->ffn_clusters[split == 2 ? 0 : split == 4 ? 1 : 2])) break;
            // (an SM takes in 64 bytes per cycle, all of them together less; pairs that run for long meet the power limit)
            const double t_kb = pair ? (tiles > 2 * units ? 0.42 : 0.36) : (tiles * split > units / 2 ? 0.33 : 0.27);
            const double t_tile = most_kb * t_kb > t_store ? most_kb * t_kb : t_store;
            const double cost = rounds * t_tile + (rest ? most_kb * t_kb / split : 0.0) + t_store + (split > 1 ? t_exchange : 0.0);
            if (best_cost < 0.0 || cost < best_cost) {
                best_cost = cost;
                best = {static_cast<Unit>(u), split > 1 ? (int)(rounds * units) : 1 << 30, split};
            }
        }
    }
    return best;
}

// block: columns that a warp stores at a time, 0 where it does so without the copy engine.
bool set_output(Problem& q, int i, void* p, int ld, int cols, int dtype, int block) {
    q.out[i] = p;
    q.ldo[i] = ld;
    q.cols[i] = cols;
    if (!p || !vec_rows(p, ld) || cols % 8 != 0) return true;
    q.vec_out |= 1 << i;
    return block == 0 || make_map2(&q.o[i], {p, q.M, cols, ld}, dtype, block, 32);
}

// What a call works on: operands as TMA can read them, copied to the workspace where they are not.
template <typename T>
struct Block {
    sama_ctx* ctx;
    const FfnShape& f;
    uint8_t* ws;
    cudaStream_t st;
    int fp;               // leading dimension of the workspace's [tokens][f] matrices
    cudaError_t err = cudaSuccess;

    void* take(size_t elements) {
        void* p = ws;
        ws += up256(elements * 2);
        return p;
    }
    // The matrix itself, or the place of a copy that align() will make.
    AlignJobs jobs = {};
    Matrix readable(const void* p, int64_t rows, int cols) {
        if (vec_rows(p, cols)) return {p, rows, cols, cols};
        const int ld = up8(cols), k = jobs.n++;
        jobs.src[k] = p;
        jobs.end[k] = reinterpret_cast<uintptr_t>(p) + (size_t)rows * cols * 2;
        jobs.dst[k] = take((size_t)rows * ld);
        jobs.cols[k] = cols;
        jobs.ld[k] = ld;
        jobs.first[k + 1] = jobs.first[k] + rows * (ld / 8);
        return {jobs.dst[k], rows, cols, ld};
    }
    void align() {
        if (jobs.n == 0 || err != cudaSuccess) return;
        int64_t blocks = (jobs.first[jobs.n] + 255) / 256;
        if (blocks > 16 * ctx->sm_count) blocks = 16 * ctx->sm_count;
        KernelScope scope(ctx, SAMA_K_FFN, -1, st);
        err = launch_dependent(align_rows_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, st, jobs);
    }
    template <int MODE, bool A_MN, bool B_MN, int G>
    void run(Params<G>& P, int kind, const TilePlan& plan) {
        if (err != cudaSuccess) return;
        err = plan.unit == PAIRED   ? launch_ffn<T, MODE, PAIRED, A_MN, B_MN, G>(ctx, P, kind, plan, st)
              : plan.unit == SHARED ? launch_ffn<T, MODE, SHARED, A_MN, B_MN, G>(ctx, P, kind, plan, st)
                                    : launch_ffn<T, MODE, SINGLE, A_MN, B_MN, G>(ctx, P, kind, plan, st);
    }
    template <int MODE, bool A_MN, bool B_MN, int G>
    void run(Params<G>& P, int kind) {
        run<MODE, A_MN, B_MN, G>(P, kind, plan_tiles(ctx, P.p, G, static_cast<Mode>(MODE)));
    }
    void check(bool ok) {
        if (!ok && err == cudaSuccess) err = cudaErrorInvalidValue;
    }

    template <bool GATE>
    void run_few(const FewArgs& a, bool vec) {
        if (err != cudaSuccess) return;
        const bool wide = a.M > 8;
        auto* kernel = vec ? (wide ? ffn_few_kernel<T, GATE, true, true> : ffn_few_kernel<T, GATE, true, false>)
                           : (wide ? ffn_few_kernel<T, GATE, false, true> : ffn_few_kernel<T, GATE, false, false>);
        ctx->ffn_path[GATE ? 0 : 1] = 16 + SAMA_FFN_FEW_TOKENS;
        KernelScope scope(ctx, SAMA_K_FFN, GATE ? 0 : 1, st);
        err = launch_dependent(kernel, dim3(blocks_of(a.N, 8)), dim3(32 * kFewWarps), 0, st, a);
    }

    void forward(const void* x, const void* wg, const void* wu, const void* wd, void* y, void* gate, void* up) {
        const int M = (int)f.n_tokens, d = f.d, n = f.f;
        void* h = take((size_t)M * fp);
        if (M <= kFewTokens) {
            FewArgs a = {};
            a.x = x;
            a.w[0] = wg;
            a.w[1] = wu;
            void* outs[3] = {gate, up, h};
            for (int i = 0; i < 3; ++i) a.out[i] = outs[i], a.ldo[i] = i < 2 ? n : fp;
            a.ldx = d;
            a.M = M;
            a.N = n;
            a.K = d;
            a.act = f.act;
            run_few<true>(a, vec_rows(x, d) && vec_rows(wg, d) && vec_rows(wu, d));
            FewArgs b = {};
            b.x = h;
            b.w[0] = b.w[1] = wd;
            b.out[0] = y;
            b.ldo[0] = d;
            b.ldx = fp;
            b.M = M;
            b.N = d;
            b.K = n;
            run_few<false>(b, vec_rows(wd, n));
            return;
        }
        const Matrix mx = readable(x, M, d), mg = readable(wg, n, d), mu = readable(wu, n, d), md = readable(wd, d, n);
        align();
        {
            Params<1> P = {};
            Problem& q = P.p[0];
            q.M = M;
            q.N = n;
            q.num_kb = q.kb_first = blocks_of(d, BK);
            const TilePlan plan = plan_tiles(ctx, &q, 1, GATE_UP);
            check(operand_map(&q.a[0], mx, f.dtype, false) && operand_map(&q.b[0], mg, f.dtype, false, plan.unit == PAIRED ? 128 : 64) &&
                  operand_map(&q.b[1], mu, f.dtype, false, plan.unit == PAIRED ? 128 : 64));
            const int block = plan.unit == PAIRED ? 64 : 32;
            check(set_output(q, 0, gate, n, n, f.dtype, block) && set_output(q, 1, up, n, n, f.dtype, block) &&
                  set_output(q, 2, h, fp, fp, f.dtype, block));
            P.act = f.act;
            run<GATE_UP, false, false, 1>(P, 0, plan);
        }
        Params<1> P = {};
        Problem& q = P.p[0];
        check(operand_map(&q.a[0], {h, M, n, fp}, f.dtype, false) && operand_map(&q.b[0], md, f.dtype, false));
        q.M = M;
        q.N = d;
        q.num_kb = q.kb_first = blocks_of(n, BK);
        check(set_output(q, 0, y, d, d, f.dtype, 64));
        run<PLAIN, false, false, 1>(P, 1);
    }

    void backward(const void* x, const void* wg, const void* wu, const void* wd, const void* gate, const void* up,
                  const void* dy, void* dx, void* dwg, void* dwu, void* dwd) {
        const int M = (int)f.n_tokens, d = f.d, n = f.f;
        void* dg = take((size_t)M * fp);
        void* du = take((size_t)M * fp);
        void* h = take((size_t)M * fp);
        const Matrix my = readable(dy, M, d), md = readable(wd, d, n), none = {};
        const Matrix mg = dx ? readable(wg, n, d) : none, mu = dx ? readable(wu, n, d) : none;
        const Matrix mx = dwg || dwu ? readable(x, M, d) : my;
        const Matrix mgate = readable(gate, M, n), mup = readable(up, M, n);
        align();
        {
            Params<1> P = {};
            Problem& q = P.p[0];
            check(operand_map(&q.a[0], my, f.dtype, false) && operand_map(&q.b[0], md, f.dtype, true));
            q.M = M;
            q.N = n;
            q.num_kb = q.kb_first = blocks_of(d, BK);
            void* outs[3] = {dg, du, h};
            for (int i = 0; i < 3; ++i) check(set_output(q, i, outs[i], fp, fp, f.dtype, 0));
            q.in[0] = mgate.p;
            q.in[1] = mup.p;
            q.ldi[0] = mgate.ld;
            q.ldi[1] = mup.ld;
            P.act = f.act;
            run<D_HIDDEN, false, true, 1>(P, 2);
        }
        const Matrix mdg = {dg, M, n, fp}, mdu = {du, M, n, fp}, mh = {h, M, n, fp};
        Params<1> I = {};
        TilePlan plan_i = {};
        if (dx) {
            Problem& q = I.p[0];
            check(operand_map(&q.a[0], mdg, f.dtype, false) && operand_map(&q.a[1], mdu, f.dtype, false) &&
                  operand_map(&q.b[0], mg, f.dtype, true) && operand_map(&q.b[1], mu, f.dtype, true));
            q.M = M;
            q.N = d;
            q.kb_first = blocks_of(n, BK);
            q.num_kb = 2 * q.kb_first;
            check(set_output(q, 0, dx, d, d, f.dtype, 64));
            plan_i = plan_tiles(ctx, &q, 1, PLAIN);
        }
        if (!dwg && !dwu && !dwd) {
            if (dx) run<PLAIN, false, true, 1>(I, 3, plan_i);
            return;
        }
        Params<3> P = {};
        struct { const Matrix* a; const Matrix* b; void* out; int rows, cols; } w[3] = {
            {&mdg, &mx, dwg, n, d}, {&mdu, &mx, dwu, n, d}, {&my, &mh, dwd, d, n}};
        for (int i = 0; i < 3; ++i) {
            Problem& q = P.p[i];
            check(operand_map(&q.a[0], *w[i].a, f.dtype, true) && operand_map(&q.b[0], *w[i].b, f.dtype, true));
            q.M = w[i].rows;
            q.N = w[i].cols;
            q.num_kb = q.kb_first = blocks_of(M, BK);
            check(set_output(q, 0, w[i].out, w[i].cols, w[i].cols, f.dtype, 64));
        }
        // (planned for all three, so that a gradient's bits do not depend on which others are wanted)
        const TilePlan plan = plan_tiles(ctx, P.p, 3, PLAIN, false);
        for (int i = 0; i < 3; ++i)
            if (!w[i].out) P.p[i].M = 0;   // no tiles
        if (dx) {
            // (not if both would leave sums in the one workspace)
            const bool apart = plan_i.split > 1 && plan_i.unit == PAIRED && plan.split > 1 && plan.unit == PAIRED;
            I.link = apart ? AFTER : LEADS;
            P.link = apart ? AFTER : BESIDE;
            run<PLAIN, false, true, 1>(I, 3, plan_i);
        }
        run<PLAIN, true, true, 3>(P, 4, plan);
    }
};

}  // namespace

// H (and dG and dU), then the copies of operands.  `copies`: some operand starts at an odd address or has rows that do.
size_t ffn_workspace(const FfnShape& f, bool grad, bool copies) {
    const size_t M = (size_t)f.n_tokens, dp = up8(f.d), fp = up8(f.f);
    const size_t hidden = (grad ? 3 : 1) * up256(M * fp * 2);
    if (!copies || (!grad && f.n_tokens <= kFewTokens)) return hidden;   // (ffn_few_kernel copies nothing)
    const size_t x_and_weights = up256(M * dp * 2) + 2 * up256((size_t)f.f * dp * 2) + up256((size_t)f.d * fp * 2);
    return hidden + x_and_weights + (grad ? up256(M * dp * 2) + 2 * up256(M * fp * 2) : 0);   // dY, G and U
}

cudaError_t launch_ffn_forward(sama_ctx* ctx, const FfnShape& f, const void* x, const void* wg, const void* wu,
                               const void* wd, void* y, void* gate, void* up, void* ws, cudaStream_t st) {
    const cudaError_t e = prepare_ffn(ctx);
    if (e != cudaSuccess) return e;
    if (f.dtype == SAMA_BF16) {
        Block<__nv_bfloat16> b{ctx, f, static_cast<uint8_t*>(ws), st, up8(f.f)};
        b.forward(x, wg, wu, wd, y, gate, up);
        return b.err;
    }
    Block<__half> b{ctx, f, static_cast<uint8_t*>(ws), st, up8(f.f)};
    b.forward(x, wg, wu, wd, y, gate, up);
    return b.err;
}

cudaError_t launch_ffn_backward(sama_ctx* ctx, const FfnShape& f, const void* x, const void* wg, const void* wu,
                                const void* wd, const void* gate, const void* up, const void* dy, void* dx, void* dwg,
                                void* dwu, void* dwd, void* ws, cudaStream_t st) {
    const cudaError_t e = prepare_ffn(ctx);
    if (e != cudaSuccess) return e;
    if (f.dtype == SAMA_BF16) {
        Block<__nv_bfloat16> b{ctx, f, static_cast<uint8_t*>(ws), st, up8(f.f)};
        b.backward(x, wg, wu, wd, gate, up, dy, dx, dwg, dwu, dwd);
        return b.err;
    }
    Block<__half> b{ctx, f, static_cast<uint8_t*>(ws), st, up8(f.f)};
    b.backward(x, wg, wu, wd, gate, up, dy, dx, dwg, dwu, dwd);
    return b.err;
}

}  // namespace sama
