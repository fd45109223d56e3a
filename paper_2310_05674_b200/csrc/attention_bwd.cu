// Attention over packed texts, backward, on the 5th-generation tensor cores:
//   P = 2^(x log2 e - lse),  dP = dO V^T,  dX = P (dP - delta) (1 - tanh^2),  delta = dO . O
//   dQ = scale dX K,   dK = scale dX^T Q,   dV = P^T dO
//
// Two launches of one kernel template.  Each CTA keeps 128 rows of two operands and streams tiles of 128 rows of the other
// two past them: d-queries keeps (Q, dO) and streams (K, V); d-keys keeps (K, V) of a key head and streams (Q, dO) of every
// head that shares it.  The products are formed with the kept rows as the lanes of tensor memory (S^T rather than S for
// the keys), so that P and dX go back to tensor memory as the left operands of the last products and no tile is
// transposed.  The sums of a row stay in one accumulator from its first tile to its last: no atomics, a fixed order.
// Forming S and dP in both launches costs seven products in place of the five of one launch that adds to dQ in memory; an
// eighth, P K, puts right what out's rounding does to dQ.
//
// The order of the products of tile i is  dP_i, dV (from P_i), S_i+1, dK (from dX_i), dP_i+1, ...:  P_i+1 is formed from
// S_i+1 while dK and dP_i+1 run, dX_i from dP_i while dV and S_i+1 run.  (d-queries: P K in dV's place, dQ in dK's.)  S, dP and
// two accumulators of 128 columns fill tensor memory.  (Tiles of 64 rows in two buffers, which the two halves of the warps took
// in turn, were slower, 1452 for 1148 us: a product 64 wide takes 48 cycles in place of 32, and each wait of the issuing thread
// leaves the tensor cores idle for some 200 cycles, since it can run ahead of them by a product or two only.)  Heads of up to 64
// columns have tiles of 64 rows and two CTAs per SM, which overlap each other.
//
// delta comes from out as the forward pass rounded it; d-queries adds up what it is off by, puts dQ right, and hands d-keys
// the exact one.
//
// What bounds it (us on one B200, bf16): one text of 8192, 32 heads of 128 over 8, causal, capped: d-queries 1060, d-keys
// 1150 in a short run (1200 and 1300 under the power limit), 620 TFLOP/s of the five products that the definition needs, 995 of
// the eight: forming P and dX between products that wait for them; tensor cores are busy 47 % of the time, as are the issue
// slots.  48 texts of up to 512, 16 heads of 64, biased: 121 and 131, the start and end of CTAs that have three to eight tiles each and the latency of a tile's way.
//
// Roles of the warps: warp 0 copies, warp 1 issues products, the other 16 (or 8) form P and dX: several share 32 rows, each
// of them has 32 of a tile's columns.  Every wait is bounded.
#include <type_traits>

#include "attention.h"

namespace sama {

namespace {

// BT rows of a streamed tile: 128, or for heads of up to 64 columns 64, which leaves room for a second CTA.
template <int D, int BT, bool KEYS> struct BwdTile {
    static constexpr int CTAS = BT == 64 ? 2 : 1;                 // per SM
    static constexpr int FORMING = BT == 64 ? 8 : 16;             // warps that form P and dX
    static constexpr int THREADS = 64 + 32 * FORMING;
    static constexpr int COLS = BT == 64 ? 256 : 512;             // of tensor memory
    // Places for tiles of the first streamed operand, which is needed until the last product of its tile, and of the second:
    // what 227 KB hold.  (Waiting for the copies of 64 KB per tile was a third of d-queries' time with two places for each.)
    static constexpr int FIRST = D == 64 ? 4 : KEYS ? 2 : 3, SECOND = D == 64 ? 4 : 2;
    static_assert(BT == 128 || D == 64, "two CTAs' accumulators");
    static_assert(COLS >= 2 * BT + 2 * D, "scores, their gradients and the sums");
    static constexpr int KEPT = kAttnRows * D * 2, TILE = BT * D * 2;
    static constexpr int STATS = KEYS ? BT * 8 : 0;      // lse and delta of a streamed tile's queries
    static constexpr int SUMS = 2 * kAttnRows * 4;       // d-queries: rows of d_out . out, and of d_out's largest; d-keys: warps of the latter
    static constexpr int SMEM = 2 * KEPT + (FIRST + SECOND) * TILE + FIRST * STATS + SUMS + 256 + 1024;
    static_assert(SMEM * CTAS + 1024 * CTAS <= 228 * 1024, "an SM's shared memory");
};

struct alignas(64) BwdParams {
    CUtensorMap kept[2], streamed[2];   // (Q, dO) and (K, V), or the other way round
    AttnShape a;
    const void *out, *dout;
    const float* lse;
    float *lse2, *delta;   // [heads][n_q]: -lse log2 e (-infinity for a query that sees nothing; fp16: lifted), and -delta
    float* largest;        // fp16: [tile of queries][heads], the largest of d_out
    void* grad[2];      // dQ, or dK and dV
    int64_t ld[2];
    int slots;
};

// What fp16 holds in full is 2^-14 to 65504.  P is lifted by 2^14, and dX by a power of two that takes d_out's largest value to
// 4 .. 8: a row's own for dQ, for dK that of the queries from the first on that sees a key of the tile.  Gradients are as exact
// for any size of d_out (without that, dQ of 2048 keys is off by 0.003 at a d_out of 1e-3, where storing it costs 0.0005).
template <typename T> constexpr float kLift = std::is_same<T, __half>::value ? 14.f : 0.f;
constexpr float kUnlift = 1.f / (1 << 14);
struct BwdPower {
    int e = 0;
    __device__ __forceinline__ BwdPower() {}
    __device__ __forceinline__ explicit BwdPower(float largest) {
        if (largest > 0.f && largest < INFINITY) e = 129 - (int)(__float_as_uint(largest) >> 23);   // (normal: 2^-24 at least)
    }
    __device__ __forceinline__ float up() const { return __uint_as_float((uint32_t)(127 + e) << 23); }
    __device__ __forceinline__ float down() const { return __uint_as_float((uint32_t)(127 - e) << 23); }
};

template <typename T, int D, int BT, AttnCap CAP, bool BIAS, bool KEYS>
__global__ void __launch_bounds__(BwdTile<D, BT, KEYS>::THREADS, BwdTile<D, BT, KEYS>::CTAS)
attn_bwd_kernel(const __grid_constant__ BwdParams P) {
    using C = BwdTile<D, BT, KEYS>;
    constexpr int FORMING = C::FORMING, MY = BT / (FORMING / 4);   // streamed rows, which are columns of P and dX, of a warp
    constexpr int N1 = C::FIRST, N2 = C::SECOND;
    constexpr bool BF16 = std::is_same<T, __nv_bfloat16>::value, HALF = !BF16;
    constexpr uint32_t IDESC_S = idesc16(BF16, false, false, kAttnRows, BT), IDESC_G = idesc16(BF16, false, true, kAttnRows, D);
    constexpr uint32_t COLS = C::COLS;
    const AttnShape& a = P.a;

    pdl_wait();
    if ((!KEYS || a.n_q == 0) && blockIdx.x == 0) attn_check_starts(a);   // (without queries d-keys is the only launch)
    // heavy tiles first: the first keys are seen by most queries, the last queries see most keys
    const int per_slot = KEYS ? a.kv_heads : a.heads, head0 = (int)blockIdx.x % per_slot;
    const int slot = KEYS ? (int)blockIdx.x / per_slot : P.slots - 1 - (int)blockIdx.x / per_slot;
    int tile;
    const int t = attn_find<kAttnRows>(KEYS ? a.k_starts : a.q_starts, a.n_texts, KEYS ? a.n_k : a.n_q, slot, &tile);
    if (t < 0) return;
    const AttnText x = attn_text(a, t);
    const int first = tile * kAttnRows, kept_rows = KEYS ? x.lk : x.lq, streamed_rows = KEYS ? x.lq : x.lk;
    if (first >= kept_rows) return;
    const int kept_base = KEYS ? x.k0 : x.q0, streamed_base = KEYS ? x.q0 : x.k0;

    // streamed tiles: those that the last query sees, or from the first that sees the first key on, for each head
    int tile0 = 0, per_head;
    if (KEYS) {
        tile0 = attn_first_query(a.causal, x, first) / BT;
        per_head = max(0, (x.lq + BT - 1) / BT - tile0);
    } else {
        per_head = (attn_seen(a.causal, x, min(first + kAttnRows, x.lq) - 1) + BT - 1) / BT;
    }
    const int n = per_head * (KEYS ? a.group : 1);

    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    const uint32_t ring1 = base + 2 * C::KEPT, ring2 = ring1 + N1 * C::TILE, stats = ring2 + N2 * C::TILE, sums = stats + N1 * C::STATS;
    const uint32_t bars = sums + C::SUMS;
    auto full1 = [&](int s) { return bars + 8u * s; };
    auto empty1 = [&](int s) { return bars + 8u * (N1 + s); };
    auto full2 = [&](int s) { return bars + 8u * (2 * N1 + s); };
    auto empty2 = [&](int s) { return bars + 8u * (2 * N1 + N2 + s); };
    const uint32_t s_bar = bars + 8u * (2 * N1 + 2 * N2), dp_bar = s_bar + 8u;   // S, dP are there
    const uint32_t p_bar = dp_bar + 8u, x_bar = p_bar + 8u;                 // P is there, over S; dX is there, over dP
    const uint32_t kept_bar = x_bar + 8u, done_bar = kept_bar + 8u;
    const uint32_t tmem_slot = done_bar + 8u;
    volatile uint32_t* tmem_ptr_slot = reinterpret_cast<volatile uint32_t*>(smem_raw + (tmem_slot - raw));
    volatile uint32_t* abort_flag = tmem_ptr_slot + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < N1; ++s) {
            mbar_init(full1(s), KEYS ? 33 : 1);   // the copy, and (d-keys) each lane's share of the statistics
            mbar_init(empty1(s), 1);
        }
        for (int s = 0; s < N2; ++s) {
            mbar_init(full2(s), 1);
            mbar_init(empty2(s), 1);
        }
        mbar_init(s_bar, 1);
        mbar_init(dp_bar, 1);
        mbar_init(p_bar, FORMING);
        mbar_init(x_bar, FORMING);
        mbar_init(kept_bar, 1);
        mbar_init(done_bar, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(tmem_slot, COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // (not before tensor memory is had: a kernel that starts early may take it and wait for this one)
    pdl_trigger();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_ptr_slot, 0);
    const uint32_t s_cols = tmem, dp_cols = tmem + BT;
    auto g_cols = [&](int i) { return tmem + (uint32_t)(2 * BT + i * D); };

    auto raise_timeout = [&]() {
        *abort_flag = 1;
        atomicOr(a.status, (int)SAMA_DEV_TIMEOUT);
    };
    // for all lanes of a warp together
    auto wait = [&](uint32_t bar, int parity) {
        const bool ok = mbar_wait(bar, (uint32_t)parity, abort_flag);
        if (__all_sync(0xffffffffu, ok)) return true;
        raise_timeout();
        return false;
    };

    if (warp == 0) {
        int i = 0;
        bool ok = true, one_ahead = false;   // (one_ahead: a tile's first copy is on its way, its second is not)
        if (n > 0 && lane == 0) {
            mbar_expect_tx(kept_bar, 2 * C::KEPT);
            for (int o = 0; o < 2; ++o)
                for (int c = 0; c < D / 64; ++c)
                    tma_load_3d(base + o * C::KEPT + c * kAttnRows * 128, &P.kept[o], kept_bar, 64 * c, head0, kept_base + first);
        }
        for (; i < n; ++i) {
            const int s1 = i % N1, s2 = i % N2;
            const int h = KEYS ? head0 * a.group + i / per_head : head0 / a.group;
            const int row = streamed_base + (tile0 + (KEYS ? i % per_head : i)) * BT;
            auto load = [&](int o, uint32_t to, uint32_t bar) {
                mbar_expect_tx(bar, C::TILE);
                for (int c = 0; c < D / 64; ++c) tma_load_3d(to + c * BT * 128, &P.streamed[o], bar, 64 * c, h, row);
            };
            if (i >= N1 && !wait(empty1(s1), (i / N1 - 1) & 1)) { ok = false; break; }
            if (lane == 0) load(0, ring1 + s1 * C::TILE, full1(s1));
            if (KEYS) {
                for (int r = lane; r < BT; r += 32) {
                    const int64_t at = (int64_t)h * a.n_q + min(row + r, a.n_q - 1);
                    const uint32_t to = stats + s1 * C::STATS + 4 * r;
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(P.lse2 + at) : "memory");
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to + 4 * BT), "l"(P.delta + at) : "memory");
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(full1(s1)) : "memory");
            }
            one_ahead = true;
            if (i >= N2 && !wait(empty2(s2), (i / N2 - 1) & 1)) { ok = false; break; }
            if (lane == 0) load(1, ring2 + s2 * C::TILE, full2(s2));
            one_ahead = false;
        }
        if (!ok || *abort_flag) {
            // let the copies already issued land before the CTA's shared memory goes away
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (n > 0) mbar_wait(kept_bar, 0);
            const int i1 = i + (one_ahead ? 1 : 0);
            for (int k = max(0, i1 - N1); k < i1; ++k) mbar_wait(full1(k % N1), (k / N1) & 1);
            for (int k = max(0, i - N2); k < i; ++k) mbar_wait(full2(k % N2), (k / N2) & 1);
        }
        __syncwarp();
    } else if (warp == 1) {
        bool ok = n > 0 && wait(kept_bar, 0);
        // S (o = 0) or dP (o = 1) of a tile: kept[o] streamed[o]^T
        auto scores = [&](int o, int s) {
            const uint64_t da = make_desc(base + o * C::KEPT), db = make_desc((o ? ring2 : ring1) + s * C::TILE);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const uint64_t at = (uint64_t)((k / 4 * kAttnRows * 128 + k % 4 * 32) >> 4);
                umma16(o ? dp_cols : s_cols, da + at, db + at, IDESC_S, k > 0);
            }
            umma_commit(o ? dp_bar : s_bar);
        };
        // dK or dQ (o = 0) from dX, dV or d-queries' sum of P K (o = 1) from P.  Each warp has left its columns, in 16 bits, in
        // the first half of its columns of fp32.
        auto gradient = [&](int o, int s, bool add) {
            const uint64_t db = attn_desc_mn((o && KEYS ? ring2 : ring1) + s * C::TILE, BT);
#pragma unroll
            for (int k = 0; k < BT / 16; ++k)
                umma16_ta(g_cols(o), (o ? s_cols : dp_cols) + (uint32_t)(k / (MY / 16) * MY + k % (MY / 16) * 8), db + (uint64_t)(k * 2048 >> 4), IDESC_G, add || k > 0);
        };
        // The first tile; for the others the warps that allow its products have seen to it that it is there.
        if (ok && (ok = wait(full1(0), 0) && wait(full2(0), 0))) {
            tc_fence_after();
            if (streamed_rows - tile0 * BT < BT) {
                attn_zero_rows<D / 64>(ring1, streamed_rows - tile0 * BT, BT, 0, 1);
                attn_zero_rows<D / 64>(ring2, streamed_rows - tile0 * BT, BT, 0, 1);
            }
            if (elect_one()) {
                scores(0, 0);
                scores(1, 0);
                if (!KEYS && N2 < n) umma_commit(empty2(0));
            }
        }
        int s1 = 0, s2 = 0, next1 = 1 % N1, next2 = 1 % N2;
        for (int i = 0; ok && i < n; ++i) {
            if (!(ok = wait(p_bar, i & 1))) break;
            tc_fence_after();
            if (elect_one()) {
                gradient(1, KEYS ? s2 : s1, i > 0);
                if (KEYS && i + N2 < n) umma_commit(empty2(s2));
                // (products are executed in order: the next scores do not overtake the weights they replace)
                if (i + 1 < n) scores(0, next1);
            }
            __syncwarp();
            if (!(ok = wait(x_bar, i & 1))) break;
            tc_fence_after();
            if (elect_one()) {
                gradient(0, s1, i > 0);
                if (i + N1 < n) umma_commit(empty1(s1));
                if (i + 1 < n) {
                    scores(1, next2);
                    if (!KEYS && i + 1 + N2 < n) umma_commit(empty2(next2));
                } else {
                    umma_commit(done_bar);
                }
            }
            __syncwarp();
            s1 = next1;
            s2 = next2;
            if (++next1 == N1) next1 = 0;
            if (++next2 == N2) next2 = 0;
        }
    } else {
        const int w = (warp - 2) >> 2, quarter = warp & 3;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const int row0 = first + quarter * 32, row = row0 + lane;   // in the text
        const bool real = row < kept_rows;
        const float c = (CAP ? a.cap : a.scale) * kLog2e;
        const AttnTanh capped(CAP ? a.scale / a.cap : 0.f, 1.f);
        bool ok = true;

        float lse2 = 0.f, delta = 0.f;   // (both negated)
        BwdPower power;                  // of dX
        volatile float* part = reinterpret_cast<volatile float*>(smem_raw + (sums - raw));
        // sum P (dP - delta), which is what delta is off by for out's rounding: it is put right in dQ by off sum P (1 - tanh^2) K,
        // which takes a product of its own, and in delta for d-keys.  (Without that, keys and values with a common offset of
        // their spread have dQ off by 0.01 to 0.02 in bf16, of four times that by a third: dQ does not grow with the offset,
        // out's rounding and the sum of P K do.)
        float2 off[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        if (!KEYS) {
            // each warp takes some rows, whose columns are added up by lanes next to one another (with a row per lane, the way
            // to delta took 6500 of a CTA's 17,000 cycles for texts of a few hundred tokens)
            constexpr int LANES = D / 8, AT_ONCE = 32 / LANES, EACH = kAttnRows / FORMING, N = EACH / AT_ONCE;
            const int r0 = (warp - 2) * EACH + lane / LANES, col = lane % LANES * 8;
            uint4 o[N], d[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int r = first + r0 + i * AT_ONCE;
                o[i] = d[i] = make_uint4(0u, 0u, 0u, 0u);
                if (r < kept_rows && col < a.dim) {
                    const int64_t at = ((int64_t)(x.q0 + r) * a.heads + head0) * a.dim + col;
                    o[i] = *reinterpret_cast<const uint4*>(static_cast<const T*>(P.out) + at);
                    d[i] = *reinterpret_cast<const uint4*>(static_cast<const T*>(P.dout) + at);
                }
            }
            if (real) {
                lse2 = P.lse[(int64_t)head0 * a.n_q + x.q0 + row] * -kLog2e;
                lse2 = lse2 == INFINITY ? -INFINITY : lse2 + kLift<T>;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t u[4] = {o[i].x, o[i].y, o[i].z, o[i].w}, v[4] = {d[i].x, d[i].y, d[i].z, d[i].w};
                float sum = 0.f, most = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 f = unpack2<T>(u[e]), g = unpack2<T>(v[e]);
                    sum = fmaf(f.x, g.x, fmaf(f.y, g.y, sum));
                    if (HALF) most = fmaxf(most, fmaxf(fabsf(g.x), fabsf(g.y)));
                }
#pragma unroll
                for (int x = 1; x < LANES; x *= 2) {
                    sum += __shfl_xor_sync(0xffffffffu, sum, x);
                    if (HALF) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, x));
                }
                if (col == 0) {
                    part[r0 + i * AT_ONCE] = sum;
                    if (HALF) part[kAttnRows + r0 + i * AT_ONCE] = most;
                }
            }
            asm volatile("bar.sync 1, %0;" ::"n"(32 * FORMING) : "memory");
            delta = -part[quarter * 32 + lane];
            if (HALF) {
                power = BwdPower(part[kAttnRows + quarter * 32 + lane]);
                if (warp == 2) {
                    float most = 0.f;
                    for (int r = lane; r < kAttnRows; r += 32) most = fmaxf(most, part[kAttnRows + r]);
#pragma unroll
                    for (int x = 16; x > 0; x /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, x));
                    if (lane == 0) P.largest[(int64_t)slot * a.heads + head0] = most;
                }
            }
            if (w == 0 && real) P.lse2[(int64_t)head0 * a.n_q + x.q0 + row] = lse2;
        }
        if (KEYS && HALF) {
            const int from = tile0 * BT / kAttnRows, tiles = max((x.lq + kAttnRows - 1) / kAttnRows - from, 0), all = tiles * a.group;
            const float* largest = P.largest + (int64_t)(x.q0 / kAttnRows + t + from) * a.heads + head0 * a.group;
            float most = 0.f;
            for (int i = threadIdx.x - 64; i < all; i += 32 * FORMING) most = fmaxf(most, largest[(int64_t)(i / a.group) * a.heads + i % a.group]);
#pragma unroll
            for (int x = 16; x > 0; x /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, x));
            if (lane == 0) part[warp - 2] = most;
            asm volatile("bar.sync 1, %0;" ::"n"(32 * FORMING) : "memory");
            for (int i = 0; i < FORMING; ++i) most = fmaxf(most, part[i]);
            power = BwdPower(most);
        }
        const float raise = HALF ? power.up() * kUnlift : 1.f, lower = HALF ? power.down() : 1.f;   // of dP, and of what comes of dX
        // d-queries: the row sees keys below `edge`; d-keys: the row is seen by queries from `edge` on
        const int edge = KEYS ? attn_first_query(a.causal, x, row) : attn_seen(a.causal, x, row);
        const int edge_of_all = KEYS ? attn_first_query(a.causal, x, row0 + 31) : attn_seen(a.causal, x, row0);

        int s1 = 0, next1 = 1 % N1, parity1 = N1 == 1, next2 = 1 % N2, parity2 = N2 == 1, tile_of_head = 0, head = KEYS ? head0 * a.group : head0;
        float slope = BIAS ? a.slopes[head] * kLog2e : 0.f;
        // The products of the next tile are allowed once it is there, and holds zeros beyond its text.  (The waits are here
        // because each one of the issuing thread's leaves the tensor cores idle.)
        auto ready = [&](int o, int i) {
            if (i + 1 >= n) return true;
            if (!wait(o ? full2(next2) : full1(next1), o ? parity2 : parity1)) return false;
            const int next_tile = tile_of_head + 1 == per_head ? 0 : tile_of_head + 1, from = streamed_rows - (tile0 + next_tile) * BT;
            if (from < BT) attn_zero_rows<D / 64>(o ? ring2 + next2 * C::TILE : ring1 + next1 * C::TILE, from, BT, warp - 2, FORMING);
            return true;
        };
        const float raised_delta = delta * raise;
        if (KEYS && n > 0) ok = wait(full1(0), 0);
        for (int i = 0; ok && i < n; ++i) {
            const int at = (tile0 + tile_of_head) * BT + w * MY;   // this warp's first streamed row, in the text
            const float* lses = reinterpret_cast<const float*>(smem_raw + (stats - raw) + s1 * C::STATS) + w * MY;
            const float* deltas = lses + BT;
            if (!(ok = wait(s_bar, i & 1))) break;
            tc_fence_after();
            const bool masked = KEYS ? at < edge_of_all || at + MY > x.lq : at + MY > edge_of_all;
            const int lo = KEYS ? edge - at : 0, hi = KEYS ? x.lq - at : edge - at;   // visible columns
            const float away = BIAS ? (float)(KEYS ? row - (x.lk - x.lq) - at : attn_position(x, row) - at) : 0.f;
            float p[MY];   // the weights, d-keys': in the end times 1 - tanh^2
            float slack_of[CAP && !KEYS ? MY : 1];
#pragma unroll
            for (int k = 0; k < MY; k += 32) tmem_ld32_nowait(s_cols + lanes + w * MY + k, p + k);
            tmem_wait_ld();
            auto weights = [&](auto form, auto some) {   // (form: of tanh; some: scores are masked)
#pragma unroll
                for (int h = 0; h < MY; h += 32) {
                    uint32_t r[16];
#pragma unroll
                    for (int k = h; k < h + 32; k += 4) {
                        float4 lse4 = make_float4(lse2, lse2, lse2, lse2);
                        if (KEYS) lse4 = *reinterpret_cast<const float4*>(lses + k);
                        const float l4[4] = {lse4.x, lse4.y, lse4.z, lse4.w};
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            float2 v = make_float2(p[k + e], p[k + e + 1]), l2 = make_float2(l4[e], l4[e + 1]), slack = both(1.f);
                            if (CAP) {
                                v = capped.of<decltype(form)::value>(v);
                                slack = fma2(mul2(v, both(-1.f)), v, both(1.f));
                            }
                            if (BIAS) l2 = fma2(make_float2(fabsf(away - (float)(k + e)), fabsf(away - (float)(k + e + 1))), both(-slope), l2);
                            v = fma2(v, both(c), l2);
                            v = make_float2(fast_exp2(v.x), fast_exp2(v.y));
                            if (decltype(some)::value && (k + e >= hi || (KEYS && k + e < lo))) v.x = slack.x = 0.f;
                            if (decltype(some)::value && (k + e + 1 >= hi || (KEYS && k + e + 1 < lo))) v.y = slack.y = 0.f;
                            const float2 flat = CAP ? mul2(v, slack) : v, operand = KEYS ? v : flat;
                            r[(k + e - h) / 2] = pack2<T>(operand.x, operand.y);
                            if (KEYS) v = flat;
                            if (CAP && !KEYS) { slack_of[k + e] = slack.x; slack_of[k + e + 1] = slack.y; }
                            p[k + e] = v.x;
                            p[k + e + 1] = v.y;
                        }
                    }
                    // over the scores that this thread has read
                    tmem_st16_nowait(s_cols + lanes + w * MY + h / 2, r);
                }
            };
            constexpr std::integral_constant<int, kNear> near;
            constexpr std::integral_constant<int, CAP == kWideCap ? kAny : kFar> far;
            if constexpr (CAP != kNoCap) {
                // (what another text has in the tile decides nothing)
                const float big = real ? attn_max<MY>([&](int k) { return fabsf(p[k]); }) : 0.f;
                if (masked || !__all_sync(0xffffffffu, capped.is_near(big))) weights(far, std::true_type());
                else weights(near, std::false_type());
            } else if (masked) {
                weights(far, std::true_type());
            } else {
                weights(far, std::false_type());
            }
            tmem_wait_st();
            tc_fence_before();
            if (!(ok = ready(0, i))) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(p_bar);
            if (!(ok = wait(dp_bar, i & 1))) break;
            tc_fence_after();
            auto slopes_of_scores = [&](auto some) {
#pragma unroll
                for (int h = 0; h < MY; h += 32) {
                    constexpr int PIECE = CAP && !KEYS ? 16 : 32;   // (16: what registers hold beside the slacks)
                    float dp[32];
                    uint32_t r[16];
#pragma unroll
                    for (int k = 0; k < 32; k += 4) {
                        if (k % PIECE == 0) {
                            if (PIECE == 16) tmem_ld16_nowait(dp_cols + lanes + w * MY + h + k, reinterpret_cast<uint32_t*>(dp) + k);
                            else tmem_ld32_nowait(dp_cols + lanes + w * MY + h, dp);
                            tmem_wait_ld();
                        }
                        float4 d4 = make_float4(raised_delta, raised_delta, raised_delta, raised_delta);
                        if (KEYS) d4 = *reinterpret_cast<const float4*>(deltas + h + k);
                        const float d[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            const int at = h + k + e;
                            float2 g = make_float2(dp[k + e], dp[k + e + 1]), d2 = make_float2(d[e], d[e + 1]);
                            if (HALF && KEYS) d2 = mul2(d2, both(raise));
                            g = mul2(make_float2(p[at], p[at + 1]), HALF ? fma2(g, both(raise), d2) : add2(g, d2));
                            if (decltype(some)::value && (at >= hi || (KEYS && at < lo))) g.x = 0.f;
                            if (decltype(some)::value && (at + 1 >= hi || (KEYS && at + 1 < lo))) g.y = 0.f;
                            if (!KEYS) off[e / 2] = add2(off[e / 2], g);
                            if (CAP && !KEYS) g = mul2(g, make_float2(slack_of[at], slack_of[at + 1]));
                            r[(k + e) / 2] = pack2<T>(g.x, g.y);
                        }
                    }
                    tmem_st16_nowait(dp_cols + lanes + w * MY + h / 2, r);
                }
            };
            if (masked) slopes_of_scores(std::true_type()); else slopes_of_scores(std::false_type());
            tmem_wait_st();
            tc_fence_before();
            if (!(ok = ready(1, i))) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(x_bar);
            s1 = next1;
            if (++next1 == N1) { next1 = 0; parity1 ^= 1; }
            if (++next2 == N2) { next2 = 0; parity2 ^= 1; }
            if (++tile_of_head == per_head && KEYS && i + 1 < n) {
                tile_of_head = 0;
                ++head;
                if (BIAS) slope = a.slopes[head] * kLog2e;
            }
        }
        if (ok && n > 0) ok = wait(done_bar, 0);
        float shift = 0.f;   // this row's, of all its warps
        if (!KEYS) {
            // d-keys gets the exact delta.  (The kept operands' place is free now.)
            volatile float* all = reinterpret_cast<volatile float*>(smem_raw + (base - raw)) + quarter * 32 + lane;
            all[w * kAttnRows] = (off[0].x + off[0].y) + (off[1].x + off[1].y);
            asm volatile("bar.sync 1, %0;" ::"n"(32 * FORMING) : "memory");
#pragma unroll
            for (int i = 0; i < FORMING / 4; ++i) shift += all[i * kAttnRows];
            if (w == 0 && real) P.delta[(int64_t)head0 * a.n_q + x.q0 + row] = delta - shift * lower;
            if (HALF) shift *= kUnlift;
        }
        // the kept operands' places, where all products are done (d-queries: the second's, the sums of `off` are in the first's)
        auto stage_of = [&](int o) { return base + (KEYS ? o : 1) * C::KEPT; };
        if (ok) {
            tc_fence_after();
            // 32 columns at a time: d-keys' warps have dK or dV
            constexpr int SHARES = FORMING / 4;
            const int which = KEYS ? w % 2 : 0, k0 = 32 * (KEYS ? w / 2 : w);
            const float f = which == 0 ? a.scale * lower : HALF ? kUnlift : 1.f;
#pragma unroll 1
            for (int k = k0; k < D; k += 32 * (KEYS ? SHARES / 2 : SHARES)) {
                float v[32];
                if (n > 0) {
                    tmem_ld32_nowait(g_cols(which) + lanes + k, v);
                    tmem_wait_ld();
                    if (!KEYS) {
                        float pk[32];
                        tmem_ld32_nowait(g_cols(1) + lanes + k, pk);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = fmaf(-shift, pk[e], v[e]);
                    }
                }
#pragma unroll
                for (int e = 0; e < 32; ++e) v[e] = n > 0 ? v[e] * f : 0.f;
#pragma unroll
                for (int e = 0; e < 32; e += 8) attn_stage<T, D>(stage_of(which), quarter * 32 + lane, k + e, v + e);
            }
        }
        asm volatile("bar.sync 1, %0;" ::"n"(32 * FORMING) : "memory");
        if (ok) {
            for (int o = 0; o < (KEYS ? 2 : 1); ++o)
                attn_unstage<T, D, FORMING>(stage_of(o), kept_rows - first, a.dim, static_cast<T*>(P.grad[o]) + (int64_t)(kept_base + first) * P.ld[o] + (int64_t)head0 * a.dim,
                                            P.ld[o], warp - 2);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem, COLS);
}

template <typename T, int D, int BT, AttnCap CAP, bool BIAS, bool KEYS>
cudaError_t launch(sama_ctx* ctx, const BwdParams& P, cudaStream_t st) {
    using C = BwdTile<D, BT, KEYS>;
    auto* kernel = attn_bwd_kernel<T, D, BT, CAP, BIAS, KEYS>;
    const uint64_t bit = 1ull << ((BT == 64 ? 32 : 0) + (std::is_same<T, __half>::value ? 16 : 0) + (D == 64 ? 8 : 0) + 2 * CAP + (BIAS ? 1 : 0));
    if (!(ctx->attn_bwd_ready[KEYS] & bit)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
        if (e != cudaSuccess) return e;
        ctx->attn_bwd_ready[KEYS] |= bit;
    }
    KernelScope scope(ctx, SAMA_K_ATTN, KEYS ? 2 : 1, st);
    const int64_t blocks = (int64_t)P.slots * (KEYS ? P.a.kv_heads : P.a.heads);
    return launch_dependent(kernel, dim3((unsigned)blocks), dim3(C::THREADS), C::SMEM, st, P);
}
template <typename T, int D, int BT, bool KEYS>
cudaError_t launch(sama_ctx* ctx, const BwdParams& P, cudaStream_t st) {
    switch (attn_cap(P.a.cap)) {
        case kNoCap: return P.a.slopes ? launch<T, D, BT, kNoCap, true, KEYS>(ctx, P, st) : launch<T, D, BT, kNoCap, false, KEYS>(ctx, P, st);
        case kCap: return P.a.slopes ? launch<T, D, BT, kCap, true, KEYS>(ctx, P, st) : launch<T, D, BT, kCap, false, KEYS>(ctx, P, st);
        default: return P.a.slopes ? launch<T, D, BT, kWideCap, true, KEYS>(ctx, P, st) : launch<T, D, BT, kWideCap, false, KEYS>(ctx, P, st);
    }
}
template <typename T, bool KEYS>
cudaError_t launch(sama_ctx* ctx, int bt, const BwdParams& P, cudaStream_t st) {
    if (P.a.dim > 64) return launch<T, 128, 128, KEYS>(ctx, P, st);
    return bt == 64 ? launch<T, 64, 64, KEYS>(ctx, P, st) : launch<T, 64, 128, KEYS>(ctx, P, st);
}
template <bool KEYS>
cudaError_t launch(sama_ctx* ctx, int dtype, int bt, const BwdParams& P, cudaStream_t st) {
    return dtype == SAMA_BF16 ? launch<__nv_bfloat16, KEYS>(ctx, bt, P, st) : launch<__half, KEYS>(ctx, bt, P, st);
}

}  // namespace

size_t attention_grad_workspace(const AttnShape& a) {
    return a.n_q == 0 ? 0 : (size_t)a.heads * ((size_t)a.n_q * 2 + a.n_q / kAttnRows + a.n_texts) * sizeof(float);
}

cudaError_t launch_attention_grad(sama_ctx* ctx, const AttnShape& a, const AttnOperands& op, const void* out, const float* lse,
                                  const void* dout, void* dq, void* dk, void* dv, void* ws, cudaStream_t st) {
    BwdParams P;
    P.a = a;
    P.out = out;
    P.dout = dout;
    P.lse = lse;
    P.lse2 = static_cast<float*>(ws);
    P.delta = P.lse2 + (size_t)a.heads * a.n_q;
    P.largest = P.delta + (size_t)a.heads * a.n_q;
    const int64_t dense = (int64_t)a.heads * a.dim;
    // Small tiles, two CTAs per SM, unless capped scores, whose arithmetic weighs more, are many (us for d-queries and d-keys,
    // 16 heads of 64: 16 texts of up to 512 38 and 41, with the large ones 48 and 49, capped 54 and 52, 61 and 61; one of 8192,
    // causal, 283 and 319, 320 and 356; but 4 of up to 2048, causal and capped, 92 and 94, 82 and 85).  Lengths are on the device, but
    // their mean is known.
    const int bt = a.dim <= 64 && (a.cap == 0.f || a.n_q <= 512 * (int64_t)a.n_texts) ? 64 : 128;
    auto query_maps = [&](CUtensorMap* m, int rows) {
        return attn_map(&m[0], op.q, op.dtype, a.dim, a.heads, a.n_q, op.q_stride, rows) &&
               attn_map(&m[1], dout, op.dtype, a.dim, a.heads, a.n_q, dense, rows);
    };
    auto key_maps = [&](CUtensorMap* m, int rows) {
        return attn_map(&m[0], op.k, op.dtype, a.dim, a.kv_heads, a.n_k, op.k_stride, rows) &&
               attn_map(&m[1], op.v, op.dtype, a.dim, a.kv_heads, a.n_k, op.v_stride, rows);
    };
    if (a.n_q > 0) {
        // (without keys nothing is loaded, but a map has to describe something)
        if (!query_maps(P.kept, kAttnRows) || !(a.n_k > 0 ? key_maps(P.streamed, bt) : query_maps(P.streamed, bt)))
            return cudaErrorInvalidValue;
        P.grad[0] = P.grad[1] = dq;
        P.ld[0] = P.ld[1] = op.q_stride;
        P.slots = a.n_q / kAttnRows + a.n_texts;
        const cudaError_t e = launch<false>(ctx, op.dtype, bt, P, st);
        if (e != cudaSuccess) return e;
    }
    if (a.n_k == 0) return cudaSuccess;
    if (!key_maps(P.kept, kAttnRows) || !(a.n_q > 0 ? query_maps(P.streamed, bt) : key_maps(P.streamed, bt))) return cudaErrorInvalidValue;
    P.grad[0] = dk;
    P.grad[1] = dv;
    P.ld[0] = op.k_stride;
    P.ld[1] = op.v_stride;
    P.slots = a.n_k / kAttnRows + a.n_texts;
    return launch<true>(ctx, op.dtype, bt, P, st);
}

}  // namespace sama
