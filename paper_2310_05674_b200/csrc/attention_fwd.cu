// Attention over packed texts, forward: out = softmax(scores) V in one pass over the keys, with the running maximum and
// sum of the softmax, on the 5th-generation tensor cores.
//
// A CTA has 128 or 256 queries of one text and head, one or two tiles of 128, and streams the keys and values that they see.
// A score tile S = Q K^T is produced in tensor memory; four warps, or eight that share its columns, turn it into weights
// P = 2^(x log2 e - m), which go back to tensor memory in 16 bits over the scores they came from, and O += P V takes them
// from there.  While one tile's weights are formed the other's products run: the other tile of the CTA, which shares the
// keys and values, or that of another CTA of the SM (heads of more than 64 columns: two CTAs; others: three).  The maximum m
// that the weights refer to is only raised when a score exceeds it by more than 8 binary orders (O and the sum are scaled
// then): the weights stay below 2^8.  bf16 rounds them relative to their size whatever they refer to; fp16, which has fewer places
// below 2^-14, gets them lifted by 2^7, so that those from 2^-21 of the largest on keep all of theirs.
//
// What bounds it (one B200, bf16): the chain from a tile's scores to its weights and their products; one text of 8192, 32
// heads of 128 over 8, causal: 466 us, 1180 TFLOP/s of the pairs that are seen (0.72 of the measured rate), 650 with a cap;
// 48 texts of up to 512, 16 heads of 64, biased: 90, where ragged tiles and the start and end of short CTAs weigh as much.
// Two prompts' next 1000 tokens behind 7000: 255 us; tensor cores and special-function units are in use for 52 % of the time,
// issue slots for 30, and 512 CTAs fill 296 places less than twice.  Exponentials by a polynomial for a quarter of the scores,
// and rounding to bf16 by integer addition, were slower (275, 254): more instructions in the chain.  For heads of 64, four
// CTAs per SM (spilled registers, 102 us for 90) and two warps per 32 rows (97) were slower.
//
// Roles of the warps: warp 0 copies (TMA, 128-byte swizzle), warp 1 issues products, the others the softmax.  Every wait is
// bounded: one that expires raises SAMA_DEV_TIMEOUT and ends the CTA's work.
#include <type_traits>

#include "attention.h"

namespace sama {

namespace {

constexpr float kRaise = 8.f;
template <typename T> constexpr float kLift = std::is_same<T, __half>::value ? 7.f : 0.f;   // (2^(8 + 7) fits)

// NW: tiles of queries of a CTA.
template <int D, int NW> struct FwdTile {
    static constexpr int HALVES = NW;                    // warps that share 32 rows of a tile, and the columns of its scores
    static constexpr int THREADS = 64 + 128 * NW * HALVES;
    static constexpr int CTAS = D == 64 ? 3 : 3 - NW;    // per SM
    static constexpr int BK = D == 64 ? 64 : 128;        // keys of a tile
    static constexpr int STAGES = D == 64 ? 4 : 2 * NW;  // tiles of keys or values in shared memory
    static constexpr int Q_BYTES = kAttnRows * D * 2, KV_BYTES = BK * D * 2;
    static constexpr int SHARED = HALVES == 1 ? 0 : 2 * NW * HALVES * kAttnRows * 4;
    static constexpr int SMEM = NW * Q_BYTES + STAGES * KV_BYTES + SHARED + 256 + 1024;
    static constexpr int COLS = NW * (BK + D);           // of tensor memory: a score tile and an output for each tile of queries
    static_assert((COLS & (COLS - 1)) == 0 && COLS * CTAS <= 512, "tensor memory is had in powers of two");
};

struct alignas(64) FwdParams {
    CUtensorMap q, k, v;
    AttnShape a;
    void* out;
    float* lse;
    int slots;
};

template <typename T, int D, int NW, AttnCap CAP, bool BIAS>
__global__ void __launch_bounds__((FwdTile<D, NW>::THREADS), (FwdTile<D, NW>::CTAS))
attn_fwd_kernel(const __grid_constant__ FwdParams P) {
    using C = FwdTile<D, NW>;
    constexpr int BK = C::BK, STAGES = C::STAGES, HALVES = C::HALVES, MY = BK / HALVES;   // MY: columns of a warp
    constexpr bool BF16 = std::is_same<T, __nv_bfloat16>::value;
    constexpr uint32_t IDESC_S = idesc16(BF16, false, false, kAttnRows, BK), IDESC_O = idesc16(BF16, false, true, kAttnRows, D);
    const AttnShape& a = P.a;

    pdl_wait();
    if (blockIdx.x == 0) attn_check_starts(a);
    // the last tiles of a text, which see the most keys, come first
    const int slot = P.slots - 1 - (int)blockIdx.x / a.heads, head = (int)blockIdx.x % a.heads;
    int tile;
    const int t = attn_find<NW * kAttnRows>(a.q_starts, a.n_texts, a.n_q, slot, &tile);
    if (t < 0) return;
    const AttnText x = attn_text(a, t);
    const int first = tile * NW * kAttnRows;
    if (first >= x.lq) return;

    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    const uint32_t ring = base + NW * C::Q_BYTES, shared = ring + STAGES * C::KV_BYTES, bars = shared + C::SHARED;
    auto full_bar = [&](int s) { return bars + 8u * s; };
    auto empty_bar = [&](int s) { return bars + 8u * (STAGES + s); };
    auto q_bar = [&](int w) { return bars + 8u * (2 * STAGES + w); };
    auto s_bar = [&](int w) { return bars + 8u * (2 * STAGES + 2 + w); };   // scores are there
    auto p_bar = [&](int w) { return bars + 8u * (2 * STAGES + 4 + w); };   // weights are there
    auto o_bar = [&](int w) { return bars + 8u * (2 * STAGES + 6 + w); };   // the output is complete
    const uint32_t tmem_slot = bars + 8u * (2 * STAGES + 8);
    volatile uint32_t* tmem_ptr_slot = reinterpret_cast<volatile uint32_t*>(smem_raw + (tmem_slot - raw));
    volatile uint32_t* abort_flag = tmem_ptr_slot + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int w = 0; w < NW; ++w) {
            mbar_init(q_bar(w), 1);
            mbar_init(s_bar(w), 1);
            mbar_init(p_bar(w), 4 * HALVES);
            mbar_init(o_bar(w), 1);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(tmem_slot, C::COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // (not before tensor memory is had: a kernel that starts early may take it and wait for this one)
    pdl_trigger();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_ptr_slot, 0);
    auto s_cols = [&](int w) { return tmem + (uint32_t)(w * BK); };
    auto o_cols = [&](int w) { return tmem + (uint32_t)(NW * BK + w * D); };

    // key tiles that the last query of each of the two tiles sees
    int n_kt[NW], n_all = 0;
    for (int w = 0; w < NW; ++w) {
        const int i0 = first + w * kAttnRows;
        n_kt[w] = i0 < x.lq ? (attn_seen(a.causal, x, min(i0 + kAttnRows, x.lq) - 1) + BK - 1) / BK : 0;
        n_all = max(n_all, n_kt[w]);
    }
    const int items = 2 * n_all;   // keys and values in turn
    const int kv_head = head / a.group;

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
        if (lane == 0 && n_all > 0) {
            auto load_q = [&](int w) {
                if (n_kt[w] == 0) return;
                mbar_expect_tx(q_bar(w), C::Q_BYTES);
                for (int c = 0; c < D / 64; ++c)
                    tma_load_3d(base + w * C::Q_BYTES + c * kAttnRows * 128, &P.q, q_bar(w), 64 * c, head, x.q0 + first + w * kAttnRows);
            };
            load_q(0);
            int item = 0;
            for (; item < items; ++item) {
                const int s = item % STAGES;
                if (item >= STAGES && !mbar_wait(empty_bar(s), (item / STAGES - 1) & 1, abort_flag)) { raise_timeout(); break; }
                mbar_expect_tx(full_bar(s), C::KV_BYTES);
                for (int c = 0; c < D / 64; ++c)
                    tma_load_3d(ring + s * C::KV_BYTES + c * BK * 128, item & 1 ? &P.v : &P.k, full_bar(s), 64 * c, kv_head, x.k0 + (item >> 1) * BK);
                if (item == 0 && NW > 1) load_q(1);
            }
            if (*abort_flag) {
                // let the copies already issued land before the CTA's shared memory goes away
                for (int w = 0; w < NW; ++w)
                    if (n_kt[w] > 0) mbar_wait(q_bar(w), 0);
                for (int i = max(0, item - STAGES); i < item; ++i) mbar_wait(full_bar(i % STAGES), (i / STAGES) & 1);
            }
        }
    } else if (warp == 1) {
        bool ok = true;
        auto wait_item = [&](int item) {
            ok = ok && wait(full_bar(item % STAGES), (item / STAGES) & 1);
            tc_fence_after();
        };
        auto release = [&](int item) {
            if (item + STAGES < items) umma_commit(empty_bar(item % STAGES));
        };
        auto scores = [&](int w, int j) {   // S_w = Q_w K_j^T
            const uint64_t dq = make_desc(base + w * C::Q_BYTES), dk = make_desc(ring + (2 * j) % STAGES * C::KV_BYTES);
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
                umma16(s_cols(w), dq + (uint64_t)((k / 4 * kAttnRows * 128 + k % 4 * 32) >> 4),
                       dk + (uint64_t)((k / 4 * BK * 128 + k % 4 * 32) >> 4), IDESC_S, k > 0);
            umma_commit(s_bar(w));
        };
        if (n_all > 0) {
            wait_item(0);
            for (int w = 0; w < NW && ok; ++w) {
                if (n_kt[w] == 0) continue;
                if (!(ok = wait(q_bar(w), 0))) break;
                tc_fence_after();
                if (elect_one()) scores(w, 0);
            }
            if (ok && elect_one()) release(0);
        }
        for (int j = 0; ok && j < n_all; ++j) {
            const int vs = (2 * j + 1) % STAGES;
            wait_item(2 * j + 1);
            if (!ok) break;
            if ((j + 1) * BK > x.lk) attn_zero_rows<D / 64>(ring + vs * C::KV_BYTES, x.lk - j * BK, BK, 0, 1);
            if (j + 1 < n_all) wait_item(2 * j + 2);
            for (int w = 0; w < NW && ok; ++w) {
                if (j >= n_kt[w]) continue;
                if (!(ok = wait(p_bar(w), j & 1))) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t dv = attn_desc_mn(ring + vs * C::KV_BYTES, BK);
#pragma unroll
                    for (int k = 0; k < BK / 16; ++k)
                        umma16_ta(o_cols(w), s_cols(w) + (uint32_t)(k / (MY / 16) * MY + k % (MY / 16) * 8), dv + (uint64_t)(k * 2048 >> 4), IDESC_O, j > 0 || k > 0);
                    // (products are executed in order: the next scores do not overtake the weights they replace)
                    if (j + 1 < n_kt[w]) scores(w, j + 1); else umma_commit(o_bar(w));
                }
            }
            if (ok && elect_one()) {
                release(2 * j + 1);
                if (j + 1 < n_all) release(2 * j + 2);
            }
            __syncwarp();
        }
    } else {
        const int w = (warp - 2) / (4 * HALVES), half = (warp - 2) / 4 % HALVES, quarter = warp & 3;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const int row0 = first + w * kAttnRows + quarter * 32, row = row0 + lane;   // in the text
        const int seen = attn_seen(a.causal, x, row), seen_by_all = attn_seen(a.causal, x, row0);
        constexpr bool RAW = !CAP && !BIAS;     // scores as they come, the factor is applied in the exponent
        const float c = RAW ? a.scale * kLog2e : 1.f;
        const float slope = BIAS ? a.slopes[head] * kLog2e : 0.f;
        const AttnTanh capped(CAP ? a.scale / a.cap : 0.f, CAP ? a.cap * kLog2e : 0.f);
        // What the other half of a row's columns has: by turns in two places, so that one barrier per exchange is enough.
        volatile float* mine = reinterpret_cast<volatile float*>(smem_raw + (shared - raw)) + (w * HALVES + half) * kAttnRows + quarter * 32 + lane;
        volatile float* other = mine + (half ? -kAttnRows : kAttnRows);
        auto exchange = [&](float v, int turn) {
            constexpr int TURN = NW * HALVES * kAttnRows;
            mine[turn * TURN] = v;
            asm volatile("bar.sync %0, 64;" ::"r"(1 + w * 4 + quarter) : "memory");
            return other[turn * TURN];
        };
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        for (int j = 0; j < n_kt[w]; ++j) {
            if (!(ok = wait(s_bar(w), j & 1))) break;
            tc_fence_after();
            float s[MY];
#pragma unroll
            for (int k = 0; k < MY; k += 32) tmem_ld32_nowait(s_cols(w) + lanes + half * MY + k, s + k);
            tmem_wait_ld();
            const bool masked = (j + 1) * BK > seen_by_all;
            const int left = seen - j * BK - half * MY;   // columns that the row sees
            if (CAP) {
                auto cap_all = [&](auto form) {
#pragma unroll
                    for (int k = 0; k < MY; k += 2) {
                        const float2 v = capped.of<decltype(form)::value>(make_float2(s[k], s[k + 1]));
                        s[k] = v.x;
                        s[k + 1] = v.y;
                    }
                };
                // (what another text has in the tile decides nothing)
                if (masked) {
#pragma unroll
                    for (int k = 0; k < MY; ++k) s[k] = k < left ? s[k] : 0.f;
                }
                const float big = row < x.lq ? attn_max<MY>([&](int k) { return fabsf(s[k]); }) : 0.f;
                if (__all_sync(0xffffffffu, capped.is_near(big))) cap_all(std::integral_constant<int, kNear>());
                else cap_all(std::integral_constant<int, CAP == kWideCap ? kAny : kFar>());
            }
            if (BIAS) {
                const int ahead = attn_position(x, row0) - j * BK - half * MY;   // of this warp's first row, over the first column
                const float away = (float)(ahead + lane);
                auto bias = [&](auto of) {
#pragma unroll
                    for (int k = 0; k < MY; k += 2) {
                        const float2 b = make_float2(of(k), of(k + 1)), v = make_float2(s[k], s[k + 1]);
                        const float2 y = CAP ? add2(v, b) : fma2(v, both(a.scale * kLog2e), b);
                        s[k] = y.x;
                        s[k + 1] = y.y;
                    }
                };
                // (one operation less where all columns lie on one side of all rows)
                const float sign = ahead >= MY - 1 ? slope : -slope, from = -sign * away;
                if (ahead >= MY - 1 || ahead + 31 <= 0) bias([&](int k) { return fmaf(sign, (float)k, from); });
                else bias([&](int k) { return -slope * fabsf(away - (float)k); });
            }
            if (masked) {
#pragma unroll
                for (int k = 0; k < MY; ++k) s[k] = k < left ? s[k] : -INFINITY;
            }
            float top = attn_max<MY>([&](int k) { return s[k]; }) * c;
            if (HALVES == 2) top = fmaxf(top, exchange(top, j & 1));
            // (a row's own scores decide: others of its warp may be another text's)
            const bool raise = top > m + kRaise || (m == -INFINITY && top > m);
            if (__any_sync(0xffffffffu, raise)) {
                const float raised = raise ? top : m;
                const float factor = raise ? fast_exp2(m - raised) : 1.f;
                m = raised;
                l *= factor;
                if (j > 0) {
#pragma unroll 1
                    for (int k = half * (D / HALVES); k < (half + 1) * (D / HALVES); k += 16) {   // (few at a time: the scores are in registers, too)
                        uint32_t r[16];
                        tmem_ld16_nowait(o_cols(w) + lanes + k, r);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * factor);
                        tmem_st16_nowait(o_cols(w) + lanes + k, r);
                    }
                }
            }
            const float from = m == -INFINITY ? 0.f : m;
            // c s - m in one operation has m rounded and the product not, which is nothing up to 2^20 (2^-4 at most, the same for the
            // whole row) and can be anything at 2^30: rows beyond are taken there in two.
            float2 c2 = both(c), from2 = both(kLift<T> - from);
            if (RAW && __any_sync(0xffffffffu, fabsf(from) > 1048576.f)) {
                if (fabsf(from) > 1048576.f) {
#pragma unroll
                    for (int k = 0; k < MY; ++k) s[k] = __fadd_rn(__fmul_rn(s[k], c), -from);
                    c2 = both(1.f);
                    from2 = both(kLift<T>);
                }
            }
            float2 sums[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
            for (int k = 0; k < MY; k += 32) {
                uint32_t r[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float2 e = RAW ? fma2(make_float2(s[k + 2 * i], s[k + 2 * i + 1]), c2, from2) : add2(make_float2(s[k + 2 * i], s[k + 2 * i + 1]), from2);
                    const float2 p = make_float2(fast_exp2(e.x), fast_exp2(e.y));
                    sums[i % 2] = add2(sums[i % 2], p);
                    r[i] = pack2<T>(p.x, p.y);
                }
                tmem_st16_nowait(s_cols(w) + lanes + half * MY + k / 2, r);
            }
            l += (sums[0].x + sums[0].y) + (sums[1].x + sums[1].y);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_bar(w));
        }
        const bool real = row < x.lq;
        const uint32_t stage = base + w * C::Q_BYTES;   // the queries' place: their products are done
        if (n_kt[w] > 0 && ok) {
            ok = wait(o_bar(w), 0);
            tc_fence_after();
        }
        // (a warp that gives up does not come to the next exchange, where its partner may already be)
        if (HALVES == 2 && !ok) asm volatile("bar.arrive %0, 64;" ::"r"(1 + w * 4 + quarter) : "memory");
        if (ok && row0 < x.lq) {
            if (HALVES == 2) l += exchange(l, n_kt[w] & 1);
            const bool empty = l == 0.f;
            const float inv = 1.f / l;
            if (real && P.lse && half == 0) P.lse[(int64_t)head * a.n_q + x.q0 + row] = empty ? -INFINITY : (m - kLift<T> + __log2f(l)) * 0.69314718f;
#pragma unroll 1
            for (int k = half * (D / HALVES); k < (half + 1) * (D / HALVES); k += 32) {
                float o[32];
                if (n_kt[w] > 0) {
                    tmem_ld32_nowait(o_cols(w) + lanes + k, o);
                    tmem_wait_ld();
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = empty ? 0.f : o[i] * inv;
#pragma unroll
                for (int i = 0; i < 32; i += 8) attn_stage<T, D>(stage, quarter * 32 + lane, k + i, o + i);
            }
        }
        asm volatile("bar.sync %0, %1;" ::"r"(9 + w), "n"(128 * HALVES) : "memory");
        const int i0 = first + w * kAttnRows;
        if (ok && i0 < x.lq)
            attn_unstage<T, D, 4 * HALVES>(stage, x.lq - i0, a.dim, static_cast<T*>(P.out) + ((int64_t)(x.q0 + i0) * a.heads + head) * a.dim,
                                           (int64_t)a.heads * a.dim, (warp - 2) % (4 * HALVES));
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem, C::COLS);
}

template <typename T, int D, int NW, AttnCap CAP, bool BIAS>
cudaError_t launch(sama_ctx* ctx, const FwdParams& P, cudaStream_t st) {
    using C = FwdTile<D, NW>;
    auto* kernel = attn_fwd_kernel<T, D, NW, CAP, BIAS>;
    const uint64_t bit = 1ull << ((NW == 2 ? 32 : 0) + (std::is_same<T, __half>::value ? 16 : 0) + (D == 64 ? 8 : 0) + 2 * CAP + (BIAS ? 1 : 0));
    if (!(ctx->attn_fwd_ready & bit)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
        if (e != cudaSuccess) return e;
        ctx->attn_fwd_ready |= bit;
    }
    KernelScope scope(ctx, SAMA_K_ATTN, 0, st);
    return launch_dependent(kernel, dim3((unsigned)((int64_t)P.slots * P.a.heads)), dim3(C::THREADS), C::SMEM, st, P);
}
template <typename T, int D, int NW>
cudaError_t launch(sama_ctx* ctx, const FwdParams& P, cudaStream_t st) {
    switch (attn_cap(P.a.cap)) {
        case kNoCap: return P.a.slopes ? launch<T, D, NW, kNoCap, true>(ctx, P, st) : launch<T, D, NW, kNoCap, false>(ctx, P, st);
        case kCap: return P.a.slopes ? launch<T, D, NW, kCap, true>(ctx, P, st) : launch<T, D, NW, kCap, false>(ctx, P, st);
        default: return P.a.slopes ? launch<T, D, NW, kWideCap, true>(ctx, P, st) : launch<T, D, NW, kWideCap, false>(ctx, P, st);
    }
}
template <typename T>
cudaError_t launch(sama_ctx* ctx, int nw, const FwdParams& P, cudaStream_t st) {
    if (P.a.dim <= 64) return launch<T, 64, 1>(ctx, P, st);
    return nw == 1 ? launch<T, 128, 1>(ctx, P, st) : launch<T, 128, 2>(ctx, P, st);
}

}  // namespace

cudaError_t launch_attention(sama_ctx* ctx, const AttnShape& a, const AttnOperands& op, void* out, float* lse, cudaStream_t st) {
    FwdParams P;
    const int bk = a.dim <= 64 ? FwdTile<64, 1>::BK : FwdTile<128, 2>::BK;
    // Two tiles per CTA, which read the keys once, for long texts; for shorter ones a CTA's start and end and the tiles that
    // a text does not fill weigh more (us with two and with one, 32 heads of 128 over 8: one text of 512 17.7 and 15.6, of 2048 78.7
    // and 78.7, of 4096, causal, 140 and 138, of 8192, causal, 466 and 476, capped 646 and 655; 8 of up to 1024 95 and 89, 32 of up
    // to 300 103 and 87; 2 of up to 4096, all heads with their own keys, 304 and 322).  Lengths are on the device, but their mean is known.
    const int nw = a.dim <= 64 || a.n_q < 2048 * (int64_t)a.n_texts ? 1 : 2;
    // (without keys nothing is loaded, but a map has to describe something)
    const bool none = a.n_k == 0;
    if (!attn_map(&P.q, op.q, op.dtype, a.dim, a.heads, a.n_q, op.q_stride, kAttnRows) ||
        !attn_map(&P.k, none ? op.q : op.k, op.dtype, a.dim, none ? a.heads : a.kv_heads, none ? a.n_q : a.n_k, none ? op.q_stride : op.k_stride, bk) ||
        !attn_map(&P.v, none ? op.q : op.v, op.dtype, a.dim, none ? a.heads : a.kv_heads, none ? a.n_q : a.n_k, none ? op.q_stride : op.v_stride, bk))
        return cudaErrorInvalidValue;
    P.a = a;
    P.out = out;
    P.lse = lse;
    P.slots = a.n_q / (nw * kAttnRows) + a.n_texts;
    return op.dtype == SAMA_BF16 ? launch<__nv_bfloat16>(ctx, nw, P, st) : launch<__half>(ctx, nw, P, st);
}

}  // namespace sama
