// Distillation from a teacher's top logits: loss and gradient of each row in one pass.
//
//   p = softmax(u / T) over the kept entries,  q = softmax(z / T) over the vocabulary,
//   loss = T^2 sum p (log p - log q),  grad = coef (q - p),  coef = grad_scale weight T
//
// The logits are read once and the gradient is written once, which is the floor: a row stays in shared memory between its
// sum and its gradient.  A row of up to 104 KB is a CTA's; longer ones are shared by a cluster of up to 8 CTAs with 64 KB each,
// which exchange maximum and sum through distributed shared memory.  A bulk copy brings the part in; the threads take
// maximum and sum of it, meet, and write q from registers straight to memory, while a warp of its own works out the teacher's
// distribution, the loss and the gradient's values at the teacher's entries, which go over q at the end.  A CTA does one
// thing after the other, and two or more of them per SM keep memory busy meanwhile.  4096 rows of 50,021 bf16 logits: 156
// to 162 us, 5.1 to 5.3 TB/s (0.77 to 0.80 of the copy rate); of 131,072 484 us, 4.4 TB/s (0.68), where a cluster meets twice per row and two
// exponentials per logit take 60 % of the special-function units.  (A persistent CTA whose groups of warps work on different
// rows of a ring was slower, 174 and 470 us at its best: it had a single copy in flight per SM most of the time.)
// Rows of up to 4 KB are a warp's each; rows that no cluster can hold, or with more than 512 entries, are read twice.
#include <type_traits>

#include "num_types.h"
#include "sama_internal.h"
#include "tc_ptx.h"

namespace sama {

namespace {

constexpr int VECS = 8, BATCH = 4;    // 16-byte vectors that a thread has in hand
constexpr int kMaxEntries = 1024;
// one row per cluster or CTA
constexpr int PART = 64 * 1024, ALONE = 104 * 1024;        // bytes of a row in a CTA of a cluster, and in one by itself
constexpr int ENTRIES = 512, BITS = 8192;                  // of the teacher's, at most; of the table that finds an id twice
constexpr int entry_bytes(int k) { return (k + 31) / 32 * 32 * 12 + BITS / 8; }
// one row per warp
constexpr int FEW_TEAMS = 8, FEW_STAGES = 3, FEW_ENTRIES = 4, FEW_CHUNK = 32 * VECS * 16, FEW_MOST = 32 * FEW_ENTRIES;
constexpr int FEW_SMEM = FEW_TEAMS * (FEW_STAGES * FEW_CHUNK + FEW_MOST * 8);

struct DistillParams {
    const void* logits;
    void* grad;                // or null: losses alone
    int64_t n_rows, ld, ld_grad;
    const void* top;
    const int32_t* ids;
    const float* weight;
    float* loss;
    int32_t* status;
    int vocab, k, top_dtype;
    int part_bytes;               // shared memory for a CTA's part of a row
    int in_place;                 // the gradient replaces the logits
    float c, temperature, coef;   // log2 e / T, T, grad_scale T
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void bulk_store(void* dst, uint32_t src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ float load_top(const DistillParams& P, int64_t i) {
    if (P.top_dtype == SAMA_F32) return static_cast<const float*>(P.top)[i];
    if (P.top_dtype == SAMA_BF16) return to_float(static_cast<const __nv_bfloat16*>(P.top)[i]);
    return to_float(static_cast<const __half*>(P.top)[i]);
}
template <typename T> __device__ __forceinline__ void unpack_vec(uint4 x, float* v) {
    const uint32_t r[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) {
            v[j] = __uint_as_float(r[j]);
        } else {
            const float2 f = unpack2<T>(r[j]);
            v[2 * j] = f.x;
            v[2 * j + 1] = f.y;
        }
    }
}

// Sums and maxima over a team, the same bits in every thread.
template <int TEAM>
struct Reduce {
    float2* slots;   // [2][warps]: used in turn, so that one barrier per reduction is enough
    int turn = 0;
    __device__ __forceinline__ void sync() { if (TEAM == 32) __syncwarp(); else __syncthreads(); }
    template <typename F>
    __device__ __forceinline__ float2 operator()(float a, float b, F&& f) {
#pragma unroll
        for (int o = 16; o > 0; o /= 2) {
            a = f(a, __shfl_xor_sync(0xffffffffu, a, o));
            b = f(b, __shfl_xor_sync(0xffffffffu, b, o));
        }
        if (TEAM == 32) return make_float2(a, b);
        constexpr int W = TEAM / 32;
        float2* s = slots + turn * W;
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) s[threadIdx.x / 32] = make_float2(a, b);
        sync();
        float2 r = s[0];
#pragma unroll
        for (int w = 1; w < W; ++w) { r.x = f(r.x, s[w].x); r.y = f(r.y, s[w].y); }
        return r;
    }
};
__device__ __forceinline__ float max_of(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float sum_of(float a, float b) { return a + b; }

// A row's vectors [v0, v1) that a CTA has, those of them that lie wholly within it, and bytes before the row in the first.
struct Span { int head, v0, v1, in0, in1; };
__device__ __forceinline__ Span span_of(const uint8_t* row, int row_bytes, int rank, int ctas) {
    Span s;
    s.head = (int)(reinterpret_cast<uintptr_t>(row) & 15u);
    const int n = (s.head + row_bytes + 15) / 16, per = ctas == 1 ? n : (n + ctas - 1) / ctas;
    s.v0 = min(rank * per, n);
    s.v1 = min(s.v0 + per, n);
    s.in0 = max(s.v0, s.head ? 1 : 0);
    s.in1 = max(s.in0, min(s.v1, (s.head + row_bytes) / 16));
    return s;
}
// The vectors at a row's two ends that are not whole: thread t < VE has a place in the first, VE <= t < 2 VE in the last.
// `place` in the CTA's vectors (-1: none), `element` in the row (outside it: nothing is there).
template <int VE>
__device__ __forceinline__ void edge_of(const Span& s, int row_bytes, int size, int t, int* place, int* element) {
    const int last = (s.head + row_bytes) / 16, v = t < VE ? 0 : last;
    const bool partial = t < VE ? s.head != 0 : (s.head + row_bytes) % 16 != 0 && !(last == 0 && s.head != 0);
    *element = v * VE + t % VE - s.head / size;
    *place = t < 2 * VE && partial && v >= s.v0 && v < s.v1 ? (v - s.v0) * VE + t % VE : -1;
}

// The largest of a vector's values (NaN aside).
template <typename T> __device__ __forceinline__ float vec_max(uint4 x) {
    if constexpr (sizeof(T) == 4) {
        return fmaxf(fmaxf(__uint_as_float(x.x), __uint_as_float(x.y)), fmaxf(__uint_as_float(x.z), __uint_as_float(x.w)));
    } else if constexpr (std::is_same<T, __half>::value) {
        const __half2* h = reinterpret_cast<const __half2*>(&x);
        const float2 f = __half22float2(__hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3])));
        return fmaxf(f.x, f.y);
    } else {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&x);
        const float2 f = __bfloat1622float2(__hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3])));
        return fmaxf(f.x, f.y);
    }
}
template <typename T> __device__ __forceinline__ uint4 vec_lowest() {
    const uint32_t w = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, __half>::value ? 0xfc00fc00u : 0xff80ff80u;
    return make_uint4(w, w, w, w);
}
// 2^(c (z - m)).  One operation less takes c z - (c m), whose second product is rounded: by up to 2^-14 up to the c m that
// `beyond` names, the same for all z, and taken back by `unrounded`; by anything for a row of nothing but masked values (-1e9, or
// the type's lowest).
__device__ __forceinline__ float power_of(float z, float m, float c) { return fast_exp2((z - m) * c); }
__device__ __forceinline__ float unrounded(float m, float c, float cm) { return fast_exp2(-fmaf(m, c, -cm)); }
__device__ __forceinline__ bool beyond(float cm) { return fabsf(cm) > 1024.f; }
// (m, l) of two parts, each a maximum and the sum of 2^(c (z - maximum)): l as seen from `top`.
__device__ __forceinline__ float rebase(float l, float m, float top, float c) { return m == -INFINITY ? l : l * fast_exp2((m - top) * c); }

// MAIN threads for the row and a warp for its entries.
template <typename T, int MAIN>
__global__ void __launch_bounds__(MAIN + 32, MAIN == 256 ? 4 : MAIN == 128 ? 7 : 11)
distill_kernel(const DistillParams P) {
    constexpr int VE = 16 / (int)sizeof(T), SIZE = (int)sizeof(T), WARPS = MAIN / 32;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t full;
    __shared__ float2 peers[8], warp_sums[WARPS];     // (maximum, sum) of the cluster's CTAs, of this one's warps
    __shared__ int no_entry;
    const int kp = (P.k + 31) / 32 * 32;
    uint32_t* bits = reinterpret_cast<uint32_t*>(smem + P.part_bytes);
    int32_t* place = reinterpret_cast<int32_t*>(bits + BITS / 32);   // of the teacher's entries: id (in the end, of those in this part),
    float *value = reinterpret_cast<float*>(place + kp), *logit = value + kp;   // weight and then gradient, logit

    unsigned ctas_u;
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas_u));
    const int ctas = (int)ctas_u, rank = ctas > 1 ? (int)cluster_ctarank() : 0;
    const int64_t row = blockIdx.x / ctas_u;
    const int t = threadIdx.x, warp = t / 32, lane = t % 32;
    const int row_bytes = P.vocab * SIZE;
    const uint8_t* z_row = static_cast<const uint8_t*>(P.logits) + row * P.ld * SIZE;
    const Span sp = span_of(z_row, row_bytes, rank, ctas);
    const int n = sp.v1 - sp.v0;
    const uint32_t bar = smem_u32(&full);
    if (t == 0) {
        mbar_init(bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_trigger();
    pdl_wait();
    if (warp == 0) {
        int at, element;
        edge_of<VE>(sp, row_bytes, SIZE, lane, &at, &element);
        if (at >= 0) reinterpret_cast<T*>(smem)[at] = element >= 0 && element < P.vocab ? reinterpret_cast<const T*>(z_row)[element] : from_float<T>(-INFINITY);
        __syncwarp();
        if (lane == 0) {
            const uint32_t bytes = (uint32_t)(sp.in1 - sp.in0) * 16u;
            mbar_expect_tx(bar, bytes);
            if (bytes) bulk_load(smem_u32(smem + (sp.in0 - sp.v0) * 16), z_row - sp.head + (int64_t)sp.in0 * 16, bytes, bar);
        }
    }
    __syncthreads();
    // (the other CTAs run before their shared memory is written: waited for only then)
    if (ctas > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");

    const float weight = P.weight ? P.weight[row] : 1.f, coef = P.coef * weight;
    float sum_u = 0.f, entropy = 0.f;
    auto over = [](float x, auto f) {
#pragma unroll
        for (int o = 16; o > 0; o /= 2) x = f(x, __shfl_xor_sync(0xffffffffu, x, o));
        return x;
    };
    if (warp == WARPS) {
        const T* z = reinterpret_cast<const T*>(z_row);
        if (ctas > 1) {
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
            if (!P.in_place) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        }
        float top = -INFINITY;
        for (int w = lane; w < BITS / 32; w += 32) bits[w] = 0;
#pragma unroll 4
        for (int j = lane; j < P.k; j += 32) {
            int32_t id = P.ids[row * P.k + j];
            float u = load_top(P, row * P.k + j);
            if (id < 0 || id >= P.vocab) {
                if (id != -1) atomicOr(P.status, (int)SAMA_DEV_BAD_INDEX);
                id = -1;
                u = -INFINITY;
            }
            place[j] = id;
            value[j] = u;
            top = fmaxf(top, u);
        }
#pragma unroll 4
        for (int j = lane; j < P.k; j += 32)
            if (place[j] >= 0) logit[j] = to_float(z[place[j]]);
        // (in place, no CTA writes before the loss has the logits that it needs)
        if (ctas > 1 && P.in_place) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        top = over(top, max_of);
        const float from_u = top == -INFINITY ? 0.f : top;
        for (int j = lane; j < P.k; j += 32) {
            const float lp = (value[j] - from_u) * P.c, p = exp2f(lp);   // log2 of p, up to the sum
            sum_u += p;
            if (p > 0.f) entropy += p * lp;
            value[j] = p;
        }
        sum_u = over(sum_u, sum_of);
        entropy = over(entropy, sum_of);
        if (lane == 0) no_entry = sum_u == 0.f;
        // Several entries with one id: the first takes them all.  An id that finds its bit set may be one of those.
        __syncwarp();
        for (int j0 = 0; j0 < P.k; j0 += 32) {
            const int j = j0 + lane;
            const int32_t id = j < P.k ? place[j] : -1;
            const uint32_t h = ((uint32_t)id * 2654435761u) >> 19, bit = 1u << (h & 31u);
            uint32_t again = __ballot_sync(0xffffffffu, id >= 0 && (atomicOr(bits + h / 32, bit) & bit) != 0);
            for (; again; again &= again - 1) {
                const int32_t it = __shfl_sync(0xffffffffu, id, __ffs(again) - 1);
                float all = 0.f;
                int leader = ENTRIES;
                for (int x = lane; x < P.k; x += 32)
                    if (place[x] == it) {
                        all += value[x];
                        leader = min(leader, x);
                    }
                all = over(all, sum_of);
                leader = __reduce_min_sync(0xffffffffu, leader);
                __syncwarp();
                for (int x = lane; x < P.k; x += 32)
                    if (place[x] == it) value[x] = x == leader ? all : 0.f;
                __syncwarp();
            }
        }
    } else {
        // (one warp asks for the copy, the others wait at a barrier: asking again and again takes issue slots)
        if (warp == 0 && !mbar_wait(bar, 0)) {
            atomicOr(P.status, (int)SAMA_DEV_TIMEOUT);
            mbar_wait(bar, 0);   // (the copy should land before the CTA's memory goes away)
        }
        asm volatile("bar.sync 1, %0;" ::"n"(MAIN) : "memory");
        const uint4* chunk = reinterpret_cast<const uint4*>(smem);
        float m = -INFINITY, l = 0.f, from = 0.f;   // from: c m as it was rounded
        auto take = [&](auto count, int b) {   // vectors b, b + MAIN, ...
            constexpr int N = decltype(count)::value;
            uint4 x[N];
            float top = -INFINITY;
#pragma unroll
            for (int v = 0; v < N; ++v) x[v] = chunk[b + v * MAIN];
#pragma unroll
            for (int v = 0; v < N; ++v) top = fmaxf(top, vec_max<T>(x[v]));
            if (top > m) {
                const float raised = top * P.c;
                l = m == -INFINITY ? l : l * fast_exp2(from - raised);
                m = top;
                from = raised;
            }
#pragma unroll
            for (int v = 0; v < N; ++v) {
                float f[VE], sum = 0.f;
                unpack_vec<T>(x[v], f);
#pragma unroll
                for (int e = 0; e < VE; ++e) sum += fast_exp2(fmaf(f[e], P.c, -from));
                l += sum;
            }
        };
        int b = t;
        for (; b + (BATCH - 1) * MAIN < n; b += MAIN * BATCH) take(std::integral_constant<int, BATCH>(), b);
        for (; b < n; b += MAIN) take(std::integral_constant<int, 1>(), b);
        if (m != -INFINITY && !beyond(from)) {
            l *= unrounded(m, P.c, from);
        } else if (m != -INFINITY) {   // once more (in the loop it would cost ordinary rows a tenth of their time)
            l = 0.f;
#pragma unroll 1
            for (b = t; b < n; b += MAIN) {
                float f[VE];
                unpack_vec<T>(chunk[b], f);
#pragma unroll
                for (int e = 0; e < VE; ++e) l += power_of(f[e], m, P.c);
            }
        }
        const float top = over(m, max_of);
        l = over(rebase(l, m, top, P.c), sum_of);
        if (lane == 0) warp_sums[warp] = make_float2(top, l);
        asm volatile("bar.sync 1, %0;" ::"n"(MAIN) : "memory");
    }
    // The row's maximum and sum, the same bits in every thread.  The warp of the entries meets the others here without
    // their waiting for it: its loads depend on one another.
    float most = -INFINITY, total = 0.f;
    if (ctas == 1) {
        // (in place they do: nothing is written before the loss has the logits that it needs)
        if (warp == WARPS || P.in_place) asm volatile("bar.sync 2, %0;" ::"n"(MAIN + 32) : "memory");
        else asm volatile("bar.arrive 2, %0;" ::"n"(MAIN + 32) : "memory");
    }
    if (ctas == 1 || warp < WARPS) {
#pragma unroll
        for (int w = 0; w < WARPS; ++w) most = fmaxf(most, warp_sums[w].x);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) total += rebase(warp_sums[w].y, warp_sums[w].x, most, P.c);
    }
    if (ctas > 1) {
        if (warp < WARPS) {
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
            if (t < ctas)
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(map_to_rank(smem_u32(&peers[rank]), (uint32_t)t)), "f"(most), "f"(total) : "memory");
            __syncwarp();
            asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        }
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        most = -INFINITY;
        total = 0.f;
        for (int c = 0; c < ctas; ++c) most = fmaxf(most, peers[c].x);
        for (int c = 0; c < ctas; ++c) total += rebase(peers[c].y, peers[c].x, most, P.c);
    }
    const float base = most == -INFINITY ? 0.f : most, whole = base * P.c, inv = 1.f / total;
    T* g_row = static_cast<T*>(P.grad) + row * P.ld_grad;
    if (warp == WARPS) {
        const bool none = sum_u == 0.f;
        const float inv_u = none ? 0.f : 1.f / sum_u;
        const int skip = sp.head / SIZE - sp.v0 * VE;
        float cross = 0.f;
        for (int j = lane; j < P.k; j += 32) {
            const int32_t id = place[j];
            const float p = value[j] * inv_u, ze = logit[j];
            if (id >= 0 && !(p == 0.f)) cross += p * ((ze - base) * P.c);
            const bool mine = id >= 0 && id + skip >= 0 && id + skip < n * VE && p != 0.f;   // (without weight the gradient is q's own)
            value[j] = coef * (power_of(ze, base, P.c) * inv - p);
            place[j] = mine ? id : -1;
        }
        if (P.loss && rank == 0) {
            // sum p (log2 p - log2 q), of which sum p = 1
            cross = over(cross, sum_of) - log2f(total);
            if (lane == 0) P.loss[row] = none ? 0.f : P.temperature * P.temperature * 0.69314718f * (entropy * inv_u - log2f(sum_u) - cross);
        }
    }
    if (!P.grad) return;
    // Vectors [in0, in1) are stored whole, the others (a row's two ends, or all where rows of the gradient start elsewhere
    // than those of the logits) by elements.
    const bool alike = (int)(reinterpret_cast<uintptr_t>(g_row) & 15u) == sp.head;
    const int element0 = sp.v0 * VE - sp.head / SIZE, in0 = alike ? sp.in0 - sp.v0 : n, in1 = alike ? sp.in1 - sp.v0 : n;
    T* g_part = g_row + element0;
    auto put_elements = [&](int b, const float* g) {
#pragma unroll
        for (int e = 0; e < VE; ++e)
            if ((uint32_t)(element0 + b * VE + e) < (uint32_t)P.vocab) g_part[b * VE + e] = from_float<T>(g[e]);
    };
    if (warp < WARPS && weight != 0.f) {
        const float f = coef * inv, near = f * unrounded(base, P.c, whole);
        const uint4* chunk = reinterpret_cast<const uint4*>(smem);
        auto gradient = [&](uint4 x, float* g) {
            unpack_vec<T>(x, g);
#pragma unroll
            for (int e = 0; e < VE; ++e) g[e] = fast_exp2(fmaf(g[e], P.c, -whole)) * near;
        };
        auto make = [&](auto count, int b) {
            constexpr int N = decltype(count)::value;
            uint4 x[N];
#pragma unroll
            for (int v = 0; v < N; ++v) x[v] = chunk[b + v * MAIN];
#pragma unroll
            for (int v = 0; v < N; ++v) {
                float g[VE];
                gradient(x[v], g);
                store_n<T, VE, true>(g_part + (b + v * MAIN) * VE, g);
            }
        };
        if (!beyond(whole)) {
            int b = in0 + t;
            for (; b + (BATCH - 1) * MAIN < in1; b += MAIN * BATCH) make(std::integral_constant<int, BATCH>(), b);
            for (; b < in1; b += MAIN) make(std::integral_constant<int, 1>(), b);
            for (int e = t; e < in0 + n - in1; e += MAIN) {
                float g[VE];
                const int at = e < in0 ? e : in1 + e - in0;
                gradient(chunk[at], g);
                put_elements(at, g);
            }
        } else {
#pragma unroll 1
            for (int b = t; b < n; b += MAIN) {
                float g[VE];
                unpack_vec<T>(chunk[b], g);
#pragma unroll
                for (int e = 0; e < VE; ++e) g[e] = power_of(g[e], base, P.c) * f;
                put_elements(b, g);
            }
        }
    }
    __syncthreads();
    if (weight == 0.f || no_entry) {   // zeros, whatever the logits
        const float g[VE] = {};
        for (int b = t; b < n; b += MAIN + 32) {
            if (b >= in0 && b < in1) store_n<T, VE>(g_part + b * VE, g);
            else put_elements(b, g);
        }
        return;
    }
    for (int j = t; j < P.k; j += MAIN + 32) {
        const int id = place[j];
        if (id >= 0) g_row[id] = from_float<T>(value[j]);
    }
}

// A row per warp: rows of up to 4 KB and teachers of up to 128 entries.  Each thread holds 8 vectors as exponentials.
template <typename T>
__global__ void __launch_bounds__(32 * FEW_TEAMS, 2)
distill_few_kernel(const DistillParams P) {
    constexpr int VE = 16 / (int)sizeof(T), SIZE = (int)sizeof(T);
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t bars[FEW_TEAMS][FEW_STAGES];
    const int team = threadIdx.x / 32, t = threadIdx.x % 32;
    uint8_t* ring = smem + team * FEW_STAGES * FEW_CHUNK;
    int32_t* e_id = reinterpret_cast<int32_t*>(smem + FEW_TEAMS * FEW_STAGES * FEW_CHUNK) + team * FEW_MOST;
    float* e_p = reinterpret_cast<float*>(smem + FEW_TEAMS * (FEW_STAGES * FEW_CHUNK + FEW_MOST * 4)) + team * FEW_MOST;
    auto bar = [&](int s) { return smem_u32(&bars[team][s]); };
    const int64_t first = (int64_t)blockIdx.x * FEW_TEAMS + team, stride = (int64_t)gridDim.x * FEW_TEAMS;
    if (t == 0) {
        for (int s = 0; s < FEW_STAGES; ++s) mbar_init(bar(s), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    pdl_trigger();
    pdl_wait();
    auto over = [](float x, auto f) {
#pragma unroll
        for (int o = 16; o > 0; o /= 2) x = f(x, __shfl_xor_sync(0xffffffffu, x, o));
        return x;
    };

    const int row_bytes = P.vocab * SIZE;
    const uint8_t* z_bytes = static_cast<const uint8_t*>(P.logits);
    auto z_row = [&](int64_t row) { return z_bytes + row * P.ld * SIZE; };
    // What a thread has at hand of a row before its turn comes: an element at the row's end, and entries of the teacher.
    T edge = from_float<T>(0.f);
    int32_t id[FEW_ENTRIES];
    float u[FEW_ENTRIES], z[FEW_ENTRIES], weight = 1.f;
    auto fetch_row = [&](int64_t row, int stage) {
        const Span s = span_of(z_row(row), row_bytes, 0, 1);
        if (t == 0) {
            const uint32_t bytes = (uint32_t)(s.in1 - s.in0) * 16u;
            mbar_expect_tx(bar(stage), bytes);
            if (bytes) bulk_load(smem_u32(ring + stage * FEW_CHUNK + s.in0 * 16), z_row(row) - s.head + s.in0 * 16, bytes, bar(stage));
        }
    };
    auto fetch_entries = [&](int64_t row) {
        int place, element;
        edge_of<VE>(span_of(z_row(row), row_bytes, 0, 1), row_bytes, SIZE, t, &place, &element);
        edge = place >= 0 && element >= 0 && element < P.vocab ? reinterpret_cast<const T*>(z_row(row))[element] : from_float<T>(-INFINITY);
#pragma unroll
        for (int i = 0; i < FEW_ENTRIES; ++i) {
            const int j = t + i * 32;
            id[i] = j < P.k ? P.ids[row * P.k + j] : -1;
            u[i] = j < P.k ? load_top(P, row * P.k + j) : -INFINITY;
        }
        if (P.weight) weight = P.weight[row];
    };
    auto fetch_targets = [&](int64_t row) {
#pragma unroll
        for (int i = 0; i < FEW_ENTRIES; ++i) {
            if (id[i] < -1 || id[i] >= P.vocab) {
                atomicOr(P.status, (int)SAMA_DEV_BAD_INDEX);
                id[i] = -1;
            }
            if (id[i] < 0) u[i] = -INFINITY;
            z[i] = id[i] >= 0 ? to_float(reinterpret_cast<const T*>(z_row(row))[id[i]]) : 0.f;
        }
    };

    for (int i = 0; i < FEW_STAGES - 1; ++i)
        if (first + i * stride < P.n_rows) fetch_row(first + i * stride, i);
    if (first < P.n_rows) {
        fetch_entries(first);
        fetch_targets(first);
    }
    int stage = 0, parity = 0;
    bool timed_out = false;
    for (int64_t row = first; row < P.n_rows; row += stride) {
        const Span s = span_of(z_row(row), row_bytes, 0, 1);
        const int n = s.v1;
        uint8_t* chunk = ring + stage * FEW_CHUNK;
        if (!mbar_wait(bar(stage), (uint32_t)parity)) {
            timed_out = true;
            mbar_wait(bar(stage), (uint32_t)parity);   // (the copy should land before the CTA's memory goes away)
        }
        int place, element;
        edge_of<VE>(s, row_bytes, SIZE, t, &place, &element);
        if (place >= 0) reinterpret_cast<T*>(chunk)[place] = edge;
        float my_u[FEW_ENTRIES], my_z[FEW_ENTRIES], top_u = -INFINITY;
        int32_t my_id[FEW_ENTRIES];
#pragma unroll
        for (int i = 0; i < FEW_ENTRIES; ++i) {
            my_id[i] = id[i];
            my_u[i] = u[i];
            my_z[i] = z[i];
            top_u = fmaxf(top_u, u[i]);
        }
        const float my_weight = weight;
        const bool more = row + stride < P.n_rows;
        if (more) fetch_entries(row + stride);
        __syncwarp();

        float v[VECS * VE], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            const uint4 x = t + i * 32 < n ? reinterpret_cast<const uint4*>(chunk)[t + i * 32] : vec_lowest<T>();
            top = fmaxf(top, vec_max<T>(x));
            unpack_vec<T>(x, v + i * VE);
        }
        top = over(top, max_of);
        top_u = over(top_u, max_of);
        const float from = top == -INFINITY ? 0.f : top, from_u = top_u == -INFINITY ? 0.f : top_u;
        float sum = 0.f, sum_u = 0.f;
#pragma unroll
        for (int i = 0; i < VECS * VE; ++i) {
            v[i] = power_of(v[i], from, P.c);
            sum += v[i];
        }
#pragma unroll
        for (int i = 0; i < FEW_ENTRIES; ++i) {
            my_u[i] = (my_u[i] - from_u) * P.c;          // log2 of p, up to the sum
            sum_u += exp2f(my_u[i]);
        }
        sum = over(sum, sum_of);
        sum_u = over(sum_u, sum_of);
        const bool none = sum_u == 0.f;                  // no entry
        const float inv = 1.f / sum, inv_u = none ? 0.f : 1.f / sum_u, log_total = log2f(sum), log_u = log2f(sum_u);
        if (P.loss) {
            float part = 0.f;
#pragma unroll
            for (int i = 0; i < FEW_ENTRIES; ++i) {
                const float p = exp2f(my_u[i]) * inv_u;
                if (my_id[i] >= 0 && !(p == 0.f)) part += p * ((my_u[i] - log_u) - ((my_z[i] - from) * P.c - log_total));
            }
            part = over(part, sum_of);
            if (t == 0) P.loss[row] = none ? 0.f : P.temperature * P.temperature * 0.69314718f * part;
        }
        if (P.grad) {
            const float coef = P.coef * my_weight, f = coef * inv;
            const bool zero = none || my_weight == 0.f;
#pragma unroll
            for (int i = 0; i < VECS; ++i)
                if (t + i * 32 < n) {
                    float g[VE];
#pragma unroll
                    for (int e = 0; e < VE; ++e) g[e] = zero ? 0.f : v[i * VE + e] * f;
                    store_n<T, VE>(reinterpret_cast<T*>(chunk) + (t + i * 32) * VE, g);
                }
#pragma unroll
            for (int i = 0; i < FEW_ENTRIES; ++i) {
                e_id[t + i * 32] = my_id[i];
                e_p[t + i * 32] = exp2f(my_u[i]) * inv_u;
            }
            __syncwarp();
            // the teacher's entries; of several with one id the first takes them all
#pragma unroll
            for (int i = 0; i < FEW_ENTRIES; ++i) {
                const int j = t + i * 32;
                if (zero || my_id[i] < 0) continue;
                float p = 0.f;
                bool is_first = true;
                for (int x = 0; x < P.k; x += 4) {
                    const int4 four = *reinterpret_cast<const int4*>(e_id + x);
                    const int32_t ids[4] = {four.x, four.y, four.z, four.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (ids[e] == my_id[i]) {
                            p += e_p[x + e];
                            is_first = is_first && x + e >= j;
                        }
                }
                if (is_first) reinterpret_cast<T*>(chunk)[my_id[i] + s.head / SIZE] = from_float<T>(coef * (power_of(my_z[i], from, P.c) * inv - p));
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            uint8_t* g_row = static_cast<uint8_t*>(P.grad) + row * P.ld_grad * SIZE;
            if ((int)(reinterpret_cast<uintptr_t>(g_row) & 15u) == s.head) {
                const uint32_t bytes = (uint32_t)(s.in1 - s.in0) * 16u;
                if (t == 0 && bytes) bulk_store(g_row - s.head + s.in0 * 16, smem_u32(chunk + s.in0 * 16), bytes);
                if (place >= 0 && element >= 0 && element < P.vocab) reinterpret_cast<T*>(g_row)[element] = reinterpret_cast<const T*>(chunk)[place];
            } else {
                // rows of the gradient start elsewhere than those of the logits
                for (int e = t; e < P.vocab; e += 32) reinterpret_cast<T*>(g_row)[e] = reinterpret_cast<const T*>(chunk)[e + s.head / SIZE];
                __syncwarp();
            }
        } else {
            // (the next copy into this place comes after the stores of the row's ends)
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
        }
        if (t == 0) asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group.read 1;" ::: "memory");
        // the row after the next takes the place of the one before this, whose gradient has left it
        const int64_t after = row + (FEW_STAGES - 1) * stride;
        if (after < P.n_rows) fetch_row(after, (stage + FEW_STAGES - 1) % FEW_STAGES);
        if (more) fetch_targets(row + stride);
        if (++stage == FEW_STAGES) { stage = 0; parity ^= 1; }
    }
    if (t == 0) {
        if (timed_out) atomicOr(P.status, (int)SAMA_DEV_TIMEOUT);
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
}

// Rows that no cluster can hold: one CTA per row, read once for the sum and once for the gradient.
template <typename T>
__global__ void __launch_bounds__(1024)
distill_long_kernel(const DistillParams P) {
    constexpr int TEAM = 1024;
    __shared__ float2 slots[2][TEAM / 32];
    __shared__ __align__(16) int32_t e_id[kMaxEntries];
    __shared__ float e_p[kMaxEntries];
    Reduce<TEAM> reduce{&slots[0][0]};
    pdl_trigger();
    pdl_wait();
    const int t = threadIdx.x;
    for (int64_t row = blockIdx.x; row < P.n_rows; row += gridDim.x) {
        const T* z = static_cast<const T*>(P.logits) + row * P.ld;
        int32_t id = t < P.k ? P.ids[row * P.k + t] : -1;
        if (id < -1 || id >= P.vocab) {
            atomicOr(P.status, (int)SAMA_DEV_BAD_INDEX);
            id = -1;
        }
        float u = id >= 0 ? load_top(P, row * P.k + t) : -INFINITY;
        const float target = id >= 0 ? to_float(z[id]) : 0.f;
        float m = -INFINITY, l = 0.f;
        for (int e0 = t; e0 < P.vocab; e0 += 8 * TEAM) {
            float v[8], top = m;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int e = e0 + i * TEAM;
                v[i] = e < P.vocab ? to_float(z[e]) : -INFINITY;
                top = fmaxf(top, v[i]);
            }
            const float from = top == -INFINITY ? 0.f : top;
            l *= m == -INFINITY ? 0.f : fast_exp2((m - top) * P.c);
            m = top;
#pragma unroll
            for (int i = 0; i < 8; ++i) l += power_of(v[i], from, P.c);
        }
        const float2 tops = reduce(m, u, max_of);
        const float from = tops.x == -INFINITY ? 0.f : tops.x, from_u = tops.y == -INFINITY ? 0.f : tops.y;
        u = (u - from_u) * P.c;
        // (a part of nothing but -infinity has a sum of 0, one with a NaN a sum of NaN)
        const float2 sums = reduce(m == -INFINITY ? l : l * fast_exp2((m - tops.x) * P.c), exp2f(u), sum_of);
        const float inv = 1.f / sums.x, inv_u = sums.y > 0.f ? 1.f / sums.y : 0.f;
        const bool none = !(sums.y > 0.f) && sums.y == sums.y;
        const float p = exp2f(u) * inv_u;
        if (P.loss) {
            const float log_q = (target - from) / P.temperature - logf(sums.x);
            const float part = reduce(id >= 0 && !(p == 0.f) ? p * ((u - log2f(sums.y)) * 0.69314718f - log_q) : 0.f, 0.f, sum_of).x;
            if (t == 0) P.loss[row] = none ? 0.f : P.temperature * P.temperature * part;
        }
        if (!P.grad) continue;
        const float weight = P.weight ? P.weight[row] : 1.f, coef = none ? 0.f : P.coef * weight;
        const bool zero = none || weight == 0.f;
        T* g = static_cast<T*>(P.grad) + row * P.ld_grad;
        for (int e = t; e < P.vocab; e += TEAM)
            g[e] = from_float<T>(zero ? 0.f : coef * (power_of(to_float(z[e]), from, P.c) * inv));
        e_id[t] = id;
        e_p[t] = p;
        __syncthreads();
        if (!zero && id >= 0) {
            float all = 0.f;
            bool is_first = true;
            for (int x = 0; x < P.k; ++x)
                if (e_id[x] == id) {
                    all += e_p[x];
                    is_first = is_first && x >= t;
                }
            if (is_first) g[id] = from_float<T>(coef * (power_of(target, from, P.c) * inv - all));
        }
        __syncthreads();   // the entries may be written again
    }
}

// Once per context: shared memory beyond the default.
template <typename T>
cudaError_t allow_memory() {
    constexpr auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
    cudaError_t e = cudaFuncSetAttribute(distill_few_kernel<T>, attr, FEW_SMEM);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(distill_kernel<T, 256>, attr, ALONE + entry_bytes(ENTRIES));
    return e;
}

template <typename T>
cudaError_t launch(sama_ctx* ctx, DistillParams& P, cudaStream_t st) {
    constexpr int SIZE = (int)sizeof(T);
    // vectors of a row: one more where rows do not all start on 16 bytes
    const bool whole = reinterpret_cast<uintptr_t>(P.logits) % 16 == 0 && (P.n_rows == 1 || P.ld * SIZE % 16 == 0);
    const int64_t vecs = ((int64_t)P.vocab * SIZE + (whole ? 0 : 16 - SIZE) + 15) / 16;
    KernelScope scope(ctx, SAMA_K_DISTILL, -1, st);
    if (vecs * 16 <= FEW_CHUNK && P.k <= FEW_MOST) {
        const int64_t wanted = (P.n_rows + FEW_TEAMS - 1) / FEW_TEAMS, most = 2 * ctx->sm_count;
        return launch_dependent(distill_few_kernel<T>, dim3((unsigned)(wanted < most ? wanted : most)), dim3(32 * FEW_TEAMS), FEW_SMEM, st, P);
    }
    // One CTA, if two of them fit an SM with such rows: to meet the others of a cluster twice costs more than a third
    // would give (100 KB: 155 us in one CTA, 185 in clusters of two, 4096 rows).  Beyond that as few as leave three per SM
    // (256 KB, 4096 rows: clusters of 4 484 us, of 3 551, of 2 609, of 8 658).  More where rows are too few for the device.
    const int64_t bytes = vecs * 16;
    int64_t ctas = bytes <= ALONE ? 1 : (bytes + PART - 1) / PART;
    while (ctas < 8 && P.n_rows * ctas * 2 <= ctx->sm_count && vecs >= 1024 * ctas) ++ctas;
    if (ctas > 8 || P.k > ENTRIES || P.n_rows * ctas > 0x7fffffff) {
        const int64_t most = 2 * ctx->sm_count;
        return launch_dependent(distill_long_kernel<T>, dim3((unsigned)(P.n_rows < most ? P.n_rows : most)), dim3(1024), 0, st, P);
    }
    const int per = (int)((vecs + ctas - 1) / ctas);
    P.part_bytes = (per * 16 + 127) / 128 * 128;
    const dim3 grid((unsigned)(P.n_rows * ctas));
    const size_t smem = (size_t)P.part_bytes + entry_bytes(P.k);
    // (as few threads as have eight vectors each: the smaller the CTA, the more of them share an SM)
    if (per <= 64 * VECS) return launch_clustered((int)ctas, distill_kernel<T, 64>, grid, dim3(64 + 32), smem, st, P);
    if (per <= 128 * VECS) return launch_clustered((int)ctas, distill_kernel<T, 128>, grid, dim3(128 + 32), smem, st, P);
    return launch_clustered((int)ctas, distill_kernel<T, 256>, grid, dim3(256 + 32), smem, st, P);
}

}  // namespace

cudaError_t launch_distill(sama_ctx* ctx, int dtype, int64_t n_rows, int vocab, const void* logits, int64_t ld, int k, int top_dtype,
                           const void* top, const int32_t* ids, float temperature, const float* weight, float grad_scale, float* loss,
                           void* grad, int64_t ld_grad, cudaStream_t st) {
    if (!ctx->distill_ready) {
        cudaError_t e = allow_memory<float>();
        if (e == cudaSuccess) e = allow_memory<__nv_bfloat16>();
        if (e == cudaSuccess) e = allow_memory<__half>();
        if (e != cudaSuccess) return e;
        ctx->distill_ready = 1;
    }
    DistillParams P;
    P.logits = logits;
    P.grad = grad;
    P.in_place = grad == logits;
    P.n_rows = n_rows;
    P.ld = ld;
    P.ld_grad = ld_grad;
    P.top = top;
    P.ids = ids;
    P.weight = weight;
    P.loss = loss;
    P.status = &ctx->scalars->status;
    P.vocab = vocab;
    P.k = k;
    P.top_dtype = top_dtype;
    P.c = 1.44269504f / temperature;
    P.temperature = temperature;
    P.coef = grad_scale * temperature;
    if (dtype == SAMA_F32) return launch<float>(ctx, P, st);
    return dtype == SAMA_BF16 ? launch<__nv_bfloat16>(ctx, P, st) : launch<__half>(ctx, P, st);
}

}  // namespace sama
