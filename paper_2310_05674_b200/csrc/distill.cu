// Distillation from a teacher's top logits: loss and gradient of each row in one pass.
//
//   p = softmax(u / T) over the kept entries,  q = softmax(z / T) over the vocabulary,
//   loss = T^2 sum p (log p - log q),  grad = coef (q - p),  coef = grad_scale weight T
//
// The logits are read once and the gradient is written once, which is the floor: a row stays in shared memory between its
// sum and its gradient.  A row is a CTA's, or that of a cluster of up to 8 CTAs with 64 KB each; rows follow one another
// through a ring, and the groups of warps of a CTA work on different rows at the same time:
//   producer   bulk copies of the rows to come; the elements at the ends of rows that do not start on 16 bytes one by one
//   sums       maximum and sum of exponentials of its part
//   send       which go to all CTAs of the cluster (distributed shared memory)
//   entries    the teacher's distribution, the loss, and the gradient's values at the teacher's entries
//   gradient   q in place of z, and the entries' values over that
//   store      bulk copies back, after which the row's place is free
// so that no group's barriers and latencies are in another's way; nothing but the arrival of the sums is waited for across
// the cluster.  (All threads on one row at a time, with a cluster barrier per row, took three times as long.)
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
constexpr int SUMS = 384, GRADS = 384, TEACHER = 128, THREADS = 32 + TEACHER + 64 + SUMS + GRADS;   // groups of threads
constexpr int STORE0 = 32 + TEACHER, SEND0 = STORE0 + 32, SUMS0 = SEND0 + 32, GRADS0 = SUMS0 + SUMS; // their first threads
constexpr int RING = 192 * 1024, MAX_STAGES = 8, MIN_STAGES = 3, PART = RING / MIN_STAGES;     // a CTA's part of a row, at most
constexpr int TEACHERS = TEACHER / 32, ENTRIES = 512, BITS = 8192;   // rows whose entries are worked on, entries at most
constexpr int ENTRY_BYTES = ENTRIES * 12 + BITS / 8;                  // of a row
constexpr int SMEM = RING + TEACHERS * ENTRY_BYTES;
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
    int stages, stage_bytes;      // of the ring
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

template <int BAR, int N> __device__ __forceinline__ void group_sync() { asm volatile("bar.sync %0, %1;" ::"n"(BAR), "n"(N) : "memory"); }

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
// Where a group is in a ring: `at` counts through `size` places, `round` the times it has gone through them.
struct Turn {
    int at = 0, round = 0;
    __device__ __forceinline__ void next(int size) {
        if (++at == size) { at = 0; ++round; }
    }
};
// (m, l) of two parts, each a maximum and the sum of 2^(c (z - maximum)): l as seen from `top`.
__device__ __forceinline__ float rebase(float l, float m, float top, float c) { return m == -INFINITY ? l : l * fast_exp2((m - top) * c); }

template <typename T>
__global__ void __launch_bounds__(THREADS, 1)
distill_kernel(const DistillParams P) {
    constexpr int VE = 16 / (int)sizeof(T), SIZE = (int)sizeof(T);
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t full[MAX_STAGES], empty[MAX_STAGES], stats[2 * MAX_STAGES], entries[TEACHERS], taken[TEACHERS], done[2], summed[MAX_STAGES];
    __shared__ float2 peers[2 * MAX_STAGES][8];       // (maximum, sum) of the cluster's CTAs, by row
    __shared__ float2 warp_sums[MAX_STAGES][SUMS / 32];
    __shared__ float row_coef[TEACHERS];
    __shared__ int4 parts[MAX_STAGES];                // of the row in a place: bytes before it, vectors, whole ones from and to
    __shared__ uint32_t abort_word;
    volatile uint32_t* abort_flag = &abort_word;
    // of the teacher's entries of a row: id and then place in the part, weight and then gradient, logit
    auto e_place = [&](int b) { return reinterpret_cast<int32_t*>(smem + RING + b * ENTRY_BYTES); };
    auto e_value = [&](int b) { return reinterpret_cast<float*>(e_place(b) + ENTRIES); };

    unsigned ctas_u;
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas_u));
    const int ctas = (int)ctas_u, rank = ctas > 1 ? (int)cluster_ctarank() : 0, S = P.stages;
    const int64_t first = blockIdx.x / ctas_u, stride = gridDim.x / ctas_u;
    const int n_rows = first < P.n_rows ? (int)((P.n_rows - first + stride - 1) / stride) : 0;   // of this cluster
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(smem_u32(&full[s]), 1);
            mbar_init(smem_u32(&summed[s]), SUMS / 32);
            mbar_init(smem_u32(&empty[s]), 2);   // (the gradient, or the sums if there is none, and the entries)
        }
        // (in place, no CTA writes before the loss has the logits that it needs)
        for (int s = 0; s < 2 * S; ++s) mbar_init(smem_u32(&stats[s]), ctas + P.in_place);
        for (int b = 0; b < TEACHERS; ++b) {
            mbar_init(smem_u32(&entries[b]), 1);
            mbar_init(smem_u32(&taken[b]), 1);
        }
        for (int b = 0; b < 2; ++b) mbar_init(smem_u32(&done[b]), GRADS / 32);
        abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (ctas > 1) cluster_sync();   // the other CTAs run before their shared memory is written
    pdl_trigger();
    pdl_wait();

    const int row_bytes = P.vocab * SIZE;
    const uint8_t* z_bytes = static_cast<const uint8_t*>(P.logits);
    auto z_row = [&](int i) { return z_bytes + (first + i * stride) * P.ld * SIZE; };
    auto chunk_of = [&](int s) { return smem + s * P.stage_bytes; };
    bool ok = true;
    auto wait = [&](uint64_t* bar, int parity) {
        if (ok && !mbar_wait(smem_u32(bar), (uint32_t)parity & 1u, abort_flag)) {
            ok = false;
            *abort_flag = 1;
            atomicOr(P.status, (int)SAMA_DEV_TIMEOUT);
        }
    };
    // A row's maximum and sum over all CTAs; the same bits in each.
    auto wait_stats = [&](const Turn& r, float* most, float* total) {
        if (ok && !mbar_wait_cluster(smem_u32(&stats[r.at]), (uint32_t)r.round & 1u, abort_flag)) {
            ok = false;
            *abort_flag = 1;
            atomicOr(P.status, (int)SAMA_DEV_TIMEOUT);
        }
        const volatile float2* p = peers[r.at];
        float m = -INFINITY, l = 0.f;
#pragma unroll 1
        for (int c = 0; c < ctas; ++c) m = fmaxf(m, p[c].x);
#pragma unroll 1
        for (int c = 0; c < ctas; ++c) l += rebase(p[c].y, p[c].x, m, P.c);
        *most = m;
        *total = l;
    };
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    if (warp == 0) {
        // ---------------------------------------------------------- producer
        auto edge = [&](int i, int* place) {
            const uint8_t* row = z_row(i);
            int element;
            edge_of<VE>(span_of(row, row_bytes, rank, ctas), row_bytes, SIZE, lane, place, &element);
            return *place >= 0 && element >= 0 && element < P.vocab ? reinterpret_cast<const T*>(row)[element] : from_float<T>(-INFINITY);
        };
        int place = -1, next_place = -1, i = 0;
        T at_edge = n_rows > 0 ? edge(0, &place) : from_float<T>(0.f);
        Turn turn;
        for (; i < n_rows; ++i, turn.next(S)) {
            const T next_edge = i + 1 < n_rows ? edge(i + 1, &next_place) : from_float<T>(0.f);
            if (turn.round > 0) wait(&empty[turn.at], turn.round - 1);
            if (!__all_sync(0xffffffffu, ok)) break;
            uint8_t* chunk = chunk_of(turn.at);
            if (place >= 0) reinterpret_cast<T*>(chunk)[place] = at_edge;
            __syncwarp();
            if (lane == 0) {
                const uint8_t* row = z_row(i);
                const Span sp = span_of(row, row_bytes, rank, ctas);
                const uint32_t bytes = (uint32_t)(sp.in1 - sp.in0) * 16u, bar = smem_u32(&full[turn.at]);
                parts[turn.at] = make_int4(sp.head, sp.v1 - sp.v0, sp.in0 - sp.v0, sp.in1 - sp.v0);
                mbar_expect_tx(bar, bytes);
                if (bytes) bulk_load(smem_u32(chunk + (sp.in0 - sp.v0) * 16), row - sp.head + (int64_t)sp.in0 * 16, bytes, bar);
            }
            at_edge = next_edge;
            place = next_place;
        }
        if (*abort_flag && lane == 0)
            // let the copies already issued land before the CTA's shared memory goes away
            for (int k = max(0, i - S); k < i; ++k) mbar_wait(smem_u32(&full[k % S]), (uint32_t)(k / S) & 1u);
        __syncwarp();
    } else if (warp <= TEACHER / 32) {
        // ---------------------------------------------------------- the teacher's entries
        // A warp has every fourth row to itself, so that its loads, which depend on one another, may take four rows' time.
        const int b = warp - 1;
        int32_t* place = e_place(b);
        float *value = e_value(b), *logit = value + ENTRIES;
        uint32_t* bits = reinterpret_cast<uint32_t*>(logit + ENTRIES);
        auto over = [](float x, auto f) {
#pragma unroll
            for (int o = 16; o > 0; o /= 2) x = f(x, __shfl_xor_sync(0xffffffffu, x, o));
            return x;
        };
        int round = 0;
        for (int i = b; i < n_rows; i += TEACHERS, ++round) {
            const Turn seat{i % S, i / S}, sums{i % (2 * S), i / (2 * S)};
            const int64_t row = first + i * stride;
            const T* z = reinterpret_cast<const T*>(z_row(i));
            const Span sp = span_of(z_row(i), row_bytes, rank, ctas);
            const int skip = sp.head / SIZE - sp.v0 * VE, places = (sp.v1 - sp.v0) * VE;
            if (P.grad && round > 0) wait(&taken[b], round - 1);
            const float weight = P.weight ? P.weight[row] : 1.f;
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
            top = over(top, max_of);
            if (P.in_place && rank == 0 && lane < ctas) mbar_arrive_cluster(map_to_rank(smem_u32(&stats[sums.at]), (uint32_t)lane));
            const float from_u = top == -INFINITY ? 0.f : top * P.c;
            float sum = 0.f, entropy = 0.f;
            for (int j = lane; j < P.k; j += 32) {
                const float lp = fmaf(value[j], P.c, -from_u), p = exp2f(lp);   // log2 of p, up to the sum
                sum += p;
                if (p > 0.f) entropy += p * lp;
                value[j] = p;
            }
            sum = over(sum, sum_of);
            const bool none = sum == 0.f, zero = none || weight == 0.f;
            const float inv_u = none ? 0.f : 1.f / sum, coef = P.coef * weight;
            // Several entries with one id: the first takes them all.  An id that finds its bit set may be one of those.
            {
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
            }
            float most, total;
            wait_stats(sums, &most, &total);
            const float base = most == -INFINITY ? 0.f : most, whole = base * P.c, inv = 1.f / total;
            float cross = 0.f;
            for (int j = lane; j < P.k; j += 32) {
                const int32_t id = place[j];
                const float p = value[j] * inv_u, ze = logit[j];
                if (id >= 0 && !(p == 0.f)) cross += p * ((ze - base) * P.c);
                int at = id >= 0 ? id + skip : -1;
                if (at >= places || p == 0.f) at = -1;   // (without weight the gradient is q's own)
                value[j] = coef * (fast_exp2(fmaf(ze, P.c, -whole)) * inv - p);
                place[j] = at;
            }
            if (lane == 0) {
                row_coef[b] = coef * inv;
                if (zero) place[0] = -2;                 // zeros, whatever the logits
            }
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(smem_u32(&entries[b]));
                mbar_arrive(smem_u32(&empty[seat.at]));
            }
            if (P.loss && rank == 0) {
                // sum p (log2 p - log2 q), of which sum p = 1
                entropy = over(entropy, sum_of) * inv_u - log2f(sum);
                cross = over(cross, sum_of) - log2f(total);
                if (lane == 0) P.loss[row] = none ? 0.f : P.temperature * P.temperature * 0.69314718f * (entropy - cross);
            }
        }
    } else if (warp == STORE0 / 32) {
        // ---------------------------------------------------------- stores
        Turn turn;
        for (int i = 0; i < n_rows && P.grad; ++i, turn.next(S)) {
            uint8_t* chunk = chunk_of(turn.at);
            uint8_t* g_row = static_cast<uint8_t*>(P.grad) + (first + i * stride) * P.ld_grad * SIZE;
            wait(&done[i & 1], i / 2);
            const int4 part = parts[turn.at];
            if ((int)(reinterpret_cast<uintptr_t>(g_row) & 15u) == part.x) {
                const Span sp = span_of(z_row(i), row_bytes, rank, ctas);
                const uint32_t bytes = (uint32_t)(part.w - part.z) * 16u;
                if (lane == 0 && bytes) bulk_store(g_row - sp.head + (int64_t)sp.in0 * 16, smem_u32(chunk + part.z * 16), bytes);
                int place, element;
                edge_of<VE>(sp, row_bytes, SIZE, lane, &place, &element);
                if (place >= 0 && element >= 0 && element < P.vocab) reinterpret_cast<T*>(g_row)[element] = reinterpret_cast<const T*>(chunk)[place];
            }
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(smem_u32(&taken[i % TEACHERS]));
                asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group.read 0;" ::: "memory");
                mbar_arrive(smem_u32(&empty[turn.at]));
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    } else if (warp == SEND0 / 32) {
        // ---------------------------------------------------------- the warps' sums, to the cluster's CTAs
        Turn turn, sums;
        for (int i = 0; i < n_rows; ++i, turn.next(S), sums.next(2 * S)) {
            const int s = turn.at, slot = sums.at;
            wait(&summed[s], turn.round);
            const volatile float2* w = warp_sums[s];
            const float m = lane < SUMS / 32 ? w[lane].x : -INFINITY;
            float most = m, total = lane < SUMS / 32 ? w[lane].y : 0.f;
#pragma unroll
            for (int o = 16; o > 0; o /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
            total = rebase(total, m, most, P.c);
#pragma unroll
            for (int o = 16; o > 0; o /= 2) total += __shfl_xor_sync(0xffffffffu, total, o);
            if (lane < ctas) {
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(map_to_rank(smem_u32(&peers[slot][rank]), (uint32_t)lane)), "f"(most), "f"(total) : "memory");
                mbar_arrive_cluster(map_to_rank(smem_u32(&stats[slot]), (uint32_t)lane));
            }
            if (!P.grad && lane == 0) mbar_arrive(smem_u32(&empty[s]));
            __syncwarp();
        }
    } else if (warp < GRADS0 / 32) {
        // ---------------------------------------------------------- maxima and sums
        const int t = threadIdx.x - SUMS0;
        Turn turn;
        for (int i = 0; i < n_rows; ++i, turn.next(S)) {
            const int s = turn.at;
            wait(&full[s], turn.round);
            const uint4* chunk = reinterpret_cast<const uint4*>(chunk_of(s));
            const int n = parts[s].y;
            float m = -INFINITY, l = 0.f;
            for (int b = t; b < n; b += SUMS * BATCH) {
                uint4 x[BATCH];
                float top = -INFINITY;
#pragma unroll
                for (int v = 0; v < BATCH; ++v) x[v] = b + v * SUMS < n ? chunk[b + v * SUMS] : vec_lowest<T>();
#pragma unroll
                for (int v = 0; v < BATCH; ++v) top = fmaxf(top, vec_max<T>(x[v]));
                if (top > m) {
                    l = m == -INFINITY ? l : l * fast_exp2((m - top) * P.c);
                    m = top;
                }
                const float from = m == -INFINITY ? 0.f : m * P.c;
#pragma unroll
                for (int v = 0; v < BATCH; ++v) {
                    float f[VE], sum = 0.f;
                    unpack_vec<T>(x[v], f);
#pragma unroll
                    for (int e = 0; e < VE; ++e) sum += fast_exp2(fmaf(f[e], P.c, -from));
                    l += sum;
                }
            }
            float top = m;
#pragma unroll
            for (int o = 16; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            l = rebase(l, m, top, P.c);
#pragma unroll
            for (int o = 16; o > 0; o /= 2) l += __shfl_xor_sync(0xffffffffu, l, o);
            if (lane == 0) {
                warp_sums[s][t / 32] = make_float2(top, l);
                mbar_arrive(smem_u32(&summed[s]));
            }
        }
    } else if (P.grad) {
        // ---------------------------------------------------------- gradients
        const int t = threadIdx.x - GRADS0;
        Turn turn, sums;
        for (int i = 0; i < n_rows; ++i, turn.next(S), sums.next(2 * S)) {
            const int s = turn.at;
            uint8_t* chunk = chunk_of(s);
            float most, total;
            wait_stats(sums, &most, &total);
            const int head = parts[s].x, n = parts[s].y;
            wait(&entries[i % TEACHERS], i / TEACHERS);
            const volatile int32_t* places = e_place(i % TEACHERS);
            const bool zero = places[0] == -2;
            const float f = *const_cast<volatile float*>(&row_coef[i % TEACHERS]), whole = most == -INFINITY ? 0.f : most * P.c;
            if (zero) {
                for (int b = t; b < n; b += GRADS) reinterpret_cast<uint4*>(chunk)[b] = make_uint4(0u, 0u, 0u, 0u);
            } else {
#pragma unroll 4
                for (int b = t; b < n; b += GRADS) {
                    float g[VE];
                    unpack_vec<T>(reinterpret_cast<const uint4*>(chunk)[b], g);
#pragma unroll
                    for (int e = 0; e < VE; ++e) g[e] = fast_exp2(fmaf(g[e], P.c, -whole)) * f;
                    store_n<T, VE>(reinterpret_cast<T*>(chunk) + b * VE, g);
                }
            }
            group_sync<3, GRADS>();
            if (!zero)
                for (int j = t; j < P.k; j += GRADS) {
                    const int place = places[j];
                    if (place >= 0) reinterpret_cast<T*>(chunk)[place] = from_float<T>(e_value(i % TEACHERS)[j]);
                }
            uint8_t* g_row = static_cast<uint8_t*>(P.grad) + (first + i * stride) * P.ld_grad * SIZE;
            if ((int)(reinterpret_cast<uintptr_t>(g_row) & 15u) != head) {
                // rows of the gradient start elsewhere than those of the logits
                group_sync<3, GRADS>();
                const int skip = head / SIZE - span_of(z_row(i), row_bytes, rank, ctas).v0 * VE, e0 = max(0, -skip), e1 = min(P.vocab, n * VE - skip);
                for (int e = e0 + t; e < e1; e += GRADS) reinterpret_cast<T*>(g_row)[e] = reinterpret_cast<const T*>(chunk)[e + skip];
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&done[i & 1]));
        }
    }
    __syncthreads();
    if (ctas > 1) cluster_sync();   // no CTA leaves while another may write to it
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
        if (!mbar_wait(bar(stage), (uint32_t)parity)) timed_out = true;
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
        const float from = top == -INFINITY ? 0.f : top * P.c, from_u = top_u == -INFINITY ? 0.f : top_u * P.c;
        float sum = 0.f, sum_u = 0.f;
#pragma unroll
        for (int i = 0; i < VECS * VE; ++i) {
            v[i] = fast_exp2(fmaf(v[i], P.c, -from));
            sum += v[i];
        }
#pragma unroll
        for (int i = 0; i < FEW_ENTRIES; ++i) {
            my_u[i] = fmaf(my_u[i], P.c, -from_u);       // log2 of p, up to the sum
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
                if (my_id[i] >= 0 && !(p == 0.f)) part += p * ((my_u[i] - log_u) - ((my_z[i] - (top == -INFINITY ? 0.f : top)) * P.c - log_total));
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
                if (is_first) reinterpret_cast<T*>(chunk)[my_id[i] + s.head / SIZE] = from_float<T>(coef * (fast_exp2(fmaf(my_z[i], P.c, -from)) * inv - p));
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
            const float from = top == -INFINITY ? 0.f : top * P.c;
            l *= m == -INFINITY ? 0.f : fast_exp2((m - top) * P.c);
            m = top;
#pragma unroll
            for (int i = 0; i < 8; ++i) l += fast_exp2(fmaf(v[i], P.c, -from));
        }
        const float2 tops = reduce(m, u, max_of);
        const float from = tops.x == -INFINITY ? 0.f : tops.x * P.c, from_u = tops.y == -INFINITY ? 0.f : tops.y * P.c;
        u = fmaf(u, P.c, -from_u);
        // (a part of nothing but -infinity has a sum of 0, one with a NaN a sum of NaN)
        const float2 sums = reduce(m == -INFINITY ? l : l * fast_exp2((m - tops.x) * P.c), exp2f(u), sum_of);
        const float inv = 1.f / sums.x, inv_u = sums.y > 0.f ? 1.f / sums.y : 0.f;
        const bool none = !(sums.y > 0.f) && sums.y == sums.y;
        const float p = exp2f(u) * inv_u;
        if (P.loss) {
            const float log_q = (target - (tops.x == -INFINITY ? 0.f : tops.x)) / P.temperature - logf(sums.x);
            const float part = reduce(id >= 0 && !(p == 0.f) ? p * ((u - log2f(sums.y)) * 0.69314718f - log_q) : 0.f, 0.f, sum_of).x;
            if (t == 0) P.loss[row] = none ? 0.f : P.temperature * P.temperature * part;
        }
        if (!P.grad) continue;
        const float weight = P.weight ? P.weight[row] : 1.f, coef = none ? 0.f : P.coef * weight;
        const bool zero = none || weight == 0.f;
        T* g = static_cast<T*>(P.grad) + row * P.ld_grad;
        for (int e = t; e < P.vocab; e += TEAM)
            g[e] = from_float<T>(zero ? 0.f : coef * (fast_exp2(fmaf(to_float(z[e]), P.c, -from)) * inv));
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
            if (is_first) g[id] = from_float<T>(coef * (fast_exp2(fmaf(target, P.c, -from)) * inv - all));
        }
        __syncthreads();   // the entries may be written again
    }
}

// Once per context: how many clusters of 2, 4 and 8 CTAs can be resident.
cudaError_t prepare(sama_ctx* ctx) {
    if (ctx->distill_clusters[0] > 0) return cudaSuccess;
    void* kernels[3] = {(void*)distill_kernel<float>, (void*)distill_kernel<__half>, (void*)distill_kernel<__nv_bfloat16>};
    void* few[3] = {(void*)distill_few_kernel<float>, (void*)distill_few_kernel<__half>, (void*)distill_few_kernel<__nv_bfloat16>};
    cudaError_t e;
    for (int i = 0; i < 3; ++i) {
        if ((e = cudaFuncSetAttribute(kernels[i], cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM)) != cudaSuccess) return e;
        if ((e = cudaFuncSetAttribute(few[i], cudaFuncAttributeMaxDynamicSharedMemorySize, FEW_SMEM)) != cudaSuccess) return e;
    }
    int found[3];
    for (int i = 0; i < 3; ++i) {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 2u << i;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.gridDim = dim3(ctx->sm_count / (2 << i) * (2 << i));
        cfg.blockDim = dim3(THREADS);
        cfg.dynamicSmemBytes = SMEM;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if ((e = cudaOccupancyMaxActiveClusters(&found[i], distill_kernel<__nv_bfloat16>, &cfg)) != cudaSuccess) return e;
        if (found[i] < 1) return cudaErrorLaunchOutOfResources;
    }
    for (int i = 2; i >= 0; --i) ctx->distill_clusters[i] = found[i];
    return cudaSuccess;
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
    if (vecs * 16 > 8 * PART || P.k > ENTRIES) {
        const int64_t most = 2 * ctx->sm_count;
        return launch_dependent(distill_long_kernel<T>, dim3((unsigned)(P.n_rows < most ? P.n_rows : most)), dim3(1024), 0, st, P);
    }
    // The fewest CTAs that can hold a row, since each of them has a row's fixed costs to bear; more where rows are too few to
    // fill the device.
    int ctas = 1;
    while (vecs * 16 > (int64_t)ctas * PART || (ctas < 8 && P.n_rows * ctas * 2 <= ctx->sm_count && vecs >= 2 * ctas * SUMS)) ctas *= 2;
    P.stage_bytes = (int)((vecs + ctas - 1) / ctas) * 16;
    P.stage_bytes = (P.stage_bytes + 127) / 128 * 128;
    P.stages = RING / P.stage_bytes < MAX_STAGES ? RING / P.stage_bytes : MAX_STAGES;
    const int64_t most = ctas == 1 ? ctx->sm_count : ctx->distill_clusters[ctas == 2 ? 0 : ctas == 4 ? 1 : 2];
    const int64_t teams = P.n_rows < most ? P.n_rows : most;
    return launch_clustered(ctas, distill_kernel<T>, dim3((unsigned)(teams * ctas)), dim3(THREADS), SMEM, st, P);
}

}  // namespace

cudaError_t launch_distill(sama_ctx* ctx, int dtype, int64_t n_rows, int vocab, const void* logits, int64_t ld, int k, int top_dtype,
                           const void* top, const int32_t* ids, float temperature, const float* weight, float grad_scale, float* loss,
                           void* grad, int64_t ld_grad, cudaStream_t st) {
    const cudaError_t e = prepare(ctx);
    if (e != cudaSuccess) return e;
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
