// Distillation from a teacher's top logits: loss and gradient of each row in one pass.
//
//   p = softmax(u / T) over the kept entries,  q = softmax(z / T) over the vocabulary,
//   loss = T^2 sum p (log p - log q),  grad = coef (q - p),  coef = grad_scale weight T
//
// The logits are read once and the gradient is written once, which is the floor: a row stays on the chip between its sum and
// its gradient.  A team works on a row: a warp (rows up to 4 KB), a CTA of 256 (32 KB), or a cluster of up to 8 CTAs of 256
// or 512 threads (256 KB, 512 KB) that exchange maximum and sum through distributed shared memory, one cluster barrier per
// row.  Rows come by bulk copies into a ring of three, two of them ahead; each thread holds 8 vectors of 16 bytes as
// exponentials in registers (one exponential per logit: at 4 bytes moved per 16-bit logit, two would take most of what the
// special-function units can do), writes the gradient over them in shared memory, and bulk copies take it out.  The
// teacher's entries are put right in shared memory before that.  Rows that do not start on 16 bytes have the elements at
// their two ends read and written one by one.  Longer rows are read twice.
#include <type_traits>

#include "num_types.h"
#include "sama_internal.h"
#include "tc_ptx.h"

namespace sama {

namespace {

constexpr int VECS = 8;        // vectors of a thread
constexpr int STAGES = 3;
constexpr int ENTRIES = 4;     // of the teacher's, of a thread
constexpr int kMaxEntries = 1024;

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
    float c, temperature, coef;   // log2 e / T, T, grad_scale T
};

template <typename T> __device__ __forceinline__ T lowest() { return from_float<T>(-INFINITY); }

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

template <int THREADS> constexpr int distill_smem() { return THREADS * VECS * 16 * STAGES + kMaxEntries * 8; }

// TEAM threads per row, or (CLUSTER) all CTAs of a cluster.
template <typename T, int TEAM, int THREADS, bool CLUSTER>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 2 : 1)
distill_kernel(const DistillParams P) {
    constexpr int VE = 16 / (int)sizeof(T), TEAMS = THREADS / TEAM, CHUNK = TEAM * VECS * 16, TEAM_ENTRIES = kMaxEntries / TEAMS;
    static_assert(ENTRIES * TEAM >= TEAM_ENTRIES, "entries of a thread");
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t bars[TEAMS][STAGES];
    __shared__ float2 slots[2][THREADS / 32];
    __shared__ float2 peers[2][8];        // (maximum, sum) of the cluster's CTAs, rows in turn
    const int team = threadIdx.x / TEAM, t = threadIdx.x % TEAM;
    uint8_t* ring = smem + team * STAGES * CHUNK;
    int32_t* e_id = reinterpret_cast<int32_t*>(smem + TEAMS * STAGES * CHUNK) + team * TEAM_ENTRIES;
    float* e_p = reinterpret_cast<float*>(e_id - team * TEAM_ENTRIES + kMaxEntries) + team * TEAM_ENTRIES;
    Reduce<TEAM> reduce{&slots[0][0]};
    auto bar = [&](int s) { return smem_u32(&bars[team][s]); };

    unsigned ctas = 1;
    if (CLUSTER) asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas));
    const int rank = CLUSTER ? (int)cluster_ctarank() : 0;
    const int64_t first = CLUSTER ? blockIdx.x / ctas : (int64_t)blockIdx.x * TEAMS + team;
    const int64_t stride = CLUSTER ? gridDim.x / ctas : (int64_t)gridDim.x * TEAMS;

    if (t == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(bar(s), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    reduce.sync();
    if (CLUSTER) cluster_sync();   // the other CTAs run before their shared memory is written
    pdl_trigger();
    pdl_wait();

    const int row_bytes = P.vocab * (int)sizeof(T);
    // This CTA's vectors [v0, v1) of a row, those of them that lie wholly within it, and bytes before the row in the first.
    struct Span { int head, v0, v1, in0, in1; };
    auto span_of = [&](const void* base, int64_t ld, int64_t row, int head_of) {
        Span s;
        s.head = head_of >= 0 ? head_of : (int)((reinterpret_cast<uintptr_t>(base) + (uintptr_t)(row * ld * (int64_t)sizeof(T))) & 15u);
        const int n = (s.head + row_bytes + 15) / 16, per = CLUSTER ? (n + (int)ctas - 1) / (int)ctas : n;
        s.v0 = min(rank * per, n);
        s.v1 = min(s.v0 + per, n);
        s.in0 = max(s.v0, s.head ? 1 : 0);
        s.in1 = max(s.in0, min(s.v1, (s.head + row_bytes) / 16));
        return s;
    };
    const uint8_t* z_bytes = static_cast<const uint8_t*>(P.logits);
    uint8_t* g_bytes = static_cast<uint8_t*>(P.grad);
    auto row_at = [&](int64_t row) { return row * P.ld * (int64_t)sizeof(T); };

    // Elements of the first and the last vector that is not whole: thread t < VE has one of the first, VE <= t < 2 VE of the last.
    auto edge_at = [&](const Span& s, int* element) {   // place in this CTA's vectors, or -1
        const int last = (s.head + row_bytes) / 16;
        const int v = t < VE ? 0 : last;
        *element = v * VE + t % VE - s.head / (int)sizeof(T);
        const bool mine = t < 2 * VE && v >= s.v0 && v < s.v1 && *element >= 0 && *element < P.vocab &&
                          (t < VE ? s.head != 0 : (s.head + row_bytes) % 16 != 0 && !(last == 0 && s.head != 0));
        return mine ? (v - s.v0) * VE + t % VE : -1;
    };
    // What a thread has at hand of a row before its turn comes: an element at the row's end, and entries of the teacher.
    float edge = 0.f;
    int32_t id[ENTRIES];
    float u[ENTRIES], z[ENTRIES];
    auto fetch_row = [&](int64_t row, int stage) {
        const Span s = span_of(P.logits, P.ld, row, -1);
        if (t == 0) {
            const uint32_t bytes = (uint32_t)(s.in1 - s.in0) * 16u;
            mbar_expect_tx(bar(stage), bytes);
            if (bytes) bulk_load(smem_u32(ring + stage * CHUNK + (s.in0 - s.v0) * 16), z_bytes + row_at(row) - s.head + (int64_t)s.in0 * 16, bytes, bar(stage));
        }
    };
    auto fetch_entries = [&](int64_t row) {
        const Span s = span_of(P.logits, P.ld, row, -1);
        int element;
        if (edge_at(s, &element) >= 0) edge = to_float(reinterpret_cast<const T*>(z_bytes + row_at(row))[element]);
#pragma unroll
        for (int i = 0; i < ENTRIES; ++i) {
            const int j = t + i * TEAM;
            id[i] = j < P.k ? P.ids[row * P.k + j] : -1;
            u[i] = j < P.k ? load_top(P, row * P.k + j) : -INFINITY;
        }
    };
    auto fetch_targets = [&](int64_t row) {
#pragma unroll
        for (int i = 0; i < ENTRIES; ++i) {
            if (id[i] < -1 || id[i] >= P.vocab) {
                atomicOr(P.status, (int)SAMA_DEV_BAD_INDEX);
                id[i] = -1;
            }
            if (id[i] < 0) u[i] = -INFINITY;
            z[i] = id[i] >= 0 ? to_float(reinterpret_cast<const T*>(z_bytes + row_at(row))[id[i]]) : 0.f;
        }
    };

    for (int i = 0; i < STAGES - 1; ++i)
        if (first + i * stride < P.n_rows) fetch_row(first + i * stride, i);
    if (first < P.n_rows) {
        fetch_entries(first);
        fetch_targets(first);
    }
    int stage = 0, parity = 0, turn = 0;
    bool timed_out = false;
    for (int64_t row = first; row < P.n_rows; row += stride) {
        const Span s = span_of(P.logits, P.ld, row, -1);
        uint8_t* chunk = ring + stage * CHUNK;
        if (!mbar_wait(bar(stage), (uint32_t)parity)) timed_out = true;
        // the row's ends: its own elements there, and nothing beside them
        const int n = s.v1 - s.v0;
        if (t < 2 * VE) {
            const int last = (s.head + row_bytes) / 16, v = t < VE ? 0 : last;
            const bool partial = t < VE ? s.head != 0 : (s.head + row_bytes) % 16 != 0 && !(last == 0 && s.head != 0);
            int element;
            const int place = edge_at(s, &element);
            if (partial && v >= s.v0 && v < s.v1) reinterpret_cast<T*>(chunk)[(v - s.v0) * VE + t % VE] = place >= 0 ? from_float<T>(edge) : lowest<T>();
        }
        float my_u[ENTRIES], my_z[ENTRIES], top_u = -INFINITY;
        int32_t my_id[ENTRIES];
#pragma unroll
        for (int i = 0; i < ENTRIES; ++i) {
            my_id[i] = id[i];
            my_u[i] = u[i];
            my_z[i] = z[i];
            top_u = fmaxf(top_u, u[i]);
        }
        const bool more = row + stride < P.n_rows;
        if (more) fetch_entries(row + stride);
        const float weight = P.weight ? P.weight[row] : 1.f;
        reduce.sync();

        float v[VECS * VE], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            const int at = t + i * TEAM;
            if (at < n) {
                unpack_vec<T>(reinterpret_cast<const uint4*>(chunk)[at], v + i * VE);
            } else {
#pragma unroll
                for (int e = 0; e < VE; ++e) v[i * VE + e] = -INFINITY;
            }
        }
#pragma unroll
        for (int i = 0; i < VECS * VE; ++i) top = fmaxf(top, v[i]);
        const float2 tops = reduce(top, top_u, max_of);
        const float from = tops.x == -INFINITY ? 0.f : tops.x * P.c, from_u = tops.y == -INFINITY ? 0.f : tops.y * P.c;
        float sum = 0.f, sum_u = 0.f;
#pragma unroll
        for (int i = 0; i < VECS * VE; ++i) {
            v[i] = fast_exp2(fmaf(v[i], P.c, -from));
            sum += v[i];
        }
#pragma unroll
        for (int i = 0; i < ENTRIES; ++i) {
            my_u[i] = fmaf(my_u[i], P.c, -from_u);       // log2 of p, up to the sum
            sum_u += exp2f(my_u[i]);
        }
        const float2 sums = reduce(sum, sum_u, sum_of);
        float most = tops.x, total = sums.x;
        if (CLUSTER) {
            const uint32_t mine = smem_u32(&peers[turn][rank]);
            if (t < (int)ctas)
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(map_to_rank(mine, (uint32_t)t)), "f"(tops.x), "f"(sums.x) : "memory");
            cluster_sync();
            most = -INFINITY;
            for (int r = 0; r < (int)ctas; ++r) most = fmaxf(most, peers[turn][r].x);
            total = 0.f;
            for (int r = 0; r < (int)ctas; ++r) {
                const float2 ml = peers[turn][r];
                total += ml.x == -INFINITY ? 0.f : ml.y * fast_exp2((ml.x - most) * P.c);
            }
            turn ^= 1;
        }
        const float whole = most == -INFINITY ? 0.f : most * P.c, inv = 1.f / total, inv_u = sums.y > 0.f ? 1.f / sums.y : 0.f;
        const bool none = !(sums.y > 0.f) && sums.y == sums.y;      // no entry
        const float log_total = logf(total), log_u = log2f(sums.y);
        // the loss, by the first CTA
        float part = 0.f;
        const bool has_loss = P.loss && rank == 0;
        if (has_loss) {
#pragma unroll
            for (int i = 0; i < ENTRIES; ++i) {
                const float p = exp2f(my_u[i]) * inv_u;
                const float log_q = (my_z[i] - (most == -INFINITY ? 0.f : most)) / P.temperature - log_total;
                if (my_id[i] >= 0 && !(p == 0.f)) part += p * ((my_u[i] - log_u) * 0.69314718f - log_q);
            }
            part = reduce(part, 0.f, sum_of).x;
            if (t == 0) P.loss[row] = none ? 0.f : P.temperature * P.temperature * part;
        }
        if (P.grad) {
            const float coef = none ? 0.f : P.coef * weight;
            const bool zero = none || weight == 0.f;
            const float f = coef * (CLUSTER && tops.x != -INFINITY ? fast_exp2((tops.x - most) * P.c) * inv : inv);
#pragma unroll
            for (int i = 0; i < VECS; ++i) {
                const int at = t + i * TEAM;
                if (at < n) {
                    float g[VE];
#pragma unroll
                    for (int e = 0; e < VE; ++e) g[e] = zero ? 0.f : v[i * VE + e] * f;
                    store_n<T, VE>(reinterpret_cast<T*>(chunk) + at * VE, g);
                }
            }
#pragma unroll
            for (int i = 0; i < ENTRIES; ++i) {
                const int j = t + i * TEAM;
                if (j < TEAM_ENTRIES) {
                    e_id[j] = my_id[i];
                    e_p[j] = exp2f(my_u[i]) * inv_u;
                }
            }
            reduce.sync();
            // the teacher's entries; of several with one id the first takes them all
#pragma unroll
            for (int i = 0; i < ENTRIES; ++i) {
                const int place = my_id[i] + s.head / (int)sizeof(T) - s.v0 * VE;
                if (zero || my_id[i] < 0 || place < 0 || place >= n * VE) continue;
                const int j = t + i * TEAM;
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
                if (is_first) reinterpret_cast<T*>(chunk)[place] = from_float<T>(coef * (fast_exp2(fmaf(my_z[i], P.c, -whole)) * inv - p));
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            reduce.sync();
            uint8_t* g_row = g_bytes + row * P.ld_grad * (int64_t)sizeof(T);
            if ((int)(reinterpret_cast<uintptr_t>(g_row) & 15u) == s.head) {
                if (t == 0) {
                    const uint32_t bytes = (uint32_t)(s.in1 - s.in0) * 16u;
                    if (bytes) bulk_store(g_row - s.head + (int64_t)s.in0 * 16, smem_u32(chunk + (s.in0 - s.v0) * 16), bytes);
                }
                int element;
                const int place = edge_at(s, &element);
                if (place >= 0) reinterpret_cast<T*>(g_row)[element] = reinterpret_cast<const T*>(chunk)[place];
            } else {
                // rows of the gradient start elsewhere than those of the logits
                const int skip = s.head / (int)sizeof(T) - s.v0 * VE;
                const int e0 = max(0, -skip), e1 = min(P.vocab, n * VE - skip);
                for (int e = e0 + t; e < e1; e += TEAM) reinterpret_cast<T*>(g_row)[e] = reinterpret_cast<const T*>(chunk)[e + skip];
                reduce.sync();
            }
        }
        if (t == 0) asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group.read 1;" ::: "memory");
        // the row after the next takes the place of the one before this, whose gradient has left it
        const int64_t after = row + (STAGES - 1) * stride;
        if (after < P.n_rows) fetch_row(after, (stage + STAGES - 1) % STAGES);
        if (more) fetch_targets(row + stride);
        if (++stage == STAGES) { stage = 0; parity ^= 1; }
    }
    if (t == 0) {
        if (timed_out) atomicOr(P.status, (int)SAMA_DEV_TIMEOUT);
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    if (CLUSTER) cluster_sync();   // no CTA leaves while another may write to it
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

template <typename T, int TEAM, int THREADS, bool CLUSTER>
cudaError_t launch(sama_ctx* ctx, const DistillParams& P, int cluster, cudaStream_t st) {
    auto* kernel = distill_kernel<T, TEAM, THREADS, CLUSTER>;
    constexpr int SMEM = distill_smem<THREADS>();
    const uint32_t bit = 1u << ((std::is_same<T, float>::value ? 0 : std::is_same<T, __half>::value ? 4 : 8) +
                                (TEAM == 32 ? 0 : !CLUSTER ? 1 : THREADS == 256 ? 2 : 3));
    if (!(ctx->distill_ready & bit)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
        if (e != cudaSuccess) return e;
        ctx->distill_ready |= bit;
    }
    const int most = (THREADS == 256 ? 2 : 1) * ctx->sm_count / cluster;            // teams that are resident, or a little more
    const int64_t wanted = CLUSTER ? P.n_rows : (P.n_rows + THREADS / TEAM - 1) / (THREADS / TEAM);
    const int64_t teams = wanted < most ? wanted : most;
    KernelScope scope(ctx, SAMA_K_DISTILL, -1, st);
    return launch_clustered(CLUSTER ? cluster : 1, kernel, dim3((unsigned)(teams * cluster)), dim3(THREADS), SMEM, st, P);
}

template <typename T>
cudaError_t launch(sama_ctx* ctx, const DistillParams& P, cudaStream_t st) {
    // vectors of a row, wherever it starts
    const int64_t vecs = ((int64_t)P.vocab * (int)sizeof(T) + 15 + 15) / 16;
    if (vecs <= 32 * VECS && P.k <= kMaxEntries / 8) return launch<T, 32, 256, false>(ctx, P, 1, st);
    if (vecs <= 256 * VECS) return launch<T, 256, 256, false>(ctx, P, 1, st);
    for (int n = 2; n <= 8; n *= 2)
        if (vecs <= (int64_t)256 * VECS * n) return launch<T, 256, 256, true>(ctx, P, n, st);
    if (vecs <= (int64_t)512 * VECS * 8) return launch<T, 512, 512, true>(ctx, P, 8, st);
    KernelScope scope(ctx, SAMA_K_DISTILL, -1, st);
    const int64_t most = 2 * ctx->sm_count;
    return launch_dependent(distill_long_kernel<T>, dim3((unsigned)(P.n_rows < most ? P.n_rows : most)), dim3(1024), 0, st, P);
}

}  // namespace

cudaError_t launch_distill(sama_ctx* ctx, int dtype, int64_t n_rows, int vocab, const void* logits, int64_t ld, int k, int top_dtype,
                           const void* top, const int32_t* ids, float temperature, const float* weight, float grad_scale, float* loss,
                           void* grad, int64_t ld_grad, cudaStream_t st) {
    DistillParams P;
    P.logits = logits;
    P.grad = grad;
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
