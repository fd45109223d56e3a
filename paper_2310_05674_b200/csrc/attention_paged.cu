// Attention of one new token per sequence over a cache in pages.
//
// Every key and value is read once for each 8 queries that share its head: 2 to 16 flops per byte, bound by memory
// (96 sequences of up to 4096 keys, 32 heads of 128 over 8: 165 to 173 us, 5.5 to 5.8 TB/s, 0.84 to 0.88 of the copy rate; one of
// 60,001, capped: 50 for 37 at that rate, the rest the way to the first keys, three loads that depend on one another, and the join).
// What is needed is bytes in flight, so the cache streams through rings in shared memory, a ring per warp, by asynchronous
// 16-byte copies that follow the page table; three tiles of 16 keys and values (8 KB each at 128 columns) are on their way per
// warp, 8 warps per SM.  The products are small (8 queries by 16 keys) and go to the warp-level matrix instructions: the
// tensor memory of the 5th generation wants 64 rows or more, of which a single token has 8 at most, and the warp-level
// ones do five times what memory can feed (without them, on the fp32 units, four queries per key head would be the limit).
//
// The work is the list of all (sequence, key head, 64 keys) steps, cut into equal parts, one per CTA, whatever the
// sequences' lengths: a CTA may finish one sequence, go through others and start on a last.  A head's keys that fall to
// several CTAs are joined by the one that arrives last, in the order of the keys, so the bits do not depend on which it is.
#include <type_traits>

#include "attention.h"

namespace sama {

namespace {

constexpr int WARPS = 4, THREADS = 32 * WARPS;
constexpr int KEYS = 16;                 // of a warp's tile
constexpr int STEP = kPagedStep;         // of a CTA's step
static_assert(STEP == KEYS * WARPS, "a tile per warp");
constexpr int ROWS = 8;                  // queries of a unit of work
constexpr int STAGES = 3;
constexpr int kMinSteps = 2;             // a CTA's share, at least: 128 keys

template <int D> struct PagedTile {
    static constexpr int TILE = KEYS * D * 2, RING = STAGES * 2 * TILE, LD = D + 4;   // LD: a row's sums, maximum and weight
};

// fp16 has fewer places below 2^-14: weights, which are 1 at most, are lifted there as operands.
template <typename T> constexpr float kLift = std::is_same<T, __half>::value ? 32768.f : 1.f;

struct PagedParams {
    PagedShape a;
    const void *q, *k_new, *v_new;
    void *k_cache, *v_cache, *out;
    float* parts;    // [2 per CTA][ROWS][LD]
    int* arrived;    // [CTA], zero between launches
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// c (8 used rows x 8) += a (8 used rows x 16) b (16 x 8)
template <typename T>
__device__ __forceinline__ void mma(float* c, uint32_t a0, uint32_t a2, uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<T, __nv_bfloat16>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(0), "r"(a2), "r"(0), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(0), "r"(a2), "r"(0), "r"(b0), "r"(b1));
}

__device__ __forceinline__ int paged_length(const PagedShape& a, int s) { return paged_keys(a.lengths[s], a.max_pages, a.page_size); }

// A place in the list of steps.
struct Place {
    int s, unit, step, len, steps;   // sequence; key head and group of ROWS queries; step of the sequence, its length and number of steps
};

template <typename T, int D, AttnCap CAP, bool BIAS>
__global__ void __launch_bounds__(THREADS, 2)
paged_kernel(const PagedParams P) {
    using C = PagedTile<D>;
    constexpr int LD = C::LD;
    const PagedShape& a = P.a;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    float* sums = reinterpret_cast<float*>(smem_raw + WARPS * C::RING);   // [WARPS][ROWS][LD], or a factor for each part and row
    __shared__ int64_t scan[WARPS];
    __shared__ int64_t start_before;
    __shared__ int start_s, last_to_arrive;
    __shared__ float row_weight[ROWS];

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t ring = smem_u32(smem_raw) + warp * C::RING;
    const int tiles_of_rows = (a.group + ROWS - 1) / ROWS, units = a.kv_heads * tiles_of_rows;

    pdl_trigger();
    pdl_wait();

    // Steps of all sequences, and the sequence in which this CTA's share begins: each thread adds up a run of sequences.
    const int run = (a.n_seqs + THREADS - 1) / THREADS, s0 = min((int)threadIdx.x * run, a.n_seqs), s1 = min(s0 + run, a.n_seqs);
    auto steps_of = [&](int s) { return paged_steps(paged_length(a, s)); };
    int64_t mine = 0;
    for (int s = s0; s < s1; ++s) mine += (int64_t)steps_of(s) * units;
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int64_t x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    if (lane == 31) scan[warp] = upto;
    __syncthreads();
    int64_t total = 0;
    for (int w = 0; w < WARPS; ++w) {
        if (w < warp) upto += scan[w];
        total += scan[w];
    }
    const int ctas = (int)min((int64_t)gridDim.x, max((int64_t)1, total / kMinSteps)), cta = (int)blockIdx.x;
    auto first_of = [&](int c) { return total / ctas * c + total % ctas * c / ctas; };   // (total * c might pass 64 bits)
    const int64_t begin = cta < ctas ? first_of(cta) : total, end = cta < ctas ? first_of(cta + 1) : total;
    if (begin < end && begin >= upto - mine && begin < upto) {
        int64_t before = upto - mine;
        int s = s0;
        for (; s < s1; ++s) {
            const int64_t n = (int64_t)steps_of(s) * units;
            if (begin < before + n) break;
            before += n;
        }
        start_s = s;
        start_before = before;
    }
    if (cta == 0) {
        bool bad = false;
        for (int s = threadIdx.x; s < a.n_seqs; s += THREADS) bad |= paged_length(a, s) != a.lengths[s];
        if (bad) atomicOr(a.status, (int)SAMA_DEV_BAD_INDEX);
    }
    // sequences without a key
    for (int s = cta; s < a.n_seqs; s += (int)gridDim.x)
        if (paged_length(a, s) == 0)
            for (int i = threadIdx.x; i < a.heads * a.dim; i += THREADS)
                static_cast<T*>(P.out)[(int64_t)s * a.heads * a.dim + i] = from_float<T>(0.f);
    __syncthreads();
    if (begin >= end) return;

    Place at;   // of the next step to be worked on
    at.s = start_s;
    at.len = paged_length(a, at.s);
    at.steps = paged_steps(at.len);
    const int64_t inside = begin - start_before;
    at.unit = (int)(inside / at.steps);
    at.step = (int)(inside - (int64_t)at.unit * at.steps);
    auto advance = [&](Place& p) {
        if (++p.step < p.steps) return;
        p.step = 0;
        if (++p.unit < units) return;
        p.unit = 0;
        do {
            if (++p.s >= a.n_seqs) { p.steps = p.len = 0; return; }
            p.len = paged_length(a, p.s);
            p.steps = paged_steps(p.len);
        } while (p.steps == 0);
    };

    // Where a tile's key of this lane (of the first 16) lies: an offset, a multiple of 8, with the new token's own row marked
    // by bit 0; or -1.
    auto locate = [&](const Place& p) -> int64_t {
        const int pos = p.step * STEP + warp * KEYS + (lane & 15), g = p.unit / tiles_of_rows;
        if (pos >= p.len) return -1;
        if (P.k_new && pos == p.len - 1) return (((int64_t)p.s * a.kv_heads + g) * a.dim) | 1;
        const uint32_t column = (uint32_t)pos / (uint32_t)a.page_size, in_page = (uint32_t)pos - column * (uint32_t)a.page_size;
        const int page = a.page_table[(int64_t)p.s * a.max_pages + column];
        if (page < 0 || page >= a.n_pages) {
            atomicOr(a.status, (int)SAMA_DEV_BAD_INDEX);
            return -1;
        }
        return page * a.page_stride + ((int64_t)in_page * a.kv_heads + g) * a.dim;
    };
    auto copy = [&](int stage, int64_t where) {
        constexpr int CHUNKS = D / 8, PER = 32 / CHUNKS;   // 16-byte chunks of a row, rows at a time
        const int c = lane % CHUNKS;
        const uint32_t base = ring + stage * 2 * C::TILE;
#pragma unroll
        for (int i = 0; i < KEYS / PER; ++i) {
            const int r = i * PER + lane / CHUNKS;
            const int64_t w = __shfl_sync(0xffffffffu, where, r);
            const bool real = w >= 0 && 8 * c < a.dim, fresh = w & 1;
            const int64_t o = real ? (w & ~(int64_t)1) + 8 * c : 0;
            const uint32_t dst = base + r * (D * 2) + ((c ^ (r & 7)) << 4);
            copy16(dst, static_cast<const T*>(fresh && real ? P.k_new : P.k_cache) + o, real);
            copy16(dst + C::TILE, static_cast<const T*>(fresh && real ? P.v_new : P.v_cache) + o, real);
        }
    };

    // The ring runs two steps ahead, and the addresses of its copies one more.
    const int n = (int)(end - begin);
    Place ahead = at;
    int64_t where[STAGES];   // of the tiles in the ring, by stage
    int64_t next = locate(ahead);
#pragma unroll
    for (int i = 0; i < STAGES; ++i) {
        if (i < STAGES - 1) {
            where[i] = next;
            if (i < n) {
                copy(i, next);
                advance(ahead);
                if (i + 1 < n) next = locate(ahead);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        } else {
            where[i] = -1;
        }
    }

    constexpr bool RAW = !CAP && !BIAS;
    const float c = RAW ? a.scale * kLog2e : 1.f;
    const AttnTanh capped(CAP ? a.scale / a.cap : 0.f, CAP ? a.cap * kLog2e : 0.f);
    uint32_t qf[D / 16][2];
    float o[D / 8][4], m = -INFINITY, l = 0.f, slope = 0.f;
    bool fresh_unit = true;
    int first_step = at.step;

    for (int i = 0; i < n; ++i) {
        const int stage = i % STAGES;
        if (fresh_unit) {
            // queries of this unit, and empty sums
            const int g = at.unit / tiles_of_rows, row = (at.unit - g * tiles_of_rows) * ROWS + lane / 4;
            const bool real = row < a.group;
            const int head = g * a.group + (real ? row : 0);
            const T* q = static_cast<const T*>(P.q) + ((int64_t)at.s * a.heads + head) * a.dim;
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int col = 16 * k + 8 * h + 2 * (lane & 3);
                    qf[k][h] = real && col < a.dim ? *reinterpret_cast<const uint32_t*>(q + col) : 0u;
                }
            if (BIAS) slope = a.slopes[head] * kLog2e;
#pragma unroll
            for (int k = 0; k < D / 8; ++k) o[k][0] = o[k][1] = o[k][2] = o[k][3] = 0.f;
            m = -INFINITY;
            l = 0.f;
            first_step = at.step;
            fresh_unit = false;
        }
        // the next tile's copies take the stage that the step before has left
        {
            const int s = (i + STAGES - 1) % STAGES;
            if (i + STAGES - 1 < n) {
                copy(s, next);
#pragma unroll
                for (int k = 0; k < STAGES; ++k)
                    if (k == s) where[k] = next;
                advance(ahead);
                if (i + STAGES < n) next = locate(ahead);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
        __syncwarp();
        int64_t here = where[0];
#pragma unroll
        for (int k = 1; k < STAGES; ++k)
            if (k == stage) here = where[k];
        const uint32_t there = __ballot_sync(0xffffffffu, here >= 0) & 0xffffu;   // keys of this tile that exist
        const uint32_t kt = ring + stage * 2 * C::TILE, vt = kt + C::TILE;
        if (there) {
            float s[2][4];
#pragma unroll
            for (int t = 0; t < 2; ++t) s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.f;
#pragma unroll
            for (int k = 0; k < D / 16; k += 2) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    // keys 8 t .. 8 t + 7 by 32 columns
                    uint32_t b[4];
                    const int r = 8 * t + (lane & 7), ch = 2 * k + lane / 8;
                    ldmatrix4(kt + r * (D * 2) + ((ch ^ (r & 7)) << 4), b);
                    mma<T>(s[t], qf[k][0], qf[k][1], b[0], b[1]);
                    mma<T>(s[t], qf[k + 1][0], qf[k + 1][1], b[2], b[3]);
                }
            }
            const int key0 = 2 * (lane & 3), pos0 = at.step * STEP + warp * KEYS;
            float top = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const float2 x = make_float2(s[t][0], s[t][1]), y = CAP == kNoCap ? x : CAP == kCap ? capped.far(x) : capped.any(x);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int key = 8 * t + key0 + e;
                    float v = e ? y.y : y.x;
                    if (BIAS) v = fmaf(-slope, (float)(at.len - 1 - (pos0 + key)), CAP ? v : v * (a.scale * kLog2e));
                    v = (there >> key) & 1u ? v * c : -INFINITY;
                    s[t][e] = v;
                    top = fmaxf(top, v);
                }
            }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            if (__any_sync(0xffffffffu, top > m)) {
                const float raised = fmaxf(m, top), factor = raised == -INFINITY ? 1.f : fast_exp2(m - raised);
                m = raised;
                l *= factor;
#pragma unroll
                for (int k = 0; k < D / 8; ++k) { o[k][0] *= factor; o[k][1] *= factor; }
            }
            const float from = m == -INFINITY ? 0.f : m;
            uint32_t p[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const float p0 = fast_exp2(s[t][0] - from), p1 = fast_exp2(s[t][1] - from);
                l += p0 + p1;
                p[t] = pack2<T>(p0 * kLift<T>, p1 * kLift<T>);
            }
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                // 16 keys by 16 columns
                uint32_t b[4];
                const int r = (lane & 7) + 8 * ((lane >> 3) & 1), ch = 2 * k + (lane >> 4);
                ldmatrix4_trans(vt + r * (D * 2) + ((ch ^ (r & 7)) << 4), b);
                mma<T>(o[2 * k], p[0], p[1], b[0], b[1]);
                mma<T>(o[2 * k + 1], p[0], p[1], b[2], b[3]);
            }
            // the new token's own row goes into the cache, by the first group of queries
            const uint32_t fresh = __ballot_sync(0xffffffffu, here >= 0 && (here & 1)) & 0xffffu;
            if (fresh && at.unit % tiles_of_rows == 0) {
                const int pos = at.len - 1, g = at.unit / tiles_of_rows;
                const int page = a.page_table[(int64_t)at.s * a.max_pages + pos / a.page_size];
                if (page >= 0 && page < a.n_pages) {
                    const int64_t to = page * a.page_stride + ((int64_t)(pos % a.page_size) * a.kv_heads + g) * a.dim;
                    const int64_t of = ((int64_t)at.s * a.kv_heads + g) * a.dim;
                    for (int k = 8 * lane; k < 2 * a.dim; k += 256) {
                        const bool v = k >= a.dim;
                        const int e = v ? k - a.dim : k;
                        *reinterpret_cast<uint4*>(static_cast<T*>(v ? P.v_cache : P.k_cache) + to + e) =
                            *reinterpret_cast<const uint4*>(static_cast<const T*>(v ? P.v_new : P.k_new) + of + e);
                    }
                } else if (lane == 0) {
                    atomicOr(a.status, (int)SAMA_DEV_BAD_INDEX);
                }
            }
        }
        __syncwarp();   // all lanes are done with this stage

        const bool unit_ends = at.step + 1 == at.steps;
        if (!unit_ends && i + 1 < n) { advance(at); continue; }

        // The four warps' sums of this unit, and, where it is shared, the other CTAs'.
        fresh_unit = true;
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        {
            float* row = sums + (warp * ROWS + lane / 4) * LD;
#pragma unroll
            for (int k = 0; k < D / 8; ++k)
                *reinterpret_cast<float2*>(row + 8 * k + 2 * (lane & 3)) = make_float2(o[k][0], o[k][1]);
            if ((lane & 3) == 0) *reinterpret_cast<float2*>(row + D) = make_float2(m, l);
        }
        __syncthreads();
        const int g = at.unit / tiles_of_rows, row0 = (at.unit - g * tiles_of_rows) * ROWS, rows = min(ROWS, a.group - row0);
        const bool shared = !unit_ends || first_step > 0;
        float* part = P.parts + (int64_t)(2 * cta + (first_step > 0 ? 0 : 1)) * ROWS * LD;
        T* out = static_cast<T*>(P.out) + ((int64_t)at.s * a.heads + g * a.group + row0) * a.dim;
        auto finish = [&](int r, int col, float x, float y, float w) {
            const float inv = 1.f / (w * kLift<T>);
            if (col < a.dim)
                *reinterpret_cast<uint32_t*>(out + (int64_t)r * a.dim + col) = w == 0.f ? 0u : pack2<T>(x * inv, y * inv);
        };
        for (int e = threadIdx.x; e < rows * (D / 2); e += THREADS) {
            const int r = e / (D / 2), col = 2 * (e - r * (D / 2));
            float top = -INFINITY;
#pragma unroll
            for (int p = 0; p < WARPS; ++p) top = fmaxf(top, sums[(p * ROWS + r) * LD + D]);
            const float from = top == -INFINITY ? 0.f : top;
            float x = 0.f, y = 0.f, w = 0.f;
#pragma unroll
            for (int p = 0; p < WARPS; ++p) {
                const float* row = sums + (p * ROWS + r) * LD;
                const float f = row[D] == -INFINITY ? 0.f : fast_exp2(row[D] - from);
                x += row[col] * f;
                y += row[col + 1] * f;
                w += row[D + 1] * f;
            }
            if (!shared) {
                finish(r, col, x, y, w);
            } else {
                __stcg(reinterpret_cast<float2*>(part + r * LD + col), make_float2(x, y));
                if (col == 0) __stcg(reinterpret_cast<float2*>(part + r * LD + D), make_float2(top, w));
            }
        }
        if (shared) {
            // the CTAs that hold this unit's first and last steps
            const int64_t unit0 = begin + i - at.step, unit1 = unit0 + at.steps - 1;
            auto holder = [&](int64_t step) {
                int h = min((int)((double)step * ctas / (double)total), ctas - 1);
                while (first_of(h) > step) --h;
                while (first_of(h + 1) <= step) ++h;
                return h;
            };
            const int h0 = holder(unit0), h1 = holder(unit1);
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) {
                last_to_arrive = atomicAdd(P.arrived + h0, 1) == h1 - h0;
                if (last_to_arrive) P.arrived[h0] = 0;
            }
            __syncthreads();
            if (last_to_arrive) {
                __threadfence();
                // Each part's factor, by the threads of a row together; then four columns per thread, several parts in flight.
                const int parts = h1 - h0 + 1;
                auto row_of = [&](int p, int r) { return P.parts + ((int64_t)(2 * (h0 + p) + (p == 0 ? 1 : 0)) * ROWS + r) * LD; };
                constexpr int SHARE = THREADS / ROWS;
                const int r0 = threadIdx.x / SHARE, q0 = threadIdx.x % SHARE;
                float top = -INFINITY, weight = 0.f;
                if (r0 < rows) {
#pragma unroll 4
                    for (int p = q0; p < parts; p += SHARE) top = fmaxf(top, __ldcg(row_of(p, r0) + D));
                }
#pragma unroll
                for (int x = 1; x < SHARE; x *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                const float from = top == -INFINITY ? 0.f : top;
                if (r0 < rows) {
#pragma unroll 4
                    for (int p = q0; p < parts; p += SHARE) {
                        // (sums of nothing are 0; a maximum that is not finite makes them NaN, as it should)
                        const float2 ml = __ldcg(reinterpret_cast<const float2*>(row_of(p, r0) + D));
                        const float f = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - from);
                        sums[p * ROWS + r0] = f;
                        weight += ml.y * f;
                    }
                }
#pragma unroll
                for (int x = 1; x < SHARE; x *= 2) weight += __shfl_xor_sync(0xffffffffu, weight, x);
                if (q0 == 0) row_weight[r0] = weight;
                __syncthreads();
                for (int e = threadIdx.x; e < rows * (D / 4); e += THREADS) {
                    const int r = e / (D / 4), col = 4 * (e - r * (D / 4));
                    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
                    for (int p = 0; p < parts; ++p) {
                        const float4 v = __ldcg(reinterpret_cast<const float4*>(row_of(p, r) + col));
                        const float f = sums[p * ROWS + r];
                        x.x += v.x * f;
                        x.y += v.y * f;
                        x.z += v.z * f;
                        x.w += v.w * f;
                    }
                    finish(r, col, x.x, x.y, row_weight[r]);
                    finish(r, col + 2, x.z, x.w, row_weight[r]);
                }
            }
        }
        __syncthreads();   // the sums may be written again
        advance(at);
    }
}

// Two CTAs per SM.
int most_ctas(const sama_ctx* ctx) { return 2 * ctx->sm_count; }

template <typename T, int D, AttnCap CAP, bool BIAS>
cudaError_t launch(sama_ctx* ctx, const PagedParams& P, int ctas, cudaStream_t st) {
    auto* kernel = paged_kernel<T, D, CAP, BIAS>;
    // the ring, and what is the larger of the warps' sums and the factors of all parts
    using C = PagedTile<D>;
    const int sums = WARPS * ROWS * C::LD * 4, factors = most_ctas(ctx) * ROWS * 4, smem = WARPS * C::RING + (sums > factors ? sums : factors);
    const uint32_t bit = 1u << ((std::is_same<T, __half>::value ? 16 : 0) + (D == 64 ? 8 : 0) + 2 * CAP + (BIAS ? 1 : 0));
    if (!(ctx->paged_ready & bit)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        ctx->paged_ready |= bit;
    }
    KernelScope scope(ctx, SAMA_K_PAGED, -1, st);
    return launch_dependent(kernel, dim3((unsigned)ctas), dim3(THREADS), (size_t)smem, st, P);
}
template <typename T, int D>
cudaError_t launch(sama_ctx* ctx, const PagedParams& P, int ctas, cudaStream_t st) {
    switch (attn_cap(P.a.cap)) {
        case kNoCap: return P.a.slopes ? launch<T, D, kNoCap, true>(ctx, P, ctas, st) : launch<T, D, kNoCap, false>(ctx, P, ctas, st);
        case kCap: return P.a.slopes ? launch<T, D, kCap, true>(ctx, P, ctas, st) : launch<T, D, kCap, false>(ctx, P, ctas, st);
        default: return P.a.slopes ? launch<T, D, kWideCap, true>(ctx, P, ctas, st) : launch<T, D, kWideCap, false>(ctx, P, ctas, st);
    }
}


}  // namespace

size_t paged_workspace(const sama_ctx* ctx) { return sizeof(float) * 2 * most_ctas(ctx) * ROWS * PagedTile<128>::LD; }

cudaError_t launch_paged(sama_ctx* ctx, const PagedShape& a, int dtype, const void* q, const void* k_new, const void* v_new,
                         void* k_cache, void* v_cache, void* out, void* ws, cudaStream_t st) {
    if (!ctx->paged_arrived) {
        const size_t bytes = sizeof(int) * most_ctas(ctx);
        cudaError_t e = cudaMalloc(&ctx->paged_arrived, bytes);
        if (e == cudaSuccess) e = cudaMemset(ctx->paged_arrived, 0, bytes);
        if (e == cudaSuccess) e = cudaDeviceSynchronize();
        if (e != cudaSuccess) {
            cudaFree(ctx->paged_arrived);
            ctx->paged_arrived = nullptr;
            return e;
        }
    }
    PagedParams P;
    P.a = a;
    P.q = q;
    P.k_new = k_new;
    P.v_new = v_new;
    P.k_cache = k_cache;
    P.v_cache = v_cache;
    P.out = out;
    P.parts = static_cast<float*>(ws);
    P.arrived = ctx->paged_arrived;
    // no more CTAs than there can be shares
    const int64_t steps = (int64_t)paged_steps((int)paged_most_keys(a.max_pages, a.page_size)) * a.n_seqs * a.kv_heads * ((a.group + ROWS - 1) / ROWS);
    const int64_t shares = steps / kMinSteps > 1 ? steps / kMinSteps : 1;
    const int ctas = shares < most_ctas(ctx) ? (int)shares : most_ctas(ctx);
    if (dtype == SAMA_BF16)
        return a.dim <= 64 ? launch<__nv_bfloat16, 64>(ctx, P, ctas, st) : launch<__nv_bfloat16, 128>(ctx, P, ctas, st);
    return a.dim <= 64 ? launch<__half, 64>(ctx, P, ctas, st) : launch<__half, 128>(ctx, P, ctas, st);
}

}  // namespace sama
