// Token embedding with scaling, and its gradient by sorted tokens.
//
//   out[t, :] = s E[id_t, :]            dE[v, :] (+)= s sum over {t : id_t = v} of dOut[t, :]
//
// Both are bound by memory traffic.  The gradient is a sum over a set of tokens that only the data knows, so the
// tokens are sorted by id first (stable: equal ids keep token order), after which every row of dE is the sum of a
// contiguous run of the sorted list.  The list, not the vocabulary, is then dealt out in equal pieces, so a token that
// makes up most of a text costs no more than any other; and a run is always added up in token order, piece by piece,
// so the result does not depend on scheduling (there is no floating-point atomic).
//
// Two launches:
//   embed_sort   : one cluster of 16 CTAs sorts (id, position) by digits of up to 10 bits, least significant first.
//                  Counts are exchanged through distributed shared memory, so the passes need only cluster barriers.
//                  Ids outside the vocabulary and the skipped id become the key `vocab`, which sorts behind all others.
//                  Meanwhile the other CTAs write zeros to the rows of dE that have no token: each takes a range of
//                  rows and finds out by reading all ids.  They stop when the list is sorted.
//   embed_reduce : a warp adds up one piece of the list for 32 threads' columns.  A run that lies inside a piece is
//                  written out; the parts of a run that crosses pieces go to the workspace in fp32, and the warps that
//                  finish last add them up, in the order of the list.  The first blocks write the zeros still missing.
// Up to 2048 tokens, where launches and round trips are what counts, one launch: every CTA sorts all tokens for itself in
// shared memory, then takes its share of the pieces and of the rows to be zeroed (lookup and gradient, 8191 rows of 256
// fp32 values: 2048 tokens 20 us, 2049 tokens, the other way, 25).  The limit is what a CTA's lists and a thread's four
// entries hold; the two ways take the same time somewhere above it, where was not looked for.
//
// Measured, gradient alone: 16,384 tokens, 50,021 rows of 1024 (bf16 in, fp32 out, 239 MB) 60 us; 131,007 tokens, 65,536
// rows of 2048 bf16 values (805 MB) 215 us, 3.8 TB/s.  The sort takes 20 to 33 us of it, its length in cluster barriers.
// The reduction keeps eight rows per thread on their way in registers: 80 of them, three blocks per SM, a third of the warp
// slots in use (32 %), and 60 to 250 bytes spilled where a thread has more than one value of a row.
// The lookup moves 5.4 and 6.8 TB/s at these sizes.
#include <type_traits>

#include "num_types.h"
#include "sama_internal.h"

namespace sama {

namespace {

// ------------------------------------------------------------------ forward

constexpr int kEmbedThreads = 256;

// A thread's columns of a row: CH chunks of PW consecutive ones, `apart` columns from chunk to chunk, so that neighbouring
// threads are on neighbouring chunks.  Rows of whole aligned 16-byte groups take one such group; others go in chunks of
// what their alignment allows, four at a time.  Against one value at a time (us, lookup / gradient): 24,596 tokens, 638
// rows of 2394 fp16 values in pairs 38 / 59 (53 / 163), of 2395 in single values 60 / 76 (53 / 163), of 2394 fp32 values
// 57 / 77 (70 / 164); 131,072 tokens, rows of 33 bf16 values 12 / 59 (21 / 63).  Up to 32 columns the further chunks would
// all lie beyond the row.  (The lookup of wide odd 16-bit rows is the one that lost, 53 to 60; the boundary is no simple one:
// 65,536 rows of 101, 401, 641, 1031 and 2395 bf16 values 12.7, 46.5, 58.6, 89, 152 us in four, 19.7, 37.3, 68.2, 81, 133 in one.)
template <int PW, int CH>
struct Columns {
    int first, apart, d;
    __device__ __forceinline__ int at(int q) const { return first + q * apart; }
    __device__ __forceinline__ bool on(int q) const { return at(q) < d; }
};
template <typename T, int PW>
__device__ __forceinline__ void put_chunk(T* p, const float* v) {
    if constexpr (PW == 2 && sizeof(T) == 4) __stcs(reinterpret_cast<float2*>(p), make_float2(v[0], v[1]));
    else if constexpr (PW == 2) __stcs(reinterpret_cast<uint32_t*>(p), pack2<T>(v[0], v[1]));
    else store_n<T, PW, true>(p, v);
}
template <typename T, int PW>
__device__ __forceinline__ void get_chunk(const T* p, float* v) {
    if constexpr (PW == 2 && sizeof(T) == 4) {
        const float2 x = *reinterpret_cast<const float2*>(p);
        v[0] = x.x; v[1] = x.y;
    } else if constexpr (PW == 2) {
        const float2 x = unpack2<T>(*reinterpret_cast<const uint32_t*>(p));
        v[0] = x.x; v[1] = x.y;
    } else {
        load_n<T, PW, true>(p, v);
    }
}

// `tpr` threads (a power of two) share a row, a thread takes ROWS of them at a time.
template <typename T, int PW, int CH, int ROWS>
__global__ void __launch_bounds__(kEmbedThreads)
embed_kernel(int64_t n_tokens, int64_t vocab, int d, int tpr, const T* table,
             const int32_t* ids, float scale, T* __restrict__ out, int32_t* status) {
    pdl_trigger();
    pdl_wait();
    const int rows = kEmbedThreads / tpr, tx = threadIdx.x & (tpr - 1);
    const int64_t t0 = (int64_t)blockIdx.x * rows * ROWS + threadIdx.x / tpr;
    int32_t id[ROWS];
    bool good[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int64_t t = t0 + (int64_t)r * rows;
        id[r] = t < n_tokens ? ids[t] : 0;
        good[r] = id[r] >= 0 && id[r] < vocab;
        if (!good[r] && tx == 0) atomicOr(status, (int)SAMA_DEV_BAD_INDEX);
    }
    for (Columns<PW, CH> c{tx * PW, tpr * PW, d}; c.first < d; c.first += tpr * PW * CH) {
        float v[ROWS][CH][PW];
#pragma unroll
        for (int r = 0; r < ROWS; ++r)  // (rows of frequent tokens are read again and again)
#pragma unroll
            for (int q = 0; q < CH; ++q)
                if (CH == 1 || c.on(q)) get_chunk<T, PW>(table + (good[r] ? (int64_t)id[r] : 0) * d + c.at(q), v[r][q]);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int64_t t = t0 + (int64_t)r * rows;
            if (t >= n_tokens) continue;
#pragma unroll
            for (int q = 0; q < CH; ++q) {
                if (CH > 1 && !c.on(q)) continue;
#pragma unroll
                for (int i = 0; i < PW; ++i) v[r][q][i] = good[r] ? v[r][q][i] * scale : 0.f;
                put_chunk<T, PW>(out + t * d + c.at(q), v[r][q]);  // (not to push the table out of L2)
            }
        }
    }
}

// ------------------------------------------------------------------ sort

constexpr int kSortCtas = 16, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kMaxBits = 10, kMaxBins = 1 << kMaxBits;
constexpr int kStage = 8192;        // elements of one CTA that fit its staging area
// One cluster of 16 fits into each of the 8 groups of SMs: one sorts, the others zero.
constexpr int kFillCtas = 7 * kSortCtas;

struct SortSmem {
    uint32_t hist[kSortWarps][kMaxBins];  // counts, then next output positions, of every warp's share
    uint32_t total[kMaxBins];             // this CTA's counts (read by the other CTAs)
    uint32_t warp_sum[2][kSortWarps];
    uint32_t shift_to[kMaxBins];          // from a place in `stage` to the place in the list, by digit
    int2 stage[kStage];                   // this CTA's elements in the order of their digit
};
static_assert(sizeof(SortSmem) <= 227 * 1024, "one CTA per SM");

// Zeroing of absent rows: kFillCtas shares of the rows, in each share warp w of 32 takes rows w, w + 32, ...
struct FillArgs {
    uint8_t* grad;          // null: nothing is zeroed
    int64_t row_bytes;
    int64_t share;          // rows per share, a multiple of 32
    uint32_t* present;      // one bit per row
    int* progress;          // [kFillCtas][32]: rows of the share's warp that are done
    int32_t vocab;
};
__device__ __forceinline__ bool zero_row_if_absent(const FillArgs& f, int64_t row, uint32_t present_word, int lane) {
    if (present_word >> (row & 31) & 1u) return false;
    uint8_t* g = f.grad + row * f.row_bytes;
    const int64_t low = f.row_bytes | (int64_t)reinterpret_cast<uintptr_t>(f.grad);   // alignment of every row
    if ((low & 15) == 0) {
        for (int64_t b = lane * 16; b < f.row_bytes; b += 512) *reinterpret_cast<uint4*>(g + b) = make_uint4(0, 0, 0, 0);
    } else if ((low & 3) == 0) {
        for (int64_t b = lane * 4; b < f.row_bytes; b += 128) *reinterpret_cast<uint32_t*>(g + b) = 0;
    } else {
        for (int64_t b = lane * 2; b < f.row_bytes; b += 64) *reinterpret_cast<uint16_t*>(g + b) = 0;
    }
    return true;
}

__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t ld_cluster_u32(const uint32_t* p, uint32_t cta) {
    uint32_t a, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(cta));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}

// The place of this lane's element among those of its digit: the warp's next places (`next`, by digit) are handed out in
// the order of the lanes.  Lanes of one digit find each other with one vote per bit (the instruction that matches whole
// values takes a step per distinct value, 200 cycles for a warp of different digits).
template <int MOST>
__device__ __forceinline__ uint32_t take_place(uint32_t* next, bool on, uint32_t digit, int bits, int lane) {
    uint32_t same = __ballot_sync(0xffffffffu, on);
#pragma unroll
    for (int b = 0; b < MOST; ++b) {
        if (b >= bits) break;
        const bool set = (digit & (1u << b)) != 0;
        same &= __ballot_sync(0xffffffffu, set) ^ (set ? 0u : 0xffffffffu);
    }
    uint32_t at = 0;
    if (on) at = next[digit] + __popc(same & ((1u << lane) - 1u));
    __syncwarp();
    if (on && lane == __ffs(same) - 1) next[digit] += __popc(same);
    __syncwarp();
    return at;
}

struct SortArgs {
    const int32_t* ids;
    int2* buf[2];       // lists of (key, position); pass p writes buf[p & 1]
    int2* span;         // [vocab]: begin and end of each present row's run in the sorted list
    int* arrived;       // [counters]: zeroed for embed_reduce
    FillArgs fill;
    int* done;          // set to `epoch` once the list is sorted
    int epoch;
    int n, counters, passes, bits;
    int32_t vocab, skip_id;
    int32_t* status;
};

// Finds the rows of this CTA's share that have a token, and zeroes the others until the list is sorted.
__device__ void fill_absent_rows(const SortArgs& a, uint8_t* smem, int cta) {
    uint32_t* present = reinterpret_cast<uint32_t*>(smem);
    constexpr int kTrack = 1 << 20;   // rows whose presence fits shared memory
    const FillArgs& f = a.fill;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t first = cta * f.share, stop = min((int64_t)f.vocab, first + f.share);
    for (int64_t r0 = first; r0 < stop; r0 += kTrack) {
        const int rows = (int)min((int64_t)kTrack, stop - r0);
        for (int i = threadIdx.x; i < (rows + 31) / 32; i += kSortThreads) present[i] = 0;
        __syncthreads();
        auto mark = [&](int32_t id) {
            const int64_t r = (int64_t)id - r0;
            if (r < 0 || r >= rows || id == a.skip_id) return;
            uint32_t* w = present + (r >> 5);
            const uint32_t bit = 1u << (r & 31);
            if (!(*w & bit)) atomicOr(w, bit);
        };
        // 16 ids per thread at a time where their address allows, the rest one by one
        const bool quads = (reinterpret_cast<uintptr_t>(a.ids) & 15u) == 0;
        const int n4 = quads ? a.n / 4 : 0;
        for (int i = threadIdx.x; i < n4; i += 4 * kSortThreads) {
            int4 id[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                id[u] = i + u * kSortThreads < n4 ? reinterpret_cast<const int4*>(a.ids)[i + u * kSortThreads] : make_int4(-1, -1, -1, -1);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                mark(id[u].x);
                mark(id[u].y);
                mark(id[u].z);
                mark(id[u].w);
            }
        }
#pragma unroll 4
        for (int i = 4 * n4 + threadIdx.x; i < a.n; i += kSortThreads) mark(a.ids[i]);
        __syncthreads();
        for (int i = threadIdx.x; i < (rows + 31) / 32; i += kSortThreads) f.present[r0 / 32 + i] = present[i];
        __syncthreads();
    }
    int64_t j = 0;
    if (stop - first <= kTrack) {
        // (a warp looks at the flag before every row; what it leaves, embed_reduce does)
        for (; first + j * 32 + warp < stop; ++j) {
            int seen = 0;
            if (lane == 0) seen = *reinterpret_cast<volatile int*>(a.done);
            if (__shfl_sync(0xffffffffu, seen, 0) == a.epoch) break;
            zero_row_if_absent(f, first + j * 32 + warp, present[j], lane);
        }
    }
    if (lane == 0) f.progress[cta * 32 + warp] = (int)j;
}

// Launched in clusters of kSortCtas.
__global__ void __launch_bounds__(kSortThreads)
embed_sort_kernel(const __grid_constant__ SortArgs a) {
    extern __shared__ uint8_t sort_raw[];
    SortSmem& sm = *reinterpret_cast<SortSmem*>(sort_raw);
    pdl_trigger();
    pdl_wait();
    if (blockIdx.x >= kSortCtas) {
        fill_absent_rows(a, sort_raw, blockIdx.x - kSortCtas);
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x;
    const int n = a.n, bins = 1 << a.bits;
    const int per_cta = ((n + kSortCtas - 1) / kSortCtas + 31) & ~31;
    const int per_warp = ((per_cta + kSortWarps - 1) / kSortWarps + 31) & ~31;
    // (n <= 2^30, so that the rounded shares stay below 2^31)
    const int cta_end = min(n, (int)(rank + 1) * per_cta);
    const int begin = (int)rank * per_cta + warp * per_warp;
    const int end = min(cta_end, begin + per_warp);
    constexpr int U = 8;  // elements in flight per thread
    // Up to 32 U elements per warp stay in registers between the two sweeps of a pass, and go through shared memory in
    // the order of their digit, so that they reach the list in runs rather than one sector each.
    const bool once = per_warp <= 32 * U;
    static_assert(kSortWarps * 32 * U <= kStage, "such a CTA's elements fit the stage");
    for (int i = (int)rank * kSortThreads + threadIdx.x; i < a.counters; i += kSortCtas * kSortThreads) a.arrived[i] = 0;
    for (int p = 0; p < a.passes; ++p) {
        const int2* src = a.buf[(p & 1) ^ 1];
        int2* dst = a.buf[p & 1];
        const int shift = a.bits * p;
        auto fetch = [&](int i) -> int2 {
            if (i >= end) return make_int2(-1, 0);   // (beyond this warp's share)
            if (p > 0) return __ldcg(src + i);
            const int32_t id = a.ids[i];
            const bool good = id >= 0 && id < a.vocab;
            if (!good) atomicOr(a.status, (int)SAMA_DEV_BAD_INDEX);
            return make_int2(good && id != a.skip_id ? id : a.vocab, i);
        };
        for (int b = lane; b < bins; b += 32) sm.hist[warp][b] = 0;
        __syncwarp();
        int2 e[U];
        for (int i = begin + lane; i - lane < end; i += 32 * U) {
#pragma unroll
            for (int u = 0; u < U; ++u) e[u] = fetch(i + 32 * u);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (e[u].x >= 0) atomicAdd(&sm.hist[warp][((uint32_t)e[u].x >> shift) & (bins - 1)], 1u);
        }
        __syncthreads();
        // thread b owns bin b
        uint32_t mine = 0;
        if (threadIdx.x < bins) {
            uint32_t c[kSortWarps];
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) c[w] = sm.hist[w][threadIdx.x];
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) {
                sm.hist[w][threadIdx.x] = mine;
                mine += c[w];
            }
            sm.total[threadIdx.x] = mine;
        }
        cluster_barrier();
        uint32_t before = 0, all = 0;
        if (threadIdx.x < bins) {
            uint32_t v[kSortCtas];
#pragma unroll
            for (uint32_t c = 0; c < kSortCtas; ++c) v[c] = ld_cluster_u32(&sm.total[threadIdx.x], c);
#pragma unroll
            for (uint32_t c = 0; c < kSortCtas; ++c) {
                if (c < rank) before += v[c];
                all += v[c];
            }
        }
        uint32_t incl = all, local = mine;   // inclusive sums over the bins: of the whole list, of this CTA's elements
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o), x = __shfl_up_sync(0xffffffffu, local, o);
            if (lane >= o) { incl += v; local += x; }
        }
        if (lane == 31) { sm.warp_sum[0][warp] = incl; sm.warp_sum[1][warp] = local; }
        __syncthreads();
        // the sums of the warps before this one
        const uint32_t past = __reduce_add_sync(0xffffffffu, lane < warp ? sm.warp_sum[0][lane] : 0u);
        const uint32_t past_here = __reduce_add_sync(0xffffffffu, lane < warp ? sm.warp_sum[1][lane] : 0u);
        if (threadIdx.x < bins) {
            const uint32_t base = past + incl - all + before, here = past_here + local - mine;
            sm.shift_to[threadIdx.x] = base - here;
            const uint32_t add = once ? here : base;
            uint32_t c[kSortWarps];
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) c[w] = sm.hist[w][threadIdx.x];
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) sm.hist[w][threadIdx.x] = c[w] + add;
        }
        __syncthreads();
        for (int i = begin + lane; i - lane < end; i += 32 * U) {
            if (!once) {
#pragma unroll
                for (int u = 0; u < U; ++u) e[u] = fetch(i + 32 * u);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i - lane + 32 * u >= end) break;
                const bool on = e[u].x >= 0;
                const uint32_t digit = on ? ((uint32_t)e[u].x >> shift) & (bins - 1) : 0u;
                const uint32_t at = take_place<kMaxBits>(sm.hist[warp], on, digit, a.bits, lane);
                if (!on) continue;
                if (once) sm.stage[at] = e[u]; else dst[at] = e[u];
            }
        }
        if (once) {
            __syncthreads();
            const int held = max(0, cta_end - (int)rank * per_cta);
#pragma unroll 4
            for (int i = threadIdx.x; i < held; i += kSortThreads) {
                const int2 v = sm.stage[i];
                dst[sm.shift_to[((uint32_t)v.x >> shift) & (bins - 1)] + i] = v;
            }
        }
        cluster_barrier();  // the pass is complete: every CTA may read all of dst, and total may be rewritten
    }
    if (rank == 0 && threadIdx.x == 0) *reinterpret_cast<volatile int*>(a.done) = a.epoch;
    const int2* list = a.buf[(a.passes - 1) & 1];
    for (int i = begin + lane; i - lane < end; i += 32 * U) {
        int32_t key[U], edge[U];   // edge: the neighbour beyond the warp's 32 entries, for the first and the last lane
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = i + 32 * u, k = lane == 0 ? j - 1 : j + 1;
            key[u] = j < n ? __ldcg(list + j).x : a.vocab;
            edge[u] = (lane == 0 || lane == 31) && k >= 0 && k < n ? __ldcg(list + k).x : -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = i + 32 * u;
            int32_t prev = __shfl_up_sync(0xffffffffu, key[u], 1), next = __shfl_down_sync(0xffffffffu, key[u], 1);
            if (lane == 0) prev = edge[u];
            if (lane == 31) next = edge[u];
            if (j >= end || key[u] >= a.vocab) continue;
            if (prev != key[u]) a.span[key[u]].x = j;
            if (next != key[u]) a.span[key[u]].y = j + 1;
        }
    }
}

// ------------------------------------------------------------------ reduction

constexpr int kJoin = 32;     // pieces per group of the join

struct ReduceArgs {
    const int2* list;         // sorted (id, position)
    const int2* span;         // each present row's run
    const void* dout;
    void* grad;
    float* head;              // [pieces][d]: the part, in this piece, of a run that began in an earlier one
    float* tail;              // [pieces][d]: the first part of a run that goes on in the next piece
    int* arrived;             // counters of stored parts: [pieces][slabs] twice, then [groups][slabs]
    int n, vocab, d;
    int piece, pieces, slabs;
    FillArgs fill;
    int fill_blocks;          // the first blocks zero what embed_sort left
    int accumulate;
    float scale;
};

template <typename TG, int PW, int CH>
__device__ __forceinline__ void put_row(const ReduceArgs& a, int row, const Columns<PW, CH>& c, const float* acc) {
#pragma unroll
    for (int q = 0; q < CH; ++q) {
        if (!c.on(q)) continue;
        TG* g = static_cast<TG*>(a.grad) + (int64_t)row * a.d + c.at(q);
        float v[PW];
#pragma unroll
        for (int i = 0; i < PW; ++i) v[i] = acc[q * PW + i] * a.scale;
        if (a.accumulate) {
            float old[PW];
            if constexpr (PW <= 2) get_chunk<TG, PW>(g, old); else load_n<TG, PW>(g, old);
#pragma unroll
            for (int i = 0; i < PW; ++i) v[i] += old[i];
        }
        if constexpr (PW <= 2) put_chunk<TG, PW>(g, v); else store_n<TG, PW>(g, v);
    }
}
template <int PW, int CH>
__device__ __forceinline__ void put_part(float* part, const Columns<PW, CH>& c, const float* acc) {
#pragma unroll
    for (int q = 0; q < CH; ++q) {
        if (!c.on(q)) continue;
        if constexpr (PW == 2) *reinterpret_cast<float2*>(part + c.at(q)) = make_float2(acc[2 * q], acc[2 * q + 1]);
        else store_n<float, PW>(part + c.at(q), acc + q * PW);
    }
}

// A thread's values of one row as they lie in memory.
template <typename T, int PW, int CH> struct Raw {
    using Chunk = std::conditional_t<PW == 1, T, std::conditional_t<PW * sizeof(T) == 4, uint32_t, std::conditional_t<PW * sizeof(T) == 8, uint2, uint4>>>;
    static_assert(sizeof(Chunk) == PW * sizeof(T), "a chunk is one access");
    Chunk r[CH] = {};
    __device__ __forceinline__ void load(const T* row, const Columns<PW, CH>& c) {
#pragma unroll
        for (int q = 0; q < CH; ++q)
            if (c.on(q)) r[q] = __ldcs(reinterpret_cast<const Chunk*>(row + c.at(q)));
    }
    __device__ __forceinline__ void add_to(float* acc) const {
#pragma unroll
        for (int q = 0; q < CH; ++q) {
            if constexpr (PW == 1) {
                acc[q] += to_float(r[q]);
            } else if constexpr (PW == 2) {
                const float2 f = unpack2<T>(r[q]);
                acc[2 * q] += f.x;
                acc[2 * q + 1] += f.y;
            } else if constexpr (sizeof(Chunk) == 8) {
                const float2 f = unpack2<T>(r[q].x), g = unpack2<T>(r[q].y);
                acc[4 * q] += f.x;
                acc[4 * q + 1] += f.y;
                acc[4 * q + 2] += g.x;
                acc[4 * q + 3] += g.y;
            } else {
                const uint32_t w[4] = {r[q].x, r[q].y, r[q].z, r[q].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (sizeof(T) == 4) {
                        acc[j] += __uint_as_float(w[j]);
                    } else {
                        const float2 f = unpack2<T>(w[j]);
                        acc[2 * j] += f.x;
                        acc[2 * j + 1] += f.y;
                    }
                }
            }
        }
    }
};

// A thread's fp32 values that another warp of this launch has stored.
template <int PW, int CH>
__device__ __forceinline__ void load_part(const float* part, const Columns<PW, CH>& c, float* v) {
#pragma unroll
    for (int q = 0; q < CH; ++q) {
        const float* p = part + (c.on(q) ? c.at(q) : 0);
        if constexpr (PW == 1) {
            v[q] = __ldcg(p);
        } else if constexpr (PW == 2) {
            const float2 x = __ldcg(reinterpret_cast<const float2*>(p));
            v[2 * q] = x.x; v[2 * q + 1] = x.y;
        } else {
#pragma unroll
            for (int i = 0; i < PW / 4; ++i) {
                const float4 x = __ldcg(reinterpret_cast<const float4*>(p) + i);
                float* o = v + q * PW + 4 * i;
                o[0] = x.x; o[1] = x.y; o[2] = x.z; o[3] = x.w;
            }
        }
    }
}

// Adds the parts at base + first + step j, j = 0 .. count - 1, to sum, in this order.
template <int PW, int CH>
__device__ __forceinline__ void add_parts(const float* base, int64_t first, int64_t step, int count,
                                          const Columns<PW, CH>& c, float* sum) {
    constexpr int VE = PW * CH, U = VE == 8 ? 4 : 8;  // (more would set the whole kernel's register count)
    for (int j = 0; j < count; j += U) {
        float v[U][VE];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (j + u < count) load_part(base + first + (j + u) * step, c, v[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (j + u < count)
#pragma unroll
                for (int q = 0; q < VE; ++q) sum[q] += v[u][q];
    }
}

// Whether this warp is the last of `parts` to get here with its part stored.
__device__ __forceinline__ bool last_to_arrive(int* counter, int parts, int lane) {
    __threadfence();
    __syncwarp();
    int before = 0;
    if (lane == 0) before = atomicAdd(counter, 1);
    before = __shfl_sync(0xffffffffu, before, 0);
    if (before != parts - 1) return false;
    if (lane == 0) *counter = 0;   // (embed_few's counters stay between calls)
    __threadfence();
    return true;
}

// The sorted list in global memory, with the rows' runs beside it, or in shared memory, where a run is quickly found.
struct GlobalList {
    const int2* list;
    const int2* span;
    __device__ __forceinline__ int2 at(int i) const { return list[i]; }
    __device__ __forceinline__ int2 run(int key) const { return span[key]; }
};
struct SharedList {
    const int2* list;
    int n;
    __device__ __forceinline__ int2 at(int i) const { return list[i]; }
    __device__ __forceinline__ int first_not_below(int key) const {
        int lo = 0, hi = n;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (list[mid].x < key) lo = mid + 1; else hi = mid;
        }
        return lo;
    }
    __device__ __forceinline__ int2 run(int key) const { return make_int2(first_not_below(key), first_not_below(key + 1)); }
};

// This warp has stored its part, in piece k, of a run over pieces k0 .. k1.  The parts are joined in groups of kJoin
// pieces, then the groups: the last to store a part adds up its group, the last to store a group's sum (in the place of
// its first part) adds up the groups.
template <typename TG, int PW, int CH, typename List>
__device__ __forceinline__ void join_run(const ReduceArgs& a, const List& list, const Columns<PW, CH>& c, int key, int k, int slab, int lane) {
    const int2 run = list.run(key);
    const int k0 = run.x / a.piece, k1 = (run.y - 1) / a.piece;
    const int g = k / kJoin, g0 = k0 / kJoin, g1 = k1 / kJoin;
    const int first = max(k0, g * kJoin), last = min(k1, g * kJoin + kJoin - 1);
    const int64_t parts = (int64_t)a.pieces * a.slabs;
    // counters: of the group a run begins in, by k0 (at most one such run per piece); of a later group, by the group
    int* in_group = g == g0 ? a.arrived + (int64_t)k0 * a.slabs + slab : a.arrived + 2 * parts + (int64_t)g * a.slabs + slab;
    if (!last_to_arrive(in_group, last - first + 1, lane)) return;
    float sum[PW * CH];
    float* slot = (g == g0 ? a.tail : a.head) + (int64_t)first * a.d;
    load_part(slot, c, sum);
    add_parts(a.head, (int64_t)(first + 1) * a.d, a.d, last - first, c, sum);
    if (g0 != g1) {
        __syncwarp();
        put_part(slot, c, sum);
        if (!last_to_arrive(a.arrived + parts + (int64_t)k0 * a.slabs + slab, g1 - g0 + 1, lane)) return;
        load_part(a.tail + (int64_t)k0 * a.d, c, sum);
        add_parts(a.head, (int64_t)(g0 + 1) * kJoin * a.d, (int64_t)kJoin * a.d, g1 - g0, c, sum);
    }
    put_row<TG>(a, key, c, sum);
}

// One warp: piece k of the list, columns [32 VE slab, 32 VE (slab + 1)), U rows in flight per thread.
template <typename T, typename TG, int PW, int CH, int U, typename List>
__device__ __forceinline__ void reduce_piece(const ReduceArgs& a, const List& list, int k, int slab, int lane) {
    const int i0 = k * a.piece, count = min(a.n - i0, a.piece);
    constexpr int VE = PW * CH;
    // (lanes beyond the last column go along for the warp's sake)
    const Columns<PW, CH> c{slab * 32 * VE + lane * PW, 32 * PW, a.d};
    const T* dout = static_cast<const T*>(a.dout);
    // the piece's entries, two per lane
    const int2 none = make_int2(a.vocab, 0);
    const int2 low = lane < count ? list.at(i0 + lane) : none, high = lane + 32 < count ? list.at(i0 + lane + 32) : none;
    const int before_key = i0 > 0 ? list.at(i0 - 1).x : -1, after_key = i0 + count < a.n ? list.at(i0 + count).x : -1;
    const int first_key = __shfl_sync(0xffffffffu, low.x, 0);
    const bool open_head = before_key == first_key && first_key < a.vocab;
    int key = first_key;
    bool in_head = open_head;   // the current run began in an earlier piece
    float acc[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) acc[j] = 0.f;

    Raw<T, PW, CH> v[U];
    auto entry = [&](int i) {
        const int2 e = i < 32 ? low : high;
        return make_int2(__shfl_sync(0xffffffffu, e.x, i & 31), __shfl_sync(0xffffffffu, e.y, i & 31));
    };
    auto fetch = [&](Raw<T, PW, CH>& r, int i) {
        if (i >= count) return;
        const int2 e = entry(i);
        if (e.x < a.vocab) r.load(dout + (int64_t)e.y * a.d, c);
    };
#pragma unroll
    for (int u = 0; u < U; ++u) fetch(v[u], u);
    for (int b = 0; b < count && key < a.vocab; b += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (b + u >= count) break;
            const int id = entry(b + u).x;
            if (id != key) {
                if (in_head) put_part(a.head + (int64_t)k * a.d, c, acc);
                else put_row<TG>(a, key, c, acc);
                in_head = false;
                key = id;
                if (key >= a.vocab) break;
#pragma unroll
                for (int j = 0; j < VE; ++j) acc[j] = 0.f;
            }
            v[u].add_to(acc);
            fetch(v[u], b + u + U);
        }
    }
    const bool open_tail = key < a.vocab && after_key == key;
    if (key < a.vocab) {
        if (in_head) put_part(a.head + (int64_t)k * a.d, c, acc);
        else if (open_tail) put_part(a.tail + (int64_t)k * a.d, c, acc);
        else put_row<TG>(a, key, c, acc);
    }
    // the run that came in, and the one that goes on where that is another
#pragma unroll 1
    for (int j = 0; j < 2; ++j) {
        const int run = j == 0 ? first_key : key;
        if (j == 0 ? open_head : (open_tail && !in_head)) join_run<TG>(a, list, c, run, k, slab, lane);
    }
}

template <typename T, typename TG, int PW, int CH>
__global__ void __launch_bounds__(kEmbedThreads, 3)
embed_reduce_kernel(const __grid_constant__ ReduceArgs a) {
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    if ((int)blockIdx.x < a.fill_blocks) {
        const FillArgs& f = a.fill;
        for (int w = (int)blockIdx.x * (kEmbedThreads / 32) + (threadIdx.x >> 5); w < kFillCtas * 32; w += a.fill_blocks * (kEmbedThreads / 32)) {
            const int64_t first = (w / 32) * f.share, stop = min((int64_t)f.vocab, first + f.share);
            for (int64_t row = first + (int64_t)f.progress[w] * 32 + w % 32; row < stop; row += 32)
                zero_row_if_absent(f, row, f.present[row / 32], lane);
        }
        return;
    }
    const int64_t unit = (int64_t)(blockIdx.x - a.fill_blocks) * (kEmbedThreads / 32) + (threadIdx.x >> 5);
    const int k = (int)(unit / a.slabs), slab = (int)(unit - (int64_t)k * a.slabs);
    // (single values: twice the rows, for half as many bytes in flight or less)
    if (k < a.pieces) reduce_piece<T, TG, PW, CH, PW * CH == 1 ? 16 : 8>(a, GlobalList{a.list, a.span}, k, slab, lane);
}

// ------------------------------------------------------------------ few tokens

// (512 threads: with 1024 the reduction's 64 registers spill a kilobyte)
constexpr int kFewTokens = 2048, kFewThreads = 512, kFewWarps = kFewThreads / 32, kFewPer = kFewTokens / kFewThreads;
constexpr int kFewBits = 9, kFewBins = 1 << kFewBits, kFewCounters = 1 << 16;
constexpr int kFewShare = 1 << 18;   // rows whose presence a CTA can track
struct FewSmem {
    uint32_t hist[kFewWarps][kFewBins];
    int2 list[2][kFewTokens];
    uint32_t warp_sum[kFewWarps];
    uint32_t present[kFewShare / 32];      // a bit per row of this CTA's share
    int next_row;
};

struct FewArgs {
    const int32_t* ids;
    int passes, bits;
    int32_t skip_id;
    int64_t share;       // rows per CTA, a multiple of 32; 0: nothing is zeroed
    int32_t* status;
};

template <typename T, typename TG, int PW, int CH>
__global__ void __launch_bounds__(kFewThreads, 1)
embed_few_kernel(const __grid_constant__ ReduceArgs a, const __grid_constant__ FewArgs f) {
    extern __shared__ uint8_t few_raw[];
    FewSmem& sm = *reinterpret_cast<FewSmem*>(few_raw);
    static_assert(sizeof(FewSmem) <= 227 * 1024, "");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = a.n, bins = 1 << f.bits;
    pdl_trigger();
    pdl_wait();
    // The sort of embed_sort, on one CTA: a warp has up to kFewPer runs of 32 consecutive elements.
    const int per_warp = ((n + kFewWarps - 1) / kFewWarps + 31) & ~31, begin = warp * per_warp, end = min(n, begin + per_warp);
    int2 e[kFewPer];
#pragma unroll
    for (int u = 0; u < kFewPer; ++u) {
        const int i = begin + 32 * u + lane;
        e[u] = make_int2(-1, 0);
        if (i < end) {
            const int32_t id = f.ids[i];
            const bool good = id >= 0 && id < a.vocab;
            if (!good && blockIdx.x == 0) atomicOr(f.status, (int)SAMA_DEV_BAD_INDEX);
            e[u] = make_int2(good && id != f.skip_id ? id : a.vocab, i);
        }
    }
    // which rows of this CTA's share have a token
    const int64_t first_row = blockIdx.x * f.share;
    const int rows = (int)max((int64_t)0, min((int64_t)a.vocab, first_row + f.share) - first_row);
    for (int i = threadIdx.x; i < (rows + 31) / 32; i += kFewThreads) sm.present[i] = 0;
    if (threadIdx.x == 0) sm.next_row = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kFewPer; ++u) {
        const int64_t r = (int64_t)e[u].x - first_row;
        if (e[u].x >= 0 && r >= 0 && r < rows) atomicOr(sm.present + (r >> 5), 1u << (r & 31));
    }
    for (int p = 0; p < f.passes; ++p) {
        const int shift = f.bits * p;
        for (int b = lane; b < bins; b += 32) sm.hist[warp][b] = 0;
        __syncwarp();
#pragma unroll
        for (int u = 0; u < kFewPer; ++u)
            if (e[u].x >= 0) atomicAdd(&sm.hist[warp][((uint32_t)e[u].x >> shift) & (bins - 1)], 1u);
        __syncthreads();
        uint32_t mine = 0;   // thread b owns bin b
        if (threadIdx.x < bins) {
            uint32_t c[kFewWarps];
#pragma unroll
            for (int w = 0; w < kFewWarps; ++w) c[w] = sm.hist[w][threadIdx.x];
#pragma unroll
            for (int w = 0; w < kFewWarps; ++w) mine += c[w];
        }
        uint32_t incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        if (lane == 31) sm.warp_sum[warp] = incl;
        __syncthreads();
        uint32_t at = __reduce_add_sync(0xffffffffu, lane < warp ? sm.warp_sum[lane] : 0u) + incl - mine;
        if (threadIdx.x < bins) {
#pragma unroll
            for (int w = 0; w < kFewWarps; ++w) {
                const uint32_t c = sm.hist[w][threadIdx.x];
                sm.hist[w][threadIdx.x] = at;
                at += c;
            }
        }
        __syncthreads();
        int2* dst = sm.list[p & 1];
#pragma unroll
        for (int u = 0; u < kFewPer; ++u) {
            if (begin + 32 * u >= end) break;
            const bool on = e[u].x >= 0;
            const uint32_t digit = on ? ((uint32_t)e[u].x >> shift) & (bins - 1) : 0u;
            const uint32_t to = take_place<kFewBits>(sm.hist[warp], on, digit, f.bits, lane);
            if (on) dst[to] = e[u];
        }
        __syncthreads();
        if (p + 1 < f.passes) {
#pragma unroll
            for (int u = 0; u < kFewPer; ++u) {
                const int i = begin + 32 * u + lane;
                if (i < end) e[u] = dst[i];
            }
        }
    }
    const SharedList list{sm.list[(f.passes - 1) & 1], n};
    // this CTA's share of the pieces, neighbouring ones on different CTAs
    const int64_t units = (int64_t)a.pieces * a.slabs;
    for (int64_t unit = (int64_t)warp * gridDim.x + blockIdx.x; unit < units; unit += (int64_t)kFewWarps * gridDim.x) {
        const int k = (int)(unit / a.slabs), slab = (int)(unit - (int64_t)k * a.slabs);
        reduce_piece<T, TG, PW, CH, 4>(a, list, k, slab, lane);
    }
    // zeros to the rows without a token, by the warps that have no piece (any more)
    for (;;) {
        int r0 = 0;
        if (lane == 0) r0 = atomicAdd(&sm.next_row, 4);
        r0 = __shfl_sync(0xffffffffu, r0, 0);
        if (r0 >= rows) break;
        for (int r = r0; r < min(r0 + 4, rows); ++r) zero_row_if_absent(a.fill, first_row + r, sm.present[r >> 5], lane);
    }
}

// Threads (a power of two, at most a block) that share a row of `chunks` vectors: the number that leaves the fewest idle in
// the last round, the larger one of equals.
int threads_per_row(int d, int ve) {
    const int chunks = (d + ve - 1) / ve;
    int best = 1;
    int64_t least = (int64_t)1 << 62;
    for (int t = 1; t <= kEmbedThreads && t < 2 * chunks; t *= 2) {
        const int64_t rounds = (chunks + t - 1) / t;
        // (a round more costs about as much as eight idle threads)
        const int64_t cost = rounds * t + 8 * rounds;
        if (cost <= least) { least = cost; best = t; }
    }
    return best;
}

// How rows of d values are taken apart: the chunks of a thread (see Columns).
enum Access { GROUPS, PAIRS, SINGLES, SINGLE };
Access access_of(int d, int dtype, uintptr_t addresses, bool wide_output) {
    const int es = (int)dtype_size(dtype);
    if (d % (16 / es) == 0 && (addresses & 15u) == 0) return GROUPS;
    if (d <= 32) return SINGLE;
    return es == 2 && d % 2 == 0 && (addresses & (wide_output ? 7u : 3u)) == 0 ? PAIRS : SINGLES;
}
inline int columns_of(Access a, int dtype) { return a == GROUPS ? 16 / (int)dtype_size(dtype) : a == PAIRS ? 8 : a == SINGLES ? 4 : 1; }
// fn<values per chunk, chunks>.  Groups of 16 bytes on both sides, so half a group of 16-bit values where the results are
// fp32: two stores of 16 bytes, each 32 bytes from its neighbour's, would write every sector of L2 twice.
template <typename T, typename TO, typename F>
auto with_access(Access a, F&& fn) {
    using std::integral_constant;
    constexpr int GROUP = 16 / sizeof(TO), GROUPS_OF = 16 / sizeof(T) / GROUP, PAIR = sizeof(T) == 2 ? 2 : 1;   // (fp32 has no pairs: its single values are as wide)
    return a == GROUPS    ? fn(integral_constant<int, GROUP>(), integral_constant<int, GROUPS_OF>())
           : a == PAIRS   ? fn(integral_constant<int, PAIR>(), integral_constant<int, 4>())
           : a == SINGLES ? fn(integral_constant<int, 1>(), integral_constant<int, 4>())
                          : fn(integral_constant<int, 1>(), integral_constant<int, 1>());
}

template <typename T>
cudaError_t embed_typed(sama_ctx* ctx, int dtype, int64_t n, int64_t vocab, int d, const void* table, const int32_t* ids,
                        float scale, void* out, cudaStream_t st) {
    const Access access = access_of(d, dtype, reinterpret_cast<uintptr_t>(table) | reinterpret_cast<uintptr_t>(out), false);
    const int tpr = threads_per_row(d, columns_of(access, dtype)), rows = kEmbedThreads / tpr;
    // Four rows per thread once one row each would be more threads than the SMs take at a time.  One row against four (us, rows
    // of 1024 bf16 values): 2100 tokens 3.0 / 3.5, 4096 4.6 / 4.1, 8192 8.0 / 5.8, 16,384 15.9 / 12.1, 131,072 104 / 70.
    // Rows in four chunks have four loads on their way as it is: not before three times as many (4821 rows of 2796 bf16 values
    // 14.1 / 20.6, 32,768 of 100 5.0 / 6.5).
    const bool chunks = access == PAIRS || access == SINGLES;
    const bool deep = n * tpr >= (int64_t)ctx->sm_count * 2048 * 4 / (chunks ? 1 : 3);
    const int64_t per_block = (int64_t)rows * (deep ? 4 : 1);
    KernelScope scope(ctx, SAMA_K_EMBED, -1, st);
    return with_access<T, T>(access, [&](auto pw, auto ch) {
        auto* kernel = deep ? embed_kernel<T, decltype(pw)::value, decltype(ch)::value, 4> : embed_kernel<T, decltype(pw)::value, decltype(ch)::value, 1>;
        return launch_dependent(kernel, dim3((unsigned)((n + per_block - 1) / per_block)), dim3(kEmbedThreads), 0, st, n, vocab,
                                d, tpr, static_cast<const T*>(table), ids, scale, static_cast<T*>(out), &ctx->scalars->status);
    });
}

// Entries per piece: as many as still give every SM 24 warps, 8 to 64.  With 8, 16, 32 and 64 (us, rows of 1024 bf16
// values): 4096 tokens 27.2, 29.0, 31.8, 41.5; 16,384 41.5, 40.1, 43.3, 50.1; 131,072 208, 145, 122, 113.
int piece_of(const sama_ctx* ctx, int64_t n, int slabs) {
    int piece = 64;
    while (piece > 8 && (n + piece - 1) / piece * slabs < (int64_t)ctx->sm_count * 24) piece /= 2;
    return piece;
}

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

// Rows of the table per share of the zeroing, and the two areas of the workspace that belong to it.
inline int64_t fill_share(int64_t vocab) { return ((vocab + kFillCtas - 1) / kFillCtas + 31) & ~(int64_t)31; }
inline size_t present_bytes(int64_t vocab) { return up256((size_t)(fill_share(vocab) / 32) * kFillCtas * 4); }
constexpr size_t kProgressBytes = sizeof(int) * kFillCtas * 32;
static_assert(kProgressBytes % 256 == 0, "what follows it is aligned");

struct GradPlan {
    bool few;
    Access access;
    int slabs, piece, pieces, counters;
    int64_t share;
    size_t list, span, arrived, present, progress, parts;  // bytes
    size_t total() const { return few ? 2 * parts : 2 * list + span + arrived + present + progress + 2 * parts; }
};
GradPlan make_plan(const sama_ctx* ctx, int dtype, int64_t n, int64_t vocab, int d, const void* dout, int grad_dtype,
                   const void* grad) {
    GradPlan g;
    g.access = access_of(d, dtype, reinterpret_cast<uintptr_t>(dout) | reinterpret_cast<uintptr_t>(grad), grad_dtype == SAMA_F32);
    const int slab = 32 * columns_of(g.access, dtype);
    g.slabs = (d + slab - 1) / slab;
    g.piece = piece_of(ctx, n, g.slabs);
    g.pieces = (int)((n + g.piece - 1) / g.piece);
    g.list = up256(sizeof(int2) * (size_t)n);
    g.span = up256(sizeof(int2) * (size_t)vocab);
    g.counters = (2 * g.pieces + (g.pieces + kJoin - 1) / kJoin) * g.slabs;
    g.few = n <= kFewTokens && g.counters <= kFewCounters && vocab <= (int64_t)ctx->sm_count * (kFewShare / 2);
    g.arrived = up256(sizeof(int) * (size_t)g.counters);
    g.share = fill_share(vocab);
    g.present = present_bytes(vocab);
    g.progress = kProgressBytes;
    g.parts = up256(sizeof(float) * (size_t)g.pieces * d);
    return g;
}

template <typename T, typename TG>
struct ReduceLaunch {
    static cudaError_t run(sama_ctx* ctx, const ReduceArgs& a, Access access, cudaStream_t st) {
        KernelScope scope(ctx, SAMA_K_EMBED_GRAD, -1, st);
        const int64_t units = (int64_t)a.pieces * a.slabs, per = kEmbedThreads / 32;
        return with_access<T, TG>(access, [&](auto pw, auto ch) {
            return launch_dependent(embed_reduce_kernel<T, TG, decltype(pw)::value, decltype(ch)::value>,
                                    dim3((unsigned)(a.fill_blocks + (units + per - 1) / per)), dim3(kEmbedThreads), 0, st, a);
        });
    }
};
template <typename T, typename TG>
struct FewLaunch {
    static cudaError_t run(sama_ctx* ctx, const ReduceArgs& a, const FewArgs& f, Access access, int ctas, cudaStream_t st) {
        KernelScope scope(ctx, SAMA_K_EMBED_GRAD, -1, st);
        return with_access<T, TG>(access, [&](auto pw, auto ch) {
            return launch_dependent(embed_few_kernel<T, TG, decltype(pw)::value, decltype(ch)::value>, dim3((unsigned)ctas),
                                    dim3(kFewThreads), sizeof(FewSmem), st, a, f);
        });
    }
    static cudaError_t prepare() {
        cudaError_t e = cudaSuccess;
        for (Access access : {GROUPS, PAIRS, SINGLES, SINGLE})
            if (e == cudaSuccess)
                e = with_access<T, TG>(access, [&](auto pw, auto ch) {
                    return cudaFuncSetAttribute(embed_few_kernel<T, TG, decltype(pw)::value, decltype(ch)::value>,
                                                cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(FewSmem));
                });
        return e;
    }
};
// Launch<type of dOut, type of the gradient>::run(args)
template <template <typename, typename> class Launch, typename... Args>
cudaError_t by_type(int dtype, int grad_dtype, Args&&... args) {
    const bool wide = grad_dtype == SAMA_F32;
    if (dtype == SAMA_F32) return Launch<float, float>::run(args...);
    if (dtype == SAMA_BF16) return wide ? Launch<__nv_bfloat16, float>::run(args...) : Launch<__nv_bfloat16, __nv_bfloat16>::run(args...);
    return wide ? Launch<__half, float>::run(args...) : Launch<__half, __half>::run(args...);
}

// Once per context: shared-memory and cluster sizes, and the counters of embed_few.
cudaError_t prepare_embed(sama_ctx* ctx) {
    cudaError_t e;
    if ((e = cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(SortSmem))) != cudaSuccess) return e;
    if ((e = cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1)) != cudaSuccess) return e;
    if ((e = FewLaunch<float, float>::prepare()) != cudaSuccess) return e;
    if ((e = FewLaunch<__nv_bfloat16, float>::prepare()) != cudaSuccess) return e;
    if ((e = FewLaunch<__nv_bfloat16, __nv_bfloat16>::prepare()) != cudaSuccess) return e;
    if ((e = FewLaunch<__half, float>::prepare()) != cudaSuccess) return e;
    if ((e = FewLaunch<__half, __half>::prepare()) != cudaSuccess) return e;
    if (!ctx->embed_counters && (e = cudaMalloc(&ctx->embed_counters, sizeof(int) * kFewCounters)) != cudaSuccess) return e;
    if ((e = cudaMemset(ctx->embed_counters, 0, sizeof(int) * kFewCounters)) != cudaSuccess) return e;
    if ((e = cudaDeviceSynchronize()) != cudaSuccess) return e;
    ctx->embed_ready = 1;
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_embed(sama_ctx* ctx, int dtype, int64_t n, int64_t vocab, int d, const void* table, const int32_t* ids,
                         float scale, void* out, cudaStream_t st) {
    if (dtype == SAMA_F32) return embed_typed<float>(ctx, dtype, n, vocab, d, table, ids, scale, out, st);
    if (dtype == SAMA_BF16) return embed_typed<__nv_bfloat16>(ctx, dtype, n, vocab, d, table, ids, scale, out, st);
    return embed_typed<__half>(ctx, dtype, n, vocab, d, table, ids, scale, out, st);
}

// Workspace: two lists of (id, position), the rows' runs, arrival counters, and two parts per piece.
size_t embed_grad_plan_bytes(const sama_ctx* ctx, int dtype, int64_t n, int64_t vocab, int d, const void* dout,
                             int grad_dtype, const void* grad) {
    return make_plan(ctx, dtype, n, vocab, d, dout, grad_dtype, grad).total();
}

// What is reserved: enough for every plan of at most these sizes, whatever its types and alignment, so that no smaller
// call needs more.  (A plan's own need is not monotone: with more tokens the pieces get longer, and their parts fewer.)
// A plan has pieces of 64 entries, or fewer than 48 pieces x slabs per SM (see piece_of), and never pieces of fewer than 8;
// a slab has 128 to 256 columns, or all of up to 32.
size_t embed_grad_workspace(const sama_ctx* ctx, int64_t n, int64_t vocab, int d) {
    const int64_t busy = (int64_t)ctx->sm_count * 48, long_pieces = (n + 63) / 64, short_pieces = (n + 7) / 8;
    const int64_t slabs = ((int64_t)d + 127) / 128;
    auto larger = [](int64_t a, int64_t b) { return a > b ? a : b; };
    int64_t part = larger(long_pieces * d, busy * 256);
    if (part > short_pieces * d) part = short_pieces * d;
    const int64_t counters = 2 * larger(long_pieces * slabs, busy) +
                             larger((long_pieces + kJoin - 1) / kJoin * slabs, busy / kJoin + slabs);
    const size_t parts = 2 * up256(sizeof(float) * (size_t)part);
    if (n <= kFewTokens && counters <= kFewCounters && vocab <= (int64_t)ctx->sm_count * (kFewShare / 2)) return parts;
    return 2 * up256(sizeof(int2) * (size_t)n) + up256(sizeof(int2) * (size_t)vocab) + up256(sizeof(int) * (size_t)counters) +
           present_bytes(vocab) + kProgressBytes + parts;
}

cudaError_t launch_embed_grad(sama_ctx* ctx, int dtype, int64_t n, int64_t vocab, int d, const int32_t* ids,
                              const void* dout, float scale, int32_t skip_id, int grad_dtype, int accumulate, void* grad,
                              void* ws, size_t ws_bytes, cudaStream_t st) {
    const GradPlan g = make_plan(ctx, dtype, n, vocab, d, dout, grad_dtype, grad);
    if (g.total() > ws_bytes) return cudaErrorInvalidValue;
    if (!ctx->embed_ready) {
        const cudaError_t e = prepare_embed(ctx);
        if (e != cudaSuccess) return e;
    }
    uint8_t* w = static_cast<uint8_t*>(ws);
    auto take = [&](size_t bytes) {
        void* p = w;
        w += bytes;
        return p;
    };
    ReduceArgs a;
    a.dout = dout;
    a.grad = grad;
    a.n = (int)n;
    a.vocab = (int)vocab;
    a.d = d;
    a.piece = g.piece;
    a.pieces = g.pieces;
    a.slabs = g.slabs;
    a.accumulate = accumulate;
    a.scale = scale;
    int bits = 1;   // of the largest key, which is `vocab` itself
    while ((vocab >> bits) != 0) ++bits;
    const int most = g.few ? kFewBits : kMaxBits, passes = (bits + most - 1) / most, digit = (bits + passes - 1) / passes;
    a.fill = {};
    a.fill.grad = accumulate ? nullptr : static_cast<uint8_t*>(grad);
    a.fill.row_bytes = (int64_t)d * dtype_size(grad_dtype);
    a.fill.vocab = (int32_t)vocab;
    if (g.few) {
        a.list = a.span = nullptr;
        a.arrived = ctx->embed_counters;
        a.head = static_cast<float*>(take(g.parts));
        a.tail = static_cast<float*>(take(g.parts));
        a.fill_blocks = 0;
        FewArgs f;
        f.ids = ids;
        f.passes = passes;
        f.bits = digit;
        f.skip_id = skip_id;
        f.status = &ctx->scalars->status;
        // enough CTAs for four pieces each, and for 32 KB of zeros
        const int64_t units = (int64_t)g.pieces * g.slabs, by_fill = accumulate ? 0 : vocab * a.fill.row_bytes / 32768;
        int64_t ctas = (units + 3) / 4 > by_fill ? (units + 3) / 4 : by_fill;
        ctas = ctas < 1 ? 1 : ctas > ctx->sm_count ? ctx->sm_count : ctas;
        // (so that the bits of a share fit, too)
        if (vocab > ctas * (kFewShare / 2)) ctas = ctx->sm_count;
        f.share = accumulate ? 0 : ((vocab + ctas - 1) / ctas + 31) & ~(int64_t)31;
        return by_type<FewLaunch>(dtype, grad_dtype, ctx, a, f, g.access, (int)ctas, st);
    }
    SortArgs s;
    s.ids = ids;
    s.buf[0] = static_cast<int2*>(take(g.list));
    s.buf[1] = static_cast<int2*>(take(g.list));
    s.span = static_cast<int2*>(take(g.span));
    s.arrived = static_cast<int*>(take(g.arrived));
    a.fill.present = static_cast<uint32_t*>(take(g.present));
    a.fill.progress = static_cast<int*>(take(g.progress));
    a.fill.share = g.share;
    s.fill = a.fill;
    s.done = &ctx->scalars->embed_done;
    // (replays of a captured call find the flag already set: then embed_reduce writes all the zeros)
    s.epoch = ++ctx->embed_epoch;
    s.n = (int)n;
    s.counters = g.counters;
    s.passes = passes;
    s.bits = digit;
    s.vocab = (int32_t)vocab;
    s.skip_id = skip_id;
    s.status = &ctx->scalars->status;
    {
        const int ctas = accumulate ? kSortCtas : kSortCtas + kFillCtas;
        KernelScope scope(ctx, SAMA_K_EMBED_GRAD, -1, st);
        const cudaError_t e = launch_clustered(kSortCtas, embed_sort_kernel, dim3(ctas), dim3(kSortThreads), sizeof(SortSmem), st, s);
        if (e != cudaSuccess) return e;
    }
    a.list = s.buf[(passes - 1) & 1];
    a.span = s.span;
    a.head = static_cast<float*>(take(g.parts));
    a.tail = static_cast<float*>(take(g.parts));
    a.arrived = s.arrived;
    a.fill_blocks = accumulate ? 0 : ctx->sm_count;
    return by_type<ReduceLaunch>(dtype, grad_dtype, ctx, a, g.access, st);
}

}  // namespace sama
