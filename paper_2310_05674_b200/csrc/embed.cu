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
// Three launches:
//   embed_sort   : one cluster of 8 CTAs sorts (id, position) by 8-bit digits, least significant first.  Counts are
//                  exchanged through distributed shared memory, so the passes need only cluster barriers.  Ids outside
//                  the vocabulary and the skipped id become the key `vocab`, which sorts behind all others.  It also
//                  leaves one bit per row of dE that has a token.
//   embed_reduce : workers of one CTA's threads each add up `piece` consecutive entries of the list.  A run that
//                  lies inside a piece is written out; the parts of runs that cross pieces go to the workspace in fp32.
//                  Further blocks write zeros to the rows without a token.
//   embed_join   : adds the parts of the runs that cross pieces, in order.
#include "num_types.h"
#include "sama_internal.h"

namespace sama {

namespace {

// ------------------------------------------------------------------ forward

constexpr int kEmbedThreads = 256;

// VE consecutive columns per thread; `tpr` threads (a power of two) share a row.
template <typename T, int VE>
__global__ void __launch_bounds__(kEmbedThreads)
embed_kernel(int64_t n_tokens, int64_t vocab, int d, int tpr, const T* __restrict__ table,
             const int32_t* __restrict__ ids, float scale, T* __restrict__ out, int32_t* status) {
    pdl_trigger();
    pdl_wait();
    const int rows = kEmbedThreads / tpr, tx = threadIdx.x & (tpr - 1);
    const int64_t t = (int64_t)blockIdx.x * rows + threadIdx.x / tpr;
    if (t >= n_tokens) return;
    const int32_t id = ids[t];
    const bool good = id >= 0 && id < vocab;
    if (!good && tx == 0) atomicOr(status, (int)SAMA_DEV_BAD_INDEX);
    const T* src = table + (good ? (int64_t)id : 0) * d;
    T* dst = out + t * d;
    for (int c = tx * VE; c < d; c += tpr * VE) {
        float v[VE];
        load_n<T, VE, true>(src + c, v);  // rows of frequent tokens are read again and again
#pragma unroll
        for (int i = 0; i < VE; ++i) v[i] = good ? v[i] * scale : 0.f;
        store_n<T, VE>(dst + c, v);
    }
}

// ------------------------------------------------------------------ sort

constexpr int kSortCtas = 8, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kDigits = 256;

struct SortSmem {
    uint32_t hist[kSortWarps][kDigits];  // counts, then next output positions, of every warp's share
    uint32_t total[kDigits];             // this CTA's counts (read by the other CTAs)
    uint32_t warp_sum[8];
};

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

// ids -> `passes` stable counting passes over (key, position), buf[0] and buf[1] in turn (pass p writes buf[p & 1]).
// present: bit v of the row map (cleared here), or null.
__global__ void __cluster_dims__(kSortCtas, 1, 1) __launch_bounds__(kSortThreads)
embed_sort_kernel(int n, int32_t vocab, int32_t skip_id, int passes, const int32_t* __restrict__ ids, int2* buf0,
                  int2* buf1, uint32_t* present, int32_t* status) {
    extern __shared__ uint8_t sort_raw[];
    SortSmem& sm = *reinterpret_cast<SortSmem*>(sort_raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x;
    const int per_cta = ((n + kSortCtas - 1) / kSortCtas + 31) & ~31;
    const int per_warp = ((per_cta + kSortWarps - 1) / kSortWarps + 31) & ~31;
    const int64_t cta_end = min((int64_t)n, (int64_t)(rank + 1) * per_cta);
    const int64_t begin = (int64_t)rank * per_cta + (int64_t)warp * per_warp;
    const int64_t end = min(cta_end, begin + per_warp);
    pdl_trigger();
    pdl_wait();
    if (present)
        for (int64_t w = (int64_t)rank * kSortThreads + threadIdx.x; w < ((int64_t)vocab + 31) / 32; w += kSortCtas * kSortThreads)
            present[w] = 0;
    for (int p = 0; p < passes; ++p) {
        const int2* src = (p & 1) ? buf0 : buf1;
        int2* dst = (p & 1) ? buf1 : buf0;
        auto fetch = [&](int64_t i) -> int2 {
            if (p > 0) return __ldcg(src + i);
            const int32_t id = ids[i];
            const bool good = id >= 0 && id < vocab;
            if (!good) atomicOr(status, (int)SAMA_DEV_BAD_INDEX);
            return make_int2(good && id != skip_id ? id : vocab, (int)i);
        };
        for (int b = lane; b < kDigits; b += 32) sm.hist[warp][b] = 0;
        __syncwarp();
        for (int64_t i = begin + lane; i - lane < end; i += 32) {
            const bool on = i < end;
            const uint32_t digit = on ? ((uint32_t)fetch(i).x >> (8 * p)) & 255u : 256u;
            const uint32_t same = __match_any_sync(0xffffffffu, digit);
            if (on && lane == __ffs(same) - 1) sm.hist[warp][digit] += __popc(same);
            __syncwarp();
        }
        __syncthreads();
        uint32_t mine = 0;
        if (threadIdx.x < kDigits) {
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t c = sm.hist[w][threadIdx.x];
                sm.hist[w][threadIdx.x] = mine;
                mine += c;
            }
            sm.total[threadIdx.x] = mine;
        }
        cluster_barrier();
        uint32_t before = 0, all = 0, incl = 0;
        if (threadIdx.x < kDigits) {
            for (uint32_t c = 0; c < kSortCtas; ++c) {
                const uint32_t v = ld_cluster_u32(&sm.total[threadIdx.x], c);
                if (c < rank) before += v;
                all += v;
            }
            incl = all;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += v;
            }
            if (lane == 31) sm.warp_sum[warp] = incl;
        }
        __syncthreads();
        if (threadIdx.x < kDigits) {
            uint32_t base = incl - all + before;
            for (int w = 0; w < warp; ++w) base += sm.warp_sum[w];
            for (int w = 0; w < kSortWarps; ++w) sm.hist[w][threadIdx.x] += base;
        }
        __syncthreads();
        for (int64_t i = begin + lane; i - lane < end; i += 32) {
            const bool on = i < end;
            int2 e = make_int2(0, 0);
            if (on) e = fetch(i);
            const uint32_t digit = on ? ((uint32_t)e.x >> (8 * p)) & 255u : 256u;
            const uint32_t same = __match_any_sync(0xffffffffu, digit);
            uint32_t at = 0;
            if (on) at = sm.hist[warp][digit] + __popc(same & ((1u << lane) - 1u));
            __syncwarp();
            if (on) {
                dst[at] = e;
                if (lane == __ffs(same) - 1) sm.hist[warp][digit] += __popc(same);
            }
            __syncwarp();
        }
        cluster_barrier();  // the pass is complete: every CTA may read all of dst, and total may be rewritten
    }
    if (present) {
        const int2* fin = ((passes - 1) & 1) ? buf1 : buf0;
        for (int64_t i = begin + lane; i < end; i += 32) {
            const int32_t key = __ldcg(fin + i).x;
            if (key < vocab && (i == 0 || __ldcg(fin + i - 1).x != key)) atomicOr(present + (key >> 5), 1u << (key & 31));
        }
    }
}

// ------------------------------------------------------------------ reduction

struct ReduceArgs {
    const int2* list;         // sorted (id, position)
    const uint32_t* present;  // row map
    const void* dout;
    void* grad;
    float* head;              // [pieces][d]: the part of a run that began in an earlier piece
    float* tail;              // [pieces][d]: the first part of a run that goes on in the next piece
    int n, vocab, d;
    int piece, pieces, tpr, reduce_blocks, fill_blocks;
    int accumulate;
    float scale;
};

template <typename TG, int VE>
__device__ __forceinline__ void put_row(const ReduceArgs& a, int row, int c, const float* acc) {
    TG* g = static_cast<TG*>(a.grad) + (int64_t)row * a.d + c;
    float v[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) v[i] = acc[i] * a.scale;
    if (a.accumulate) {
        float old[VE];
        load_n<TG, VE>(g, old);
#pragma unroll
        for (int i = 0; i < VE; ++i) v[i] += old[i];
    }
    store_n<TG, VE>(g, v);
}

template <typename T, typename TG, int VE>
__global__ void __launch_bounds__(kEmbedThreads)
embed_reduce_kernel(const __grid_constant__ ReduceArgs a) {
    pdl_trigger();
    pdl_wait();
    constexpr int U = 4;  // rows in flight per thread
    const T* dout = static_cast<const T*>(a.dout);
    if ((int)blockIdx.x >= a.reduce_blocks) {
        // rows without a token: one warp per word of the row map
        const int warps = kEmbedThreads / 32, lane = threadIdx.x & 31;
        const int words = (a.vocab + 31) / 32;
        float z[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) z[i] = 0.f;
        for (int w = ((int)blockIdx.x - a.reduce_blocks) * warps + (threadIdx.x >> 5); w < words; w += a.fill_blocks * warps) {
            uint32_t absent = ~a.present[w];
            if (w == words - 1 && (a.vocab & 31)) absent &= (1u << (a.vocab & 31)) - 1u;
            while (absent) {
                const int r = __ffs(absent) - 1;
                absent &= absent - 1;
                TG* g = static_cast<TG*>(a.grad) + ((int64_t)w * 32 + r) * a.d;
                for (int c = lane * VE; c < a.d; c += 32 * VE) store_n<TG, VE>(g + c, z);
            }
        }
        return;
    }
    const int tx = threadIdx.x & (a.tpr - 1);
    const int k = blockIdx.x * (kEmbedThreads / a.tpr) + threadIdx.x / a.tpr;
    if (k >= a.pieces) return;
    const int i0 = k * a.piece, i1 = min(a.n, i0 + a.piece);
    const int first = a.list[i0].x;
    const bool open_head = i0 > 0 && a.list[i0 - 1].x == first;
    for (int c = tx * VE; c < a.d; c += a.tpr * VE) {
        int key = first;
        bool from_head = open_head;
        float acc[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) acc[i] = 0.f;
        for (int i = i0; i < i1 && key < a.vocab; i += U) {
            int2 e[U];
            float v[U][VE];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                e[u] = i + u < i1 ? a.list[i + u] : make_int2(a.vocab, 0);
                if (e[u].x < a.vocab) load_n<T, VE>(dout + (int64_t)e[u].y * a.d + c, v[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i + u >= i1) break;
                if (e[u].x != key) {
                    if (from_head) store_n<float, VE>(a.head + (int64_t)k * a.d + c, acc);
                    else put_row<TG, VE>(a, key, c, acc);
                    from_head = false;
                    key = e[u].x;
#pragma unroll
                    for (int j = 0; j < VE; ++j) acc[j] = 0.f;
                }
                if (key >= a.vocab) break;
#pragma unroll
                for (int j = 0; j < VE; ++j) acc[j] += v[u][j];
            }
        }
        if (key < a.vocab) {
            if (from_head) store_n<float, VE>(a.head + (int64_t)k * a.d + c, acc);
            else if (i1 < a.n && a.list[i1].x == key) store_n<float, VE>(a.tail + (int64_t)k * a.d + c, acc);
            else put_row<TG, VE>(a, key, c, acc);
        }
    }
}

// One worker per piece in which a run begins that does not end there.
template <typename TG, int VE>
__global__ void __launch_bounds__(kEmbedThreads)
embed_join_kernel(const __grid_constant__ ReduceArgs a) {
    pdl_trigger();
    pdl_wait();
    const int tx = threadIdx.x & (a.tpr - 1);
    const int k = blockIdx.x * (kEmbedThreads / a.tpr) + threadIdx.x / a.tpr;
    if (k >= a.pieces - 1) return;
    const int i1 = (k + 1) * a.piece;
    const int key = a.list[i1 - 1].x;
    if (key >= a.vocab || a.list[i1].x != key) return;
    const int i0 = k * a.piece;
    if (i0 > 0 && a.list[i0].x == key && a.list[i0 - 1].x == key) return;  // began earlier
    int last = k + 1;                                                       // the piece the run ends in
    while ((last + 1) * (int64_t)a.piece < a.n && a.list[(last + 1) * a.piece].x == key) ++last;
    for (int c = tx * VE; c < a.d; c += a.tpr * VE) {
        float acc[VE], v[VE];
        load_n<float, VE>(a.tail + (int64_t)k * a.d + c, acc);
        for (int j = k + 1; j <= last; ++j) {
            load_n<float, VE>(a.head + (int64_t)j * a.d + c, v);
#pragma unroll
            for (int i = 0; i < VE; ++i) acc[i] += v[i];
        }
        put_row<TG, VE>(a, key, c, acc);
    }
}

int threads_per_row(int d, int ve) {
    int t = 1;
    while (t < kEmbedThreads && t * ve < d) t *= 2;
    return t;
}

template <typename T>
cudaError_t embed_typed(sama_ctx* ctx, int64_t n, int64_t vocab, int d, const void* table, const int32_t* ids, float scale,
                        void* out, cudaStream_t st) {
    constexpr int VE = 16 / sizeof(T);
    const bool vec = d % VE == 0 && ((reinterpret_cast<uintptr_t>(table) | reinterpret_cast<uintptr_t>(out)) & 15u) == 0;
    const int tpr = threads_per_row(d, vec ? VE : 1), rows = kEmbedThreads / tpr;
    const dim3 grid((unsigned)((n + rows - 1) / rows));
    KernelScope scope(ctx, SAMA_K_EMBED, -1, st);
    auto* kernel = vec ? embed_kernel<T, VE> : embed_kernel<T, 1>;
    return launch_dependent(kernel, grid, dim3(kEmbedThreads), 0, st, n, vocab, d, tpr, static_cast<const T*>(table), ids,
                            scale, static_cast<T*>(out), &ctx->scalars->status);
}

constexpr int kPiece = 32;

template <typename T, typename TG>
cudaError_t reduce_typed(sama_ctx* ctx, ReduceArgs a, cudaStream_t st) {
    constexpr int VE = 16 / (sizeof(T) < sizeof(TG) ? sizeof(T) : sizeof(TG));
    const bool vec = a.d % VE == 0 && ((reinterpret_cast<uintptr_t>(a.dout) | reinterpret_cast<uintptr_t>(a.grad)) & 15u) == 0;
    a.tpr = threads_per_row(a.d, vec ? VE : 1);
    const int workers = kEmbedThreads / a.tpr;
    a.reduce_blocks = (a.pieces + workers - 1) / workers;
    a.fill_blocks = a.accumulate ? 0 : 2 * ctx->sm_count;
    {
        KernelScope scope(ctx, SAMA_K_EMBED_GRAD, -1, st);
        auto* kernel = vec ? embed_reduce_kernel<T, TG, VE> : embed_reduce_kernel<T, TG, 1>;
        const cudaError_t e = launch_dependent(kernel, dim3(a.reduce_blocks + a.fill_blocks), dim3(kEmbedThreads), 0, st, a);
        if (e != cudaSuccess) return e;
    }
    KernelScope scope(ctx, SAMA_K_EMBED_GRAD, -1, st);
    auto* kernel = vec ? embed_join_kernel<TG, VE> : embed_join_kernel<TG, 1>;
    return launch_dependent(kernel, dim3(a.reduce_blocks), dim3(kEmbedThreads), 0, st, a);
}

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

cudaError_t launch_embed(sama_ctx* ctx, int dtype, int64_t n, int64_t vocab, int d, const void* table, const int32_t* ids,
                         float scale, void* out, cudaStream_t st) {
    if (dtype == SAMA_F32) return embed_typed<float>(ctx, n, vocab, d, table, ids, scale, out, st);
    if (dtype == SAMA_BF16) return embed_typed<__nv_bfloat16>(ctx, n, vocab, d, table, ids, scale, out, st);
    return embed_typed<__half>(ctx, n, vocab, d, table, ids, scale, out, st);
}

// Workspace: two lists of (id, position), the row map, and two parts per piece.
size_t embed_grad_workspace(int64_t n, int64_t vocab, int d) {
    const size_t pieces = ((size_t)n + kPiece - 1) / kPiece;
    return 2 * up256(sizeof(int2) * (size_t)n) + up256((size_t)(vocab + 31) / 32 * 4) + 2 * up256(pieces * (size_t)d * 4);
}

cudaError_t launch_embed_grad(sama_ctx* ctx, int dtype, int64_t n, int64_t vocab, int d, const int32_t* ids,
                              const void* dout, float scale, int32_t skip_id, int grad_dtype, int accumulate, void* grad,
                              void* ws, cudaStream_t st) {
    uint8_t* w = static_cast<uint8_t*>(ws);
    int2* buf[2];
    for (int i = 0; i < 2; ++i) {
        buf[i] = reinterpret_cast<int2*>(w);
        w += up256(sizeof(int2) * (size_t)n);
    }
    uint32_t* present = reinterpret_cast<uint32_t*>(w);
    w += up256((size_t)(vocab + 31) / 32 * 4);
    ReduceArgs a;
    a.piece = kPiece;
    a.pieces = (int)((n + a.piece - 1) / a.piece);
    a.head = reinterpret_cast<float*>(w);
    a.tail = reinterpret_cast<float*>(w + up256((size_t)a.pieces * d * 4));
    int passes = 1;  // 8 bits each; the largest key is `vocab` itself
    while (passes < 4 && (vocab >> (8 * passes)) != 0) ++passes;
    {
        KernelScope scope(ctx, SAMA_K_EMBED_GRAD, -1, st);
        // (the cluster shape is part of the kernel's declaration)
        const cudaError_t e = launch_dependent(embed_sort_kernel, dim3(kSortCtas), dim3(kSortThreads), sizeof(SortSmem), st,
                                               (int)n, (int32_t)vocab, skip_id, passes, ids, buf[0], buf[1],
                                               accumulate ? (uint32_t*)nullptr : present, &ctx->scalars->status);
        if (e != cudaSuccess) return e;
    }
    a.list = buf[(passes - 1) & 1];
    a.present = present;
    a.dout = dout;
    a.grad = grad;
    a.n = (int)n;
    a.vocab = (int)vocab;
    a.d = d;
    a.accumulate = accumulate;
    a.scale = scale;
    const bool wide = grad_dtype == SAMA_F32;
    if (dtype == SAMA_F32) return reduce_typed<float, float>(ctx, a, st);
    if (dtype == SAMA_BF16)
        return wide ? reduce_typed<__nv_bfloat16, float>(ctx, a, st) : reduce_typed<__nv_bfloat16, __nv_bfloat16>(ctx, a, st);
    return wide ? reduce_typed<__half, float>(ctx, a, st) : reduce_typed<__half, __half>(ctx, a, st);
}

}  // namespace sama
