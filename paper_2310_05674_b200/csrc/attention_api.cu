// Host side of attention: argument checks, workspace, launch sequencing.
#include "api_util.h"
#include "attention.h"

using namespace sama;

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 30, kMaxStride = (int64_t)1 << 32;

// Rows of `width` bytes, `stride` bytes apart.
struct Rows {
    const void* p;
    int64_t n;
    size_t width, stride;
    size_t span() const { return n > 0 ? (size_t)(n - 1) * stride + width : 0; }
};
// Rows that lie in the gaps of others, as parts of one buffer do, share no byte with them.
bool rows_overlap(const Rows& a, const Rows& b) {
    if (!overlaps(a.p, a.span(), b.p, b.span())) return false;
    if (a.stride != b.stride) return true;
    const intptr_t s = (intptr_t)a.stride;
    intptr_t d = (reinterpret_cast<intptr_t>(b.p) - reinterpret_cast<intptr_t>(a.p)) % s;
    if (d < 0) d += s;
    return !((size_t)d >= a.width && (size_t)d + b.width <= a.stride);
}

int check_heads(int32_t dtype, int32_t heads, int32_t kv_heads, int32_t dim, float scale, float cap) {
    if (heads < 1 || heads > 65535 || kv_heads < 1 || heads % kv_heads != 0 || dim < 8 || dim > 128 || dim % 8 != 0) return SAMA_ERR_SIZE;
    if ((dtype != SAMA_BF16 && dtype != SAMA_F16) || !moderate(scale)) return SAMA_ERR_PARAM;
    // (the polynomial of a capped score has (scale / cap)^9)
    if (cap != 0.f && (!moderate(cap) || scale / cap > 8192.f)) return SAMA_ERR_PARAM;
    return SAMA_OK;
}

struct AttnCall {
    AttnShape shape;
    AttnOperands op;
    Rows q, k, v, out;
};
// Checks shared by both directions, and the call's geometry.
int check_attn(sama_ctx* ctx, const sama_attn_t* a, const void* q, const void* k, const void* v, const void* out, AttnCall* c) {
    if (!ctx || !a) return SAMA_ERR_NULL;
    const int rc = check_heads(a->dtype, a->heads, a->kv_heads, a->head_dim, a->scale, a->cap);
    if (rc != SAMA_OK) return rc;
    if (a->n_q < 0 || a->n_q > kMaxRows || a->n_k < 0 || a->n_k > kMaxRows || a->n_texts < 0 || a->n_texts > (1 << 20)) return SAMA_ERR_SIZE;
    if (!a->k_starts && a->n_k != a->n_q) return SAMA_ERR_SIZE;
    if (a->causal != 0 && a->causal != 1) return SAMA_ERR_PARAM;
    const int64_t wq = (int64_t)a->heads * a->head_dim, wk = (int64_t)a->kv_heads * a->head_dim;
    const int64_t strides[3] = {a->q_stride ? a->q_stride : wq, a->k_stride ? a->k_stride : wk, a->v_stride ? a->v_stride : wk};
    for (int i = 0; i < 3; ++i)
        if (strides[i] < (i == 0 ? wq : wk) || strides[i] > kMaxStride || strides[i] % 8 != 0) return SAMA_ERR_SIZE;
    // blocks are numbered in 31 bits
    if ((a->n_q / kAttnRows + a->n_texts) * a->heads > 0x7fffffffLL || (a->n_k / kAttnRows + a->n_texts) * a->heads > 0x7fffffffLL)
        return SAMA_ERR_SIZE;
    if (a->n_texts > 0 && (!a->q_starts || (a->n_q > 0 && (!q || !out)) || (a->n_k > 0 && (!k || !v)))) return SAMA_ERR_NULL;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(a->q_starts, 4) || !aligned(a->k_starts, 4) ||
        !aligned(a->prefix, 4) || !aligned(a->slopes, 4))
        return SAMA_ERR_ALIGN;
    c->q = {q, a->n_q, (size_t)wq * 2, (size_t)strides[0] * 2};
    c->k = {k, a->n_k, (size_t)wk * 2, (size_t)strides[1] * 2};
    c->v = {v, a->n_k, (size_t)wk * 2, (size_t)strides[2] * 2};
    c->out = {out, a->n_q, (size_t)wq * 2, (size_t)wq * 2};
    c->op = {q, k, v, strides[0], strides[1], strides[2], a->dtype};
    AttnShape& s = c->shape;
    s.q_starts = a->q_starts;
    s.k_starts = a->k_starts ? a->k_starts : a->q_starts;
    s.prefix = a->prefix;
    s.slopes = a->slopes;
    s.status = &ctx->scalars->status;
    s.n_texts = a->n_texts;
    s.n_q = (int)a->n_q;
    s.n_k = (int)a->n_k;
    s.heads = a->heads;
    s.kv_heads = a->kv_heads;
    s.group = a->heads / a->kv_heads;
    s.dim = a->head_dim;
    s.causal = a->causal;
    s.scale = a->scale;
    s.cap = a->cap;
    return SAMA_OK;
}

// Small arrays that a call reads, against an output.
bool hits_arrays(const sama_attn_t* a, const Rows& o) {
    const size_t starts = ((size_t)a->n_texts + 1) * 4;
    return overlaps(o.p, o.span(), a->q_starts, starts) || overlaps(o.p, o.span(), a->k_starts, starts) ||
           overlaps(o.p, o.span(), a->prefix, (size_t)a->n_texts * 4) || overlaps(o.p, o.span(), a->slopes, (size_t)a->heads * 4);
}

}  // namespace

extern "C" {

int sama_attention(sama_ctx* ctx, const sama_attn_t* a, const void* q, const void* k, const void* v, void* out,
                   float* lse_out, void* stream) {
    AttnCall c;
    const int rc = check_attn(ctx, a, q, k, v, out, &c);
    if (rc != SAMA_OK) return rc;
    if (!aligned(lse_out, 4)) return SAMA_ERR_ALIGN;
    const Rows lse = {lse_out, lse_out ? a->heads : 0, (size_t)a->n_q * 4, (size_t)a->n_q * 4};
    const Rows outs[2] = {c.out, lse}, ins[3] = {c.q, c.k, c.v};
    for (const Rows& o : outs) {
        for (const Rows& i : ins)
            if (rows_overlap(o, i)) return SAMA_ERR_OVERLAP;
        if (hits_arrays(a, o)) return SAMA_ERR_OVERLAP;
    }
    if (rows_overlap(c.out, lse)) return SAMA_ERR_OVERLAP;
    if (a->n_texts == 0 || a->n_q == 0) return SAMA_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SAMA_ERR_CUDA;
    SAMA_CUDA(ctx, launch_attention(ctx, c.shape, c.op, out, lse_out, (cudaStream_t)stream));
    return SAMA_OK;
}

int sama_attention_grad(sama_ctx* ctx, const sama_attn_t* a, const void* q, const void* k, const void* v, const void* out,
                        const float* lse, const void* d_out, void* dq, void* dk, void* dv, void* stream) {
    AttnCall c;
    int rc = check_attn(ctx, a, q, k, v, out, &c);
    if (rc != SAMA_OK) return rc;
    if (a->n_texts > 0 && ((a->n_q > 0 && (!lse || !d_out || !dq)) || (a->n_k > 0 && (!dk || !dv)))) return SAMA_ERR_NULL;
    if (!aligned(lse, 4) || !aligned(d_out, 16) || !aligned(dq, 16) || !aligned(dk, 16) || !aligned(dv, 16)) return SAMA_ERR_ALIGN;
    const Rows r_lse = {lse, a->heads, (size_t)a->n_q * 4, (size_t)a->n_q * 4};
    Rows r_dout = c.out, outs[3] = {c.q, c.k, c.v};
    r_dout.p = d_out;
    outs[0].p = dq;
    outs[1].p = dk;
    outs[2].p = dv;
    const Rows ins[6] = {c.q, c.k, c.v, c.out, r_dout, r_lse};
    for (int i = 0; i < 3; ++i) {
        for (const Rows& in : ins)
            if (rows_overlap(outs[i], in)) return SAMA_ERR_OVERLAP;
        for (int j = 0; j < i; ++j)
            if (rows_overlap(outs[i], outs[j])) return SAMA_ERR_OVERLAP;
        if (hits_arrays(a, outs[i])) return SAMA_ERR_OVERLAP;
    }
    if (a->n_texts == 0 || (a->n_q == 0 && a->n_k == 0)) return SAMA_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SAMA_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)stream;
    if ((rc = need_workspace(ctx, attention_grad_workspace(c.shape), true, st)) != SAMA_OK) return rc;
    SAMA_CUDA(ctx, launch_attention_grad(ctx, c.shape, c.op, out, lse, d_out, dq, dk, dv, ctx->op_ws, st));
    return SAMA_OK;
}

int sama_paged_attention(sama_ctx* ctx, const sama_paged_t* a, const void* q, const void* k_new, const void* v_new,
                         void* k_cache, void* v_cache, void* out, void* stream) {
    if (!ctx || !a) return SAMA_ERR_NULL;
    int rc = check_heads(a->dtype, a->heads, a->kv_heads, a->head_dim, a->scale, a->cap);
    if (rc != SAMA_OK) return rc;
    if (a->n_seqs < 0 || a->n_seqs > (1 << 20) || a->max_pages < 1 || a->max_pages > (1 << 24) || a->page_size < 1 ||
        a->page_size > (1 << 20) || a->n_pages < 1 || a->n_pages > 0x7fffffff)
        return SAMA_ERR_SIZE;
    // (a CTA's steps of 64 keys are numbered in 31 bits)
    const int64_t longest = paged_most_keys(a->max_pages, a->page_size);
    if (longest * a->n_seqs > ((int64_t)1 << 44) / a->heads) return SAMA_ERR_SIZE;
    const int64_t row = (int64_t)a->kv_heads * a->head_dim, page = row * a->page_size, stride = a->page_stride ? a->page_stride : page;
    if (stride < page || stride % 8 != 0 || stride > ((int64_t)1 << 40)) return SAMA_ERR_SIZE;
    if (a->n_seqs > 0 && (!q || !k_cache || !v_cache || !out || !a->page_table || !a->lengths)) return SAMA_ERR_NULL;
    if ((k_new == nullptr) != (v_new == nullptr)) return SAMA_ERR_NULL;
    const void* wide[6] = {q, k_new, v_new, k_cache, v_cache, out};
    for (const void* p : wide)
        if (!aligned(p, 16)) return SAMA_ERR_ALIGN;
    if (!aligned(a->page_table, 4) || !aligned(a->lengths, 4) || !aligned(a->slopes, 4)) return SAMA_ERR_ALIGN;
    const Rows rk = {k_cache, a->n_pages, (size_t)page * 2, (size_t)stride * 2}, rv = {v_cache, a->n_pages, (size_t)page * 2, (size_t)stride * 2};
    const size_t nq = (size_t)a->n_seqs * a->heads * a->head_dim * 2, nn = (size_t)a->n_seqs * row * 2;
    const Rows ro = {out, a->n_seqs > 0 ? 1 : 0, nq, nq};
    const struct { const void* p; size_t bytes; } ins[6] = {{q, nq}, {k_new, nn}, {v_new, nn},
        {a->page_table, (size_t)a->n_seqs * a->max_pages * 4}, {a->lengths, (size_t)a->n_seqs * 4}, {a->slopes, (size_t)a->heads * 4}};
    for (const auto& in : ins) {
        const Rows ri = {in.p, in.bytes > 0 ? 1 : 0, in.bytes, in.bytes};
        if (rows_overlap(ro, ri)) return SAMA_ERR_OVERLAP;
        // the caches are written where there are new tokens
        if (k_new && (overlaps(in.p, in.bytes, k_cache, rk.span()) || overlaps(in.p, in.bytes, v_cache, rv.span()))) return SAMA_ERR_OVERLAP;
    }
    if (overlaps(out, nq, k_cache, rk.span()) || overlaps(out, nq, v_cache, rv.span()) || (k_new && rows_overlap(rk, rv))) return SAMA_ERR_OVERLAP;
    if (a->n_seqs == 0) return SAMA_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SAMA_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)stream;
    if ((rc = need_workspace(ctx, paged_workspace(ctx), ctx->paged_arrived != nullptr, st)) != SAMA_OK) return rc;
    PagedShape s;
    s.page_table = a->page_table;
    s.lengths = a->lengths;
    s.slopes = a->slopes;
    s.status = &ctx->scalars->status;
    s.n_pages = a->n_pages;
    s.page_stride = stride;
    s.n_seqs = a->n_seqs;
    s.max_pages = a->max_pages;
    s.page_size = a->page_size;
    s.heads = a->heads;
    s.kv_heads = a->kv_heads;
    s.group = a->heads / a->kv_heads;
    s.dim = a->head_dim;
    s.scale = a->scale;
    s.cap = a->cap;
    SAMA_SETUP(ctx, launch_paged(ctx, s, a->dtype, q, k_new, v_new, k_cache, v_cache, out, ctx->op_ws, st));
    return SAMA_OK;
}

}  // extern "C"
