// Host side of the text-model operators: argument checks, workspace, launch sequencing.
#include <cmath>

#include "api_util.h"
#include "num_types.h"
#include "sama_internal.h"

using namespace sama;

namespace {

constexpr int64_t kMaxTokens = (int64_t)1 << 30;

// The operators' workspace, at least `bytes` large.  Growing it waits for the work that may still use the old one.
// `ready`: the operator's kernels are set up; the first call does that, and allocates for it.  Neither is possible while
// the stream is being captured, and trying would break the capture: the call is refused before.
int need_workspace(sama_ctx* ctx, size_t bytes, bool ready, cudaStream_t st) {
    if (ready && ctx->op_ws_bytes >= bytes) return SAMA_OK;
    cudaStreamCaptureStatus capture;
    SAMA_CUDA(ctx, cudaStreamIsCapturing(st, &capture));
    if (capture != cudaStreamCaptureStatusNone) return SAMA_ERR_NOMEM;
    if (ctx->op_ws_bytes >= bytes) return SAMA_OK;
    SAMA_CUDA(ctx, cudaStreamSynchronize(st));
    cudaFree(ctx->op_ws);
    ctx->op_ws = nullptr;
    ctx->op_ws_bytes = 0;
    if (cudaMalloc(&ctx->op_ws, bytes) != cudaSuccess) { cudaGetLastError(); return SAMA_ERR_NOMEM; }
    ctx->op_ws_bytes = bytes;
    return SAMA_OK;
}

// The kernels step through a row's columns in 32 bits, up to 8192 beyond its end.  With this limit on d, n_tokens * d and
// vocab * d elements of at most 4 bytes stay within 2^63 bytes, too.
constexpr int32_t kMaxColumns = 1 << 30;
bool embed_sizes_ok(int64_t n_tokens, int64_t vocab, int32_t d) {
    return n_tokens >= 0 && n_tokens <= kMaxTokens && vocab >= 1 && vocab < 0x7fffffff && d >= 1 && d <= kMaxColumns;
}

struct Span {
    const void* p;
    size_t bytes;
};

// Checks shared by the block's two directions: `ins` are all required, `outs` may be NULL; no output overlaps anything.
int check_ffn(const FfnShape& s, const Span* ins, int n_in, const Span* outs, int n_out, bool* copies) {
    if (s.n_tokens < 0 || s.n_tokens > ((int64_t)1 << 24) || s.d < 1 || s.d > (1 << 20) || s.f < 1 || s.f > (1 << 20))
        return SAMA_ERR_SIZE;
    if ((s.dtype != SAMA_BF16 && s.dtype != SAMA_F16) || s.act < SAMA_ACT_SILU || s.act > SAMA_ACT_RELU) return SAMA_ERR_PARAM;
    *copies = s.d % 8 != 0 || s.f % 8 != 0;
    for (int i = 0; i < n_in; ++i) {
        if (!ins[i].p && ins[i].bytes > 0) return SAMA_ERR_NULL;
        if (!aligned(ins[i].p, 2)) return SAMA_ERR_ALIGN;
        if (!aligned(ins[i].p, 16)) *copies = true;
    }
    for (int i = 0; i < n_out; ++i) {
        if (!aligned(outs[i].p, 2)) return SAMA_ERR_ALIGN;
        for (int j = 0; j < n_in; ++j)
            if (overlaps(outs[i].p, outs[i].bytes, ins[j].p, ins[j].bytes)) return SAMA_ERR_OVERLAP;
        for (int j = 0; j < i; ++j)
            if (overlaps(outs[i].p, outs[i].bytes, outs[j].p, outs[j].bytes)) return SAMA_ERR_OVERLAP;
    }
    return SAMA_OK;
}

}  // namespace

extern "C" {

int sama_embed(sama_ctx* ctx, int32_t dtype, int64_t n_tokens, int64_t vocab, int32_t d, const void* table,
               const int32_t* ids, float scale, void* out, void* stream) {
    if (!ctx || !table) return SAMA_ERR_NULL;
    if (!embed_sizes_ok(n_tokens, vocab, d)) return SAMA_ERR_SIZE;
    if (n_tokens > 0 && (!ids || !out)) return SAMA_ERR_NULL;
    if (!dtype_valid(dtype) || !std::isfinite(scale)) return SAMA_ERR_PARAM;
    const size_t es = dtype_size(dtype);
    if (!aligned(table, es) || !aligned(out, es) || !aligned(ids, 4)) return SAMA_ERR_ALIGN;
    const size_t ob = (size_t)n_tokens * d * es;
    if (overlaps(out, ob, table, (size_t)vocab * d * es) || overlaps(out, ob, ids, (size_t)n_tokens * 4))
        return SAMA_ERR_OVERLAP;
    if (n_tokens == 0) return SAMA_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SAMA_ERR_CUDA;
    SAMA_CUDA(ctx, launch_embed(ctx, dtype, n_tokens, vocab, d, table, ids, scale, out, (cudaStream_t)stream));
    return SAMA_OK;
}

int sama_embed_grad(sama_ctx* ctx, int32_t dtype, int64_t n_tokens, int64_t vocab, int32_t d, const int32_t* ids,
                    const void* d_out, float scale, int32_t skip_id, int32_t grad_dtype, int32_t accumulate,
                    void* grad, void* stream) {
    if (!ctx || !grad) return SAMA_ERR_NULL;
    if (!embed_sizes_ok(n_tokens, vocab, d)) return SAMA_ERR_SIZE;
    if (n_tokens > 0 && (!ids || !d_out)) return SAMA_ERR_NULL;
    if (!dtype_valid(dtype) || (grad_dtype != dtype && grad_dtype != SAMA_F32) || !std::isfinite(scale) ||
        (accumulate != 0 && accumulate != 1))
        return SAMA_ERR_PARAM;
    const size_t es = dtype_size(dtype), gs = dtype_size(grad_dtype);
    if (!aligned(d_out, es) || !aligned(grad, gs) || !aligned(ids, 4)) return SAMA_ERR_ALIGN;
    const size_t gb = (size_t)vocab * d * gs;
    if (overlaps(grad, gb, d_out, (size_t)n_tokens * d * es) || overlaps(grad, gb, ids, (size_t)n_tokens * 4))
        return SAMA_ERR_OVERLAP;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SAMA_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)stream;
    if (n_tokens == 0) {
        if (!accumulate) SAMA_CUDA(ctx, cudaMemsetAsync(grad, 0, gb, st));
        return SAMA_OK;
    }
    const int rc = need_workspace(ctx, embed_grad_workspace(ctx, n_tokens, vocab, d), ctx->embed_ready != 0, st);
    if (rc != SAMA_OK) return rc;
    SAMA_SETUP(ctx, launch_embed_grad(ctx, dtype, n_tokens, vocab, d, ids, d_out, scale, skip_id, grad_dtype, accumulate,
                                      grad, ctx->op_ws, ctx->op_ws_bytes, st));
    return SAMA_OK;
}

int sama_clip_grads(sama_ctx* ctx, const sama_tensor_t* tensors, int32_t n_tensors, float max_norm, float* norm_out,
                    void* stream) {
    if (!ctx || (n_tensors > 0 && !tensors)) return SAMA_ERR_NULL;
    if (n_tensors < 0 || n_tensors > 65536) return SAMA_ERR_SIZE;
    if (!(max_norm > 0.f)) return SAMA_ERR_PARAM;
    if (!aligned(norm_out, 4)) return SAMA_ERR_ALIGN;
    for (int i = 0; i < n_tensors; ++i) {
        const sama_tensor_t& t = tensors[i];
        if (t.n < 0 || t.n > ((int64_t)1 << 40)) return SAMA_ERR_SIZE;
        if (t.n > 0 && !t.in) return SAMA_ERR_NULL;
        if (!dtype_valid(t.dtype) || (t.out && !dtype_valid(t.out_dtype))) return SAMA_ERR_PARAM;
        const size_t es = dtype_size(t.dtype), os = dtype_size(t.out_dtype);
        if (!aligned(t.in, es) || !aligned(t.out, os)) return SAMA_ERR_ALIGN;
        const size_t ib = (size_t)t.n * es, ob = (size_t)t.n * os;
        const bool in_place = t.out == t.in && t.out_dtype == t.dtype;
        if ((!in_place && overlaps(t.out, ob, t.in, ib)) || overlaps(norm_out, 4, t.in, ib) || overlaps(norm_out, 4, t.out, ob))
            return SAMA_ERR_OVERLAP;
    }
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SAMA_ERR_CUDA;
    SAMA_CUDA(ctx, launch_clip_grads(ctx, tensors, n_tensors, max_norm, norm_out, (cudaStream_t)stream));
    return SAMA_OK;
}

int sama_gated_ffn(sama_ctx* ctx, int32_t dtype, int32_t act, int64_t n_tokens, int32_t d, int32_t f, const void* x,
                   const void* w_gate, const void* w_up, const void* w_down, void* y, void* gate_out, void* up_out,
                   void* stream) {
    if (!ctx) return SAMA_ERR_NULL;
    const FfnShape s{n_tokens, d, f, dtype, act};
    const size_t t = (size_t)n_tokens * d * 2, h = (size_t)n_tokens * f * 2, w = (size_t)d * f * 2;
    const Span ins[4] = {{x, t}, {w_gate, w}, {w_up, w}, {w_down, w}}, outs[3] = {{y, t}, {gate_out, h}, {up_out, h}};
    bool copies = false;
    int rc = check_ffn(s, ins, 4, outs, 3, &copies);
    if (rc != SAMA_OK) return rc;
    if (n_tokens == 0) return SAMA_OK;
    if (!y || (gate_out == nullptr) != (up_out == nullptr)) return SAMA_ERR_NULL;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SAMA_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)stream;
    if ((rc = need_workspace(ctx, ffn_workspace(s, false, copies), ctx->ffn_pair_units > 0, st)) != SAMA_OK) return rc;
    SAMA_SETUP(ctx, launch_ffn_forward(ctx, s, x, w_gate, w_up, w_down, y, gate_out, up_out, ctx->op_ws, st));
    return SAMA_OK;
}

int sama_gated_ffn_grad(sama_ctx* ctx, int32_t dtype, int32_t act, int64_t n_tokens, int32_t d, int32_t f, const void* x,
                        const void* w_gate, const void* w_up, const void* w_down, const void* gate, const void* up,
                        const void* dy, void* dx, void* dw_gate, void* dw_up, void* dw_down, void* stream) {
    if (!ctx) return SAMA_ERR_NULL;
    const FfnShape s{n_tokens, d, f, dtype, act};
    const size_t t = (size_t)n_tokens * d * 2, h = (size_t)n_tokens * f * 2, w = (size_t)d * f * 2;
    const Span ins[7] = {{x, t}, {w_gate, w}, {w_up, w}, {w_down, w}, {gate, h}, {up, h}, {dy, t}};
    const Span outs[4] = {{dx, t}, {dw_gate, w}, {dw_up, w}, {dw_down, w}};
    bool copies = false;
    int rc = check_ffn(s, ins, 7, outs, 4, &copies);
    if (rc != SAMA_OK) return rc;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SAMA_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)stream;
    if (n_tokens == 0) {
        void* dw[3] = {dw_gate, dw_up, dw_down};
        for (void* p : dw)
            if (p) SAMA_CUDA(ctx, cudaMemsetAsync(p, 0, w, st));
        return SAMA_OK;
    }
    if ((rc = need_workspace(ctx, ffn_workspace(s, true, copies), ctx->ffn_pair_units > 0, st)) != SAMA_OK) return rc;
    SAMA_SETUP(ctx, launch_ffn_backward(ctx, s, x, w_gate, w_up, w_down, gate, up, dy, dx, dw_gate, dw_up, dw_down,
                                        ctx->op_ws, st));
    return SAMA_OK;
}

int sama_last_ffn_path(sama_ctx* ctx, int32_t launch) { return ctx && launch >= 0 && launch < 5 ? ctx->ffn_path[launch] : 0; }

}  // extern "C"
