// Prints, for each line of the standard input, what the text-model operators compute on the host, for a GPU of 148 SMs.
//   embed DTYPE N VOCAB D DOUT GRAD_DTYPE GRAD  ->  bytes that are reserved, bytes that this call's plan needs
//   ffn N D F GRAD COPIES                       ->  bytes that are reserved
//   setup CUDA_ERROR                            ->  status of an operator whose set-up failed so, the error it left
#include <cstdio>
#include <cstring>

#include "api_util.h"
#include "sama_internal.h"

int main() {
    static sama_ctx ctx;
    std::memset(static_cast<void*>(&ctx), 0, sizeof ctx);
    ctx.sm_count = 148;
    char what[16];
    while (std::scanf("%15s", what) == 1) {
        long long n, vocab, dout, grad;
        int dtype, d, f, grad_dtype, copies, error;
        if (std::strcmp(what, "embed") == 0 &&
            std::scanf("%d %lld %lld %d %lld %d %lld", &dtype, &n, &vocab, &d, &dout, &grad_dtype, &grad) == 7) {
            std::printf("%zu %zu\n", sama::embed_grad_workspace(&ctx, n, vocab, d),
                        sama::embed_grad_plan_bytes(&ctx, dtype, n, vocab, d, reinterpret_cast<void*>(dout), grad_dtype,
                                                    reinterpret_cast<void*>(grad)));
        } else if (std::strcmp(what, "ffn") == 0 && std::scanf("%lld %d %d %d %d", &n, &d, &f, &grad_dtype, &copies) == 5) {
            std::printf("%zu\n", sama::ffn_workspace({n, d, f, SAMA_BF16, SAMA_ACT_SILU}, grad_dtype != 0, copies != 0));
        } else if (std::strcmp(what, "setup") == 0 && std::scanf("%d", &error) == 1) {
            const int status = sama::setup_fail(&ctx, static_cast<cudaError_t>(error));
            std::printf("%d %d\n", status, ctx.last_cuda_error);
        } else {
            return 1;
        }
    }
    return 0;
}
