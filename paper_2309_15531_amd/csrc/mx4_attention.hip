// Attention over a paged cache in mx4: which form a call gets, and its launch.
#include "mx4_attention.h"

namespace mx4 {
int launch_attention_f16(adadim_ctx* ctx, const Attention& a);
int launch_attention_bf16(adadim_ctx* ctx, const Attention& a);
}

int launch_mx4_attention(adadim_ctx* ctx, const mx4::Attention& a, int q_type) {
    return q_type == ADADIM_TYPE_F16 ? mx4::launch_attention_f16(ctx, a) : mx4::launch_attention_bf16(ctx, a);
}

int attention_shares(adadim_ctx* ctx, size_t bytes, void*& shared);

namespace {
__global__ void mx4_attend_zero(unsigned* tickets) { tickets[blockIdx.x * 256 + threadIdx.x] = 0u; }
}

// The counters and room for `bytes` of partial sums.
int attention_shares(adadim_ctx* ctx, size_t bytes, void*& shared) {
    shared = adadim_workspace(ctx, WS_ATTEND, mx4::AT_TICKETS * 4 + bytes);
    if (!shared) return ADADIM_EHIP;
    if (!ctx->ws_cleared[WS_ATTEND]) {
        hipLaunchKernelGGL(mx4_attend_zero, dim3(mx4::AT_TICKETS / 256), dim3(256), 0, ctx->stream, static_cast<unsigned*>(shared));
        ADADIM_LAUNCH_CHECK(ctx, "mx4_attend_zero");
        adadim_workspace_cleared(ctx, WS_ATTEND);
    }
    return ADADIM_OK;
}
