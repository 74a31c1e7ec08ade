// C-ABI entry points of the microscaled 4-bit operators and of the experts' routing: argument validation.  As in api.hip every
// check runs before the first HIP call.
#include "mx4_matmul.h"

int launch_mx4_quantize(adadim_ctx* ctx, const void* X, int x_type, int64_t rows, int64_t cols, int64_t ldx, uint8_t* codes,
                        uint8_t* scales, void* dW, int dW_dtype, const float* colscale);
int launch_mx4_dequantize(adadim_ctx* ctx, const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* Y,
                          int y_type, int64_t ldy);
int launch_mx4_matmul(adadim_ctx* ctx, const mx4::Product& a, int x_type);
int launch_expert_route(adadim_ctx* ctx, const void* logits, int type, int64_t tokens, int64_t ldl, int experts, int k, int renormalize,
                        int32_t* chosen, float* weights, int32_t* offsets, int32_t* rows, int32_t* slots);
int launch_expert_combine(adadim_ctx* ctx, const void* Z, int z_type, int64_t n_rows, int64_t cols, int64_t ldz, const int32_t* slots,
                          const float* weights, int64_t tokens, int k, void* Y, int y_type, int64_t ldy);

static bool is_float_type(int t) { return t == ADADIM_TYPE_F16 || t == ADADIM_TYPE_BF16 || t == ADADIM_TYPE_F32; }
static int type_size(int t) { return t == ADADIM_TYPE_F32 ? 4 : 2; }
static bool aligned_to(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

constexpr int64_t MOST_ROWS = int64_t(1) << 30, MOST_COLS = int64_t(1) << 24;

extern "C" {

int64_t adadim_mx4_code_bytes(int64_t rows, int64_t cols) {
    return rows <= 0 || cols <= 0 ? 0 : rows * mx4::pieces(cols) * mx4::PIECE_BYTES;
}
int64_t adadim_mx4_scale_bytes(int64_t rows, int64_t cols) { return rows <= 0 || cols <= 0 ? 0 : rows * mx4::pieces(cols) * 4; }

int adadim_mx4_quantize(adadim_ctx* ctx, const void* X, int x_type, int64_t rows, int64_t cols, int64_t ldx, uint8_t* codes,
                        uint8_t* scales, void* dW, int dW_dtype, const float* colscale) {
    if (!ctx) return ADADIM_ENULL;
    const char* me = "adadim_mx4_quantize";
    if (!is_float_type(x_type)) return adadim_fail(ctx, ADADIM_EINVAL, "%s: x_type must be F16, BF16 or F32, got %d", me, x_type);
    if (rows < 0 || cols <= 0 || ldx < cols || rows > MOST_ROWS || cols > MOST_COLS || !launchable((rows + 15) / 16 * ((cols + 511) / 512), 256))
        return adadim_fail(ctx, ADADIM_EINVAL, "%s: need rows >= 0, cols > 0, ldx >= cols in range (rows=%lld cols=%lld ldx=%lld)", me,
                           (long long)rows, (long long)cols, (long long)ldx);
    if (dW && dW_dtype != ADADIM_DW_F32 && dW_dtype != ADADIM_DW_F16 && dW_dtype != ADADIM_DW_F16_SCALED)
        return adadim_fail(ctx, ADADIM_EINVAL, "%s: unknown dW_dtype %d", me, dW_dtype);
    if (rows == 0) return ADADIM_OK;
    if (!X || !codes || !scales) return adadim_fail(ctx, ADADIM_ENULL, "%s: X, codes or scales is NULL", me);
    if (dW && dW_dtype == ADADIM_DW_F16_SCALED && !colscale)
        return adadim_fail(ctx, ADADIM_ENULL, "%s: colscale is NULL with dW_dtype F16_SCALED", me);
    if (!aligned16(codes) || !aligned_to(scales, 4) || !aligned_to(X, type_size(x_type)) ||
        (dW && !aligned_to(dW, dW_dtype == ADADIM_DW_F32 ? 4 : 2)) || (dW && dW_dtype == ADADIM_DW_F16_SCALED && !aligned_to(colscale, 4)))
        return adadim_fail(ctx, ADADIM_EALIGN, "%s: codes must be 16-byte, scales 4-byte, X and dW element aligned", me);
    return launch_mx4_quantize(ctx, X, x_type, rows, cols, ldx, codes, scales, dW, dW_dtype, colscale);
}

int adadim_mx4_dequantize(adadim_ctx* ctx, const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* Y, int y_type,
                          int64_t ldy) {
    if (!ctx) return ADADIM_ENULL;
    const char* me = "adadim_mx4_dequantize";
    if (!is_float_type(y_type)) return adadim_fail(ctx, ADADIM_EINVAL, "%s: y_type must be F16, BF16 or F32, got %d", me, y_type);
    if (rows < 0 || cols <= 0 || ldy < cols || rows > MOST_ROWS || cols > MOST_COLS || !launchable((rows + 15) / 16 * ((cols + 511) / 512), 256))
        return adadim_fail(ctx, ADADIM_EINVAL, "%s: need rows >= 0, cols > 0, ldy >= cols in range (rows=%lld cols=%lld ldy=%lld)", me,
                           (long long)rows, (long long)cols, (long long)ldy);
    if (rows == 0) return ADADIM_OK;
    if (!codes || !scales || !Y) return adadim_fail(ctx, ADADIM_ENULL, "%s: codes, scales or Y is NULL", me);
    if (!aligned16(codes) || !aligned_to(scales, 4) || !aligned_to(Y, type_size(y_type)))
        return adadim_fail(ctx, ADADIM_EALIGN, "%s: codes must be 16-byte, scales 4-byte, Y element aligned", me);
    return launch_mx4_dequantize(ctx, codes, scales, rows, cols, Y, y_type, ldy);
}

// what the two products have in common; n_rows: rows of Y
static int product_checked(adadim_ctx* ctx, const char* me, int x_type, const mx4::Product& a) {
    if (x_type != ADADIM_TYPE_F16 && x_type != ADADIM_TYPE_BF16 && x_type != ADADIM_TYPE_MX4)
        return adadim_fail(ctx, ADADIM_EINVAL, "%s: x_type must be F16, BF16 or MX4, got %d", me, x_type);
    if (!is_float_type(a.y_type)) return adadim_fail(ctx, ADADIM_EINVAL, "%s: y_type must be F16, BF16 or F32, got %d", me, a.y_type);
    if (a.tokens < 0 || a.n_rows < 0 || a.out <= 0 || a.in <= 0 || a.tokens > MOST_ROWS || a.n_rows > MOST_ROWS || a.out > MOST_COLS ||
        a.in > MOST_COLS || (x_type != ADADIM_TYPE_MX4 && (a.ldx < a.in || a.ldx > INT32_MAX)) || a.ldy < a.out || a.ldy > INT32_MAX)
        return adadim_fail(ctx, ADADIM_EINVAL,
                           "%s: need rows >= 0, out, in > 0 in range, ldx >= in, ldy >= out (tokens=%lld rows=%lld out=%lld in=%lld "
                           "ldx=%lld ldy=%lld)",
                           me, (long long)a.tokens, (long long)a.n_rows, (long long)a.out, (long long)a.in, (long long)a.ldx, (long long)a.ldy);
    if (a.n_rows == 0) return ADADIM_OK;
    if ((a.tokens > 0 && !a.X) || !a.codes || !a.scales || !a.Y) return adadim_fail(ctx, ADADIM_ENULL, "%s: X, codes, scales or Y is NULL", me);
    if (a.tokens > 0 && x_type == ADADIM_TYPE_MX4 && !a.x_scales)
        return adadim_fail(ctx, ADADIM_ENULL, "%s: x_scales is NULL with x_type MX4", me);
    if (!aligned16(a.codes) || !aligned_to(a.scales, 4) || !aligned_to(a.Y, type_size(a.y_type)) ||
        (x_type == ADADIM_TYPE_MX4 ? !aligned16(a.X) || !aligned_to(a.x_scales, 4) : !aligned_to(a.X, 2)))
        return adadim_fail(ctx, ADADIM_EALIGN, "%s: codes must be 16-byte, scales 4-byte, X and Y element aligned", me);
    return launch_mx4_matmul(ctx, a, x_type);
}

int adadim_mx4_matmul(adadim_ctx* ctx, const void* X, const uint8_t* x_scales, int x_type, int64_t tokens, int64_t ldx,
                      const uint8_t* codes, const uint8_t* scales, int64_t out, int64_t in, void* Y, int y_type, int64_t ldy) {
    if (!ctx) return ADADIM_ENULL;
    const mx4::Product a{X, reinterpret_cast<const uint32_t*>(x_scales), tokens, ldx, tokens, nullptr, false, nullptr, tokens, 1, codes,
                         reinterpret_cast<const uint32_t*>(scales), out, in, Y, y_type, ldy};
    return product_checked(ctx, "adadim_mx4_matmul", x_type, a);
}

int adadim_mx4_matmul_experts(adadim_ctx* ctx, const void* X, const uint8_t* x_scales, int x_type, int64_t tokens, int64_t ldx,
                              const int32_t* rows, int64_t n_rows, const int32_t* offsets, int experts, const uint8_t* codes,
                              const uint8_t* scales, int64_t out, int64_t in, void* Y, int y_type, int64_t ldy) {
    if (!ctx) return ADADIM_ENULL;
    const char* me = "adadim_mx4_matmul_experts";
    if (experts <= 0 || experts > 1024) return adadim_fail(ctx, ADADIM_EINVAL, "%s: experts must be in [1,1024], got %d", me, experts);
    if (!rows && n_rows != tokens && n_rows > 0)
        return adadim_fail(ctx, ADADIM_EINVAL, "%s: without rows X has as many rows as Y (tokens=%lld n_rows=%lld)", me, (long long)tokens,
                           (long long)n_rows);
    if (!offsets) return adadim_fail(ctx, ADADIM_ENULL, "%s: offsets is NULL", me);
    if (!aligned_to(offsets, 4) || !aligned_to(rows, 4)) return adadim_fail(ctx, ADADIM_EALIGN, "%s: offsets and rows must be 4-byte aligned", me);
    const mx4::Product a{X, reinterpret_cast<const uint32_t*>(x_scales), tokens, ldx, tokens, rows, rows != nullptr, offsets, n_rows, experts, codes,
                         reinterpret_cast<const uint32_t*>(scales), out, in, Y, y_type, ldy};
    return product_checked(ctx, me, x_type, a);
}

int adadim_expert_route(adadim_ctx* ctx, const void* logits, int type, int64_t tokens, int64_t ldl, int experts, int k, int renormalize,
                        int32_t* chosen, float* weights, int32_t* offsets, int32_t* rows, int32_t* slots) {
    if (!ctx) return ADADIM_ENULL;
    const char* me = "adadim_expert_route";
    if (!is_float_type(type)) return adadim_fail(ctx, ADADIM_EINVAL, "%s: type must be F16, BF16 or F32, got %d", me, type);
    if (experts <= 0 || experts > 1024 || k <= 0 || k > 32 || k > experts || tokens < 0 || ldl < experts || tokens > MOST_ROWS ||
        tokens * k > INT32_MAX || !launchable((tokens + 63) / 64, 1024) || (renormalize != 0 && renormalize != 1))
        return adadim_fail(ctx, ADADIM_EINVAL,
                           "%s: need 1..1024 experts, 1 <= k <= min(32, experts), ldl >= experts, tokens < 2^28, tokens * k < 2^31, renormalize 0 or 1 "
                           "(tokens=%lld ldl=%lld experts=%d k=%d renormalize=%d)",
                           me, (long long)tokens, (long long)ldl, experts, k, renormalize);
    if (!offsets || (tokens > 0 && (!logits || !chosen || !weights || !rows || !slots)))
        return adadim_fail(ctx, ADADIM_ENULL, "%s: a required pointer is NULL", me);
    if (!aligned_to(logits, type_size(type)) || !aligned_to(chosen, 4) || !aligned_to(weights, 4) || !aligned_to(offsets, 4) ||
        !aligned_to(rows, 4) || !aligned_to(slots, 4))
        return adadim_fail(ctx, ADADIM_EALIGN, "%s: arrays must be element aligned", me);
    return launch_expert_route(ctx, logits, type, tokens, ldl, experts, k, renormalize, chosen, weights, offsets, rows, slots);
}

int adadim_expert_combine(adadim_ctx* ctx, const void* Z, int z_type, int64_t n_rows, int64_t cols, int64_t ldz, const int32_t* slots,
                          const float* weights, int64_t tokens, int k, void* Y, int y_type, int64_t ldy) {
    if (!ctx) return ADADIM_ENULL;
    const char* me = "adadim_expert_combine";
    if (!is_float_type(z_type) || !is_float_type(y_type))
        return adadim_fail(ctx, ADADIM_EINVAL, "%s: types must be F16, BF16 or F32, got %d and %d", me, z_type, y_type);
    if (n_rows < 0 || cols <= 0 || tokens < 0 || k <= 0 || k > 1024 || ldz < cols || ldy < cols || n_rows > MOST_ROWS || tokens > MOST_ROWS ||
        cols > MOST_COLS || !launchable(tokens * ((cols + 2047) / 2048), 256))
        return adadim_fail(ctx, ADADIM_EINVAL,
                           "%s: need n_rows, tokens >= 0, cols > 0, k in [1,1024], ldz, ldy >= cols in range (n_rows=%lld cols=%lld tokens=%lld "
                           "k=%d ldz=%lld ldy=%lld)",
                           me, (long long)n_rows, (long long)cols, (long long)tokens, k, (long long)ldz, (long long)ldy);
    if (tokens == 0) return ADADIM_OK;
    if ((n_rows > 0 && !Z) || !slots || !weights || !Y) return adadim_fail(ctx, ADADIM_ENULL, "%s: Z, slots, weights or Y is NULL", me);
    if (!aligned_to(Z, type_size(z_type)) || !aligned_to(Y, type_size(y_type)) || !aligned_to(slots, 4) || !aligned_to(weights, 4))
        return adadim_fail(ctx, ADADIM_EALIGN, "%s: arrays must be element aligned", me);
    return launch_expert_combine(ctx, Z, z_type, n_rows, cols, ldz, slots, weights, tokens, k, Y, y_type, ldy);
}

}  // extern "C"
