// Rows of 16- or 32-bit values to microscaled 4-bit codes and back.
//
// Block of 32 values, amax the largest magnitude:  e = floor(log2 amax) - 2 (so that amax / 2^e lies in [4, 8)), at least
// -127; code = sign and the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 to |x| / 2^e, ties to the even mantissa, at most 6; the
// stored scale is e + 127.  floor(log2) is the exponent field of amax as fp32 (every fp16 value is a normal fp32 number;
// an fp32 subnormal has field 0 and ends at e = -127 as it must).  A block of zeros has scale 1.  A block with an
// infinity or a NaN has the scale NaN (255) and codes of 0.
//
// Bound by HBM: 2 (4) bytes read and 17/32 written per value.  A workgroup owns 512 columns x 4 or 16 rows; a lane
// holds 8 consecutive values, so a wave's load is one contiguous KB (two for fp32), a block lives in a quad (its amax meets by
// DPP), a piece in a row of 16 lanes, and codes leave as 256 contiguous bytes.  The scale words of the tile are
// collected in LDS and leave as runs along the rows, the way they are stored.
// 28672 x 8192 fp16: 102 us there, one call behind the other (5.8 TB/s; a large copy reaches 5.06, with half of its bytes written), 126 us there and
// 92 us back in turn; 16 x 4096 2.5 and 2.3 us.  With dW: 183 us for F16, 294 for F32 (5.8, 5.2 TB/s); 486 for F16_SCALED (2.2 TB/s), whose
// layout takes 64 bytes of a row at a time, rows apart from wave to wave.
#include "mx4.h"

namespace {

using namespace mx4;

constexpr int QT_COLS = 512, QT_WAVES = 4;

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xF, 0xF, false));
}
constexpr int QUAD_XOR1 = 0xB1, QUAD_XOR2 = 0x4E, ROW_ROR4 = 0x124, ROW_ROR8 = 0x128;

// dW = x - value, one rounding, in the type and layout of adadim_quantize.
struct DwOut {
    void* p;
    int type;
    const float* colscale;
    int64_t rows;
};

template <class T, int ITER, bool DW>
__global__ __launch_bounds__(64 * QT_WAVES) void mx4_quantize_rows(const T* __restrict__ X, int64_t rows, int64_t cols, int64_t ldx,
                                                                   uint32_t col_tiles, uint8_t* __restrict__ codes,
                                                                   uint32_t* __restrict__ scales, DwOut dw) {
    constexpr int ROWS = QT_WAVES * ITER;
    __shared__ uint32_t s_word[4][ROWS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t np = pieces(cols), row0 = int64_t(blockIdx.x / col_tiles) * ROWS, c0 = int64_t(blockIdx.x % col_tiles) * QT_COLS;
    const int64_t c = c0 + 8 * lane;
    const bool inside = c < np * PIECE;
    const int have = static_cast<int>(min(int64_t(8), max(int64_t(0), cols - c)));
    typename Chunk<T, 8>::vec x[ITER];
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int64_t row = row0 + wave + QT_WAVES * i;
        x[i] = row < rows && have > 0 ? Chunk<T, 8>::load(X + row * ldx + c, have) : typename Chunk<T, 8>::vec{};
    }
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int64_t row = row0 + wave + QT_WAVES * i;
        float f[8];
        uint32_t big = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f[j] = static_cast<float>(x[i][j]);
            big = max(big, __float_as_uint(f[j]) & 0x7fffffffu);
        }
        big = max(big, dpp<QUAD_XOR1>(big));
        big = max(big, dpp<QUAD_XOR2>(big));
        const uint32_t field = big >> 23;
        const uint32_t byte = big == 0 ? 127u : field == 255u ? 255u : max(field, 2u) - 2u;
        const float s = scale_operand(byte);
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], s, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], s, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], s, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], s, 3);
        if (byte == 255u) w = 0;
        uint32_t word = byte << (8 * ((lane >> 2) & 3));
        word |= dpp<ROW_ROR4>(word);
        word |= dpp<ROW_ROR8>(word);
        if ((lane & 15) == 0) s_word[lane >> 4][wave + QT_WAVES * i] = word;
        if (row < rows && inside) {
            *reinterpret_cast<uint32_t*>(codes + row * (np * PIECE_BYTES) + (c >> 1)) = w;
            if constexpr (DW) {
                if (have > 0) {
                    float v[8];
                    values8(w, s, v);
                    if (dw.type == ADADIM_DW_F32) {
                        Chunk<float, 8>::vec d;
#pragma unroll
                        for (int j = 0; j < 8; ++j) d[j] = f[j] - v[j];
                        Chunk<float, 8>::store(static_cast<float*>(dw.p) + row * cols + c, have, d);
                    } else {
                        Chunk<_Float16, 8>::vec d;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            float r = f[j] - v[j];
                            if (dw.type == ADADIM_DW_F16_SCALED && j < have) r *= dw.colscale[c + j];
                            d[j] = static_cast<_Float16>(r);
                        }
                        // eight columns from a multiple of 8 lie together in the scoring layout too
                        const int64_t at = dw.type == ADADIM_DW_F16_SCALED ? score_index(row, c, dw.rows, cols) : row * cols + c;
                        Chunk<_Float16, 8>::store(static_cast<_Float16*>(dw.p) + at, have, d);
                    }
                }
            }
        }
    }
    __syncthreads();
    const int p = threadIdx.x / ROWS, r = threadIdx.x % ROWS;
    if (p < 4 && c0 / PIECE + p < np && row0 + r < rows) scales[(c0 / PIECE + p) * rows + row0 + r] = s_word[p][r];
}

// The way back: a lane takes a word of codes, writes eight values.
template <class T, int ITER>
__global__ __launch_bounds__(64 * QT_WAVES) void mx4_dequantize_rows(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                                     int64_t rows, int64_t cols, uint32_t col_tiles,
                                                                     T* __restrict__ Y, int64_t ldy) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t np = pieces(cols), row0 = int64_t(blockIdx.x / col_tiles) * (QT_WAVES * ITER);
    const int64_t c = int64_t(blockIdx.x % col_tiles) * QT_COLS + 8 * lane;
    if (c >= cols) return;
    const int have = static_cast<int>(min(int64_t(8), cols - c));
    uint32_t w[ITER], byte[ITER];
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int64_t row = min(row0 + wave + QT_WAVES * i, rows - 1);
        w[i] = *reinterpret_cast<const uint32_t*>(codes + row * (np * PIECE_BYTES) + (c >> 1));
        byte[i] = scales[((c / PIECE) * rows + row) * 4 + ((c >> 5) & 3)];
    }
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int64_t row = row0 + wave + QT_WAVES * i;
        if (row >= rows) return;
        float v[8];
        values8(w[i], scale_operand(byte[i]), v);
        typename Chunk<T, 8>::vec o;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = static_cast<T>(v[j]);
        Chunk<T, 8>::store(Y + row * ldy + c, have, o);
    }
}

}  // namespace

// 16 rows per workgroup where that leaves at least 1024 of them (four a compute unit), else 4.
static inline bool deep_tiles(int64_t rows, int64_t col_tiles) { return (rows + 15) / 16 * col_tiles >= 1024; }

int launch_mx4_quantize(adadim_ctx* ctx, const void* X, int x_type, int64_t rows, int64_t cols, int64_t ldx, uint8_t* codes,
                        uint8_t* scales, void* dW, int dW_dtype, const float* colscale) {
    const int64_t ct = (cols + QT_COLS - 1) / QT_COLS;
    const bool deep = deep_tiles(rows, ct);
    const dim3 grid(static_cast<unsigned>((rows + (deep ? 15 : 3)) / (deep ? 16 : 4) * ct)), block(64 * QT_WAVES);
    const DwOut dw{dW, dW_dtype, colscale, rows};
    uint32_t* sw = reinterpret_cast<uint32_t*>(scales);
    ProfScope prof(ctx, "mx4_quantize_rows");
#define MX4_Q(T, ITER, DW) \
    hipLaunchKernelGGL((mx4_quantize_rows<T, ITER, DW>), grid, block, 0, ctx->stream, static_cast<const T*>(X), rows, cols, ldx, static_cast<uint32_t>(ct), codes, sw, dw)
#define MX4_QT(T)                                                              \
    do {                                                                       \
        if (deep) { if (dW) MX4_Q(T, 4, true); else MX4_Q(T, 4, false); }      \
        else      { if (dW) MX4_Q(T, 1, true); else MX4_Q(T, 1, false); }      \
    } while (0)
    if (x_type == ADADIM_TYPE_F16) MX4_QT(_Float16);
    else if (x_type == ADADIM_TYPE_BF16) MX4_QT(__bf16);
    else MX4_QT(float);
#undef MX4_QT
#undef MX4_Q
    ADADIM_LAUNCH_CHECK(ctx, "mx4_quantize_rows");
    return ADADIM_OK;
}

int launch_mx4_dequantize(adadim_ctx* ctx, const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* Y,
                          int y_type, int64_t ldy) {
    const int64_t ct = (cols + QT_COLS - 1) / QT_COLS;
    const bool deep = deep_tiles(rows, ct);
    const dim3 grid(static_cast<unsigned>((rows + (deep ? 15 : 3)) / (deep ? 16 : 4) * ct)), block(64 * QT_WAVES);
    ProfScope prof(ctx, "mx4_dequantize_rows");
#define MX4_D(T, ITER) \
    hipLaunchKernelGGL((mx4_dequantize_rows<T, ITER>), grid, block, 0, ctx->stream, codes, scales, rows, cols, static_cast<uint32_t>(ct), static_cast<T*>(Y), ldy)
#define MX4_DT(T) do { if (deep) MX4_D(T, 4); else MX4_D(T, 1); } while (0)
    if (y_type == ADADIM_TYPE_F16) MX4_DT(_Float16);
    else if (y_type == ADADIM_TYPE_BF16) MX4_DT(__bf16);
    else MX4_DT(float);
#undef MX4_DT
#undef MX4_D
    ADADIM_LAUNCH_CHECK(ctx, "mx4_dequantize_rows");
    return ADADIM_OK;
}
