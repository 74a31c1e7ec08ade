// Products with microscaled 4-bit weights: Y = X W^T, alone or grouped by expert.
#include "mx4_matmul.h"

#include <type_traits>

namespace {

using namespace mx4;

constexpr int XF16 = ADADIM_TYPE_F16, XBF16 = ADADIM_TYPE_BF16, XMX4 = ADADIM_TYPE_MX4;

// One lane's share of a piece of X for v_mfma_*_16x16x*: row (lane & 15), block g = lane >> 4 of the piece.
template <int XT>
struct XFrag {
    uint4v v[4];                                  // 32 values of 16 bits
};
template <>
struct XFrag<XMX4> {
    uint4v v[1];
    uint32_t scale;                               // in the low byte
};

template <int XT>
__device__ __forceinline__ XFrag<XT> load_x(const Product& a, int64_t src, int64_t piece, int g) {
    XFrag<XT> x = {};
    if constexpr (XT == XMX4) {
        x.scale = 127u;
        if (src >= 0) {
            x.v[0] = *reinterpret_cast<const uint4v*>(static_cast<const uint8_t*>(a.X) + (src * pieces(a.in) + piece) * PIECE_BYTES + 16 * g);
            x.scale = (a.x_scales[piece * a.tokens + src] >> (8 * g)) & 255u;
        }
    } else if (src >= 0) {
        const int64_t k = piece * PIECE + 32 * g;
        const uint16_t* p = static_cast<const uint16_t*>(a.X) + src * a.ldx + k;
        if (k + 32 <= a.in) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x.v[i] = load_any<uint4v>(p + 8 * i);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const auto c = Chunk<uint16_t, 8>::load(p + 8 * i, static_cast<int>(max(int64_t(0), min(int64_t(8), a.in - k - 8 * i))));
                x.v[i] = __builtin_bit_cast(uint4v, c);
            }
        }
    }
    return x;
}

// acc += W X for one piece.  With 16-bit X the four instructions take elements 8 i .. 8 i + 7 of every lane's block.
template <int XT>
__device__ __forceinline__ float4v step16(uint4v w, uint32_t ws, const XFrag<XT>& x, bool wide, float4v acc) {
    if constexpr (XT == XMX4) {
        int8v a = {}, b = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = static_cast<int>(w[i]);
            b[i] = static_cast<int>(x.v[0][i]);
        }
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, 0, static_cast<int>(ws), 0, static_cast<int>(x.scale));
    } else if constexpr (XT == XBF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values8_bf16(w[i], scale_operand(ws)), __builtin_bit_cast(bf8v, x.v[i]), acc, 0, 0, 0);
        return acc;
    } else {
        if (wide) {                                           // some weight of the step is no fp16 number: both operands in bf16, X in two parts
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                bf8v hi, lo;
                split_f16(__builtin_bit_cast(half8v, x.v[i]), hi, lo);
                const bf8v v = values8_bf16(w[i], scale_operand(ws));
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, hi, acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, lo, acc, 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(values8_f16(w[i], scale_operand(ws)), __builtin_bit_cast(half8v, x.v[i]), acc, 0, 0, 0);
        }
        return acc;
    }
}

// Few rows.  A workgroup owns 16 outputs of one expert and walks the group's rows 16 at a time; its waves deal out the
// pieces of the contraction and add up in LDS, in the order of the waves.
constexpr int RW_WAVES = 8;

template <int XT>
__global__ __launch_bounds__(64 * RW_WAVES) void mx4_rows(Product a) {
    __shared__ float4v s_part[RW_WAVES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4;
    const Group gr = group_of(a, blockIdx.y);
    const int64_t np = pieces(a.in), o0 = int64_t(blockIdx.x) * 16, o = min(o0 + (lane & 15), a.out - 1);
    for (int64_t r0 = gr.lo; r0 < gr.hi; r0 += 16) {
        const int64_t src = source_row(a, r0 + (lane & 15), gr.hi);
        float4v acc = {};
        for (int64_t p = wave; p < np; p += RW_WAVES) {
            const uint4v w = *reinterpret_cast<const uint4v*>(gr.codes + (o * np + p) * PIECE_BYTES + 16 * g);
            const uint32_t ws = (gr.scales[p * a.out + o] >> (8 * g)) & 255u;
            const XFrag<XT> x = load_x<XT>(a, src, p, g);
            acc = step16<XT>(w, ws, x, XT == XF16 && __any(beyond_f16(ws)), acc);
        }
        s_part[wave][lane] = acc;
        __syncthreads();
        if (threadIdx.x < 256) {
            // thread t: output t & 15 of row t >> 4; lane 16 q + row held outputs 4 q .. 4 q + 3 of that row
            const int oo = threadIdx.x & 15, rr = threadIdx.x >> 4;
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < RW_WAVES; ++w) sum += s_part[w][16 * (oo >> 2) + rr][oo & 3];
            if (r0 + rr < gr.hi && o0 + oo < a.out) store_y(a, r0 + rr, o0 + oo, sum);
        }
        __syncthreads();
    }
}

// Rows of X that the tiles' 16-byte transfers cannot take as they lie: copied once, in the order of Y's rows where rows[] is given, to rows of
// whole pieces filled up with zeros.
__global__ __launch_bounds__(256) void mx4_align_rows(Product a, int64_t n, int64_t pitch, uint16_t* __restrict__ to) {
    const int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 8, row = i / pitch, c = i % pitch;
    if (row >= n) return;
    const int64_t src = source_row(a, row, n);
    Chunk<uint16_t, 8>::vec v = {};
    if (c < a.in && src >= 0)
        v = Chunk<uint16_t, 8>::load(static_cast<const uint16_t*>(a.X) + src * a.ldx + c, static_cast<int>(min(int64_t(8), a.in - c)));
    *reinterpret_cast<Chunk<uint16_t, 8>::vec*>(to + i) = v;
}

}  // namespace

#include "mx4_tiles.h"

namespace {

PerDeviceOnce g_tiles_once;

template <int XT, int BM, int BN, int WT, int WO>
constexpr int tile_lds() {
    return 2 * (BM * (XT == XMX4 ? 128 : 256) + (XT == XMX4 ? BN * 128 : 0));
}

template <int XT>
hipError_t raise_lds() {
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&mx4_tiles<XT, 256, 256, 2, 4>), hipFuncAttributeMaxDynamicSharedMemorySize, tile_lds<XT, 256, 256, 2, 4>());
    if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void*>(&mx4_tiles<XT, 128, 128, 2, 2>), hipFuncAttributeMaxDynamicSharedMemorySize, tile_lds<XT, 128, 128, 2, 2>());
    return e;
}

// Row tiles that the launch has to have workgroups for: each group may end in a tile of its own.
inline int64_t most_row_tiles(const Product& a, int bm) {
    return a.offsets ? a.n_rows / bm + min(int64_t(a.experts), a.n_rows) : (a.n_rows + bm - 1) / bm;
}

template <int XT, int BM, int BN, int WT, int WO>
int launch_tiles(adadim_ctx* ctx, const Product& a) {
    const int64_t tiles = most_row_tiles(a, BM) * ((a.out + BN - 1) / BN);
    if (tiles > INT32_MAX - 8) return adadim_fail(ctx, ADADIM_EINVAL, "mx4 product: more tiles than a launch has workgroups");
    ProfScope prof(ctx, "mx4_tiles");
    hipLaunchKernelGGL((mx4_tiles<XT, BM, BN, WT, WO>), dim3(static_cast<unsigned>((tiles + 7) / 8 * 8)), dim3(64 * WT * WO),
                       (tile_lds<XT, BM, BN, WT, WO>()), ctx->stream, a);
    ADADIM_LAUNCH_CHECK(ctx, "mx4_tiles");
    return ADADIM_OK;
}

// Rows of X (those of a tile, or all that rows[] may name) that 32-bit offsets do not reach.
inline bool far_rows(const Product& a, int x_type) {
    return (a.rows ? a.tokens : 256) * (x_type == XMX4 ? pieces(a.in) * PIECE_BYTES : 2 * a.ldx) > int64_t(UINT32_MAX);
}

template <int XT>
int launch_many(adadim_ctx* ctx, Product a) {
    ADADIM_HIP_TRY(ctx, g_tiles_once.run([] {
        hipError_t e = raise_lds<XF16>();
        if (e == hipSuccess) e = raise_lds<XBF16>();
        if (e == hipSuccess) e = raise_lds<XMX4>();
        return e;
    }));
    if (XT != XMX4 && (!aligned16(a.X) || a.ldx % 8 != 0 || a.in % 8 != 0 || far_rows(a, XT))) {
        const int64_t pitch = pieces(a.in) * PIECE, blocks = (a.n_rows * pitch / 8 + 255) / 256;
        if (blocks > INT32_MAX) return adadim_fail(ctx, ADADIM_EINVAL, "mx4 product: X too large to be copied to aligned rows");
        uint16_t* to = static_cast<uint16_t*>(adadim_workspace(ctx, WS_MX4_X, size_t(a.n_rows) * size_t(pitch) * 2));
        if (!to) return ADADIM_EHIP;
        ProfScope prof(ctx, "mx4_align_rows");
        hipLaunchKernelGGL(mx4_align_rows, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, ctx->stream, a, a.n_rows, pitch, to);
        ADADIM_LAUNCH_CHECK(ctx, "mx4_align_rows");
        a.X = to;
        a.ldx = pitch;
        a.tokens = a.n_rows;
        a.rows = nullptr;
    }
    const int64_t wide = most_row_tiles(a, 256) * ((a.out + 255) / 256);
    return wide >= 200 ? launch_tiles<XT, 256, 256, 2, 4>(ctx, a) : launch_tiles<XT, 128, 128, 2, 2>(ctx, a);
}

}  // namespace

int launch_mx4_matmul(adadim_ctx* ctx, const mx4::Product& a, int x_type) {
    if (a.tokens > 0 && a.n_rows / a.experts > 64 && !(x_type == XMX4 && far_rows(a, x_type))) {
        if (x_type == XF16) return launch_many<XF16>(ctx, a);
        if (x_type == XBF16) return launch_many<XBF16>(ctx, a);
        return launch_many<XMX4>(ctx, a);
    }
    const dim3 grid(static_cast<unsigned>((a.out + 15) / 16), static_cast<unsigned>(a.experts)), block(64 * RW_WAVES);
    ProfScope prof(ctx, "mx4_rows");
    if (x_type == XF16) hipLaunchKernelGGL((mx4_rows<XF16>), grid, block, 0, ctx->stream, a);
    else if (x_type == XBF16) hipLaunchKernelGGL((mx4_rows<XBF16>), grid, block, 0, ctx->stream, a);
    else hipLaunchKernelGGL((mx4_rows<XMX4>), grid, block, 0, ctx->stream, a);
    ADADIM_LAUNCH_CHECK(ctx, "mx4_rows");
    return ADADIM_OK;
}
