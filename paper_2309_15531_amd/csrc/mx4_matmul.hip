// Products with microscaled 4-bit weights: Y = X W^T, alone or grouped by expert.
#include "mx4_matmul.h"
#include "mx4_plan.h"

#include <type_traits>

namespace {

using namespace mx4;

constexpr int XF16 = ADADIM_TYPE_F16, XBF16 = ADADIM_TYPE_BF16, XMX4 = ADADIM_TYPE_MX4;

// Few rows.  A workgroup owns 16 NT outputs of one expert and walks the group's rows 16 MT at a time.  Its eight waves deal out the pieces of
// the contraction and add up in LDS in the order of the waves.  With shares (one weight, all rows in one pass) gridDim.z workgroups
// split the contraction: each leaves its sums in `part`, and the last to finish adds them up in the order of the shares.  Partial sums travel
// as relaxed atomics at device scope, past the XCDs' caches; a workgroup waits for its stores before it counts itself in, and
// the last one clears the counter.
//
// v_mfma_*_16x16x*: lane (r = lane & 15, g = lane >> 4) holds block g of a piece of row r of W, and of X.  With 16-bit X four instructions
// take values 8 i .. 8 i + 7 of every lane's block.
//
// Bound by the read of W while the rows are few.  What a wave issues a piece counts too: the piece's number is the same in all lanes, so
// addresses are made in scalar registers, and X is read through a buffer descriptor, in which an offset behind the end stands for a row that
// does not exist: it costs no access and reads as zeros.
//
// Eight waves, so that a wave has few pieces one after the other (4 at 4096 deep); NT by the estimates of mx4_plan.h: more outputs of a
// workgroup read X less often, fewer give more workgroups.  With weights that come from memory: 1 token, 28672 -> 8192, mx4 X 24.6 to
// 28.7 us (4.4 to 5.1 TB/s), 8192 -> 28672 fp16 30.5 us (4.1 TB/s), 4096 -> 11008 8.2 to 9.0 us (2.7 to 2.9 TB/s: a launch's start is 3 us of it); 16
// tokens x 2 of 8 experts, 4096 -> 11008 fp16 45 us (4.2 TB/s).  Where there are more rows every workgroup draws all of X through the L2: 16 tokens,
// 4096 -> 11008, 11.8 us.  Deeper unrolling, a second set of registers for the next piece, and X turned in LDS gained
// nothing.
constexpr int RW_WAVES = 8;
constexpr uint32_t NO_ROW = 0x80000000u;          // an offset that no X has (the host copies X where it is larger)

template <int XT>
struct XFrag {
    uint4v v[XT == XMX4 ? 1 : 4];
    uint32_t scale;                               // mx4: of the four blocks
};

// acc += W X for one piece.  wide: a weight has gone by that no fp16 number holds.
template <int XT, int NT, int MT>
__device__ __forceinline__ void piece16(const uint4v (&w)[NT], const uint32_t (&word)[NT], const XFrag<XT> (&x)[MT], int g, float4v (&acc)[NT][MT], bool& wide) {
    if constexpr (XT == XMX4) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                int8v av = {}, bv = {};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    av[i] = static_cast<int>(w[n][i]);
                    bv[i] = static_cast<int>(x[m].v[0][i]);
                }
                acc[n][m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, acc[n][m], 4, 4, 0, static_cast<int>(word[n] >> (8 * g)), 0,
                                                                             static_cast<int>(x[m].scale >> (8 * g)));
            }
    } else {
        float sc[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint32_t byte = (word[n] >> (8 * g)) & 255u;
            sc[n] = scale_operand(byte);
            if constexpr (XT == XF16) wide |= beyond_f16(byte);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if constexpr (XT == XF16) {
                    const half8v v = values8_f16(w[n][i], sc[n]);
#pragma unroll
                    for (int m = 0; m < MT; ++m)
                        acc[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, __builtin_bit_cast(half8v, x[m].v[i]), acc[n][m], 0, 0, 0);
                } else {
                    const bf8v v = values8_bf16(w[n][i], sc[n]);
#pragma unroll
                    for (int m = 0; m < MT; ++m)
                        acc[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf8v, x[m].v[i]), acc[n][m], 0, 0, 0);
                }
            }
    }
}

// The n-th of the groups that have rows; -1 behind the last.  Where there are fewer rows than experts the launch has workgroups for as many groups
// as there are rows: 2 tokens x 2 of 64 experts, 768 -> 9984, mx4, took 22.9 us with workgroups for all 64, 8.1 so.
__device__ __forceinline__ int filled_group(const Product& a, int n, int lane) {
    for (int e0 = 0; e0 < a.experts; e0 += 64) {
        bool has = false;
        if (e0 + lane < a.experts) {
            const Group g = group_of(a, e0 + lane);
            has = g.hi > g.lo;
        }
        const uint64_t all = __ballot(has);
        const uint64_t mine = __ballot(has && __popcll(all & ((uint64_t(1) << lane) - 1)) == n);
        if (mine) return e0 + __builtin_ctzll(mine);
        n -= __popcll(all);
    }
    return -1;
}

// SHIFT: rows of 16-bit X that begin in the middle of a word.  They are read from the word's begin on, one word more, and moved into place.
template <int XT, int NT, int MT, bool SHIFT>
__global__ __launch_bounds__(64 * RW_WAVES) void mx4_rows(ProductArgs args, void* shared) {
    const Product a = args.open();
    float* const part = parts_of(shared);
    unsigned* const ticket = tickets_of(shared);
    constexpr int TILES = NT * MT, ROUND = TILES < 4 ? TILES : 4;                // tiles added up at a time
    __shared__ float4v s_part[RW_WAVES][ROUND][64];
    __shared__ unsigned s_ticket;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    const int expert = gridDim.y < static_cast<unsigned>(a.experts) ? filled_group(a, blockIdx.y, lane) : static_cast<int>(blockIdx.y);
    if (expert < 0) return;
    const Group gr = group_of(a, expert);
    const int np = static_cast<int>(pieces(a.in));
    const int64_t o0 = int64_t(blockIdx.x) * (16 * NT);
    const int p_lo = static_cast<int>(int64_t(np) * blockIdx.z / gridDim.z), p_hi = static_cast<int>(int64_t(np) * (blockIdx.z + 1) / gridDim.z);
    const int p_full = XT == XMX4 ? p_hi : min(p_hi, static_cast<int>(a.in / PIECE));          // pieces whose X is whole
    const uint8_t* const w_base = gr.codes + o0 * np * PIECE_BYTES;
    const uint32_t* const s_base = gr.scales + o0;
    uint32_t wo[NT], so[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        so[n] = static_cast<uint32_t>(min(int64_t(16 * n + (lane & 15)), a.out - 1 - o0));
        wo[n] = so[n] * (static_cast<uint32_t>(np) * PIECE_BYTES) + 16 * g;
    }
    const uint32_t x_pitch = XT == XMX4 ? np * PIECE_BYTES : static_cast<uint32_t>(2 * a.ldx);

    for (int64_t r0 = gr.lo; r0 < gr.hi; r0 += 16 * MT) {
        const int64_t first = a.gather ? 0 : r0;              // the row of X that offsets are taken from
        const char* x_base = static_cast<const char*>(a.X) + first * x_pitch;
        uint32_t skew = 0;
        if constexpr (SHIFT) {
            skew = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(x_base) & 2u);
            x_base -= skew;
        }
        const auto x_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(x_base), 0, NO_ROW, 0x00027000);
        uint32_t xo[MT], xso[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int64_t src = source_row(a, r0 + 16 * m + (lane & 15), gr.hi);
            xso[m] = src < 0 ? 0u : static_cast<uint32_t>(src - first);
            xo[m] = src < 0 ? NO_ROW : xso[m] * x_pitch + (XT == XMX4 ? 16 : 64) * g + skew;
        }
        float4v acc[NT][MT];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[n][m] = float4v{};
        bool wide = false;
        for (int p = p_lo + wave; p < p_full; p += RW_WAVES) {
            uint4v w[NT];
            uint32_t word[NT];
            XFrag<XT> x[MT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                w[n] = *reinterpret_cast<const uint4v*>(w_base + int64_t(p) * PIECE_BYTES + wo[n]);
                word[n] = (s_base + int64_t(p) * a.out)[so[n]];
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if constexpr (XT == XMX4) {
                    x[m].v[0] = __builtin_bit_cast(uint4v, __builtin_amdgcn_raw_buffer_load_b128(x_rsrc, xo[m], p * PIECE_BYTES, 0));
                    x[m].scale = (a.x_scales + int64_t(p) * a.x_rows + first)[xso[m]];
                } else if constexpr (SHIFT) {
                    const uint32_t at = xo[m] & ~3u, shift = 8 * (xo[m] & 2u);
                    uint32_t d[17];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint4v q = __builtin_bit_cast(uint4v, __builtin_amdgcn_raw_buffer_load_b128(x_rsrc, at + 16 * i, p * (2 * PIECE), 0));
#pragma unroll
                        for (int j = 0; j < 4; ++j) d[4 * i + j] = q[j];
                    }
                    d[16] = __builtin_amdgcn_raw_buffer_load_b32(x_rsrc, shift ? at + 64 : NO_ROW, p * (2 * PIECE), 0);
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[m].v[i / 4][i % 4] = __builtin_amdgcn_alignbit(d[i + 1], d[i], shift);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        x[m].v[i] = __builtin_bit_cast(uint4v, __builtin_amdgcn_raw_buffer_load_b128(x_rsrc, xo[m] + 16 * i, p * (2 * PIECE), 0));
                }
            }
            piece16<XT, NT, MT>(w, word, x, g, acc, wide);
        }
        if constexpr (XT != XMX4) {
            if (p_full < p_hi && wave == (p_full - p_lo) % RW_WAVES) {           // the piece in which the rows end
                uint4v w[NT];
                uint32_t word[NT];
                XFrag<XT> x[MT];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    w[n] = *reinterpret_cast<const uint4v*>(w_base + int64_t(p_full) * PIECE_BYTES + wo[n]);
                    word[n] = (s_base + int64_t(p_full) * a.out)[so[n]];
                }
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int left = static_cast<int>(a.in - int64_t(p_full) * PIECE) - 32 * g - 8 * i;
                        Chunk<uint16_t, 8>::vec c = {};
                        if (xo[m] != NO_ROW)
                            c = Chunk<uint16_t, 8>::load(reinterpret_cast<const uint16_t*>(x_base) + xo[m] / 2 + int64_t(p_full) * PIECE + 8 * i, min(8, max(0, left)));
                        x[m].v[i] = __builtin_bit_cast(uint4v, c);
                    }
                piece16<XT, NT, MT>(w, word, x, g, acc, wide);
            }
        }
        if constexpr (XT == XF16) {
            if (__any(wide)) {                                // this wave's share once more with both operands in bf16, X in two parts
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int m = 0; m < MT; ++m) acc[n][m] = float4v{};
                for (int p = p_lo + wave; p < p_hi; p += RW_WAVES)
#pragma unroll 1
                    for (int i = 0; i < 4; ++i) {
                        bf8v hi[MT], lo[MT];
#pragma unroll
                        for (int m = 0; m < MT; ++m) {
                            const int64_t left = a.in - int64_t(p) * PIECE - 32 * g - 8 * i;
                            Chunk<_Float16, 8>::vec x = {};
                            if (xo[m] != NO_ROW)
                                x = Chunk<_Float16, 8>::load(reinterpret_cast<const _Float16*>(x_base) + xo[m] / 2 + int64_t(p) * PIECE + 8 * i, static_cast<int>(min(int64_t(8), max(int64_t(0), left))));
                            split_f16(x, hi[m], lo[m]);
                        }
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const uint32_t w = *reinterpret_cast<const uint32_t*>(w_base + int64_t(p) * PIECE_BYTES + wo[n] + 4 * i);
                            const bf8v v = values8_bf16(w, scale_operand(((s_base + int64_t(p) * a.out)[so[n]] >> (8 * g)) & 255u));
#pragma unroll
                            for (int m = 0; m < MT; ++m) {
                                acc[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, hi[m], acc[n][m], 0, 0, 0);
                                acc[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, lo[m], acc[n][m], 0, 0, 0);
                            }
                        }
                    }
            }
        }
        // the sums of the waves: a thread takes output oo of row rr, which lane 16 (oo / 4) + rr of every wave holds
        auto place = [&](int t, int v, int64_t& row, int64_t& col) {
            const int oo = v & 15, rr = (v >> 4) & 15;
            row = r0 + 16 * (t % MT) + rr;
            col = o0 + 16 * (t / MT) + oo;
        };
#pragma unroll
        for (int t0 = 0; t0 < TILES; t0 += ROUND) {
            if (t0 > 0 || r0 > gr.lo) __syncthreads();
#pragma unroll
            for (int t = 0; t < ROUND; ++t) s_part[wave][t][lane] = acc[(t0 + t) / MT][(t0 + t) % MT];
            __syncthreads();
            for (int v = threadIdx.x; v < 256 * ROUND; v += 64 * RW_WAVES) {
                const int t = v >> 8, oo = v & 15, rr = (v >> 4) & 15;
                float sum = 0.0f;
#pragma unroll
                for (int w = 0; w < RW_WAVES; ++w) sum += s_part[w][t][16 * (oo >> 2) + rr][oo & 3];
                int64_t row, col;
                place(t0 + t, v, row, col);
                if (row >= gr.hi || col >= a.out) continue;
                if (gridDim.z > 1)
                    __hip_atomic_store(part + (int64_t(blockIdx.z) * a.n_rows + row) * a.out + col, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                else
                    store_y(a, row, col, a.rows && source_row(a, row, gr.hi) < 0 ? 0.0f : sum);
            }
        }
        if (gridDim.z > 1) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (threadIdx.x == 0) s_ticket = __hip_atomic_fetch_add(ticket + blockIdx.x, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __syncthreads();
            if (s_ticket != gridDim.z - 1) return;
            if (threadIdx.x == 0) __hip_atomic_store(ticket + blockIdx.x, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            for (int v = threadIdx.x; v < 256 * TILES; v += 64 * RW_WAVES) {
                int64_t row, col;
                place(v >> 8, v, row, col);
                if (row >= gr.hi || col >= a.out) continue;
                const float* p = part + row * a.out + col;
                float sum = 0.0f;
                for (unsigned z0 = 0; z0 < gridDim.z; z0 += 8) {
                    float q[8];
#pragma unroll
                    for (unsigned z = 0; z < 8; ++z)
                        q[z] = z0 + z < gridDim.z ? __hip_atomic_load(p + int64_t(z0 + z) * a.n_rows * a.out, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0f;
#pragma unroll
                    for (unsigned z = 0; z < 8; ++z) sum += q[z];
                }
                store_y(a, row, col, sum);
            }
        }
    }
}

// X in the order of Y's rows, for kernels that read 16 bytes at a time, reach rows by 32-bit offsets and read another row in place of one that
// does not exist: copied where it does not lie so.
// 16-bit rows become whole pieces, filled up with zeros.  PITCH: bytes of a row.
template <bool MX>
__global__ __launch_bounds__(256) void mx4_copy_rows(ProductArgs args, int64_t pitch, uint8_t* __restrict__ to, uint32_t* __restrict__ to_scales) {
    const Product a = args.open();
    const int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 16, row = i / pitch, c = i % pitch;
    if (row >= a.n_rows) return;
    const int64_t src = source_row(a, row, a.n_rows);
    uint4v v = {};
    if constexpr (MX) {
        if (src >= 0) v = *reinterpret_cast<const uint4v*>(static_cast<const uint8_t*>(a.X) + src * pitch + c);
        if (c % PIECE_BYTES == 0) {
            const int64_t p = c / PIECE_BYTES;
            to_scales[p * a.n_rows + row] = src >= 0 ? a.x_scales[p * a.x_rows + src] : ONE_WORD;
        }
    } else if (c < 2 * a.in && src >= 0)
        v = __builtin_bit_cast(uint4v, Chunk<uint16_t, 8>::load(static_cast<const uint16_t*>(a.X) + src * a.ldx + c / 2, static_cast<int>(min(int64_t(8), a.in - c / 2))));
    *reinterpret_cast<uint4v*>(to + i) = v;
}

}  // namespace

#include "mx4_ring.h"

namespace {

static_assert(MOST_SHARED <= SHARE_TICKETS, "a counter for each tile that is shared");
__global__ void mx4_zero_tickets(unsigned* ticket) { ticket[threadIdx.x] = 0u; }

// The counters and room for `bytes` of sums.
int shares(adadim_ctx* ctx, size_t bytes, void*& shared) {
    shared = adadim_workspace(ctx, WS_MX4_PART, SHARE_TICKETS * 4 + bytes);
    if (!shared) return ADADIM_EHIP;
    if (!ctx->ws_cleared[WS_MX4_PART]) {
        hipLaunchKernelGGL(mx4_zero_tickets, dim3(1), dim3(SHARE_TICKETS), 0, ctx->stream, static_cast<unsigned*>(shared));
        ADADIM_LAUNCH_CHECK(ctx, "mx4_zero_tickets");
        adadim_workspace_cleared(ctx, WS_MX4_PART);
    }
    return ADADIM_OK;
}

template <int BM, int BN, int WT, int WO>
hipError_t raise_tiles() {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&mx4_tiles<BM, BN, WT, WO>), hipFuncAttributeMaxDynamicSharedMemorySize, Tiles<BM, BN, WT, WO>::LDS);
}

// Row tiles that the launch has to have workgroups for: each group may end in a tile of its own.
inline int64_t most_row_tiles(const Product& a, int bm) {
    return a.offsets ? a.n_rows / bm + min(int64_t(a.experts), a.n_rows) : (a.n_rows + bm - 1) / bm;
}

template <int BM, int BN, int WT, int WO>
int launch_tiles(adadim_ctx* ctx, const Product& a) {
    const int64_t tiles = most_row_tiles(a, BM) * ((a.out + BN - 1) / BN);
    if (!launchable(tiles + 7, 64 * WT * WO)) return adadim_fail(ctx, ADADIM_EINVAL, "mx4 product: more tiles than a launch has workgroups");
    ProfScope prof(ctx, "mx4_tiles");
    hipLaunchKernelGGL((mx4_tiles<BM, BN, WT, WO>), dim3(static_cast<unsigned>((tiles + 7) / 8 * 8)), dim3(64 * WT * WO),
                       (Tiles<BM, BN, WT, WO>::LDS), ctx->stream, ProductArgs(a));
    ADADIM_LAUNCH_CHECK(ctx, "mx4_tiles");
    return ADADIM_OK;
}

template <int XT, int BM, int BN, int WT, int WO, int NS>
hipError_t raise_ring() {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&mx4_ring<XT, BM, BN, WT, WO, NS>), hipFuncAttributeMaxDynamicSharedMemorySize, Ring<XT, BM, BN, WT, WO, NS>::LDS);
}

template <int XT, int BM, int BN, int WT, int WO, int NS>
int launch_ring(adadim_ctx* ctx, const Product& a, int splits) {
    const int64_t tiles = most_row_tiles(a, BM) * ((a.out + BN - 1) / BN), grid = (tiles + 7) / 8 * 8;
    if (!launchable(tiles + 7, 64 * WT * WO)) return adadim_fail(ctx, ADADIM_EINVAL, "mx4 product: more tiles than a launch has workgroups");
    void* shared = nullptr;
    if (splits > 1) {
        const int rc = shares(ctx, size_t(splits) * size_t(grid) * BM * BN * 4, shared);
        if (rc != ADADIM_OK) return rc;
    }
    ProfScope prof(ctx, "mx4_ring");
    hipLaunchKernelGGL((mx4_ring<XT, BM, BN, WT, WO, NS>), dim3(static_cast<unsigned>(grid), static_cast<unsigned>(splits)), dim3(64 * WT * WO),
                       (Ring<XT, BM, BN, WT, WO, NS>::LDS), ctx->stream, ProductArgs(a), shared);
    ADADIM_LAUNCH_CHECK(ctx, "mx4_ring");
    return ADADIM_OK;
}

// ---- few rows
template <int XT, int NT, int MT>
int launch_rows(adadim_ctx* ctx, const Product& a, int splits) {
    const bool shift = XT != XMX4 && ((reinterpret_cast<uintptr_t>(a.X) & 3u) != 0 || (a.ldx % 2 != 0 && a.tokens > 1));
    const int64_t tiles = (a.out + 16 * NT - 1) / (16 * NT);
    void* shared = nullptr;
    if (splits > 1) {
        const int rc = shares(ctx, size_t(splits) * size_t(a.n_rows) * size_t(a.out) * 4, shared);
        if (rc != ADADIM_OK) return rc;
    }
    ProfScope prof(ctx, "mx4_rows");
    const dim3 grid(static_cast<unsigned>(tiles), static_cast<unsigned>(a.offsets ? min(int64_t(a.experts), a.n_rows) : 1), static_cast<unsigned>(splits)), block(64 * RW_WAVES);
    if constexpr (XT != XMX4) {
        if (shift) {
            hipLaunchKernelGGL((mx4_rows<XT, NT, MT, true>), grid, block, 0, ctx->stream, ProductArgs(a), shared);
            ADADIM_LAUNCH_CHECK(ctx, "mx4_rows");
            return ADADIM_OK;
        }
    }
    hipLaunchKernelGGL((mx4_rows<XT, NT, MT, false>), grid, block, 0, ctx->stream, ProductArgs(a), shared);
    ADADIM_LAUNCH_CHECK(ctx, "mx4_rows");
    return ADADIM_OK;
}


template <int XT, int NT>
int launch_rows_of(adadim_ctx* ctx, const Product& a, const Plan& p) {
    if constexpr (NT < 4) {
        if (p.row_tiles == 4) return launch_rows<XT, NT, 4>(ctx, a, p.shares);
        if (p.row_tiles == 2) return launch_rows<XT, NT, 2>(ctx, a, p.shares);
    }
    return launch_rows<XT, NT, 1>(ctx, a, p.shares);
}

// The kernel of a form.
template <int XT>
int launch_form(adadim_ctx* ctx, const Product& a, const Plan& p) {
    constexpr bool MX = XT == XMX4;
    switch (p.form) {
        case Form::rows: return p.out_tiles == 1 ? launch_rows_of<XT, 1>(ctx, a, p) : p.out_tiles == 2 ? launch_rows_of<XT, 2>(ctx, a, p) : launch_rows_of<XT, 4>(ctx, a, p);
        case Form::ring32: return launch_ring<XT, 32, MX ? 128 : 256, 1, MX ? 4 : 8, MX ? 6 : 4>(ctx, a, p.shares);
        case Form::ring64: return launch_ring<XT, 64, 64, 2, 2, MX ? 4 : 3>(ctx, a, p.shares);
        case Form::ring64w: return launch_ring<XT, 64, 128, MX ? 2 : 1, MX ? 2 : 4, MX ? 4 : 3>(ctx, a, p.shares);
        case Form::mid:
            if constexpr (MX) return launch_tiles<128, 128, 2, 2>(ctx, a);
            else return launch_ring<XT, 128, 128, 2, 4, 3>(ctx, a, p.shares);
        default:                                              // big
            if constexpr (MX) return launch_tiles<256, 256, 2, 4>(ctx, a);
            else return launch_ring<XT, 128, 256, 2, 4, 3>(ctx, a, p.shares);
    }
}

template <int XT>
hipError_t raise_lds() {
    constexpr bool MX = XT == XMX4;
    hipError_t e = raise_ring<XT, 32, MX ? 128 : 256, 1, MX ? 4 : 8, MX ? 6 : 4>();
    if (e == hipSuccess) e = raise_ring<XT, 64, 64, 2, 2, MX ? 4 : 3>();
    if (e == hipSuccess) e = raise_ring<XT, 64, 128, MX ? 2 : 1, MX ? 2 : 4, MX ? 4 : 3>();
    if constexpr (MX) {
        if (e == hipSuccess) e = raise_tiles<128, 128, 2, 2>();
        if (e == hipSuccess) e = raise_tiles<256, 256, 2, 4>();
    } else {
        if (e == hipSuccess) e = raise_ring<XT, 128, 128, 2, 4, 3>();
        if (e == hipSuccess) e = raise_ring<XT, 128, 256, 2, 4, 3>();
    }
    return e;
}

template <int XT>
int launch_product(adadim_ctx* ctx, Product a) {
    constexpr bool MX = XT == XMX4;
    const bool odd = !MX && (!aligned16(a.X) || (a.tokens > 1 && a.ldx % 8 != 0) || a.in % 8 != 0);
    const Plan p = mx4_plan(a.n_rows, a.out, a.in, a.offsets ? a.experts : 0, MX, odd);
    // offsets are taken from token 0 where rows[] is given, from a tile's first row otherwise
    const int64_t pitch = MX ? pieces(a.in) * PIECE_BYTES : 2 * a.ldx;
    const bool far = (a.gather ? a.tokens : min(a.n_rows, int64_t(256))) * pitch >= int64_t(NO_ROW);
    // Without tokens there is no row 0 for the kernels to read in place of those that rows[] does not name: the copy is made of zeros alone.
    const bool none = a.tokens == 0;
    if ((odd && p.form != Form::rows) || (far && (a.gather || !MX)) || none) {
        const int64_t to_pitch = MX ? pitch : pieces(a.in) * (2 * PIECE), blocks = (a.n_rows * to_pitch / 16 + 255) / 256;
        if (!launchable(blocks, 256)) return adadim_fail(ctx, ADADIM_EINVAL, "mx4 product: X too large to be copied");
        const size_t codes = size_t(a.n_rows) * size_t(to_pitch);
        uint8_t* to = static_cast<uint8_t*>(adadim_workspace(ctx, WS_MX4_X, codes + (MX ? codes / 16 : 0)));
        if (!to) return ADADIM_EHIP;
        uint32_t* to_scales = reinterpret_cast<uint32_t*>(to + codes);
        ProfScope prof(ctx, "mx4_copy_rows");
        hipLaunchKernelGGL((mx4_copy_rows<MX>), dim3(static_cast<unsigned>(blocks)), dim3(256), 0, ctx->stream, ProductArgs(a), to_pitch, to, to_scales);
        ADADIM_LAUNCH_CHECK(ctx, "mx4_copy_rows");
        a.X = to;
        a.gather = false;
        if (MX) {
            a.x_scales = to_scales;
            a.x_rows = a.n_rows;
        } else a.ldx = to_pitch / 2;
    }
    return launch_form<XT>(ctx, a, p);
}

}  // namespace

int launch_mx4_matmul(adadim_ctx* ctx, const mx4::Product& a, int x_type) {
    static PerDeviceOnce once;
    ADADIM_HIP_TRY(ctx, once.run([] {
        hipError_t e = raise_lds<XF16>();
        if (e == hipSuccess) e = raise_lds<XBF16>();
        if (e == hipSuccess) e = raise_lds<XMX4>();
        return e;
    }));
    if (x_type == XF16) return launch_product<XF16>(ctx, a);
    if (x_type == XBF16) return launch_product<XBF16>(ctx, a);
    return launch_product<XMX4>(ctx, a);
}
