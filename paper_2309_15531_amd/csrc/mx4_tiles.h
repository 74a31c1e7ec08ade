// Product tiles of microscaled 4-bit weights on the matrix cores, for many rows.  Included by mx4_matmul.hip.
#pragma once

#include "mx4_matmul.h"

namespace {

using namespace mx4;

namespace tiles {

__device__ __forceinline__ void g2l16(const void* g, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(g) : "memory", "m0");
}
__device__ __forceinline__ uint4v lds_read16(uint32_t addr) {
    typedef uint4v __attribute__((address_space(3))) * lds_ptr;
    return *reinterpret_cast<lds_ptr>(uintptr_t(addr));
}
template <class V>
__device__ __forceinline__ void lds_write(uint32_t addr, const V& v) {
    typedef V __attribute__((address_space(3))) * lds_ptr;
    *reinterpret_cast<lds_ptr>(uintptr_t(addr)) = v;
}

// Rows of 128 bytes (8 chunks of 16) or 256 bytes (16 chunks) in LDS; chunk c of row r lies at slot c ^ swizzle(r), so that
// a fragment read (32 consecutive rows, one chunk each) touches every bank evenly.
template <int CHUNKS>
__device__ __forceinline__ int swizzle(int row) { return CHUNKS == 8 ? (row ^ (row >> 3)) & 7 : row & 15; }

template <int J>
__device__ __forceinline__ float16v mma_mx4(uint4v w, uint32_t ws, uint4v x, uint32_t xs, float16v acc) {
    int8v a = {}, b = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = static_cast<int>(w[i]);
        b[i] = static_cast<int>(x[i]);
    }
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc, 4, 4, J, static_cast<int>(ws), J, static_cast<int>(xs));
}

__device__ const uint4v zero_chunk = {0u, 0u, 0u, 0u};   // what the transfers of chunks that do not exist read

constexpr int WAIT_VM0 = 0x0F70;                  // s_waitcnt vmcnt(0), nothing else

// The tile (expert, first row, first output) of a workgroup.  Tiles are counted out on the device: every group has
// ceil(rows / BM) of them, in the order of the experts.  Workgroups go to the eight XCDs in turn; each XCD takes a contiguous eighth
// of the tiles, listed in strips of 8 row tiles, so that the 32 that run together share 8 panels of X and 4 of W in its L2.
struct Tile {
    int expert;
    int64_t row0, out0;
};
template <int BM, int BN>
__device__ __forceinline__ bool tile_of(const Product& a, Tile& t) {
    const int lane = threadIdx.x & 63;
    const uint32_t n_tiles = static_cast<uint32_t>((a.out + BN - 1) / BN);
    int64_t m_tiles = (a.n_rows + BM - 1) / BM;
    auto count = [&](int e) {
        if (e >= a.experts) return 0;
        const Group g = group_of(a, e);
        return static_cast<int>((max(g.hi - g.lo, int64_t(0)) + BM - 1) / BM);
    };
    if (a.offsets) {
        int n = 0;
        for (int e = lane; e < a.experts; e += 64) n += count(e);
        for (int d = 1; d < 64; d *= 2) n += __shfl_xor(n, d);
        m_tiles = n;
    }
    const int64_t all = m_tiles * n_tiles;
    if (all <= 0 || all > int64_t(gridDim.x)) return false;   // (more only where the offsets decrease)
    const uint32_t total = static_cast<uint32_t>(all), per = (total + 7) / 8;
    const uint32_t id = blockIdx.x % 8 * per + blockIdx.x / 8;
    if (blockIdx.x / 8 >= per || id >= total) return false;
    const uint32_t strip = id / (8 * n_tiles), in_strip = id % (8 * n_tiles);
    const uint32_t high = min(8u, static_cast<uint32_t>(m_tiles) - 8 * strip);
    const int m = static_cast<int>(8 * strip + in_strip % high);
    t.out0 = int64_t(in_strip / high) * BN;
    t.expert = 0;
    t.row0 = int64_t(m) * BM;
    if (a.offsets) {
        int before = 0;
        for (int e0 = 0; e0 < a.experts; e0 += 64) {
            int n = count(e0 + lane), sum = n;
            for (int d = 1; d < 64; d *= 2) {
                const int o = __shfl_up(sum, d);
                if (lane >= d) sum += o;
            }
            const uint64_t past = __ballot(before + sum > m);
            if (past) {
                const int l = __builtin_ctzll(past);
                t.expert = e0 + l;
                t.row0 = int64_t(m - before - __shfl(sum - n, l)) * BM;
                break;
            }
            before += __shfl(sum, 63);
        }
    }
    return true;
}

}  // namespace tiles

// Y tile of BM rows x BN outputs by WT x WO waves (along the rows, along the outputs).
//
// mx4 X: a stage is 256 k, 128 bytes of every row of both operands, brought to LDS by DMA; the lane (row r, half h) of the
// 32x32x64 instruction number j takes chunk j + 4 h, so that its scale is byte j of one word: half 0 works through the stage's first
// piece while half 1 works through the second.
// 16-bit X: a stage is 128 k, 256 bytes of every row of X; the weights' codes go straight to registers (32 bytes a lane and row tile: half
// h takes blocks 2 h and 2 h + 1) and become 16-bit numbers there, two a conversion, next to the 32x32x16 instructions that
// need them; instruction j takes values 64 h + 8 j .. + 7.
// Two stages of LDS: one is computed while the other arrives.
template <int XT, int BM, int BN, int WT, int WO>
__global__ __launch_bounds__(64 * WT * WO) void mx4_tiles(Product a) {
    using namespace tiles;
    constexpr bool MX = XT == XMX4;
    constexpr int NW = WT * WO, TT = BM / WT / 32, TO = BN / WO / 32;
    constexpr int CH = MX ? 8 : 16, ROWB = 16 * CH, ROWS_PER = 64 / CH;           // chunks and bytes of a row, rows of a transfer
    constexpr int X_BYTES = BM * ROWB, STAGE = X_BYTES + (MX ? BN * ROWB : 0);
    constexpr int XL = BM / ROWS_PER / NW, WL = MX ? BN / ROWS_PER / NW : 0;       // transfers of a wave and stage
    static_assert(BM % (ROWS_PER * NW) == 0 && (!MX || BN % (ROWS_PER * NW) == 0), "transfers");
    extern __shared__ __align__(16) char smem[];
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));
    Tile t;
    if (!tile_of<BM, BN>(a, t)) return;
    Group gr = group_of(a, t.expert);
    const int64_t r_first = gr.lo + t.row0, np = pieces(a.in);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wt = wave / WO, wo = wave % WO, fr = lane & 31, fh = lane >> 5;
    const int n_st = static_cast<int>(MX ? (np + 1) / 2 : np);

    // a row of X to read in place of one that does not exist: its products are not stored, or stored as zeros
    auto x_row = [&](int i) {
        const int64_t s = source_row(a, r_first + i, gr.hi);
        return s < 0 ? int64_t(0) : s;
    };
    const char* xp[XL];
    const char* wp[WL > 0 ? WL : 1];
    int xc[XL], wc[WL > 0 ? WL : 1];
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int row = ROWS_PER * (wave + NW * i) + lane / CH;
        xc[i] = (lane % CH) ^ swizzle<CH>(row);
        xp[i] = static_cast<const char*>(a.X) + x_row(row) * (MX ? np * PIECE_BYTES : 2 * a.ldx) + 16 * xc[i];
    }
    if constexpr (MX) {
#pragma unroll
        for (int i = 0; i < WL; ++i) {
            const int row = ROWS_PER * (wave + NW * i) + lane / CH;
            wc[i] = (lane % CH) ^ swizzle<CH>(row);
            wp[i] = reinterpret_cast<const char*>(gr.codes) + min(t.out0 + row, a.out - 1) * np * PIECE_BYTES + 16 * wc[i];
        }
    }
    // chunks of a row that exist in stage s
    auto have = [&](int s) {
        if constexpr (MX) return static_cast<int>(min(int64_t(8), 4 * (np - 2 * s)));
        else return static_cast<int>(min(int64_t(16), (a.in - int64_t(PIECE) * s + 7) / 8));
    };
    auto fetch = [&](int s, int buf) {
        const int n = have(s);
        if (n == CH) {
#pragma unroll
            for (int i = 0; i < XL; ++i) g2l16(xp[i], lds0 + buf * STAGE + (wave + NW * i) * 1024);
#pragma unroll
            for (int i = 0; i < WL; ++i) g2l16(wp[i], lds0 + buf * STAGE + X_BYTES + (wave + NW * i) * 1024);
        } else {
            const char* none = reinterpret_cast<const char*>(&zero_chunk);
#pragma unroll
            for (int i = 0; i < XL; ++i) g2l16(xc[i] < n ? xp[i] : none, lds0 + buf * STAGE + (wave + NW * i) * 1024);
#pragma unroll
            for (int i = 0; i < WL; ++i) g2l16(wc[i] < n ? wp[i] : none, lds0 + buf * STAGE + X_BYTES + (wave + NW * i) * 1024);
        }
#pragma unroll
        for (int i = 0; i < XL; ++i) xp[i] += ROWB;
#pragma unroll
        for (int i = 0; i < WL; ++i) wp[i] += ROWB;
    };

    int64_t w_row[TO];
#pragma unroll
    for (int o = 0; o < TO; ++o) w_row[o] = min(t.out0 + (wo * TO + o) * 32 + fr, a.out - 1);

    float16v acc[TO][TT];
#pragma unroll
    for (int o = 0; o < TO; ++o)
#pragma unroll
        for (int i = 0; i < TT; ++i) acc[o][i] = float16v{};

    // ---- what a wave needs of a stage besides LDS, fetched one stage ahead
    struct Side {
        uint32_t ws[TO], xs[MX ? TT : 1];
        uint4v w[MX ? 1 : TO][2];
    };
    int64_t x_src[MX ? TT : 1];
    if constexpr (MX) {
#pragma unroll
        for (int i = 0; i < TT; ++i) x_src[i] = x_row((wt * TT + i) * 32 + fr);
    }
    auto side = [&](int s) {
        Side d;
        if constexpr (MX) {
            const int64_t p = 2 * s + fh, q = min(p, np - 1);
#pragma unroll
            for (int o = 0; o < TO; ++o) d.ws[o] = gr.scales[q * a.out + w_row[o]];
#pragma unroll
            for (int i = 0; i < TT; ++i) d.xs[i] = a.x_scales[q * a.tokens + x_src[i]];
            if (p >= np) {                                    // half a stage: zeros from the zero page, of scale 1
#pragma unroll
                for (int o = 0; o < TO; ++o) d.ws[o] = ONE_WORD;
#pragma unroll
                for (int i = 0; i < TT; ++i) d.xs[i] = ONE_WORD;
            }
        } else {
#pragma unroll
            for (int o = 0; o < TO; ++o) {
                d.ws[o] = gr.scales[s * a.out + w_row[o]] >> (16 * fh);
                const uint4v* p = reinterpret_cast<const uint4v*>(gr.codes + (w_row[o] * np + s) * PIECE_BYTES + 32 * fh);
                d.w[o][0] = p[0];
                d.w[o][1] = p[1];
            }
        }
        return d;
    };

    const uint32_t xf = lds0 + (wt * TT * 32 + fr) * ROWB, wf = lds0 + X_BYTES + (wo * TO * 32 + fr) * ROWB;
    const int fsw = swizzle<CH>(fr);                          // (rows 32 apart have swizzles that differ by a constant)
    auto x_frag = [&](int buf, int i, int c) { return lds_read16(xf + buf * STAGE + i * 32 * ROWB + ((c ^ fsw ^ swizzle<CH>(32 * (wt * TT + i))) << 4)); };
    auto w_frag = [&](int buf, int o, int c) { return lds_read16(wf + buf * STAGE + o * 32 * ROWB + ((c ^ fsw ^ swizzle<CH>(32 * (wo * TO + o))) << 4)); };

    bool wide = false;                                        // fp16 X: a weight has gone by that no fp16 number holds
    auto compute = [&](int buf, const Side& d) {
        if constexpr (MX) {
            auto step = [&](auto tag) {
                constexpr int J = decltype(tag)::value;
                uint4v w[TO], x[TT];
#pragma unroll
                for (int o = 0; o < TO; ++o) w[o] = w_frag(buf, o, J + 4 * fh);
#pragma unroll
                for (int i = 0; i < TT; ++i) x[i] = x_frag(buf, i, J + 4 * fh);
#pragma unroll
                for (int o = 0; o < TO; ++o)
#pragma unroll
                    for (int i = 0; i < TT; ++i) acc[o][i] = mma_mx4<J>(w[o], d.ws[o], x[i], d.xs[i], acc[o][i]);
            };
            step(std::integral_constant<int, 0>{});
            step(std::integral_constant<int, 1>{});
            step(std::integral_constant<int, 2>{});
            step(std::integral_constant<int, 3>{});
        } else {
            float sc[TO][2];
#pragma unroll
            for (int o = 0; o < TO; ++o)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const uint32_t byte = (d.ws[o] >> (8 * b)) & 255u;
                    sc[o][b] = scale_operand(byte);
                    wide |= beyond_f16(byte);
                }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint4v x[TT];
#pragma unroll
                for (int i = 0; i < TT; ++i) x[i] = x_frag(buf, i, j + 8 * fh);
#pragma unroll
                for (int o = 0; o < TO; ++o) {
                    const uint32_t word = d.w[o][j >> 2][j & 3];
                    if constexpr (XT == XF16) {
                        const half8v w = values8_f16(word, sc[o][j >> 2]);
#pragma unroll
                        for (int i = 0; i < TT; ++i)
                            acc[o][i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(w, __builtin_bit_cast(half8v, x[i]), acc[o][i], 0, 0, 0);
                    } else {
                        const bf8v w = values8_bf16(word, sc[o][j >> 2]);
#pragma unroll
                        for (int i = 0; i < TT; ++i)
                            acc[o][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, __builtin_bit_cast(bf8v, x[i]), acc[o][i], 0, 0, 0);
                    }
                }
            }
        }
    };

    Side now = side(0);
    fetch(0, 0);
    __builtin_amdgcn_s_waitcnt(WAIT_VM0);
    __syncthreads();
    for (int s = 0; s < n_st; ++s) {
        Side next = now;
        if (s + 1 < n_st) {
            next = side(s + 1);
            fetch(s + 1, (s + 1) & 1);
        }
        compute(s & 1, now);
        __builtin_amdgcn_s_waitcnt(WAIT_VM0);
        __syncthreads();
        now = next;
    }
    if constexpr (XT == XF16) {
        if (__syncthreads_or(wide)) {
            // The tile once more with both operands in bf16, X in two parts.  Rare: a stage at a time.
#pragma unroll
            for (int o = 0; o < TO; ++o)
#pragma unroll
                for (int i = 0; i < TT; ++i) acc[o][i] = float16v{};
#pragma unroll
            for (int i = 0; i < XL; ++i) xp[i] -= int64_t(n_st) * ROWB;
            for (int s = 0; s < n_st; ++s) {
                fetch(s, 0);
                const Side d = side(s);
                __builtin_amdgcn_s_waitcnt(WAIT_VM0);
                __syncthreads();
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    bf8v w[TO];
#pragma unroll
                    for (int o = 0; o < TO; ++o) w[o] = values8_bf16(d.w[o][j >> 2][j & 3], scale_operand((d.ws[o] >> (8 * (j >> 2))) & 255u));
#pragma unroll
                    for (int i = 0; i < TT; ++i) {
                        bf8v hi, lo;
                        split_f16(__builtin_bit_cast(half8v, x_frag(0, i, j + 8 * fh)), hi, lo);
#pragma unroll
                        for (int o = 0; o < TO; ++o) {
                            acc[o][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[o], hi, acc[o][i], 0, 0, 0);
                            acc[o][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[o], lo, acc[o][i], 0, 0, 0);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                __syncthreads();
            }
        }
    }

    // ---- Y: a lane holds, of each 32 x 32 block, token fr and outputs 8 q + 4 h .. + 3.  A wave turns 32 tokens x its outputs through LDS of
    // its own and stores rows of 16 bytes a lane.
    auto store = [&](auto tag) {
        typedef decltype(tag) TY;
        constexpr int N = 16 / sizeof(TY), COLS = TO * 32, PITCH = COLS * sizeof(TY) + 16, LANES = COLS / N, PER = 64 / LANES;
        static_assert(NW * 32 * PITCH <= 2 * STAGE, "room");
        typedef TY outv __attribute__((ext_vector_type(N)));
        typedef TY quad __attribute__((ext_vector_type(4)));
        const uint32_t mine = lds0 + wave * 32 * PITCH;
#pragma unroll
        for (int i = 0; i < TT; ++i) {
#pragma unroll
            for (int o = 0; o < TO; ++o)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    quad v;
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = static_cast<TY>(acc[o][i][4 * q + r]);
                    lds_write(mine + fr * PITCH + (32 * o + 8 * q + 4 * fh) * sizeof(TY), v);
                }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += PER) {
                const int row = r0 + lane / LANES, col = (lane % LANES) * N;
                const int64_t r = r_first + (wt * TT + i) * 32 + row, c = t.out0 + wo * COLS + col;
                uint4v v = lds_read16(mine + row * PITCH + col * sizeof(TY));
                if (r < gr.hi && c < a.out) {
                    if (a.rows && source_row(a, r, gr.hi) < 0) v = uint4v{};
                    Chunk<TY, N>::store(static_cast<TY*>(a.Y) + r * a.ldy + c, static_cast<int>(min(int64_t(N), a.out - c)),
                                        __builtin_bit_cast(outv, v));
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    };
    if (a.y_type == ADADIM_TYPE_F16) store(_Float16{});
    else if (a.y_type == ADADIM_TYPE_BF16) store(__bf16{});
    else store(float{});
}

}  // namespace
