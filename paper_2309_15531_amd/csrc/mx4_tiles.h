// What the product kernels with tiles of both operands share, and the one for many rows of mx4 X.  Included by mx4_matmul.hip.
#pragma once

#include "mx4_matmul.h"

namespace {

using namespace mx4;

namespace tiles {

__device__ __forceinline__ void g2l16(const void* g, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(g) : "memory", "m0");
}
__device__ __forceinline__ void g2l16_s(const void* sbase, uint32_t voff, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(voff), "s"(sbase) : "memory", "m0");
}
// The same value in every lane, told to the compiler.
__device__ __forceinline__ const char* uniform(const void* p) {
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(b)), hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(b >> 32));
    return reinterpret_cast<const char*>(uintptr_t(hi) << 32 | lo);
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

// Rows of 128 bytes (8 chunks of 16) in LDS; chunk c of row r lies at slot c ^ swizzle(r), so that a fragment read
// (32 consecutive rows, one chunk each) touches every bank evenly.  The same for rows 32 apart.
__device__ __forceinline__ int swizzle(int row) { return (row & 7) ^ ((row >> 3) & 3); }

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
__device__ const uint32_t one_word = ONE_WORD;            // ... and of their scales

constexpr int WAIT_VM0 = 0x0F70, WAIT_ALL = 0x0070;       // s_waitcnt vmcnt(0); vmcnt(0) lgkmcnt(0)

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

// Y of a wave: TT x 32 rows from `row0`, TO x 32 outputs from `out0`.  Of each 32 x 32 block a lane holds row lane & 31 and outputs
// 8 q + 4 (lane >> 5) .. + 3.  32 rows at a time are turned through LDS of the wave's own, and stored 16 bytes a lane.
template <int TO, int TT, int NW>
__device__ __forceinline__ void store_tile(const Product& a, const float16v (&acc)[TO][TT], uint32_t lds0, int wave, int lane, int64_t row0,
                                           int64_t row_end, int64_t out0) {
    const int fr = lane & 31, fh = lane >> 5;
    auto store = [&](auto tag) {
        typedef decltype(tag) TY;
        constexpr int N = 16 / sizeof(TY), COLS = TO * 32, PITCH = COLS * sizeof(TY) + 16, LANES = COLS / N, PER = 64 / LANES;
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
                const int64_t r = row0 + i * 32 + row, c = out0 + col;
                uint4v v = lds_read16(mine + row * PITCH + col * sizeof(TY));
                if (r < row_end && c < a.out) {
                    if (a.rows && source_row(a, r, row_end) < 0) v = uint4v{};
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

}  // namespace tiles

// Y tile of BM rows x BN outputs by WT x WO waves (along the rows, along the outputs), X in mx4.
//
// A stage is 256 k, 128 bytes of every row of both operands, brought to LDS by DMA; the lane (row r, half h) of the 32x32x64 instruction
// number j takes chunk j + 4 h, so that its scale is byte j of one word: half 0 works through the stage's first piece while half 1
// works through the second.  Two stages of LDS: one is computed while the other arrives.
//
// Bound by the matrix cores at the clock that the power limit leaves, and by what a tile does outside its loop (its first stage and its output: 6 us
// of 55 at 8192 deep).  256 x 256: 8192 x 8192 x 8192 248 us with one set of operands, 263 to 285 with several in turn (4.43 and 3.9 to 4.2 PFLOP/s;
// instructions on registers alone reach 6.4 with such operands), 8192 x 8192 -> 28672 868 to 911 us, 4096 tokens x 2 of 16 experts, 5120 -> 4096, 139 to
// 156 us.  128 x 128: 2048 x 4096 -> 4096 24.6 us.  Between them, 128 x 256
// and 256 x 128 by four waves took 1.2 to 1.4 times 256 x 256: LDS gives them too few operands.  Scales read from memory by each wave took
// 3 to 10 % longer than those brought to LDS with the codes.  Prefetching a stage further into the L2 took 5 % longer.  Workgroups that go on to
// further tiles, the next one's first stage under the output of the last, gained nothing (258 us both; the experts 152 against 144): the time saved goes
// into a lower clock.
template <int BM, int BN, int WT, int WO>
struct Tiles {
    static constexpr int NW = WT * WO, TT = BM / WT / 32, TO = BN / WO / 32;
    static constexpr int CH = 8, ROWB = 16 * CH, ROWS_PER = 64 / CH, STEPS = CH / 2;      // chunks and bytes of a row, rows of a transfer, steps of a stage
    static constexpr int X_BYTES = BM * ROWB, W_BYTES = BN * ROWB, S_BYTES = 2 * (BM + BN) * 4, STAGE = X_BYTES + W_BYTES + S_BYTES, LDS = 2 * STAGE;
    static constexpr int XL = BM / ROWS_PER / NW, WL = BN / ROWS_PER / NW;                // transfers of a wave and stage, and two of scales
    static_assert(BM % 64 == 0 && BM + BN == 64 * NW, "a wave brings the scales of 64 rows, a transfer for each of the stage's pieces");
    static_assert(BM % (ROWS_PER * NW) == 0 && BN % (ROWS_PER * NW) == 0, "transfers");
    static_assert(NW % 4 == 0, "the swizzle is the same for all transfers of a wave");
    static_assert(NW * 32 * (TO * 32 * 4 + 16) <= LDS, "room for the outputs");
};

template <int BM, int BN, int WT, int WO>
__global__ __launch_bounds__(64 * WT * WO) void mx4_tiles(ProductArgs args) {
    const Product a = args.open();
    using namespace tiles;
    using S = Tiles<BM, BN, WT, WO>;
    constexpr int NW = S::NW, TT = S::TT, TO = S::TO, CH = S::CH, ROWB = S::ROWB, ROWS_PER = S::ROWS_PER, STEPS = S::STEPS;
    constexpr int X_BYTES = S::X_BYTES, W_BYTES = S::W_BYTES, STAGE = S::STAGE, XL = S::XL, WL = S::WL;
    extern __shared__ __align__(16) char smem[];
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));
    Tile t;
    if (!tile_of<BM, BN>(a, t)) return;
    const Group gr = group_of(a, t.expert);
    const int64_t r_first = gr.lo + t.row0, np = pieces(a.in);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wt = wave / WO, wo = wave % WO, fr = lane & 31, fh = lane >> 5;
    const int n_st = static_cast<int>((np + 1) / 2);

    // where rows are gathered: a row of X, the first in place of one that does not exist (its products are not stored, or stored as zeros)
    auto x_row = [&](int i) {
        const int64_t s = source_row(a, r_first + i, gr.hi);
        return s < 0 ? int64_t(0) : s;
    };
    // Transfers.  Number i of a wave takes ROWS_PER rows; every lane has the same chunk in all of them.  They are given as 32-bit offsets
    // from a row that all share: the tile's first (W; X in Y's order) or that of token 0, which the host holds within 4 GB.
    const int t_row = ROWS_PER * wave + lane / CH, t_chunk = (lane % CH) ^ swizzle(t_row);
    const int64_t x_pitch = np * PIECE_BYTES, x_first = a.gather ? 0 : r_first;
    uint32_t xo[XL], wofs[WL];
    const char* x_base = uniform(static_cast<const char*>(a.X) + x_first * x_pitch);
    const char* w_base = uniform(gr.codes + t.out0 * np * PIECE_BYTES);
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int row = t_row + ROWS_PER * NW * i;
        xo[i] = static_cast<uint32_t>((a.gather ? x_row(row) : min(int64_t(row), gr.hi - 1 - r_first)) * x_pitch + 16 * t_chunk);
    }
#pragma unroll
    for (int i = 0; i < WL; ++i)
        wofs[i] = static_cast<uint32_t>(min(int64_t(t_row + ROWS_PER * NW * i), a.out - 1 - t.out0) * np * PIECE_BYTES + 16 * t_chunk);
    const bool s_of_x = wave < BM / 64;
    const int s_row = 64 * wave + lane - (s_of_x ? 0 : BM);
    const uint32_t so = static_cast<uint32_t>(4 * (!s_of_x ? min(int64_t(s_row), a.out - 1 - t.out0)
                                                  : a.gather ? x_row(s_row) : min(int64_t(s_row), gr.hi - 1 - r_first)));
    const int64_t s_pitch = 4 * (s_of_x ? a.x_rows : a.out);
    const char* s_base = uniform(s_of_x ? a.x_scales + x_first : gr.scales + t.out0);
    auto g2l4_s = [](const char* sbase, uint32_t voff, uint32_t lds) {
        asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(voff), "s"(sbase) : "memory", "m0");
    };
    // The last stage along k, which may be shorter, is computed first: stage q > 0 in the order of computation is number q - 1 along k.
    // The chunks that stage 0 lacks, and all of the stages behind the last (nothing branches on them), read zeros.
    auto fetch_first = [&]() {
        const int64_t k = n_st - 1;
        const int n = static_cast<int>(min(int64_t(CH), 4 * (np - 2 * k)));
        const char* none = reinterpret_cast<const char*>(&zero_chunk);
        const uint32_t to = lds0 + wave * 1024;
#pragma unroll
        for (int i = 0; i < XL; ++i) g2l16(t_chunk < n ? x_base + xo[i] + k * ROWB : none, to + NW * i * 1024);
#pragma unroll
        for (int i = 0; i < WL; ++i) g2l16(t_chunk < n ? w_base + wofs[i] + k * ROWB : none, to + X_BYTES + NW * i * 1024);
        const bool whole = 2 * k + 1 < np;                    // of the piece that stage 0 may lack: scales 1
        const uint32_t s_to = lds0 + X_BYTES + W_BYTES + wave * 256;
        g2l4_s(uniform(s_base + 2 * k * s_pitch), so, s_to);
        g2l4_s(uniform(whole ? s_base + (2 * k + 1) * s_pitch : reinterpret_cast<const char*>(&one_word)), whole ? so : 0u, s_to + (BM + BN) * 4);
    };
    const char *xb, *wb, *sb;
    uint32_t mask = ~0u;
    auto fetch_one = [&](int buf, int i) {
        const uint32_t to = lds0 + buf * STAGE + wave * 1024;
        if (i < XL) g2l16_s(xb, xo[i < XL ? i : 0] & mask, to + NW * i * 1024);
        else if (i < XL + WL) g2l16_s(wb, wofs[i < XL || i >= XL + WL ? 0 : i - XL] & mask, to + X_BYTES + NW * (i - XL) * 1024);
        else g2l4_s(i == XL + WL ? sb : uniform(sb + (mask ? s_pitch : 0)), so & mask, lds0 + buf * STAGE + X_BYTES + W_BYTES + wave * 256 + (i - XL - WL) * (BM + BN) * 4);
    };

    float16v acc[TO][TT];
#pragma unroll
    for (int o = 0; o < TO; ++o)
#pragma unroll
        for (int i = 0; i < TT; ++i) acc[o][i] = float16v{};

    // ---- the scales of a wave's rows in a stage, a word for its half's piece
    struct Side {
        uint32_t ws[TO], xs[TT];
    };
    uint32_t s_at = lds0 + X_BYTES + W_BYTES + 4 * (fh * (BM + BN) + fr);
    auto lds_read4 = [](uint32_t addr) {
        typedef uint32_t __attribute__((address_space(3))) * lds_ptr;
        return *reinterpret_cast<lds_ptr>(uintptr_t(addr));
    };
    auto read_scale = [&](Side& d, int k) {
        if (k < TO) d.ws[k] = lds_read4(s_at + 4 * (BM + 32 * (wo * TO + k)));
        else d.xs[k - TO] = lds_read4(s_at + 4 * 32 * (wt * TT + k - TO));
    };

    // Fragment addresses: step j of half h reads chunk j + CH / 2 * h of its row.  They move between the two stages: those of step 0 a
    // step before the others, since a stage's first operands are read during the last step of the one before.
    uint32_t xa[STEPS], wa[STEPS];
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
        const uint32_t slot = static_cast<uint32_t>((j + STEPS * fh) ^ swizzle(fr)) << 4;
        xa[j] = lds0 + (wt * TT * 32 + fr) * ROWB + slot;
        wa[j] = lds0 + X_BYTES + (wo * TO * 32 + fr) * ROWB + slot;
    }

    // ---- the pipeline.  A stage is four steps of TO x TT matrix instructions; a step's operands are read during the step before.
    // Before the last step of a stage all its reads have ended: there the wave waits for the next stage's transfers, meets the others,
    // reads the next stage's first operands and sends for the one after it, into the buffer that has become free.
    struct Frags {
        uint4v w[TO], x[TT];
    };
    // operand number k of a step: TO of W, then TT of X
    auto read_one = [&](Frags& f, int step, int k) {
        if (k >= TO) f.x[k - TO] = lds_read16(xa[step] + (k - TO) * 32 * ROWB);
        else f.w[k] = lds_read16(wa[step] + k * 32 * ROWB);
    };
    auto mma = [&](auto step_tag, const Frags& f, const Side& d, int m) {
        constexpr int J = decltype(step_tag)::value;
        const int o = m / TT, i = m % TT;
        acc[o][i] = mma_mx4<J>(f.w[o], d.ws[o], f.x[i], d.xs[i], acc[o][i]);
    };
    constexpr int M = TO * TT, R = TO + TT, F = XL + WL + 2;
    // a step: its instructions with the next step's operands read between them, in this order
    auto step = [&](auto step_tag, const Frags& f, const Side& d, Frags& nf, int nstep) {
#pragma unroll
        for (int m = 0; m < (M > R ? M : R); ++m) {
            if (m < R) read_one(nf, nstep, m);
            if (m < M) mma(step_tag, f, d, m);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    int to_fetch = 1;
    auto next_fetch = [&]() {                                 // where the next stage's transfers come from
        const bool real = to_fetch < n_st;
        const char* none = reinterpret_cast<const char*>(&zero_chunk);
        xb = uniform(real ? x_base : none);
        wb = uniform(real ? w_base : none);
        sb = uniform(real ? s_base : none);
        mask = real ? ~0u : 0u;
        ++to_fetch;
        x_base += ROWB;
        w_base += ROWB;
        s_base += 2 * s_pitch;
    };
    fetch_first();
    if (r_first + wt * TT * 32 >= gr.hi || t.out0 + wo * TO * 32 >= a.out) {
        // A wave beyond the group's last row or the last output only brings its part of the operands: what shares its SIMD has the matrix cores
        // to itself.
        __builtin_amdgcn_s_waitcnt(WAIT_VM0);
        __syncthreads();
        for (int q = 0; q <= n_st; ++q) {
            next_fetch();
#pragma unroll
            for (int i = 0; i < F; ++i) fetch_one((q + 1) & 1, i);
            __builtin_amdgcn_s_waitcnt(WAIT_ALL);
            __builtin_amdgcn_s_barrier();
        }
        return;
    }
    __builtin_amdgcn_s_waitcnt(WAIT_VM0);
    __syncthreads();
    Side now, next;
    Frags f0, f1;
#pragma unroll
    for (int k = 0; k < R; ++k) read_scale(now, k);
#pragma unroll
    for (int k = 0; k < R; ++k) read_one(f0, 0, k);
    xa[0] += STAGE;
    wa[0] += STAGE;
    s_at += STAGE;
    next_fetch();
#pragma unroll
    for (int i = 0; i < F; ++i) fetch_one(1, i);
    for (int q = 0; q < n_st; ++q) {
        const int buf = q & 1;
        step(std::integral_constant<int, 0>{}, f0, now, f1, 1);
        step(std::integral_constant<int, 1>{}, f1, now, f0, 2);
        step(std::integral_constant<int, 2>{}, f0, now, f1, 3);
        __builtin_amdgcn_s_waitcnt(WAIT_ALL);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        next_fetch();
#pragma unroll
        for (int m = 0; m < (M > R ? M : R); ++m) {
            if (m < R) {
                read_one(f0, 0, m);
                read_scale(next, m);
            }
#pragma unroll
            for (int i = m * F / M; i < (m < M ? (m + 1) * F / M : 0); ++i) fetch_one(buf, i);
            if (m < M) mma(std::integral_constant<int, STEPS - 1>{}, f1, now, m);
            __builtin_amdgcn_sched_barrier(0);
        }
        const uint32_t move = buf ? -STAGE : STAGE;
        s_at -= move;
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
            xa[j] += j ? move : -move;
            wa[j] += j ? move : -move;
        }
        now = next;
    }
    __builtin_amdgcn_s_waitcnt(WAIT_ALL);
    __syncthreads();
    store_tile<TO, TT, NW>(a, acc, lds0, wave, lane, r_first + wt * TT * 32, gr.hi, t.out0 + wo * TO * 32);
}

}  // namespace
