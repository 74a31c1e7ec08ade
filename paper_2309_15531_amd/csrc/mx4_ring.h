// Product tiles whose operands all come through a ring of LDS stages.  Included by mx4_matmul.hip behind mx4_tiles.h.
#pragma once

#include "mx4_tiles.h"

namespace {

using namespace mx4;

// Y tile of BM rows x BN outputs by WT x WO waves, over one of gridDim.y shares of the contraction.
//
// A stage is one piece (128 k) of BM rows of X (64 bytes each in mx4, 256 in 16 bits) and of BN rows of W, and their scale words, brought
// by DMA into one of NS slots: NS - 1 stages are on their way while one is computed, so that a tile with little to compute a stage
// does not wait a memory latency for each.  Shares of the contraction leave their sums in `part`, and the one that finishes last adds
// them up in the order of the shares (as in mx4_rows).
//
// The lane (row r, half h) of instruction number j of a stage takes, of mx4 X, chunk j + 2 h (so that its scale is byte j of the word
// shifted by 16 h) and, of 16-bit X, values 64 h + 8 j .. + 7.
//
// 16-bit X: bound by the matrix cores at the clock that the power limit leaves (2048 x 11008 -> 4096 fp16: pipes busy 62 % of the time at
// 1.8 GHz).  128 x 256, 8192 x 8192 x 8192: bf16 848 to 889 us, fp16 886 to 921 us (1.24 to 1.30 and 1.19 to 1.24 PFLOP/s); 2048 x 11008 -> 4096
// fp16 148 to 157 us among other passes (1.17 to 1.25 PFLOP/s), 170 to 176 each by itself under a profiler; 256 x 256 in two stages
// took 1.0 to 1.9 times as long, 128 x 128 through the same ring 1.2 to 1.26 times at these sizes.
// mx4 X: for tiles too small for the two-stage kernel; 256 x 256 through the ring, in rows of 64 bytes a stage, took 298 us for 8192 x 8192 x 8192 where
// two stages of 128 bytes a row take 248 (both with one set of operands).
// NS: of the small tiles, as many slots as leave two to four workgroups to a compute unit's 160 KB; of the large ones, what fits.
template <int XT, int BM, int BN, int WT, int WO, int NS>
struct Ring {
    static constexpr bool MX = XT == XMX4;
    static constexpr int NW = WT * WO, TT = BM / WT / 32, TO = BN / WO / 32;
    static constexpr int CH = MX ? 4 : 16, STEPS = MX ? 2 : 8;
    static constexpr int X_BYTES = BM * CH * 16, W_BYTES = BN * 64, S_BYTES = (BN + (MX ? (BM + 63) / 64 * 64 : 0)) * 4;
    static constexpr int SLOT = X_BYTES + W_BYTES + S_BYTES;
    static constexpr int XN = X_BYTES / 1024, WN = W_BYTES / 1024, SN = S_BYTES / 256;                // transfers of a stage ...
    static constexpr int XL = (XN + NW - 1) / NW, WL = (WN + NW - 1) / NW, SL = (SN + NW - 1) / NW;    // ... and of a wave: where the waves outnumber them some bring the same
    static constexpr int LOADS = XL + WL + SL;
    // what the epilogue needs: 32 rows of a wave's outputs, in fp32 at most
    static constexpr int OUT_BYTES = NW * 32 * (TO * 32 * 4 + 16);
    static constexpr int LDS = NS * SLOT > OUT_BYTES ? NS * SLOT : OUT_BYTES;
    static_assert(X_BYTES % 1024 == 0 && W_BYTES % 1024 == 0 && S_BYTES % 128 == 0 && NS >= 3 && (NS - 2) * LOADS < 64, "transfers");
};

// s_waitcnt vmcnt(n) lgkmcnt(0)
constexpr int wait_vm_lgkm0(int n) { return (n & 15) | ((n >> 4) << 14) | 0x0070; }

template <int XT, int BM, int BN, int WT, int WO, int NS>
__global__ __launch_bounds__(64 * WT * WO) void mx4_ring(ProductArgs args, void* shared) {
    const Product a = args.open();
    using namespace tiles;
    using R = Ring<XT, BM, BN, WT, WO, NS>;
    constexpr bool MX = R::MX;
    constexpr int NW = R::NW, TT = R::TT, TO = R::TO, CH = R::CH, STEPS = R::STEPS, ROWB = CH * 16, SLOT = R::SLOT;
    extern __shared__ __align__(16) char smem[];
    __shared__ unsigned s_ticket;
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));
    Tile t;
    if (!tile_of<BM, BN>(a, t)) return;
    const Group gr = group_of(a, t.expert);
    const int64_t r_first = gr.lo + t.row0, np = pieces(a.in);
    const int p_lo = static_cast<int>(np * blockIdx.y / gridDim.y), n_st = static_cast<int>(np * (blockIdx.y + 1) / gridDim.y) - p_lo;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wt = wave / WO, wo = wave % WO, fr = lane & 31, fh = lane >> 5;

    auto x_row = [&](int i) {                                 // a row to read in place of one that does not exist, too
        const int64_t s = source_row(a, r_first + i, gr.hi);
        return s < 0 ? int64_t(0) : s;
    };
    // Transfers as 32-bit offsets from a row that all share (see mx4_tiles)
    auto chunk_of = [](int ch, int row, int slot) { return slot ^ (ch == 4 ? (row >> 2) & 3 : row & 15); };
    const int64_t x_pitch = MX ? np * PIECE_BYTES : 2 * a.ldx, x_first = a.gather ? 0 : r_first;
    const char* x_base = uniform(static_cast<const char*>(a.X) + x_first * x_pitch + int64_t(p_lo) * ROWB);
    const char* w_base = uniform(gr.codes + (t.out0 * np + p_lo) * PIECE_BYTES);
    const char* ws_base = uniform(gr.scales + int64_t(p_lo) * a.out + t.out0);
    const char* xs_base = MX ? uniform(a.x_scales + int64_t(p_lo) * a.x_rows + x_first) : nullptr;
    uint32_t xo[R::XL], wofs[R::WL], so[R::SL];
    int x_chunk[R::XL];
    bool s_of_x[R::SL];
#pragma unroll
    for (int i = 0; i < R::XL; ++i) {
        const int row = (64 / CH) * ((wave + NW * i) % R::XN) + lane / CH;
        x_chunk[i] = chunk_of(CH, row, lane % CH);
        xo[i] = static_cast<uint32_t>((a.gather ? x_row(row) : min(int64_t(row), gr.hi - 1 - r_first)) * x_pitch + 16 * x_chunk[i]);
    }
#pragma unroll
    for (int i = 0; i < R::WL; ++i) {
        const int row = 16 * ((wave + NW * i) % R::WN) + lane / 4;
        wofs[i] = static_cast<uint32_t>(min(int64_t(row), a.out - 1 - t.out0) * np * PIECE_BYTES + 16 * chunk_of(4, row, lane % 4));
    }
    // scale words: 64 rows a transfer, first those of W, then those of X
    int s_slot[R::SL];
#pragma unroll
    for (int i = 0; i < R::SL; ++i) {
        s_slot[i] = (wave + NW * i) % R::SN;
        s_of_x[i] = 64 * s_slot[i] >= BN;
        const int row = 64 * s_slot[i] + lane - (s_of_x[i] ? BN : 0);
        if (s_of_x[i]) so[i] = static_cast<uint32_t>((a.gather ? x_row(min(row, BM - 1)) : min(int64_t(row), gr.hi - 1 - r_first)) * 4);
        else so[i] = static_cast<uint32_t>(min(int64_t(row), a.out - 1 - t.out0) * 4);
    }
    auto g2l4_s = [](const char* sbase, uint32_t voff, uint32_t lds) {
        asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(voff), "s"(sbase) : "memory", "m0");
    };
    // The share's last piece, which may end early, is computed first: stage q > 0 is piece p_lo + q - 1.  Stages behind the last
    // read zeros, so that nothing branches on them.
    const char *xb, *wb, *wsb, *xsb;
    uint32_t mask = ~0u;
    int to_fetch = 0;
    auto next_fetch = [&]() {
        const int64_t k = to_fetch == 0 ? n_st - 1 : to_fetch - 1;
        const bool real = to_fetch < n_st;
        const char* none = reinterpret_cast<const char*>(&zero_chunk);
        xb = uniform(real ? x_base + k * ROWB : none);
        wb = uniform(real ? w_base + k * PIECE_BYTES : none);
        wsb = uniform(real ? ws_base + 4 * k * a.out : none);
        if constexpr (MX) xsb = uniform(real ? xs_base + 4 * k * a.x_rows : none);
        mask = real ? ~0u : 0u;
        ++to_fetch;
    };
    auto fetch_one = [&](uint32_t slot, int i) {
        const uint32_t to = lds0 + slot;
        if (i < R::XL) g2l16_s(xb, xo[i < R::XL ? i : 0] & mask, to + (wave + NW * i) % R::XN * 1024);
        else if (i < R::XL + R::WL) {
            const int j = i < R::XL ? 0 : i < R::XL + R::WL ? i - R::XL : 0;
            g2l16_s(wb, wofs[j] & mask, to + R::X_BYTES + (wave + NW * j) % R::WN * 1024);
        } else {
            const int j = i < R::XL + R::WL ? 0 : i - R::XL - R::WL;
            g2l4_s(MX && s_of_x[j] ? xsb : wsb, so[j] & mask, lds0 + slot + R::X_BYTES + R::W_BYTES + s_slot[j] * 256);
        }
    };

    float16v acc[TO][TT];
#pragma unroll
    for (int o = 0; o < TO; ++o)
#pragma unroll
        for (int i = 0; i < TT; ++i) acc[o][i] = float16v{};

    // ---- what a wave holds of a stage: scales, and with 16-bit X the codes of its rows of W
    struct Side {
        uint32_t ws[TO], xs[MX ? TT : 1];
        uint4v w[MX ? 1 : TO][2];
    };
    const uint32_t s_at = lds0 + R::X_BYTES + R::W_BYTES + 4 * fr;
    const uint32_t w_swz = (fr >> 2) & 3, w_at = lds0 + R::X_BYTES + (wo * TO * 32 + fr) * 64;
    auto lds_read4 = [](uint32_t addr) {
        typedef uint32_t __attribute__((address_space(3))) * lds_ptr;
        return *reinterpret_cast<lds_ptr>(uintptr_t(addr));
    };
    auto side_of = [&](uint32_t slot) {
        Side d;
#pragma unroll
        for (int o = 0; o < TO; ++o) {
            d.ws[o] = lds_read4(s_at + slot + 4 * 32 * (wo * TO + o)) >> (16 * fh);
            if constexpr (!MX) {
                d.w[o][0] = lds_read16(w_at + slot + o * 32 * 64 + (((2 * fh) ^ w_swz) << 4));
                d.w[o][1] = lds_read16(w_at + slot + o * 32 * 64 + (((2 * fh + 1) ^ w_swz) << 4));
            }
        }
        if constexpr (MX) {
#pragma unroll
            for (int i = 0; i < TT; ++i) d.xs[i] = lds_read4(s_at + slot + 4 * (BN + 32 * (wt * TT + i))) >> (16 * fh);
        }
        return d;
    };
    uint32_t xa[STEPS], wa[MX ? STEPS : 1];
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
        xa[j] = lds0 + (wt * TT * 32 + fr) * ROWB + (static_cast<uint32_t>(chunk_of(CH, fr, j + STEPS * fh)) << 4);
        if constexpr (MX) wa[j] = w_at + ((static_cast<uint32_t>(j + 2 * fh) ^ w_swz) << 4);
    }
    bool wide = false;                                        // fp16 X: a weight has gone by that no fp16 number holds
    constexpr int M = TO * TT;

    // ---- stage 0: the chunks it lacks are zeros (16-bit X; mx4 rows are whole pieces)
    {
        next_fetch();
        const int have = MX ? 4 : static_cast<int>(min(int64_t(16), (a.in - PIECE * (p_lo + int64_t(n_st) - 1) + 7) / 8));
#pragma unroll
        for (int i = 0; i < R::XL; ++i)
            g2l16(x_chunk[i] < have ? xb + xo[i] : reinterpret_cast<const char*>(&zero_chunk), lds0 + (wave + NW * i) % R::XN * 1024);
#pragma unroll
        for (int i = R::XL; i < R::LOADS; ++i) fetch_one(0, i);
    }
#pragma unroll
    for (int s = 1; s < NS; ++s) {
        next_fetch();
#pragma unroll
        for (int i = 0; i < R::LOADS; ++i) fetch_one(s * SLOT, i);
    }
    __builtin_amdgcn_s_waitcnt(wait_vm_lgkm0((NS - 1) * R::LOADS < 63 ? (NS - 1) * R::LOADS : 63));
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    uint32_t slot = 0;
    auto after = [](uint32_t s) { return s == (NS - 1) * SLOT ? 0u : s + SLOT; };
    // The stage behind the one at hand has arrived, and every wave has read what it needs of the one at hand: its slot is free.
    auto meet = [&]() {
        __builtin_amdgcn_s_waitcnt(wait_vm_lgkm0((NS - 2) * R::LOADS));
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        next_fetch();
    };
    if constexpr (MX) {
        // Little to compute a stage: all of the next stage is read while one is computed from registers.
        struct Stage {
            Side side;
            uint4v w[2][TO], x[2][TT];
        };
        constexpr int READS = 2 * (TO + TT);
        auto read_one = [&](Stage& st, uint32_t at, int k) {
            const int j = k / (TO + TT), n = k % (TO + TT);
            if (n < TO) st.w[j][n] = lds_read16(wa[j] + at + n * 32 * 64);
            else st.x[j][n - TO] = lds_read16(xa[j] + at + (n - TO) * 32 * ROWB);
        };
        Stage s0, s1;
        s0.side = side_of(0);
#pragma unroll
        for (int k = 0; k < READS; ++k) read_one(s0, 0, k);
        auto body = [&](const Stage& st, Stage& next) {
            meet();
            const uint32_t next_slot = after(slot);
            next.side = side_of(next_slot);
#pragma unroll
            for (int m = 0; m < 2 * M; ++m) {
#pragma unroll
                for (int k = m * READS / (2 * M); k < (m + 1) * READS / (2 * M); ++k) read_one(next, next_slot, k);
#pragma unroll
                for (int i = m * R::LOADS / (2 * M); i < (m + 1) * R::LOADS / (2 * M); ++i) fetch_one(slot, i);
                const int j = m / M, o = m % M / TT, i = m % TT;
                if (j == 0) acc[o][i] = mma_mx4<0>(st.w[0][o], st.side.ws[o], st.x[0][i], st.side.xs[i], acc[o][i]);
                else acc[o][i] = mma_mx4<1>(st.w[1][o], st.side.ws[o], st.x[1][i], st.side.xs[i], acc[o][i]);
                __builtin_amdgcn_sched_barrier(0);
            }
            slot = next_slot;
        };
        for (int q = 0; q < n_st; q += 2) {                   // (the surplus stage of an odd number multiplies zeros)
            body(s0, s1);
            body(s1, s0);
        }
    } else {
        // X is read two steps ahead, W's codes become numbers one step ahead.  The waves meet two steps before a stage's end, so that
        // what is read of the next stage has two steps' instructions to arrive.
        uint4v xf[4][TT], wf[2][TO];
        float sc[TO][2];
        auto scales_of = [&](const Side& d, bool real) {
#pragma unroll
            for (int o = 0; o < TO; ++o)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const uint32_t byte = (d.ws[o] >> (8 * b)) & 255u;
                    sc[o][b] = scale_operand(byte);
                    wide |= real && beyond_f16(byte);
                }
        };
        auto read_x = [&](int b, uint32_t at, int step, int i) { xf[b][i] = lds_read16(xa[step] + at + i * 32 * ROWB); };
        auto number_w = [&](int b, const Side& d, int step, int o) {
            if constexpr (XT == XF16) wf[b][o] = __builtin_bit_cast(uint4v, values8_f16(d.w[o][step >> 2][step & 3], sc[o][step >> 2]));
            else wf[b][o] = __builtin_bit_cast(uint4v, values8_bf16(d.w[o][step >> 2][step & 3], sc[o][step >> 2]));
        };
        auto mma = [&](int step, int m) {
            const int o = m / TT, i = m % TT;
            if constexpr (XT == XF16)
                acc[o][i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8v, wf[step & 1][o]), __builtin_bit_cast(half8v, xf[step & 3][i]), acc[o][i], 0, 0, 0);
            else
                acc[o][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8v, wf[step & 1][o]), __builtin_bit_cast(bf8v, xf[step & 3][i]), acc[o][i], 0, 0, 0);
        };
        constexpr int SLOTS = M > TT ? (M > TO ? M : TO) : (TT > TO ? TT : TO);
        Side now = side_of(0);
        scales_of(now, true);
#pragma unroll
        for (int i = 0; i < TT; ++i) {
            read_x(0, 0, 0, i);
            read_x(1, 0, 1, i);
        }
#pragma unroll
        for (int o = 0; o < TO; ++o) number_w(0, now, 0, o);
        for (int q = 0; q < n_st; ++q) {
#pragma unroll
            for (int j = 0; j < 6; ++j)
#pragma unroll
                for (int m = 0; m < SLOTS; ++m) {
                    if (m < TT) read_x((j + 2) & 3, slot, j + 2, m);
                    if (m < M) mma(j, m);
                    if (m < TO) number_w((j + 1) & 1, now, j + 1, m);
                    __builtin_amdgcn_sched_barrier(0);
                }
            meet();
            const uint32_t next_slot = after(slot);
            const Side next = side_of(next_slot);
#pragma unroll
            for (int m = 0; m < SLOTS; ++m) {
                if (m < TT) read_x(0, next_slot, 0, m);
#pragma unroll
                for (int i = m * R::LOADS / (2 * SLOTS); i < (m + 1) * R::LOADS / (2 * SLOTS); ++i) fetch_one(slot, i);
                if (m < M) mma(6, m);
                if (m < TO) number_w(1, now, 7, m);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int m = 0; m < SLOTS; ++m) {
                if (m < TT) read_x(1, next_slot, 1, m);
#pragma unroll
                for (int i = (SLOTS + m) * R::LOADS / (2 * SLOTS); i < (SLOTS + m + 1) * R::LOADS / (2 * SLOTS); ++i) fetch_one(slot, i);
                if (m < M) mma(7, m);
                __builtin_amdgcn_sched_barrier(0);
            }
            scales_of(next, q + 1 < n_st);
#pragma unroll
            for (int o = 0; o < TO; ++o) number_w(0, next, 0, o);
            now = next;
            slot = next_slot;
        }
    }
    __builtin_amdgcn_s_waitcnt(WAIT_ALL);                     // no transfer may outlive the workgroup, or meet what follows in LDS
    __syncthreads();
    if constexpr (XT == XF16) {
        if (__syncthreads_or(wide)) {
            // The share once more with both operands in bf16, X in two parts.  Rare: a stage at a time.
#pragma unroll
            for (int o = 0; o < TO; ++o)
#pragma unroll
                for (int i = 0; i < TT; ++i) acc[o][i] = float16v{};
            to_fetch = 0;
            for (int q = 0; q < n_st; ++q) {
                next_fetch();
                const int have = static_cast<int>(q == 0 ? min(int64_t(16), (a.in - PIECE * (p_lo + int64_t(n_st) - 1) + 7) / 8) : 16);
#pragma unroll
                for (int i = 0; i < R::XL; ++i)
                    g2l16(x_chunk[i] < have ? xb + xo[i] : reinterpret_cast<const char*>(&zero_chunk), lds0 + (wave + NW * i) % R::XN * 1024);
#pragma unroll
                for (int i = R::XL; i < R::LOADS; ++i) fetch_one(0, i);
                __builtin_amdgcn_s_waitcnt(WAIT_ALL);
                __syncthreads();
                const Side d = side_of(0);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    bf8v w[TO];
#pragma unroll
                    for (int o = 0; o < TO; ++o) w[o] = values8_bf16(d.w[o][j >> 2][j & 3], scale_operand((d.ws[o] >> (8 * (j >> 2))) & 255u));
#pragma unroll
                    for (int i = 0; i < TT; ++i) {
                        bf8v hi, lo;
                        split_f16(__builtin_bit_cast(half8v, lds_read16(xa[j] + i * 32 * ROWB)), hi, lo);
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

    if (gridDim.y > 1) {
        float* const part = parts_of(shared);
        unsigned* const ticket = tickets_of(shared);
        // this share's sums, a lane's four consecutive outputs at a time, in the order in which the lanes hold them: whoever adds them up
        // holds the same places
        float* mine = part + (int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * (BM * BN) + tid;
#pragma unroll
        for (int o = 0; o < TO; ++o)
#pragma unroll
            for (int i = 0; i < TT; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    __hip_atomic_store(mine + ((o * TT + i) * 16 + r) * (64 * NW), acc[o][i][r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) s_ticket = __hip_atomic_fetch_add(ticket + blockIdx.x, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (s_ticket != gridDim.y - 1) return;
        if (tid == 0) __hip_atomic_store(ticket + blockIdx.x, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const float* all = part + int64_t(blockIdx.x) * (BM * BN) + tid;
#pragma unroll
        for (int o = 0; o < TO; ++o)
#pragma unroll
            for (int i = 0; i < TT; ++i) {
                float16v sum = {};
                for (unsigned z = 0; z < gridDim.y; ++z) {
                    const float* p = all + int64_t(z) * gridDim.x * (BM * BN);
                    float16v v;
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        v[r] = __hip_atomic_load(p + ((o * TT + i) * 16 + r) * (64 * NW), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
                    for (int r = 0; r < 16; ++r) sum[r] += v[r];
                }
                acc[o][i] = sum;
            }
    }
    store_tile<TO, TT, NW>(a, acc, lds0, wave, lane, r_first + wt * TT * 32, gr.hi, t.out0 + wo * TO * 32);
}

}  // namespace
