// Attention over a paged cache in mx4:  y = sum_j softmax_j(scale q . k_j) v_j  over the positions j that a query sees.
//
// A tile is 16 NT rows (a row: one query head of one new token) of a sequence that share a key-value head.  A wave goes over records of 32
// positions:  S^T = K Q^T, 2 tiles of 16 positions by NT tiles of 16 rows, keys converted in registers to the queries' type (exact:
// 2 bits and fp16's or bf16's exponents), then p = 2^(scale log2(e) s - m + 8) in fp32, rounded to fp16 (11 bits; with the
// 2^8 the smallest number that fp16 still holds is 2^-33 of the row's largest), and O^T += V^T P^T with the values in fp16 (exact).  Positions
// lie along a lane's registers and rows along the lanes in S^T and in O^T: neither is turned round, and a row's maximum and
// sum are numbers of its lanes.  The maximum m is only raised (and O^T and the sum scaled) where a score passes it by more than 7:
// p stays below 2^15.  The sum is of p before rounding.  Scores, sums and O^T are fp32.
//
// KEYS: the four waves of a workgroup have the same rows and take records in turn (few rows: the read of the cache bounds it); their sums meet
// in LDS.  Otherwise each wave has 16 NT rows of its own and all go over the same records, which the L1 then holds.
// Either way a tile's records may be shared between workgroups (gridDim.y); partial sums travel as relaxed atomics at device scope, and
// the workgroup that finishes last joins them in their order: same bits every run.
#pragma once

#include "mx4_cache.h"

namespace mx4 {

constexpr int AT_WAVES = 4;
constexpr int AT_TICKETS = 8192;                  // tiles that may be shared
constexpr float LOWEST = -3e38f;                  // a maximum before the first score
constexpr float RAISE = 7.0f, HEAD = 8.0f;

struct AttentionArgs {
    Attention a;
    int tiles;                                    // row tiles, of which each sequence has one that may not exist
    int least;                                    // records that a share has at least
    unsigned* tickets;
    float* parts;
};

template <class T> struct Dots;
template <> struct Dots<_Float16> {
    typedef half8v vec;
    static __device__ __forceinline__ vec keys(uint32_t w, float s) { return values8_f16(w, s); }
    static __device__ __forceinline__ float4v mfma(vec a, vec b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Dots<__bf16> {
    typedef bf8v vec;
    static __device__ __forceinline__ vec keys(uint32_t w, float s) { return values8_bf16(w, s); }
    static __device__ __forceinline__ float4v mfma(vec a, vec b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

// The bytes of a record that a lane needs.
template <int D>
struct Bytes {
    static constexpr int W = D / 32, VW = D / 16;             // words of a key's quarter, of 8 positions' values
    uint32_t k[2][W], v[VW], ks[2], vs[2];
    __device__ __forceinline__ void load(const uint8_t* r, int lane) {
        typedef Record<D> R;
        const int m = lane & 15, g = lane >> 4;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = 16 * t + m;
            const uint32_t* p = reinterpret_cast<const uint32_t*>(r + key * (D / 2) + g * (D / 8));
#pragma unroll
            for (int c = 0; c < W; ++c) k[t][c] = p[c];
            if constexpr (D == 256) ks[t] = *reinterpret_cast<const uint16_t*>(r + R::KEY_SCALES + key * 8 + 2 * g);
            else ks[t] = r[R::KEY_SCALES + key * W + g * W / 4];
        }
        const uint32_t* p = reinterpret_cast<const uint32_t*>(r + R::VALUES + (g * 16 + m) * (8 * R::UNIT));
#pragma unroll
        for (int c = 0; c < VW; ++c) v[c] = p[c];
        const uint32_t* s = reinterpret_cast<const uint32_t*>(r + R::VALUE_SCALES + (g * W + m * W / 16) * 8);
        vs[0] = s[0];
        vs[1] = s[1];
    }
};

// max and sum over the four lane quarters
template <class F>
__device__ __forceinline__ float quarters(float v, F f) {
    v = f(v, __shfl_xor(v, 16));
    return f(v, __shfl_xor(v, 32));
}

template <class T, int D, int NT>
struct Rows {
    static constexpr int W = D / 32, TILES = D / 16;
    typedef typename Dots<T>::vec vec;
    vec q[NT][W];
    float4v o[NT][TILES];
    float m[NT], l[NT];                           // m: largest score so far, times c, of all quarters; l: sum of this lane's p
    float c;                                      // scale log2(e)

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n] = LOWEST;
            l[n] = 0.0f;
#pragma unroll
            for (int j = 0; j < TILES; ++j) o[n][j] = float4v{0, 0, 0, 0};
        }
    }

    // lo, hi: the positions that the rows see, counted from the record's first; have: how many of it exist
    template <bool MASK>
    __device__ __forceinline__ void add(const Bytes<D>& b, int lane, const int (&lo)[NT], const int (&hi)[NT], int have) {
        const int g = lane >> 4;
        float4v s[NT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int n = 0; n < NT; ++n) s[n][t] = float4v{0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const uint32_t byte = D == 256 ? w < 4 ? b.ks[t] & 255u : b.ks[t] >> 8 : b.ks[t];
                const vec k = Dots<T>::keys(b.k[t][w], scale_operand(byte));
#pragma unroll
                for (int n = 0; n < NT; ++n) s[n][t] = Dots<T>::mfma(k, q[n][w], s[n][t]);
            }
        }
        float top[NT];
        bool raise = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if constexpr (MASK) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int at = 16 * t + 4 * g + i;
                        s[n][t][i] = at >= lo[n] && at < hi[n] ? s[n][t][i] : -INFINITY;
                    }
            }
            top[n] = fmaxf(fmaxf(fmaxf(s[n][0][0], s[n][0][1]), fmaxf(s[n][0][2], s[n][0][3])),
                           fmaxf(fmaxf(s[n][1][0], s[n][1][1]), fmaxf(s[n][1][2], s[n][1][3]))) * c;
            raise = raise || top[n] > m[n] + RAISE;
        }
        if (__any(raise)) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float up = fmaxf(m[n], quarters(top[n], [](float x, float y) { return fmaxf(x, y); }));
                const float by = __builtin_amdgcn_exp2f(m[n] - up);
                m[n] = up;
                l[n] *= by;
#pragma unroll
                for (int j = 0; j < TILES; ++j) o[n][j] *= by;
            }
        }
        half8v p[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float base = HEAD - m[n];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][t][i], c, base));
                    l[n] += e;
                    p[n][4 * t + i] = static_cast<_Float16>(e);
                }
        }
        float vs[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            vs[i] = scale_operand((b.vs[i >> 2] >> (8 * (i & 3))) & 255u);
            if constexpr (MASK) vs[i] = 4 * g + (i < 4 ? i : 12 + i) < have ? vs[i] : 0.0f;        // (2^-127: zeros in fp16)
        }
#pragma unroll
        for (int u = 0; u < D / 32; ++u) {
            half8v even, odd;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = i * (D / 32) + u;
                half2v v;
                switch (at & 3) {
                    case 0: v = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(b.v[at >> 2], vs[i], 0); break;
                    case 1: v = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(b.v[at >> 2], vs[i], 1); break;
                    case 2: v = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(b.v[at >> 2], vs[i], 2); break;
                    default: v = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(b.v[at >> 2], vs[i], 3); break;
                }
                even[i] = v.x;
                odd[i] = v.y;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                o[n][2 * u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(even, p[n], o[n][2 * u], 0, 0, 0);
                o[n][2 * u + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(odd, p[n], o[n][2 * u + 1], 0, 0, 0);
            }
        }
    }
};

// `count` consecutive elements of a row of Y from d on, of which those below dim exist.
template <int N>
__device__ __forceinline__ void store_row(const Attention& a, int64_t at, int d, const float (&v)[N]) {
    const int have = min(N, a.dim - d);
    if (have <= 0) return;
    if (a.y_type == ADADIM_TYPE_F32) {
        typename Chunk<float, N>::vec o;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = v[i];
        Chunk<float, N>::store(static_cast<float*>(a.Y) + at + d, have, o);
    } else if (a.y_type == ADADIM_TYPE_F16) {
        typename Chunk<_Float16, N>::vec o;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = static_cast<_Float16>(v[i]);
        Chunk<_Float16, N>::store(static_cast<_Float16*>(a.Y) + at + d, have, o);
    } else {
        typename Chunk<__bf16, N>::vec o;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = static_cast<__bf16>(v[i]);
        Chunk<__bf16, N>::store(static_cast<__bf16*>(a.Y) + at + d, have, o);
    }
}

__device__ __forceinline__ void put(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float get(const float* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// The rows of tile `tile` of R rows: sequence s has the tiles from offsets[s] * group / R + s on (enough for it: each begins one of its own).
struct TileRows {
    int64_t first;                                // token of row 0
    int rows;                                     // rows of the tile, 0: no such tile
    int token;                                    // of row 0 within the sequence's new ones
    int rest;                                     // its head within the group
    int added;                                    // the sequence's new tokens
    int sequence;
};
template <int R>
__device__ __forceinline__ TileRows tile_rows(const Attention& a, int tile) {
    const int lane = threadIdx.x & 63;
    auto offset = [&](int s) { return min(max(int64_t(a.offsets[s]), int64_t(0)), a.tokens); };
    auto begin = [&](int s) { return offset(s) * a.group / R + s; };
    int lo = 0, n = a.sequences;                  // the last of the n from lo on that begins at or before the tile
    while (n > 1) {
        const int step = (n + 63) / 64, s = lo + lane * step;
        const uint64_t at = __ballot(s < lo + n && begin(min(s, a.sequences)) <= tile);
        const int last = at ? 63 - __builtin_clzll(at) : 0;
        n = min(step, n - last * step);
        lo += last * step;
    }
    const int64_t o0 = offset(lo), o1 = offset(lo + 1);
    const int64_t r0 = (tile - begin(lo)) * R, have = (o1 - o0) * a.group;
    TileRows t;
    t.sequence = __builtin_amdgcn_readfirstlane(lo);
    t.added = __builtin_amdgcn_readfirstlane(static_cast<int>(max(o1 - o0, int64_t(0))));
    const bool ok = r0 >= 0 && r0 < have;
    t.rows = __builtin_amdgcn_readfirstlane(ok ? static_cast<int>(min(int64_t(R), have - r0)) : 0);
    t.token = __builtin_amdgcn_readfirstlane(ok ? static_cast<int>(r0 / a.group) : 0);
    t.rest = __builtin_amdgcn_readfirstlane(ok ? static_cast<int>(r0 % a.group) : 0);
    t.first = o0 + t.token;
    return t;
}

template <class T, int D, int NT, bool KEYS>
__global__ __launch_bounds__(64 * AT_WAVES) void mx4_attend(AttentionArgs args) {
    const Attention& a = args.a;
    constexpr int WROWS = 16 * NT, R = KEYS ? WROWS : AT_WAVES * WROWS;
    constexpr int TILES = D / 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    const int head = blockIdx.x % a.heads, tile = args.tiles - 1 - static_cast<int>(blockIdx.x / a.heads);        // (the longest rows first)
    const TileRows tr = tile_rows<R>(a, tile);
    if (tr.rows == 0) return;
    const int64_t most = a.width << a.log_page;
    const int length = static_cast<int>(min(max(int64_t(a.lengths[tr.sequence]), int64_t(0)), most));
    // the position of new token t is before + t
    const int before = length - tr.added;
    auto token_of = [&](int row) { return tr.token + (tr.rest + row) / a.group; };
    auto sees_to = [&](int token) { return a.causal ? min(max(before + token + 1, 0), length) : length; };
    auto sees_from = [&](int token) { return a.window ? static_cast<int>(max(int64_t(before) + token + 1 - a.window, int64_t(0))) : 0; };

    // ---- the records of the tile, of the workgroup's share, of the wave
    const int t_last = token_of(tr.rows - 1);
    const int r_begin = sees_from(tr.token) >> 5, r_end = (sees_to(t_last) + 31) >> 5;
    const int n_records = max(r_end - r_begin, 0);
    const int share = max((n_records + static_cast<int>(gridDim.y) - 1) / static_cast<int>(gridDim.y), args.least);
    const int shares = max((n_records + share - 1) / share, 1);
    if (static_cast<int>(blockIdx.y) >= shares) return;
    const int w_row = KEYS ? 0 : WROWS * wave;                // the wave's first row
    const int w_rows = min(WROWS, tr.rows - w_row);           // (not positive: none)
    int b = r_begin + share * blockIdx.y, e = min(b + share, r_end);
    const int w_first = token_of(w_row), w_last = token_of(max(w_row + w_rows - 1, w_row));
    if constexpr (KEYS) b += wave;
    else {
        if (w_rows <= 0) e = b;
        b = max(b, sees_from(w_first) >> 5);
        e = min(e, (sees_to(w_last) + 31) >> 5);
    }
    constexpr int STEP = KEYS ? AT_WAVES : 1;
    // records from all_from to before all_to hide nothing from any row
    const int all_from = (sees_from(w_last) + 31) >> 5, all_to = sees_to(w_first) >> 5;

    // ---- the wave's rows
    Rows<T, D, NT> rows;
    rows.c = a.scale * 1.44269504088896340736f;
    rows.clear();
    int row_token[NT], lo[NT], hi[NT];
    int64_t row_at[NT];                           // (token, head) of the lane's row, as the place of its element 0 in units of a pitch and elements
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = min(w_row + 16 * n + (lane & 15), tr.rows - 1);       // (rows that are not there repeat the last one)
        const int t = token_of(row), h = (tr.rest + row) % a.group;
        row_token[n] = t;
        lo[n] = sees_from(t);
        hi[n] = sees_to(t);
        row_at[n] = int64_t(head) * a.group + h;
        const T* q = static_cast<const T*>(a.Q) + (tr.first - tr.token + t) * a.ldq + row_at[n] * a.dim;
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
            const int d = (D / 4) * g + 8 * w;
            rows.q[n][w] = d < a.dim ? __builtin_bit_cast(typename Dots<T>::vec, Chunk<T, 8>::load(q + d, a.dim - d)) : typename Dots<T>::vec{};
        }
    }
    const int32_t* const table = a.table + int64_t(tr.sequence) * a.width;
    const int per_page = a.log_page - 5;
    auto page_of = [&](int r) { return r < e ? table[r >> per_page] : -1; };
    auto record = [&](int page, int r) {
        const int64_t p = uint32_t(page) < uint64_t(a.pages) ? page : 0;      // (a page that is not there is not used; page 0 is)
        return a.cache + (((p * a.heads + head) << per_page) + (r & ((1 << per_page) - 1))) * Record<D>::BYTES;
    };
    Bytes<D> now, next;
    int page = page_of(b), page1 = page_of(b + STEP);
    if (b < e) now.load(record(page, b), lane);
    for (; b < e; b += STEP) {
        const int page2 = page_of(b + 2 * STEP);
        if (b + STEP < e) next.load(record(page1, b + STEP), lane);
        if (uint32_t(page) < uint64_t(a.pages)) {
            int from[NT], to[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                from[n] = lo[n] - 32 * b;
                to[n] = hi[n] - 32 * b;
            }
            if (b >= all_from && b < all_to) rows.template add<false>(now, lane, from, to, 32);
            else rows.template add<true>(now, lane, from, to, length - 32 * b);
        }
        now = next;
        page = page1;
        page1 = page2;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) rows.l[n] = quarters(rows.l[n], [](float x, float y) { return x + y; });

    // ---- out.  parts: per shared tile and head [share][R rows][D + 2]: sums, then m and l
    constexpr int PITCH = D + 2;
    const int64_t item = int64_t(blockIdx.x);
    float* const mine = args.parts + (item * gridDim.y + blockIdx.y) * (R * PITCH);
    __shared__ unsigned s_ticket;
    if constexpr (KEYS) {
        constexpr int PARTS = D > 128 ? 2 : 1, JT = TILES / PARTS;             // (a part of D's elements at a time: 64 KB)
        __shared__ float s_o[AT_WAVES][16][16 * JT + 4];
        __shared__ float s_m[AT_WAVES][WROWS], s_l[AT_WAVES][WROWS];
        if (lane < 16)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                s_m[wave][16 * n + lane] = rows.m[n];
                s_l[wave][16 * n + lane] = rows.l[n];
            }
        __syncthreads();
        const int r = threadIdx.x >> 4, x = threadIdx.x & 15;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int rn = 16 * n + (lane & 15), row = 16 * n + r;
            float top = s_m[0][rn], m = s_m[0][row], l = 0.0f;
#pragma unroll
            for (int w = 1; w < AT_WAVES; ++w) {
                top = fmaxf(top, s_m[w][rn]);
                m = fmaxf(m, s_m[w][row]);
            }
            const float by = __builtin_amdgcn_exp2f(rows.m[n] - top);
#pragma unroll
            for (int w = 0; w < AT_WAVES; ++w) l += s_l[w][row] * __builtin_amdgcn_exp2f(s_m[w][row] - m);
            const float by1 = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
                if (n > 0 || part > 0) __syncthreads();
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < JT; ++j) s_o[wave][lane & 15][JT * (4 * g + i) + j] = rows.o[n][part * JT + j][i] * by;
                __syncthreads();
                if (row >= tr.rows) continue;
                const int d0 = TILES * x + part * JT;
                float v[JT];
#pragma unroll
                for (int j = 0; j < JT; ++j) {
                    v[j] = 0.0f;
#pragma unroll
                    for (int w = 0; w < AT_WAVES; ++w) v[j] += s_o[w][r][JT * x + j];
                }
                if (shares > 1) {
#pragma unroll
                    for (int j = 0; j < JT; ++j) put(mine + row * PITCH + d0 + j, v[j]);
                    if (d0 == 0) {
                        put(mine + row * PITCH + D, m);
                        put(mine + row * PITCH + D + 1, l);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < JT; ++j) v[j] = l == 0.0f ? 0.0f : v[j] * by1;
                    store_row(a, (tr.first - tr.token + token_of(row)) * a.ldy + (int64_t(head) * a.group + (tr.rest + row) % a.group) * a.dim, d0, v);
                }
            }
        }
    } else {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int row = w_row + 16 * n + (lane & 15);
            if (row >= tr.rows) continue;
            const float l = rows.l[n], by = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v[TILES];
#pragma unroll
                for (int j = 0; j < TILES; ++j) v[j] = rows.o[n][j][i];
                const int d = TILES * (4 * g + i);
                if (shares > 1) {
#pragma unroll
                    for (int j = 0; j < TILES; ++j) put(mine + row * PITCH + d + j, v[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < TILES; ++j) v[j] = l == 0.0f ? 0.0f : v[j] * by;
                    store_row(a, (tr.first - tr.token + row_token[n]) * a.ldy + row_at[n] * a.dim, d, v);
                }
            }
            if (shares > 1 && g == 0) {
                put(mine + row * PITCH + D, rows.m[n]);
                put(mine + row * PITCH + D + 1, l);
            }
        }
    }
    if (shares == 1) return;

    // ---- who finishes last joins the shares
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) s_ticket = __hip_atomic_fetch_add(args.tickets + item, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (s_ticket != unsigned(shares) - 1) return;
    if (threadIdx.x == 0) __hip_atomic_store(args.tickets + item, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const float* const all = args.parts + item * gridDim.y * (R * PITCH);
    const int d0 = (threadIdx.x & 15) * TILES;
    for (int row = threadIdx.x >> 4; row < tr.rows; row += 16) {
        const float* const p = all + row * PITCH;
        float m = LOWEST, l = 0.0f, v[TILES];
        for (int z = 0; z < shares; ++z) m = fmaxf(m, get(p + int64_t(z) * (R * PITCH) + D));
#pragma unroll
        for (int j = 0; j < TILES; ++j) v[j] = 0.0f;
        for (int z = 0; z < shares; ++z) {
            const float* const q = p + int64_t(z) * (R * PITCH);
            const float by = __builtin_amdgcn_exp2f(get(q + D) - m);
            l += get(q + D + 1) * by;
#pragma unroll
            for (int j = 0; j < TILES; ++j) v[j] += get(q + d0 + j) * by;
        }
#pragma unroll
        for (int j = 0; j < TILES; ++j) v[j] = l == 0.0f ? 0.0f : v[j] / l;
        store_row(a, (tr.first - tr.token + token_of(row)) * a.ldy + (int64_t(head) * a.group + (tr.rest + row) % a.group) * a.dim, d0, v);
    }
}

}  // namespace mx4
