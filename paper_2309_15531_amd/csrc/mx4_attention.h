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
// Few rows (this file): the four waves of a workgroup have the same rows and take records in turn; their sums meet in LDS.  Many rows:
// mx4_attention_tiles.h.  Either way a tile's records may be shared between workgroups (gridDim.y); partial sums travel as relaxed atomics at
// device scope, and the workgroup that finishes last joins them in their order: same bits every run.
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

// The bytes of a record's keys that a lane of row m and quarter g needs: of positions m and 16 + m the elements (D/4) g ...
template <int D>
struct KeyBytes {
    static constexpr int W = D / 32;
    uint32_t words[2][W], scale_bytes[2];
    __device__ __forceinline__ void load(const uint8_t* r, int lane) {
        const int m = lane & 15, g = lane >> 4;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = 16 * t + m;
            const uint32_t* p = reinterpret_cast<const uint32_t*>(r + key * (D / 2) + g * (D / 8));
#pragma unroll
            for (int c = 0; c < W; ++c) words[t][c] = p[c];
            if constexpr (D == 256) scale_bytes[t] = *reinterpret_cast<const uint16_t*>(r + Record<D>::KEY_SCALES + key * 8 + 2 * g);
            else scale_bytes[t] = r[Record<D>::KEY_SCALES + key * W + g * W / 4];
        }
    }
    __device__ __forceinline__ float scale(int t, int w) const {
        return scale_operand(D == 256 ? w < 4 ? scale_bytes[t] & 255u : scale_bytes[t] >> 8 : scale_bytes[t]);
    }
};

// Of its values: the elements m D/16 .. of the 8 positions of quarter g.
template <int D>
struct ValueBytes {
    static constexpr int W = D / 32;
    uint32_t words[D / 16], scale_words[2];
    __device__ __forceinline__ void load(const uint8_t* r, int lane) {
        const int m = lane & 15, g = lane >> 4;
        const uint32_t* p = reinterpret_cast<const uint32_t*>(r + Record<D>::VALUES + (g * 16 + m) * (8 * Record<D>::UNIT));
#pragma unroll
        for (int c = 0; c < D / 16; ++c) words[c] = p[c];
        const uint32_t* s = reinterpret_cast<const uint32_t*>(r + Record<D>::VALUE_SCALES + (g * W + m * W / 16) * 8);
        scale_words[0] = s[0];
        scale_words[1] = s[1];
    }
    // the 8 positions' scales; those that do not exist (have: how many do) become zeros whatever their codes: 2^-127 in fp16
    __device__ __forceinline__ void scales(float (&v)[8], int g, int have) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = scale_operand((scale_words[i >> 2] >> (8 * (i & 3))) & 255u);
        if (have < RECORD) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 4 * g + (i < 4 ? i : 12 + i) < have ? v[i] : 0.0f;
        }
    }
    // elements 2 u and 2 u + 1 of position i
    __device__ __forceinline__ half2v pair(int i, int u, float scale) const {
        const int at = i * W + u;
        switch (at & 3) {
            case 0: return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(words[at >> 2], scale, 0);
            case 1: return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(words[at >> 2], scale, 1);
            case 2: return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(words[at >> 2], scale, 2);
            default: return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(words[at >> 2], scale, 3);
        }
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
    __device__ __forceinline__ void add(const KeyBytes<D>& kb, const ValueBytes<D>& vb, int lane, bool mask, const int (&lo)[NT], const int (&hi)[NT], int have) {
        const int g = lane >> 4;
        float4v s[NT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int n = 0; n < NT; ++n) s[n][t] = float4v{0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const vec k = Dots<T>::keys(kb.words[t][w], kb.scale(t, w));
#pragma unroll
                for (int n = 0; n < NT; ++n) s[n][t] = Dots<T>::mfma(k, q[n][w], s[n][t]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);        // (keys' and values' operands are not held at the same time)
        if (mask) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int at = 16 * t + 4 * g + i;
                        s[n][t][i] = at >= lo[n] && at < hi[n] ? s[n][t][i] : -INFINITY;
                    }
        }
        float top[NT];
        bool raise = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
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
        __builtin_amdgcn_sched_barrier(0);
        float vs[8];
        vb.scales(vs, g, have);
#pragma unroll
        for (int u = 0; u < D / 32; ++u) {
            half8v even, odd;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const half2v v = vb.pair(i, u, vs[i]);
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

// What a workgroup has to do: its rows, the records of its share, how many shares there are (0: nothing to do).
struct Work {
    TileRows tr;
    int head, length, before;                     // before + t: the position of new token t
    int begin, end, shares;
    __device__ __forceinline__ int token_of(const Attention& a, int row) const { return tr.token + (tr.rest + row) / a.group; }
    __device__ __forceinline__ int head_of(const Attention& a, int row) const { return head * a.group + (tr.rest + row) % a.group; }
    __device__ __forceinline__ int sees_to(const Attention& a, int token) const { return a.causal ? min(max(before + token + 1, 0), length) : length; }
    __device__ __forceinline__ int sees_from(const Attention& a, int token) const {
        return a.window ? static_cast<int>(max(int64_t(before) + token + 1 - a.window, int64_t(0))) : 0;
    }
    __device__ __forceinline__ int64_t row_of_y(const Attention& a, int row) const {
        return (tr.first - tr.token + token_of(a, row)) * a.ldy + int64_t(head_of(a, row)) * a.dim;
    }
};
template <int R>
__device__ __forceinline__ Work work_of(const AttentionArgs& args) {
    const Attention& a = args.a;
    Work w;
    w.shares = 0;
    w.head = blockIdx.x % a.heads;
    w.tr = tile_rows<R>(a, args.tiles - 1 - static_cast<int>(blockIdx.x / a.heads));         // (the longest rows first)
    if (w.tr.rows == 0) return w;
    w.length = static_cast<int>(min(max(int64_t(a.lengths[w.tr.sequence]), int64_t(0)), a.width << a.log_page));
    w.before = w.length - w.tr.added;
    const int begin = w.sees_from(a, w.tr.token) >> 5, end = (w.sees_to(a, w.token_of(a, w.tr.rows - 1)) + 31) >> 5;
    const int records = max(end - begin, 0), y = static_cast<int>(blockIdx.y), ny = static_cast<int>(gridDim.y);
    const int share = max((records + ny - 1) / ny, args.least);
    const int shares = max((records + share - 1) / share, 1);
    w.shares = y < shares ? shares : 0;
    w.begin = begin + share * y;
    w.end = min(w.begin + share, end);
    return w;
}

// Partial sums: per tile, head and share [R rows][D + 2], the sums, then m and l.  Who finishes last joins the shares.
template <int D> constexpr int PART = D + 2;
template <int R, int D, int WAVES>
__device__ __forceinline__ void join(const AttentionArgs& args, const Work& w) {
    constexpr int N = D / 16;
    __shared__ unsigned s_ticket;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) s_ticket = __hip_atomic_fetch_add(args.tickets + blockIdx.x, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (s_ticket != unsigned(w.shares) - 1) return;
    if (threadIdx.x == 0) __hip_atomic_store(args.tickets + blockIdx.x, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const float* const all = args.parts + int64_t(blockIdx.x) * gridDim.y * (R * PART<D>);
    const int d0 = (threadIdx.x & 15) * N;
    for (int row = threadIdx.x >> 4; row < w.tr.rows; row += 4 * WAVES) {
        const float* const p = all + row * PART<D>;
        float m = LOWEST, l = 0.0f, v[N];
        for (int z = 0; z < w.shares; ++z) m = fmaxf(m, get(p + int64_t(z) * (R * PART<D>) + D));
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = 0.0f;
        for (int z = 0; z < w.shares; ++z) {
            const float* const q = p + int64_t(z) * (R * PART<D>);
            const float by = __builtin_amdgcn_exp2f(get(q + D) - m);
            l += get(q + D + 1) * by;
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] += get(q + d0 + j) * by;
        }
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = l == 0.0f ? 0.0f : v[j] / l;
        store_row(args.a, w.row_of_y(args.a, row), d0, v);
    }
}

// Waves of a SIMD that the registers have to leave room for.
template <int D, int NT> constexpr int FEW_WAVES = NT == 1 ? (D == 64 ? 4 : D == 128 ? 3 : 1) : D == 64 ? 3 : 2;

template <class T, int D, int NT>
__global__ __launch_bounds__(64 * AT_WAVES, (FEW_WAVES<D, NT>)) void mx4_attend_few(AttentionArgs args) {
    const Attention& a = args.a;
    constexpr int R = 16 * NT, TILES = D / 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    const Work w = work_of<R>(args);
    if (w.shares == 0) return;
    int b = w.begin + wave;
    const int e = w.end;
    const int t_last = w.token_of(a, w.tr.rows - 1);
    // records from all_from to before all_to hide nothing from any row
    const int all_from = (w.sees_from(a, t_last) + 31) >> 5, all_to = w.sees_to(a, w.tr.token) >> 5;

    Rows<T, D, NT> rows;
    rows.c = a.scale * 1.44269504088896340736f;
    rows.clear();
    int lo[NT], hi[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = min(16 * n + (lane & 15), w.tr.rows - 1);             // (rows that are not there repeat the last one)
        const int t = w.token_of(a, row);
        lo[n] = w.sees_from(a, t);
        hi[n] = w.sees_to(a, t);
        const T* q = static_cast<const T*>(a.Q) + (w.tr.first - w.tr.token + t) * a.ldq + int64_t(w.head_of(a, row)) * a.dim;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            const int d = (D / 4) * g + 8 * k;
            rows.q[n][k] = d < a.dim ? __builtin_bit_cast(typename Dots<T>::vec, Chunk<T, 8>::load(q + d, a.dim - d)) : typename Dots<T>::vec{};
        }
    }
    const int32_t* const table = a.table + int64_t(w.tr.sequence) * a.width;
    const int per_page = a.log_page - 5;
    auto page_of = [&](int r) { return r < e ? table[r >> per_page] : -1; };
    auto record = [&](int page, int r) {
        const int64_t p = uint32_t(page) < uint64_t(a.pages) ? page : 0;      // (a page that is not there is not used; page 0 is)
        return a.cache + (((p * a.heads + w.head) << per_page) + (r & ((1 << per_page) - 1))) * Record<D>::BYTES;
    };
    KeyBytes<D> k_now, k_next;
    ValueBytes<D> v_now, v_next;
    int page = page_of(b), page1 = page_of(b + AT_WAVES);
    if (b < e) {
        k_now.load(record(page, b), lane);
        v_now.load(record(page, b), lane);
    }
    for (; b < e; b += AT_WAVES) {
        const int page2 = page_of(b + 2 * AT_WAVES);
        if (b + AT_WAVES < e) {
            k_next.load(record(page1, b + AT_WAVES), lane);
            v_next.load(record(page1, b + AT_WAVES), lane);
        }
        if (uint32_t(page) < uint64_t(a.pages)) {
            int from[NT], to[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                from[n] = lo[n] - 32 * b;
                to[n] = hi[n] - 32 * b;
            }
            rows.add(k_now, v_now, lane, b < all_from || b >= all_to, from, to, w.length - 32 * b);
        }
        k_now = k_next;
        v_now = v_next;
        page = page1;
        page1 = page2;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) rows.l[n] = quarters(rows.l[n], [](float x, float y) { return x + y; });

    // ---- the four waves' sums
    float* const mine = args.parts + (int64_t(blockIdx.x) * gridDim.y + blockIdx.y) * (R * PART<D>);
    constexpr int PARTS = D > 128 ? 2 : 1, JT = TILES / PARTS;             // (a part of D's elements at a time: 64 KB)
    __shared__ float s_o[AT_WAVES][16][16 * JT + 4];
    __shared__ float s_m[AT_WAVES][R], s_l[AT_WAVES][R];
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
        for (int i = 1; i < AT_WAVES; ++i) {
            top = fmaxf(top, s_m[i][rn]);
            m = fmaxf(m, s_m[i][row]);
        }
        const float by = __builtin_amdgcn_exp2f(rows.m[n] - top);
#pragma unroll
        for (int i = 0; i < AT_WAVES; ++i) l += s_l[i][row] * __builtin_amdgcn_exp2f(s_m[i][row] - m);
        const float by1 = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
            if (n > 0 || part > 0) __syncthreads();
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < JT; ++j) s_o[wave][lane & 15][JT * (4 * g + i) + j] = rows.o[n][part * JT + j][i] * by;
            __syncthreads();
            if (row >= w.tr.rows) continue;
            const int d0 = TILES * x + part * JT;
            float v[JT];
#pragma unroll
            for (int j = 0; j < JT; ++j) {
                v[j] = 0.0f;
#pragma unroll
                for (int i = 0; i < AT_WAVES; ++i) v[j] += s_o[i][r][JT * x + j];
            }
            if (w.shares > 1) {
#pragma unroll
                for (int j = 0; j < JT; ++j) put(mine + row * PART<D> + d0 + j, v[j]);
                if (d0 == 0) {
                    put(mine + row * PART<D> + D, m);
                    put(mine + row * PART<D> + D + 1, l);
                }
            } else {
#pragma unroll
                for (int j = 0; j < JT; ++j) v[j] = l == 0.0f ? 0.0f : v[j] * by1;
                store_row(a, w.row_of_y(a, row), d0, v);
            }
        }
    }
    if (w.shares > 1) join<R, D, AT_WAVES>(args, w);
}

}  // namespace mx4
