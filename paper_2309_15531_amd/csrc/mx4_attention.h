// Attention over a paged cache in mx4:  y = sum_j softmax_j(scale q . k_j) v_j  over the positions j that a query sees.
//
// A tile is a number of rows (a row: one query head of one new token) of a sequence that share a key-value head.  A wave goes over records of 32
// positions:  S^T = K Q^T, keys converted in registers to the queries' type (exact: 2 bits and a scale that fp16 and bf16 have), then
// p = 2^(c (s - m) + 8) with c = scale log2(e) in fp32, rounded to fp16 (half a step of 11 bits; with the 2^8 the smallest number that fp16 still
// holds is 2^-33 of the row's largest), and O^T += V^T P^T with the values in fp16 (exact).  Positions lie along a lane's registers and rows
// along the lanes in S^T and in O^T: neither is turned round, and a row's maximum and sum are numbers of its lanes.  The maximum m, a score, is only
// raised (and O^T and the sum scaled) where a score passes it by more than 7 / c: p stays below 2^15.2.  The sum is of p before rounding.
// Scores, sums and O^T are fp32.
//
// Few rows (this file): the waves of a workgroup have the same rows and take records in turn; their sums meet in LDS.  Many rows:
// mx4_attention_tiles.h.  Either way a tile's records may be shared between workgroups (gridDim.y), whose partial sums are joined in their order:
// same bits every run.  Here they travel as relaxed atomics at device scope, and the workgroup that finishes last joins them.
//
// Few rows are bound by the read of the cache: 2 sequences to 100003 positions of 32 heads (674 MB) 126 us, 5.4 TB/s; 64 sequences of 1024 to 8192, 64
// heads over 8 (354 MB) 86 us, 4.1 TB/s.  A record takes a wave 0.85 us by itself (conversions, dependent products, exponentials), so a SIMD
// wants four of them: the bytes of one record at a time in registers and the queries in LDS leave 128 (149 registers and three waves with the
// next record's bytes beside them, in workgroups of four waves: 94 us, where this took 92).  16 rows to a tile, not 32: those take 250 registers and
// two waves (17 sequences, 6 tokens of 40 heads over 8: 36 us, 30 so).
#pragma once

#include "mx4_cache.h"

namespace mx4 {

constexpr int AT_WAVES = 8;                       // of a workgroup of few rows
constexpr int AT_TICKETS = 8192;                  // tiles that may be shared
constexpr float RAISE = 7.0f, HEAD = 8.0f;
constexpr float LARGEST = 3.402823466e38f;
constexpr float FAR = 1048576.0f;                 // |c m| from which on a wave weighs by differences of scores

struct AttentionArgs {
    Attention a;
    int tiles;                                    // row tiles, of which each sequence has one that may not exist
    int least;                                    // records that a share has at least
    int most;                                     // shares of a tile at most
    int round;                                    // workgroups that run at a time, where shares are to be alike over all sequences; or 0
    float c, step;                                // scale log2(e); RAISE / c, or 0 where fp32 does not hold that
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

// The bytes of a record's keys that a lane of row m and quarter g needs: of position 16 t + m the elements (D/4) g ..
template <int D>
struct KeyBytes {
    static constexpr int W = D / 32;
    uint32_t words[W], scale_bytes;
    __device__ __forceinline__ void load(const uint8_t* r, int t, int lane) {
        const int key = 16 * t + (lane & 15), g = lane >> 4;
        const uint32_t* p = reinterpret_cast<const uint32_t*>(r + key * (D / 2) + g * (D / 8));
#pragma unroll
        for (int c = 0; c < W; ++c) words[c] = p[c];
        if constexpr (D == 256) scale_bytes = *reinterpret_cast<const uint16_t*>(r + Record<D>::KEY_SCALES + key * 8 + 2 * g);
        else scale_bytes = r[Record<D>::KEY_SCALES + key * W + g * W / 4];
    }
    __device__ __forceinline__ float scale(int w) const {
        return scale_operand(D == 256 ? w < 4 ? scale_bytes & 255u : scale_bytes >> 8 : scale_bytes);
    }
};

// Of its values: the elements m D/16 .. of the positions 16 t + 4 g .. (four).
template <int D>
struct ValueBytes {
    static constexpr int W = D / 32;
    uint32_t words[W], scale_word;
    // dim: elements that are not filled up; lanes of units behind them (nobody stores what these come to) read the first unit's bytes again, not their own
    __device__ __forceinline__ void load(const uint8_t* r, int t, int lane, int dim) {
        const int m = (lane & 15) * (D / 16) < dim ? lane & 15 : 0, g = lane >> 4;
        const uint32_t* p = reinterpret_cast<const uint32_t*>(r + Record<D>::VALUES + ((g * 16 + m) * 8 + 4 * t) * Record<D>::UNIT);
#pragma unroll
        for (int c = 0; c < W; ++c) words[c] = p[c];
        scale_word = *reinterpret_cast<const uint32_t*>(r + Record<D>::VALUE_SCALES + (g * W + m * W / 16) * 8 + 4 * t);
    }
    // the positions' scales; those that do not exist (have: how many of the record do) become zeros whatever their codes: 2^-127 in fp16
    __device__ __forceinline__ void scales(float (&v)[4], int t, int g, int have) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = scale_operand((scale_word >> (8 * i)) & 255u);
        if (have < RECORD) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = 4 * g < have - 16 * t - i ? v[i] : 0.0f;            // (one register for all four)
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

// A difference from a row's maximum: finite also where there is none yet (m = -infinity), so that what is hidden stays -infinity.
__device__ __forceinline__ float from_top(float s, float m) { return s - fmaxf(m, -LARGEST); }

// A row's maximum m and how a wave takes weights from scores: by fma(s, c, base), in one of two ways that it chooses anew with each raise.
//   near  |c m| < 2^20 in all its rows: base = 8 - c m, of whose roundings (at most 3/32 together) all of a row's weights have the same share
//   far   the rounding of c m would be whole units of the exponent in the end: scores are taken as differences from m first (exact at the top), base = 8
struct Maximum {
    float limit, base;                            // a score beyond limit raises m: m + step when near, m itself when far; -infinity: no score yet
    bool far;                                     // the same in all lanes
    __device__ __forceinline__ void none() {
        limit = -INFINITY;
        base = HEAD;
        far = false;
    }
    // (near it may be off by a rounding of limit, or by up to step where that would be beyond fp32: weights go by base, and are related to m by it)
    __device__ __forceinline__ float m(float step) const { return far ? limit : limit - step; }
    __device__ __forceinline__ float exponent(float s, float c) const { return __builtin_fmaf(far ? from_top(s, limit) : s, c, base); }
    // top: the largest of a lane's new scores
    __device__ __forceinline__ bool passed(float top) const { return __any(top > limit); }
    // top: the row's; returns what sums so far are to be multiplied with
    __device__ __forceinline__ float raise(float top, float c, float step) {
        const float up = top > limit ? top : m(step), was = exponent(up, c), at = up * c;
        const bool had = limit > -INFINITY, has = up > -INFINITY;
        far = __any(has && !(fabsf(at) < FAR));
        base = HEAD - (far || !has ? 0.0f : at);
        limit = far ? up : fminf(up + step, LARGEST);
        const float now = __builtin_fmaf(far ? 0.0f : up, c, base);
        return had ? __builtin_amdgcn_exp2f(now - was) : 0.0f;
    }
    // what brings a row's sums to a weight of 2^8 for m
    __device__ __forceinline__ float settled(float c, float step) const {
        return far || !(limit > -INFINITY) ? 1.0f : __builtin_amdgcn_exp2f(HEAD - exponent(m(step), c));
    }
};

template <class T, int D>
struct Rows {
    static constexpr int W = D / 32, TILES = D / 16;
    typedef typename Dots<T>::vec vec;
    float4v o[TILES];
    Maximum top;
    float l;                                      // sum of this lane's p

    // q: the rows of Q in LDS, 64 lanes' 16 bytes for each of the W instructions
    static __device__ __forceinline__ void scores(const KeyBytes<D> (&b)[2], const vec* q, int lane, float4v (&s)[2]) {
        s[0] = s[1] = float4v{0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const vec x = q[w * 64 + lane];
#pragma unroll
            for (int t = 0; t < 2; ++t) s[t] = Dots<T>::mfma(Dots<T>::keys(b[t].words[w], b[t].scale(w)), x, s[t]);
        }
    }
    // what lies outside lo .. hi; first: the record's first position
    static __device__ __forceinline__ void hide(float4v (&s)[2], int g, int lo, int hi, int first) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = first + 16 * t + 4 * g + i;
                s[t][i] = at >= lo && at < hi ? s[t][i] : -INFINITY;
            }
    }
    __device__ __forceinline__ void weigh(float4v (&s)[2], float c, float step, half8v& p) {
        const float most = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        const bool passed = top.passed(most);
        if (passed || top.far) {
            if (passed) {
                const float by = top.raise(quarters(most, [](float x, float y) { return fmaxf(x, y); }), c, step);
                l *= by;
#pragma unroll
                for (int j = 0; j < TILES; ++j) o[j] *= by;
            }
            if (top.far) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[t][i] = from_top(s[t][i], top.limit);
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], c, top.base));
                l += e;
                p[4 * t + i] = static_cast<_Float16>(e);
            }
    }
    // have: how many positions of the record exist
    __device__ __forceinline__ void values(const ValueBytes<D> (&b)[2], int g, int have, const half8v& p) {
        float vs[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t) b[t].scales(vs[t], t, g, have);
#pragma unroll
        for (int u = 0; u < D / 32; ++u) {
            half8v even, odd;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const half2v v = b[i >> 2].pair(i & 3, u, vs[i >> 2][i & 3]);
                even[i] = v.x;
                odd[i] = v.y;
            }
            o[2 * u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(even, p, o[2 * u], 0, 0, 0);
            o[2 * u + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(odd, p, o[2 * u + 1], 0, 0, 0);
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

// Partial sums on their way past the L2s, where all XCDs meet: two numbers at a time.
typedef float float2p __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void put(float* p, float x, float y) {
    __hip_atomic_store(reinterpret_cast<uint64_t*>(p), __builtin_bit_cast(uint64_t, float2p{x, y}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2p get(const float* p) {
    return __builtin_bit_cast(float2p, __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// What all lanes have the same goes into a scalar register: branches and loads by it are scalar then.  (Quotients come from the vector unit.)
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// The rows of tile `tile` of R rows: the first `sequences` tiles are each sequence's first one; the further ones of sequence s are those from
// offsets[s] * group / R on behind them (enough for it: its rows are R times as many, and one tile is there already).
struct TileRows {
    int64_t first;                                // token of row 0
    int rows;                                     // rows of the tile, 0: no such tile
    int token;                                    // of row 0 within the sequence's new ones
    int rest;                                     // its head within the group
    int added;                                    // the sequence's new tokens
    int sequence;
    int length;                                   // its positions
};
template <int R>
__device__ __forceinline__ TileRows tile_rows(const Attention& a, int tile) {
    const int lane = threadIdx.x & 63;
    auto offset = [&](int s) { return static_cast<int>(min(max(int64_t(a.offsets[s]), int64_t(0)), a.tokens)); };
    int lo = tile, o0, o1, length;
    int64_t r0 = 0;
    if (tile < a.sequences) {                     // one load of each array
        const int o = offset(lo + (lane & 1));
        length = a.lengths[lo];
        o0 = __builtin_amdgcn_readlane(o, 0);
        o1 = __builtin_amdgcn_readlane(o, 1);
    } else {
        const int extra = tile - a.sequences;
        auto begin = [&](int o) { return static_cast<int>(int64_t(o) * a.group / R); };
        int n = a.sequences;                      // the last of the n from lo on whose further tiles begin at or before this one
        lo = 0;
        while (n > 63) {
            const int step = (n + 63) / 64, s = min(lo + lane * step, a.sequences);
            const uint64_t at = __ballot(s < lo + n && begin(offset(s)) <= extra);
            const int last = at ? 63 - __builtin_clzll(at) : 0;
            n = min(step, n - last * step);
            lo += last * step;
        }
        const int s = lo + min(lane, n), o = offset(s), l = a.lengths[min(s, a.sequences - 1)];
        const uint64_t at = __ballot(lane < n && begin(o) <= extra);
        const int last = at ? 63 - __builtin_clzll(at) : 0;
        o0 = __builtin_amdgcn_readlane(o, last);
        o1 = __builtin_amdgcn_readlane(o, last + 1);
        length = __builtin_amdgcn_readlane(l, last);
        lo += last;
        r0 = int64_t(extra - begin(o0) + 1) * R;
    }
    const int64_t have = int64_t(o1 - o0) * a.group;
    const bool ok = r0 >= 0 && r0 < have;
    TileRows t;
    t.sequence = uniform(lo);
    t.length = uniform(static_cast<int>(min(max(int64_t(length), int64_t(0)), a.width << a.log_page)));
    t.added = uniform(max(o1 - o0, 0));
    t.rows = uniform(ok ? static_cast<int>(min(int64_t(R), have - r0)) : 0);
    t.token = uniform(ok ? static_cast<int>(r0 / a.group) : 0);
    t.rest = uniform(ok ? static_cast<int>(r0 % a.group) : 0);
    t.first = uniform(o0) + t.token;
    return t;
}

// What a workgroup has to do: its rows, the records of its share, how many shares there are (0: nothing to do).
struct Work {
    TileRows tr;
    int head, length, before;                     // before + t: the position of new token t
    int shares, begin, end;
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
template <int R, bool LAST_FIRST>
__device__ __forceinline__ Work work_of(const AttentionArgs& args, int y) {
    const Attention& a = args.a;
    Work w;
    w.shares = 0;
    w.head = blockIdx.x % a.heads;
    const int tile = blockIdx.x / a.heads;
    w.tr = tile_rows<R>(a, LAST_FIRST && tile >= a.sequences ? args.tiles - 1 - (tile - a.sequences) : tile);
    if (w.tr.rows == 0) return w;
    w.length = w.tr.length;
    w.before = w.length - w.tr.added;
    const int begin = uniform(w.sees_from(a, w.tr.token) >> 5), end = uniform((w.sees_to(a, w.token_of(a, w.tr.rows - 1)) + 31) >> 5);
    const int records = max(end - begin, 0);
    int least = args.least;
    if constexpr (!LAST_FIRST) {
        // Shares as long in one sequence as in the other, so long that all of them (those that are not divisible among them) are whole rounds
        // of workgroups; one sequence to a lane.  2 sequences to 100003: 126 us, 147 with as many shares for each.
        if (args.round > 0) {
            const int lane = threadIdx.x & 63, s = min(lane, a.sequences - 1);
            const int o0 = min(max(a.offsets[s], 0), static_cast<int>(a.tokens)), o1 = min(max(a.offsets[s + 1], o0), static_cast<int>(a.tokens));
            const int64_t length = min(max(int64_t(a.lengths[s]), int64_t(0)), a.width << a.log_page);
            const int64_t from = a.window ? max(length - (o1 - o0) + 1 - a.window, int64_t(0)) : 0;
            float tiles = lane < a.sequences ? static_cast<float>((int64_t(o1 - o0) * a.group + R - 1) / R) : 0.0f;
            float all = tiles * static_cast<float>(((length + 31) >> 5) - (from >> 5));
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                tiles += __shfl_xor(tiles, d);
                all += __shfl_xor(all, d);
            }
            const float items = tiles * a.heads, rounds = args.round * fmaxf(ceilf(1.5f * items / args.round), 1.0f);
            least = uniform(max(static_cast<int>(all * a.heads / (rounds - 0.5f * items)) + 1, args.least));
        }
    }
    const int share = uniform(max((records + args.most - 1) / args.most, least));
    const int shares = uniform(max((records + share - 1) / share, 1));
    if (y >= shares) return w;
    w.shares = shares;
    w.begin = begin + share * y;
    w.end = min(w.begin + share, end);
    return w;
}

// Partial sums: per tile, head and share [R rows][D + 2], the sums, then m and l.  Joining them: 16 lanes a row, whose lane x has the elements
// 64 j + 4 x .. and first the m and l of the shares x, x + 16, ..; `at_once` rows from row0 on, one for each 16 threads.
template <int D> constexpr int PART = D + 2;
constexpr int MOST_SHARES = 64;
template <int R, int D>
__device__ __forceinline__ void join_rows(const AttentionArgs& args, const Work& w, int row_begin, int row_end, int at_once) {
    constexpr int N = D / 64, AT_ONCE = 4;
    const float* const all = args.parts + int64_t(blockIdx.x) * args.most * (R * PART<D>);
    const int x = threadIdx.x & 15, lane0 = threadIdx.x & 48;
    for (int row0 = row_begin; row0 < row_end; row0 += at_once) {
        const int row = min(row0 + static_cast<int>(threadIdx.x >> 4), row_end - 1);
        const float* const p = all + row * PART<D>;
        float by[MOST_SHARES / 16], m = -INFINITY, l = 0.0f;
        float2p ml[MOST_SHARES / 16];
#pragma unroll
        for (int i = 0; i < MOST_SHARES / 16; ++i) ml[i] = 16 * i + x < w.shares ? get(p + int64_t(16 * i + x) * (R * PART<D>) + D) : float2p{-INFINITY, 0.0f};
#pragma unroll
        for (int i = 0; i < MOST_SHARES / 16; ++i) m = fmaxf(m, ml[i].x);
#pragma unroll
        for (int d = 1; d < 16; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
#pragma unroll
        for (int i = 0; i < MOST_SHARES / 16; ++i) {
            by[i] = __builtin_amdgcn_exp2f(from_top(ml[i].x, m) * args.c);
            l += ml[i].y * by[i];
        }
#pragma unroll
        for (int d = 1; d < 16; d *= 2) l += __shfl_xor(l, d);
        float v[N][4];
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) v[j][k] = 0.0f;
#pragma unroll
        for (int i = 0; i < MOST_SHARES / 16; ++i)
            for (int z0 = 16 * i; z0 < min(16 * i + 16, w.shares); z0 += AT_ONCE) {
                float2p part[AT_ONCE][N][2];
#pragma unroll
                for (int z = 0; z < AT_ONCE; ++z)
#pragma unroll
                    for (int j = 0; j < N; ++j)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            part[z][j][k] = float2p{0.0f, 0.0f};
                            if (z0 + z < w.shares) part[z][j][k] = get(p + int64_t(z0 + z) * (R * PART<D>) + 64 * j + 4 * x + 2 * k);
                        }
#pragma unroll
                for (int z = 0; z < AT_ONCE; ++z) {
                    const float f = __shfl(by[i], lane0 + ((z0 + z) & 15));
#pragma unroll
                    for (int j = 0; j < N; ++j)
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[j][k] += part[z][j][k >> 1][k & 1] * f;
                }
            }
        if (row0 + static_cast<int>(threadIdx.x >> 4) >= row_end) continue;
        const int64_t y = w.row_of_y(args.a, row);
#pragma unroll
        for (int j = 0; j < N; ++j) {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[j][k] = l == 0.0f ? 0.0f : v[j][k] / l;
            store_row(args.a, y, 64 * j + 4 * x, v[j]);
        }
    }
}

// The workgroup that finishes last joins.
template <int R, int D, int WAVES>
__device__ __forceinline__ void join(const AttentionArgs& args, const Work& w) {
    __shared__ unsigned s_ticket;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) s_ticket = __hip_atomic_fetch_add(args.tickets + blockIdx.x, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (s_ticket != unsigned(w.shares) - 1) return;
    if (threadIdx.x == 0) __hip_atomic_store(args.tickets + blockIdx.x, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    join_rows<R, D>(args, w, 0, w.tr.rows, 4 * WAVES);
}

// Waves of a SIMD that the registers have to leave room for.
template <int D> constexpr int FEW_WAVES = D <= 128 ? 4 : 2;

template <class T, int D>
__global__ __launch_bounds__(64 * AT_WAVES, FEW_WAVES<D>) void mx4_attend_few(AttentionArgs args) {
    const Attention& a = args.a;
    constexpr int R = 16, TILES = D / 16, W = D / 32;
    typedef typename Dots<T>::vec vec;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    const Work w = work_of<R, false>(args, blockIdx.y);
    if (w.shares == 0) return;
    int b = w.begin + wave;
    const int e = w.end;
    const int32_t* const table = a.table + int64_t(w.tr.sequence) * a.width;
    const int per_page = a.log_page - 5;
    auto page_of = [&](int r) { return r < e ? table[r >> per_page] : -1; };
    auto there = [&](int page) { return uint32_t(page) < uint64_t(a.pages); };
    auto record = [&](int page, int r) {
        const int64_t p = there(page) ? page : 0;             // (a page that is not there is not used; page 0 is)
        return a.cache + (((p * a.heads + w.head) << per_page) + (r & ((1 << per_page) - 1))) * Record<D>::BYTES;
    };
    int page = page_of(b), page1 = page_of(b + AT_WAVES);
    KeyBytes<D> kb[2];
    ValueBytes<D> vb[2];
    auto load_keys = [&](const uint8_t* r) { kb[0].load(r, 0, lane); kb[1].load(r, 1, lane); };
    auto load_values = [&](const uint8_t* r) { vb[0].load(r, 0, lane, a.dim); vb[1].load(r, 1, lane, a.dim); };
    if (b < e) {
        load_keys(record(page, b));
        load_values(record(page, b));
    }

    // ---- the rows: every wave has the same
    __shared__ vec s_q[W * 64];
    Rows<T, D> rows;
    rows.top.none();
    rows.l = 0.0f;
#pragma unroll
    for (int j = 0; j < TILES; ++j) rows.o[j] = float4v{0, 0, 0, 0};
    const int my_row = min(lane & 15, w.tr.rows - 1), token = w.token_of(a, my_row);        // (rows that are not there repeat the last one)
    const int lo = w.sees_from(a, token), hi = w.sees_to(a, token);
    if (wave < W) {
        const T* q = static_cast<const T*>(a.Q) + (w.tr.first - w.tr.token + token) * a.ldq + int64_t(w.head_of(a, my_row)) * a.dim;
        const int d = (D / 4) * g + 8 * wave;
        s_q[wave * 64 + lane] = d < a.dim ? __builtin_bit_cast(vec, Chunk<T, 8>::load(q + d, a.dim - d)) : vec{};
    }
    // records from all_from to before all_to hide nothing from any row
    const int all_from = uniform((w.sees_from(a, w.token_of(a, w.tr.rows - 1)) + 31) >> 5), all_to = uniform(w.sees_to(a, w.tr.token) >> 5);
    __syncthreads();

    for (; b < e; b += AT_WAVES) {
        // the next record's keys come while this one's scores are weighed, its values while the next one's scores are computed: bytes of
        // one record at a time, in favour of more waves
        const int next = b + AT_WAVES, page2 = page_of(next + AT_WAVES);
        const bool use = there(page);
        float4v s[2];
        half8v p;
        if (use) rows.scores(kb, s_q, lane, s);
        __builtin_amdgcn_sched_barrier(0);
        if (next < e) load_keys(record(page1, next));
        if (use) {
            if (b < all_from || b >= all_to) rows.hide(s, g, lo, hi, RECORD * b);
            rows.weigh(s, args.c, args.step, p);
            __builtin_amdgcn_sched_barrier(0);
            rows.values(vb, g, w.length - RECORD * b, p);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (next < e) load_values(record(page1, next));
        page = page1;
        page1 = page2;
    }
    const float settled = rows.top.settled(args.c, args.step), m_wave = rows.top.m(args.step);
    rows.l = quarters(rows.l, [](float x, float y) { return x + y; }) * settled;

    // ---- the waves' sums, in PASSES of 64 elements (35 KB): of the TILES elements of a unit the four from 4 pass on (all with D = 64)
    float* const mine = args.parts + (int64_t(blockIdx.x) * args.most + blockIdx.y) * (R * PART<D>);
    constexpr int PASSES = D / 64;
    __shared__ __attribute__((aligned(16))) float s_o[AT_WAVES][16][64 + 4];
    __shared__ float s_m[AT_WAVES][R], s_l[AT_WAVES][R];
    if (lane < 16) {
        s_m[wave][lane] = m_wave;
        s_l[wave][lane] = rows.l;
    }
    __syncthreads();
    const int row = threadIdx.x >> 5, x = threadIdx.x & 31;   // 32 lanes a row, two elements each
    float top = s_m[0][lane & 15], m = s_m[0][row], l = 0.0f;
#pragma unroll
    for (int i = 1; i < AT_WAVES; ++i) {
        top = fmaxf(top, s_m[i][lane & 15]);
        m = fmaxf(m, s_m[i][row]);
    }
    const float by = __builtin_amdgcn_exp2f(from_top(m_wave, top) * args.c) * settled;
#pragma unroll
    for (int i = 0; i < AT_WAVES; ++i) l += s_l[i][row] * __builtin_amdgcn_exp2f(from_top(s_m[i][row], m) * args.c);
    const float by1 = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
        if (pass > 0) __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float4v v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = rows.o[4 * pass + j][i] * by;
            *reinterpret_cast<float4v*>(&s_o[wave][lane & 15][4 * (4 * g + i)]) = v;
        }
        __syncthreads();
        if (row >= w.tr.rows) continue;
        float v[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < AT_WAVES; ++i) {
            const float2v o = *reinterpret_cast<const float2v*>(&s_o[i][row][2 * x]);
            v[0] += o.x;
            v[1] += o.y;
        }
        const int d = (x >> 1) * TILES + 4 * pass + 2 * (x & 1);
        if (w.shares > 1) {
            put(mine + row * PART<D> + d, v[0], v[1]);
            if (x == 0 && pass == 0) put(mine + row * PART<D> + D, m, l);
        } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) v[k] = l == 0.0f ? 0.0f : v[k] * by1;
            store_row(a, w.row_of_y(a, row), d, v);
        }
    }
    if (w.shares > 1) join<R, D, AT_WAVES>(args, w);
}

}  // namespace mx4
