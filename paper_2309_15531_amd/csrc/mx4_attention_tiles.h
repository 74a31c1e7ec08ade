// Attention of many rows over a paged cache in mx4 (the mathematics: mx4_attention.h).
//
// A workgroup has eight waves, two a SIMD, of 32 rows each: while one weighs scores on the vector unit the other multiplies.  Its records go
// through LDS four at a time, converted by one or two of the waves each: what costs most to prepare, the values of codes with their
// scales, is done once for all 256 rows.  They lie there as the 32-row instruction takes
// its left operand, lane by lane in 16 bytes (no bank is met twice in a read): keys [step][half][position], with step s of half h the
// elements h D/2 + 8 s ..; values [tile jj][step][half][row r], with row r of tile jj the element (D/16) (r % 16) + (D/32) (r / 16) + jj, and
// the step's positions 4 h .. and 8 + 4 h .. of 16 as S^T leaves them in a lane of half h.
//
// Neither unit is full: over the launch of chunks below the matrix pipe is busy 48 % and the vector unit 46 % of the clocks (16 exponentials, 16 sums,
// 16 fma, 8 roundings, maxima of a record and its share of the conversion), and waves wait 30 % of their time, for LDS and for each other: within
// a wave products and weights follow one another, and the SIMD's other wave does not fill the gaps.  4096 tokens into an empty cache, 32 heads of 128:
// 147 us, 935 TFLOP/s; 2 x 2048 tokens over 16384, 64 heads over 8: 1375 us, 1080 TFLOP/s.  Heads of 64: 107 and 865 us (vector unit 65 %), of
// 256, whose stages have one buffer: 331 and 2680 (waits 61 %).  What did not help there (the chunks, beside 1420 to 1490 as the cards went):
// scores one record ahead in a wave, 1850 (in order or left to the compiler); operands read from LDS ahead of use, 1500; waves' priorities, 1490;
// workgroups of six waves, three a SIMD, 1940, of four 1600; one buffer for two, 1480.  Every wave converting for itself, 64 rows of 16-row tiles: 5400.
#pragma once

#include "mx4_attention.h"

namespace mx4 {

template <class T> struct Dots32;
template <> struct Dots32<_Float16> {
    static __device__ __forceinline__ float16v mfma(half8v a, half8v b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Dots32<__bf16> {
    static __device__ __forceinline__ float16v mfma(bf8v a, bf8v b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

constexpr int TL_WAVES = 8;

template <int D>
struct Stage {
    static constexpr int KEYS = 64 * D, BYTES = 128 * D;      // of a record: its keys' part, all
    static constexpr int RECORDS = 4, BUFFERS = D > 128 ? 1 : 2;
    static constexpr int LDS = BUFFERS * RECORDS * BYTES;
};

// Half a record, its positions 16 t .. 16 t + 15, to its places in LDS.
template <class T, int D>
__device__ __forceinline__ void convert_keys(const KeyBytes<D>& b, uint8_t* to, int t, int lane) {
    constexpr int W = D / 32;
    const int m = lane & 15, g = lane >> 4;
#pragma unroll
    for (int w = 0; w < W; ++w)
        *reinterpret_cast<typename Dots<T>::vec*>(to + ((((g & 1) * W + w) * 2 + (g >> 1)) * 32 + 16 * t + m) * 16) = Dots<T>::keys(b.words[w], b.scale(w));
}
template <int D>
__device__ __forceinline__ void convert_values(const ValueBytes<D>& b, uint8_t* to, int t, int lane, int have) {
    const int m = lane & 15, g = lane >> 4;
    typedef _Float16 half4v __attribute__((ext_vector_type(4)));
    float vs[4];
    b.scales(vs, t, g, have);
    uint8_t* const v0 = to + Stage<D>::KEYS + (t * 64 + (g & 1) * 32 + m) * 16 + (g >> 1) * 8;
#pragma unroll
    for (int u = 0; u < D / 32; ++u) {
        half4v both[2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const half2v v = b.pair(i, u, vs[i]);
            both[0][i] = v.x;
            both[1][i] = v.y;
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int j = 2 * u + x, jj = j % (D / 32), high = j / (D / 32);                              // the unit's element j
            *reinterpret_cast<half4v*>(v0 + (jj * 128 + high * 16) * 16) = both[x];
        }
    }
}

template <class T, int D>
struct Tiles32 {
    static constexpr int STEPS = D / 16, OT = D / 32;
    typedef typename Dots<T>::vec vec;
    vec q[STEPS];
    float16v o[OT];
    Maximum top;
    float l;

    __device__ __forceinline__ float16v scores(const uint8_t* r, int lane) const {
        float16v s = {};
#pragma unroll
        for (int k = 0; k < STEPS; ++k) s = Dots32<T>::mfma(*reinterpret_cast<const vec*>(r + (k * 64 + lane) * 16), q[k], s);
        return s;
    }
    __device__ __forceinline__ void raise(float16v& s, float c, float step) {
        float most = fmaxf(s[0], s[1]);
#pragma unroll
        for (int i = 2; i < 16; ++i) most = fmaxf(most, s[i]);
        const bool passed = top.passed(most);
        if (passed || top.far) {
            if (passed) {
                const float by = top.raise(fmaxf(most, __shfl_xor(most, 32)), c, step);
                l *= by;
#pragma unroll
                for (int j = 0; j < OT; ++j) o[j] *= by;
            }
            if (top.far) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = from_top(s[i], top.limit);
            }
        }
    }
    __device__ __forceinline__ void weigh(const float16v& s, float c, half8v (&p)[2]) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, top.base));
            l += e;
            p[i >> 3][i & 7] = static_cast<_Float16>(e);
        }
    }
    __device__ __forceinline__ void values(const uint8_t* r, int lane, const half8v (&p)[2]) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < OT; ++j)
                o[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const half8v*>(r + Stage<D>::KEYS + ((j * 2 + k) * 64 + lane) * 16), p[k], o[j], 0, 0, 0);
    }
};

template <class T, int D>
__global__ __launch_bounds__(64 * TL_WAVES, 2) void mx4_attend_tiles(AttentionArgs args) {
    const Attention& a = args.a;
    constexpr int WROWS = 32, R = TL_WAVES * WROWS, N = D / 16;
    constexpr int BUFFERS = Stage<D>::BUFFERS, RECORDS = Stage<D>::RECORDS, BYTES = Stage<D>::BYTES;
    extern __shared__ __attribute__((aligned(16))) uint8_t s_stage[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const Work w = work_of<R, true>(args, blockIdx.y);                                        // (behind the first tiles those that see most first)
    if (w.shares == 0) return;

    // ---- the wave's rows and the records that they see
    const int w_row = WROWS * wave, w_last = min(w_row + WROWS, w.tr.rows) - 1;                           // (w_last < w_row: none)
    const int row = min(w_row + (lane & 31), w.tr.rows - 1), token = w.token_of(a, row);                  // (rows that are not there repeat the last one)
    const int t_first = uniform(w.token_of(a, min(w_row, w.tr.rows - 1))), t_last = uniform(w.token_of(a, max(w_last, 0)));
    const int from = w_last < w_row ? w.end : w.sees_from(a, t_first) >> 5;
    const int to = w_last < w_row ? w.begin : min((w.sees_to(a, t_last) + 31) >> 5, w.end);
    const int all_from = (w.sees_from(a, t_last) + 31) >> 5, all_to = w.sees_to(a, t_first) >> 5;         // (these hide nothing from any row)
    const int lo = w.sees_from(a, token), hi = w.sees_to(a, token);
    Tiles32<T, D> t;
    t.top.none();
    t.l = 0.0f;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) t.o[j] = float16v{};
    {
        const T* q = static_cast<const T*>(a.Q) + (w.tr.first - w.tr.token + token) * a.ldq + int64_t(w.head_of(a, row)) * a.dim;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            const int d = (D / 2) * h + 8 * k;
            t.q[k] = d < a.dim ? __builtin_bit_cast(typename Dots<T>::vec, Chunk<T, 8>::load(q + d, a.dim - d)) : typename Dots<T>::vec{};
        }
    }

    const int32_t* const table = a.table + int64_t(w.tr.sequence) * a.width;
    const int per_page = a.log_page - 5;
    auto page_of = [&](int r) { return r < w.end ? table[r >> per_page] : -1; };
    auto there = [&](int page) { return uint32_t(page) < uint64_t(a.pages); };
    // whether all the pages are there, looked up once for all: a scalar load for each record would be waited for
    bool whole = true;
    for (int p = (w.begin >> per_page) + lane, end = w.begin < w.end ? (w.end - 1) >> per_page : -1; __any(p <= end); p += 64) whole = whole && !__any(p <= end && !there(table[p]));
    // The first four waves convert a record of a stage each: they are issued first and would wait for the others, which are left more of the
    // vector unit so (4 % less time than with half a record to each of eight).  With 256 elements that takes too many registers: half a record each.
    constexpr int OWN = D > 128 ? 1 : 2;          // halves of a record
    const int part = wave & 3, own = OWN == 2 ? 0 : wave >> 2;
    const bool converts = OWN == 1 || wave < 4;
    KeyBytes<D> kb[OWN];
    ValueBytes<D> vb[OWN];
    // (the page's number a stage ahead, by a vector load: waiting for a scalar one would wait for LDS, too, and the other way)
    auto page_ahead = [&](int r) {
        int i = r < w.end ? r >> per_page : 0;
        asm volatile("" : "+v"(i));
        return table[i];
    };
    int page = page_ahead(w.begin + part);
    auto fetch = [&](int first) {
        const int r = first + part;
        if (r >= w.end || !converts) return;
        const int id = uniform(page);
        const int64_t p = there(id) ? id : 0;                 // (a page that is not there is not used; page 0 is)
        const uint8_t* const rec = a.cache + (((p * a.heads + w.head) << per_page) + (r & ((1 << per_page) - 1))) * Record<D>::BYTES;
        page = page_ahead(r + RECORDS);
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            kb[i].load(rec, own + i, lane);
            vb[i].load(rec, own + i, lane, a.dim);
        }
    };
    auto bring = [&](int first, int buffer) {
        const int r = first + part;
        if (r >= w.end || !converts) return;
        uint8_t* const at = s_stage + (buffer * RECORDS + part) * BYTES;
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            convert_keys<T, D>(kb[i], at, own + i, lane);
            convert_values<D>(vb[i], at, own + i, lane, w.length - RECORD * r);
        }
    };
    auto hide = [&](float16v& s, int r) {
        if (r >= all_from && r < all_to) return;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int key = RECORD * r + 8 * (i >> 2) + 4 * h + (i & 3);
            s[i] = key >= lo && key < hi ? s[i] : -INFINITY;
        }
    };
    auto stage = [&](int first, int buffer) {
        const uint8_t* const at = s_stage + buffer * RECORDS * BYTES;
        const int r1 = min(first + RECORDS, to);
        for (int r = max(first, from); r < r1; ++r) {
            if (!whole && !there(page_of(r))) continue;
            const uint8_t* const rec = at + (r - first) * BYTES;
            float16v s = t.scores(rec, lane);
            hide(s, r);
            t.raise(s, args.c, args.step);
            half8v p[2];
            t.weigh(s, args.c, p);
            t.values(rec, lane, p);
        }
    };
    fetch(w.begin);
    bring(w.begin, 0);
    fetch(w.begin + RECORDS);
    __syncthreads();
    int buffer = 0;
    for (int first = w.begin; first < w.end; first += RECORDS) {
        if constexpr (BUFFERS == 2) {
            bring(first + RECORDS, buffer ^ 1);
            fetch(first + 2 * RECORDS);
            stage(first, buffer);
            __syncthreads();
            buffer ^= 1;
        } else {
            stage(first, 0);
            __syncthreads();
            bring(first + RECORDS, 0);
            fetch(first + 2 * RECORDS);
            __syncthreads();
        }
    }

    // ---- out
    float* const mine = args.parts + (int64_t(blockIdx.x) * args.most + blockIdx.y) * (R * PART<D>);
    const float l = t.l + __shfl_xor(t.l, 32), by = l == 0.0f ? 0.0f : 1.0f / l, settled = t.top.settled(args.c, args.step);
    if (w_row + (lane & 31) <= w_last) {
        int out = row;                            // (worked out anew: no registers for it in the loop)
        asm volatile("" : "+v"(out));
        const int64_t y = w.row_of_y(a, out);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int d = N * (8 * (i >> 2) + 4 * h + (i & 3));
            float v[N];
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = t.o[j % (D / 32)][i + 8 * (j / (D / 32))];
            if (w.shares > 1) {
#pragma unroll
                for (int j = 0; j < N; j += 2) *reinterpret_cast<float2v*>(mine + row * PART<D> + d + j) = float2v{v[j] * settled, v[j + 1] * settled};
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) v[j] = l == 0.0f ? 0.0f : v[j] * by;
                store_row(a, y, d, v);
            }
        }
        if (w.shares > 1 && h == 0) *reinterpret_cast<float2v*>(mine + row * PART<D> + D) = float2v{t.top.m(args.step), l * settled};
    }
}

// The shares of the tiles that have several: a launch of its own, in which a tile's rows are spread over as many workgroups as it had waves.
// (Joined by the workgroup that finishes last, 20000 positions and 32 tokens of 64 heads over 8 took 198 us.)
template <int D>
__global__ __launch_bounds__(512) void mx4_attend_join(AttentionArgs args) {
    constexpr int R = 32 * TL_WAVES;
    const Work w = work_of<R, true>(args, 0);
    const int row = 32 * blockIdx.y;
    if (w.shares > 1 && row < w.tr.rows) join_rows<R, D>(args, w, row, min(row + 32, w.tr.rows), 32);
}

}  // namespace mx4
