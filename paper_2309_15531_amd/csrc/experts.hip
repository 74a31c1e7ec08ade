// A router's scores to its choice of experts and the rows sorted by expert, and the experts' outputs back to the tokens.
//
// Choice: the k largest scores of a token, the lowest index first among equal ones; a score of -infinity or NaN is never
// chosen (a token may have fewer than k experts, or none: -1 in the free places, their weight 0).  Weights in fp32:
//     exp(l_j - max) / sum   over the chosen (renormalize) or over all scores;  +infinite scores share among themselves.
// Order: the rows of expert e are those tokens that chose it, in the order of the tokens: a counting sort whose ranks come
// from one bit per (token, expert), so that no order of arrival is visible in the result.
#include "common.h"

namespace {

// Larger number, larger key; -infinity and NaN have key 0 and never win.  (-0 and +0 are equal scores.)  A 16-bit score's key has its place
// below it, the lower the larger: one comparison finds both.
template <class T>
struct Keys {
    static constexpr bool WITH_PLACE = sizeof(T) == 2;
    static __device__ __forceinline__ uint32_t of(float f, uint32_t place) {
        if (!(f > -INFINITY)) return 0u;
        if constexpr (WITH_PLACE) {
            const uint32_t u = __builtin_bit_cast(uint16_t, static_cast<T>(f + 0.0f));
            return (u & 0x8000u ? ~u : u | 0x8000u) << 16 | (0xffffu - place);
        } else {
            const uint32_t u = __float_as_uint(f + 0.0f);
            return u & 0x80000000u ? ~u : u | 0x80000000u;
        }
    }
    static __device__ __forceinline__ float score(uint32_t key) {
        if constexpr (WITH_PLACE) {
            const uint32_t u = key >> 16;
            return static_cast<float>(__builtin_bit_cast(T, static_cast<uint16_t>(u & 0x8000u ? u & 0x7fffu : ~u)));
        } else return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
    }
};

constexpr int RT_TOKENS = 64;                     // tokens of a chunk: one bit each of an expert's mask
constexpr int RT_THREADS = 1024;
constexpr int RT_GROUPS = 256;                    // workgroups that place rows, at most

struct Route {
    const void* logits;
    int64_t tokens, ldl;
    int experts, k, renormalize;
    int32_t* chosen;
    float* weights;
    int32_t *offsets, *rows, *slots;
    uint64_t* masks;                              // [chunks][experts]: the tokens of the chunk that chose the expert
    uint8_t* counts;                              // [chunks][experts, up to the next multiple of 4]: how many
};

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xF, 0xF, false));
}
constexpr int QUAD_XOR1 = 0xB1, QUAD_XOR2 = 0x4E, HALF_MIRROR = 0x141, ROW_MIRROR = 0x140;
// f over the W (8 or 16) lanes of a token, the result in all of them
template <int W, class F>
__device__ __forceinline__ uint32_t over_lanes(uint32_t v, F f) {
    v = f(v, dpp<QUAD_XOR1>(v));
    v = f(v, dpp<QUAD_XOR2>(v));
    v = f(v, dpp<HALF_MIRROR>(v));
    if constexpr (W == 16) v = f(v, dpp<ROW_MIRROR>(v));
    return v;
}

// The sums of n (at most RT_THREADS) numbers in front of each, and of all; s_sum: RT_THREADS / 64 words.
__device__ __forceinline__ int32_t sum_before(int32_t n, int32_t& all, int32_t* s_sum) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t sum = n;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int32_t o = __shfl_up(sum, d);
        if (lane >= d) sum += o;
    }
    if (lane == 63) s_sum[wave] = sum;
    __syncthreads();
    int32_t before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < RT_THREADS / 64; ++w) {
        if (w < wave) before += s_sum[w];
        all += s_sum[w];
    }
    return before + sum - n;
}

// The rows and slots of chunk c, whose rows of expert e begin at base[e].
__device__ __forceinline__ void place_chunk(const Route& a, int64_t c, const uint64_t* mask, const int32_t* base) {
    const int64_t t0 = c * RT_TOKENS;
    const int n = static_cast<int>(min(int64_t(RT_TOKENS), a.tokens - t0)) * a.k;
    for (int i = threadIdx.x; i < n; i += RT_THREADS) {
        const int tt = i / a.k;
        const int32_t e = a.chosen[t0 * a.k + i];
        int32_t slot = -1;
        if (e >= 0) {
            slot = base[e] + __popcll(mask[e] & ((uint64_t(1) << tt) - 1));
            a.rows[slot] = static_cast<int32_t>(t0 + tt);
        }
        a.slots[t0 * a.k + i] = slot;
    }
}

// A chunk of 64 tokens.  W lanes a token, V consecutive scores each: k times the largest left, over a lane's own and then over the lanes by DPP,
// its lowest index the same way.  Fewer lanes with more scores each would be less work still, but the loads would no longer be whole
// lines.  Where the chunk is all there is, the rows are placed too, in the same launch.
// 16 tokens of 8 experts: 2.9 us, bound by latency (its waves wait for 74 % of their time).  16384 of 128 in bf16: 7.3 us, bound by issue: 570 vector
// instructions a wave and four waves on a SIMD keep it issuing for 68 % of their time (k = 8 rounds; the scores, 4.2 MB, would take 1 us).
template <class T, int W, int V>
__global__ __launch_bounds__(RT_THREADS) void route_choose(Route a) {
    extern __shared__ uint64_t s_mask[];          // [experts], then int32 [experts]
    __shared__ int32_t s_sum[RT_THREADS / 64];
    const int sub = threadIdx.x % W;
    for (int i = threadIdx.x; i < a.experts; i += RT_THREADS) s_mask[i] = 0u;
    __syncthreads();
    for (int tt = threadIdx.x / W; tt < RT_TOKENS; tt += RT_THREADS / W) {
        const int64_t t = int64_t(blockIdx.x) * RT_TOKENS + tt;
        const bool real = t < a.tokens;           // (all lanes go through the moves between lanes)
        float f[V];
        uint32_t key[V];
        const T* l = static_cast<const T*>(a.logits) + (real ? t : 0) * a.ldl + sub * V;
        const int have = a.experts - sub * V;
        typedef T vec __attribute__((ext_vector_type(V)));
        if (have >= V) {
            vec v;
            __builtin_memcpy(&v, l, sizeof(v));
#pragma unroll
            for (int v_ = 0; v_ < V; ++v_) f[v_] = static_cast<float>(v[v_]);
        } else {
#pragma unroll
            for (int v_ = 0; v_ < V; ++v_) f[v_] = v_ < have ? static_cast<float>(l[v_]) : -INFINITY;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = Keys<T>::of(f[v], sub * V + v);
        float top = 0.0f, sum = 0.0f, mine[2] = {};           // lane j (and j + W): exp(l - max) of the j-th chosen
        int32_t index[2] = {-1, -1};
        for (int j = 0; j < a.k; ++j) {
            uint32_t best = 0u;
#pragma unroll
            for (int v = 0; v < V; ++v) best = max(best, key[v]);
            best = over_lanes<W>(best, [](uint32_t x, uint32_t y) { return max(x, y); });
            if (__ballot(best != 0u) == 0) break;             // nothing left of any of the wave's tokens
            uint32_t at = 0xffffu - (best & 0xffffu);
            if constexpr (Keys<T>::WITH_PLACE) {
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (key[v] == best) key[v] = 0u;
            } else {
                at = 0xffffffffu;
#pragma unroll
                for (int v = V - 1; v >= 0; --v)
                    if (key[v] == best) at = sub * V + v;
                at = over_lanes<W>(at, [](uint32_t x, uint32_t y) { return min(x, y); });
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (at == static_cast<uint32_t>(sub * V + v)) key[v] = 0u;
            }
            if (best != 0u) {
                const float val = Keys<T>::score(best);
                if (j == 0) top = val;
                const float p = val == top ? 1.0f : expf(val - top);
                sum += p;
                if (sub == j % W) {
                    mine[W == 16 && j >= W] = p;
                    index[W == 16 && j >= W] = static_cast<int32_t>(at);
                }
                if (sub == 0 && real) atomicOr(reinterpret_cast<unsigned long long*>(&s_mask[at]), 1ull << tt);
            }
        }
        if (!a.renormalize) {
            sum = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (f[v] > -INFINITY) sum += f[v] == top ? 1.0f : expf(f[v] - top);
            sum = __uint_as_float(over_lanes<W>(__float_as_uint(sum), [](uint32_t x, uint32_t y) {
                return __float_as_uint(__uint_as_float(x) + __uint_as_float(y));
            }));
            sum = __shfl(sum, (threadIdx.x & 63) & ~(W - 1));         // (the lanes added in different orders)
        }
#pragma unroll
        for (int h = 0; h < (W == 16 ? 2 : 1); ++h)
            if (real && sub + h * W < a.k) {
                a.chosen[t * a.k + sub + h * W] = index[h];
                a.weights[t * a.k + sub + h * W] = index[h] >= 0 ? mine[h] / sum : 0.0f;
            }
    }
    __syncthreads();
    const int e = threadIdx.x;
    const int32_t n = e < a.experts ? __popcll(s_mask[e]) : 0;
    if (gridDim.x > 1) {
        const int pitch = (a.experts + 3) & ~3;
        if (e < a.experts) a.masks[int64_t(blockIdx.x) * a.experts + e] = s_mask[e];
        if (e < pitch) a.counts[int64_t(blockIdx.x) * pitch + e] = static_cast<uint8_t>(n);
        return;
    }
    int32_t all, *s_base = reinterpret_cast<int32_t*>(s_mask + a.experts);
    const int32_t at = sum_before(n, all, s_sum);
    if (e < a.experts) {
        s_base[e] = at;
        a.offsets[e] = at;
        if (e == a.experts - 1) a.offsets[a.experts] = all;
    }
    __syncthreads();                              // (the choices above are visible to the workgroup, too)
    place_chunk(a, 0, s_mask, s_base);
    for (int64_t i = all + e; i < a.tokens * a.k; i += RT_THREADS) a.rows[i] = -1;
}

// Several chunks: workgroup g places the rows of `per` of them.  It adds up the counts of all chunks (four experts to a word, the
// rows of counts dealt to the threads), once for those in front of its own and once for all.  131072 rows of 128 experts: 6.5 us, bound by
// latency (its waves wait for 59 % of their time, and issue for 49 %).
__global__ __launch_bounds__(RT_THREADS) void route_place(Route a, int64_t chunks, int64_t per) {
    extern __shared__ int32_t s_total[];          // [2][experts up to 4]: of all chunks, of those in front
    __shared__ int32_t s_sum[RT_THREADS / 64];
    const int pitch = (a.experts + 3) & ~3, words = pitch / 4;
    int32_t* const s_before = s_total + pitch;
    const int64_t first = blockIdx.x * per, last = min(first + per, chunks);
    for (int i = threadIdx.x; i < 2 * pitch; i += RT_THREADS) s_total[i] = 0;
    __syncthreads();
    const int lanes = RT_THREADS / words;         // rows of counts at a time (words <= 256)
    if (static_cast<int>(threadIdx.x) < lanes * words) {
        const int w = threadIdx.x % words;
        const uint32_t* counts = reinterpret_cast<const uint32_t*>(a.counts) + w;
        int32_t total[4] = {}, before[4] = {};
        for (int64_t c0 = threadIdx.x / words; c0 < chunks; c0 += 8 * lanes) {
            uint32_t q[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) q[u] = c0 + u * lanes < chunks ? counts[(c0 + u * lanes) * words] : 0u;
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const int32_t n = (q[u] >> (8 * b)) & 255u;
                    total[b] += n;
                    if (c0 + u * lanes < first) before[b] += n;
                }
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            atomicAdd(&s_total[4 * w + b], total[b]);         // (whole numbers: the order does not show)
            atomicAdd(&s_before[4 * w + b], before[b]);
        }
    }
    __syncthreads();
    const int e = threadIdx.x;
    int32_t all;
    const int32_t at = sum_before(e < a.experts ? s_total[e] : 0, all, s_sum);
    if (e < a.experts) {
        s_before[e] += at;
        if (blockIdx.x == 0) {
            a.offsets[e] = at;
            if (e == a.experts - 1) a.offsets[a.experts] = all;
        }
    }
    __syncthreads();
    for (int64_t c = first; c < last; ++c) {
        place_chunk(a, c, a.masks + c * a.experts, s_before);
        __syncthreads();
        if (e < a.experts) s_before[e] += __popcll(a.masks[c * a.experts + e]);
        __syncthreads();
    }
    // the places that no row takes
    const int64_t end = min(last * RT_TOKENS, a.tokens) * a.k;
    for (int64_t i = max(first * RT_TOKENS * a.k, int64_t(all)) + e; i < end; i += RT_THREADS) a.rows[i] = -1;
}

__global__ void route_none(int32_t* offsets, int experts) {
    for (int e = threadIdx.x; e <= experts; e += blockDim.x) offsets[e] = 0;
}

// Y[t] = sum_j weights[t, j] Z[slots[t, j]]: fp32, in the order of j, rounded once.  Bound by HBM: every row of Z is
// read once.  A lane takes eight columns of a token.  8192 tokens x 8, 4096 columns of bf16: 121 us, 5.0 TB/s (a large copy: 5.06).
template <class T, int N>
struct Pack {
    typedef T vec __attribute__((ext_vector_type(N)));
};

template <class TZ, class TY>
__global__ __launch_bounds__(256) void combine_rows(const TZ* __restrict__ Z, int64_t n_rows, int64_t cols, int64_t ldz,
                                                    const int32_t* __restrict__ slots, const float* __restrict__ weights,
                                                    int64_t tokens, int k, uint32_t col_tiles, TY* __restrict__ Y, int64_t ldy) {
    const int64_t t = blockIdx.x / col_tiles, c = (int64_t(blockIdx.x % col_tiles) * 256 + threadIdx.x) * 8;
    if (c >= cols) return;
    const int have = static_cast<int>(min(int64_t(8), cols - c));
    float acc[8] = {};
    for (int j = 0; j < k; ++j) {
        const int32_t s = slots[t * k + j];
        if (s < 0 || s >= n_rows) continue;
        const float w = weights[t * k + j];
        const TZ* z = Z + int64_t(s) * ldz + c;
        typename Pack<TZ, 8>::vec v = {};
        if (have == 8) __builtin_memcpy(&v, z, sizeof(v));
        else
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < have) v[i] = z[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = fmaf(w, static_cast<float>(v[i]), acc[i]);
    }
    TY* y = Y + t * ldy + c;
    typename Pack<TY, 8>::vec o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = static_cast<TY>(acc[i]);
    if (have == 8) __builtin_memcpy(y, &o, sizeof(o));
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) y[i] = o[i];
}

}  // namespace

int launch_expert_route(adadim_ctx* ctx, const void* logits, int type, int64_t tokens, int64_t ldl, int experts, int k, int renormalize,
                        int32_t* chosen, float* weights, int32_t* offsets, int32_t* rows, int32_t* slots) {
    if (tokens == 0) {
        hipLaunchKernelGGL(route_none, dim3(1), dim3(256), 0, ctx->stream, offsets, experts);
        ADADIM_LAUNCH_CHECK(ctx, "route_none");
        return ADADIM_OK;
    }
    const int64_t chunks = (tokens + RT_TOKENS - 1) / RT_TOKENS, pitch = (experts + 3) & ~3;
    Route a{logits, tokens, ldl, experts, k, renormalize, chosen, weights, offsets, rows, slots, nullptr, nullptr};
    if (chunks > 1) {
        char* ws = static_cast<char*>(adadim_workspace(ctx, WS_ROUTE, size_t(chunks) * size_t(experts * 8 + pitch)));
        if (!ws) return ADADIM_EHIP;
        a.masks = reinterpret_cast<uint64_t*>(ws);
        a.counts = reinterpret_cast<uint8_t*>(ws + chunks * experts * 8);
    }
    {
        ProfScope prof(ctx, "route_choose");
        const dim3 grid(static_cast<unsigned>(chunks)), block(RT_THREADS);
        const size_t lds = size_t(experts) * 12;
#define RT_GO(T, W, V) hipLaunchKernelGGL((route_choose<T, W, V>), grid, block, lds, ctx->stream, a)
#define RT_V(T)                                    \
    do {                                           \
        if (experts <= 8) RT_GO(T, 8, 1);          \
        else if (experts <= 16) RT_GO(T, 16, 1);   \
        else if (experts <= 32) RT_GO(T, 16, 2);   \
        else if (experts <= 64) RT_GO(T, 16, 4);   \
        else if (experts <= 128) RT_GO(T, 16, 8);  \
        else if (experts <= 256) RT_GO(T, 16, 16); \
        else if (experts <= 512) RT_GO(T, 16, 32); \
        else RT_GO(T, 16, 64);                     \
    } while (0)
        if (type == ADADIM_TYPE_F16) RT_V(_Float16);
        else if (type == ADADIM_TYPE_BF16) RT_V(__bf16);
        else RT_V(float);
#undef RT_V
#undef RT_GO
    }
    ADADIM_LAUNCH_CHECK(ctx, "route_choose");
    if (chunks > 1) {
        const int64_t per = (chunks + RT_GROUPS - 1) / RT_GROUPS;
        ProfScope prof(ctx, "route_place");
        hipLaunchKernelGGL(route_place, dim3(static_cast<unsigned>((chunks + per - 1) / per)), dim3(RT_THREADS), size_t(pitch) * 8, ctx->stream, a, chunks, per);
        ADADIM_LAUNCH_CHECK(ctx, "route_place");
    }
    return ADADIM_OK;
}

int launch_expert_combine(adadim_ctx* ctx, const void* Z, int z_type, int64_t n_rows, int64_t cols, int64_t ldz, const int32_t* slots,
                          const float* weights, int64_t tokens, int k, void* Y, int y_type, int64_t ldy) {
    const int64_t ct = (cols + 2047) / 2048;
    const dim3 grid(static_cast<unsigned>(tokens * ct)), block(256);
    ProfScope prof(ctx, "combine_rows");
#define CB_GO(TZ, TY) \
    hipLaunchKernelGGL((combine_rows<TZ, TY>), grid, block, 0, ctx->stream, static_cast<const TZ*>(Z), n_rows, cols, ldz, slots, weights, tokens, k, static_cast<uint32_t>(ct), static_cast<TY*>(Y), ldy)
#define CB_Y(TZ)                                              \
    do {                                                      \
        if (y_type == ADADIM_TYPE_F16) CB_GO(TZ, _Float16);   \
        else if (y_type == ADADIM_TYPE_BF16) CB_GO(TZ, __bf16); \
        else CB_GO(TZ, float);                                \
    } while (0)
    if (z_type == ADADIM_TYPE_F16) CB_Y(_Float16);
    else if (z_type == ADADIM_TYPE_BF16) CB_Y(__bf16);
    else CB_Y(float);
#undef CB_Y
#undef CB_GO
    ADADIM_LAUNCH_CHECK(ctx, "combine_rows");
    return ADADIM_OK;
}
