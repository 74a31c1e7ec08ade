// A router's scores to its choice of experts and the rows sorted by expert, and the experts' outputs back to the tokens.
//
// Choice: the k largest scores of a token, the lowest index first among equal ones; a score of -infinity or NaN is never
// chosen (a token may have fewer than k experts, or none: -1 in the free places, their weight 0).  Weights in fp32:
//     exp(l_j - max) / sum   over the chosen (renormalize) or over all scores;  +infinite scores share among themselves.
// Order: the rows of expert e are those tokens that chose it, in the order of the tokens: a counting sort whose ranks come
// from one bit per (token, expert), so that no order of arrival is visible in the result.
#include "common.h"

namespace {

// Larger number, larger key; -infinity and NaN have key 0 and never win.  (-0 and +0 are equal scores.)
__device__ __forceinline__ uint32_t score_key(float f) {
    if (!(f > -INFINITY)) return 0u;
    const uint32_t u = __float_as_uint(f + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <class T>
__device__ __forceinline__ float score(const T* p) { return static_cast<float>(*p); }

constexpr int RT_TOKENS = 64;                     // tokens of a chunk: one bit each of an expert's mask
constexpr int RT_WAVES = 8;

struct Route {
    const void* logits;
    int64_t tokens, ldl;
    int experts, k, renormalize;
    int32_t* chosen;
    float* weights;
    int32_t *offsets, *rows, *slots;
    uint64_t* masks;                              // [chunks][experts]
    int32_t* bases;                               // [chunks][experts]
};

// A wave per token: every lane holds the scores lane, lane + 64, ..; k times the largest one left.
template <class T, int V>
__global__ __launch_bounds__(64 * RT_WAVES) void route_choose(Route a) {
    extern __shared__ uint32_t s_mask[];          // [experts][2]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < 2 * a.experts; i += 64 * RT_WAVES) s_mask[i] = 0u;
    __syncthreads();
    for (int tt = wave; tt < RT_TOKENS; tt += RT_WAVES) {
        const int64_t t = int64_t(blockIdx.x) * RT_TOKENS + tt;
        if (t >= a.tokens) break;
        const T* l = static_cast<const T*>(a.logits) + t * a.ldl;
        float f[V];
        uint32_t key[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = lane + 64 * v;
            f[v] = e < a.experts ? score(l + e) : -INFINITY;
            key[v] = score_key(f[v]);
        }
        float top = 0.0f, sum = 0.0f;
        float mine = 0.0f;                        // lane j: exp(l - max) of the j-th chosen
        int32_t index = -1;
        for (int j = 0; j < a.k; ++j) {
            uint32_t best = 0u;
            int at = 0x7fffffff;
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (key[v] > best) {
                    best = key[v];
                    at = lane + 64 * v;
                }
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const uint32_t ob = __shfl_xor(best, d);
                const int oa = __shfl_xor(at, d);
                if (ob > best || (ob == best && oa < at)) {
                    best = ob;
                    at = oa;
                }
            }
            if (best == 0u) break;                // nothing left (the same in every lane)
            float val = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (at == lane + 64 * v) {
                    key[v] = 0u;
                    val = f[v];
                }
            val = __shfl(val, at & 63);
            if (j == 0) top = val;
            const float p = val == top ? 1.0f : expf(val - top);
            sum += p;
            if (lane == j) {
                mine = p;
                index = at;
            }
            if (lane == 0) atomicOr(&s_mask[2 * at + (tt >> 5)], 1u << (tt & 31));
        }
        if (!a.renormalize) {
            sum = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (f[v] > -INFINITY) sum += f[v] == top ? 1.0f : expf(f[v] - top);
#pragma unroll
            for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        }
        if (lane < a.k) {
            a.chosen[t * a.k + lane] = index;
            a.weights[t * a.k + lane] = index >= 0 ? mine / sum : 0.0f;
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += 64 * RT_WAVES)
        a.masks[int64_t(blockIdx.x) * a.experts + e] = uint64_t(s_mask[2 * e]) | uint64_t(s_mask[2 * e + 1]) << 32;
}

// One workgroup: the experts' totals and their sums, then where each chunk's rows of each expert begin.
__global__ __launch_bounds__(1024) void route_bases(Route a, int64_t chunks) {
    __shared__ int32_t s_sum[1024];
    const int e = threadIdx.x;
    int32_t n = 0;
    if (e < a.experts)
        for (int64_t c = 0; c < chunks; ++c) n += __popcll(a.masks[c * a.experts + e]);
    s_sum[e] = n;
    __syncthreads();
    for (int d = 1; d < 1024; d *= 2) {
        const int32_t before = e >= d ? s_sum[e - d] : 0;
        __syncthreads();
        s_sum[e] += before;
        __syncthreads();
    }
    if (e < a.experts) {
        int32_t at = s_sum[e] - n;
        if (e == 0) a.offsets[0] = 0;
        a.offsets[e + 1] = s_sum[e];
        for (int64_t c = 0; c < chunks; ++c) {
            a.bases[c * a.experts + e] = at;
            at += __popcll(a.masks[c * a.experts + e]);
        }
    }
    // the places that no row takes
    const int64_t all = a.tokens * a.k;
    for (int64_t i = s_sum[1023] + int64_t(e); i < all; i += 1024) a.rows[i] = -1;
}

__global__ __launch_bounds__(256) void route_place(Route a) {
    const int64_t t0 = int64_t(blockIdx.x) * RT_TOKENS;
    const int n = static_cast<int>(min(int64_t(RT_TOKENS), a.tokens - t0)) * a.k;
    for (int i = threadIdx.x; i < n; i += 256) {
        const int tt = i / a.k;
        const int32_t e = a.chosen[t0 * a.k + i];
        int32_t slot = -1;
        if (e >= 0) {
            const int64_t at = int64_t(blockIdx.x) * a.experts + e;
            slot = a.bases[at] + __popcll(a.masks[at] & ((uint64_t(1) << tt) - 1));
            a.rows[slot] = static_cast<int32_t>(t0 + tt);
        }
        a.slots[t0 * a.k + i] = slot;
    }
}

__global__ void route_none(int32_t* offsets, int experts) {
    for (int e = threadIdx.x; e <= experts; e += blockDim.x) offsets[e] = 0;
}

// Y[t] = sum_j weights[t, j] Z[slots[t, j]]: fp32, in the order of j, rounded once.  Bound by HBM: every row of Z is
// read once.  A lane takes eight columns of a token.
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
    const int64_t chunks = (tokens + RT_TOKENS - 1) / RT_TOKENS;
    char* ws = static_cast<char*>(adadim_workspace(ctx, WS_ROUTE, size_t(chunks) * size_t(experts) * 12));
    if (!ws) return ADADIM_EHIP;
    uint64_t* masks = reinterpret_cast<uint64_t*>(ws);
    const Route a{logits, tokens, ldl, experts, k, renormalize, chosen, weights, offsets, rows, slots, masks,
                  reinterpret_cast<int32_t*>(masks + chunks * experts)};
    const dim3 grid(static_cast<unsigned>(chunks));
    {
        ProfScope prof(ctx, "route_choose");
        const size_t lds = size_t(experts) * 8;
#define RT_GO(T, V) hipLaunchKernelGGL((route_choose<T, V>), grid, dim3(64 * RT_WAVES), lds, ctx->stream, a)
#define RT_V(T)                                    \
    do {                                           \
        if (experts <= 64) RT_GO(T, 1);            \
        else if (experts <= 128) RT_GO(T, 2);      \
        else if (experts <= 256) RT_GO(T, 4);      \
        else RT_GO(T, 16);                         \
    } while (0)
        if (type == ADADIM_TYPE_F16) RT_V(_Float16);
        else if (type == ADADIM_TYPE_BF16) RT_V(__bf16);
        else RT_V(float);
#undef RT_V
#undef RT_GO
    }
    ADADIM_LAUNCH_CHECK(ctx, "route_choose");
    {
        ProfScope prof(ctx, "route_bases");
        hipLaunchKernelGGL(route_bases, dim3(1), dim3(1024), 0, ctx->stream, a, chunks);
    }
    ADADIM_LAUNCH_CHECK(ctx, "route_bases");
    {
        ProfScope prof(ctx, "route_place");
        hipLaunchKernelGGL(route_place, grid, dim3(256), 0, ctx->stream, a);
    }
    ADADIM_LAUNCH_CHECK(ctx, "route_place");
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
