// Rows of keys and values to their slots in a paged cache in mx4, and back.
//
// The scale of a block is the power of two that brings its largest magnitude into [4, 8), held to 2^-23 .. 2^13 (at most 6 x 2^13 = 49152 is
// kept of a value: no less than fp16's largest leaves; blocks below 2^-21 lose digits: fp16's subnormals lose none); codes as in mx4_quantize.hip.
//
// Bound by HBM: 2 (4) bytes read and 17/32 written a value.  A lane takes 8 elements of a position's key and the same of its value, D / 8
// lanes a position: a block is a quad of lanes, whether all is finite is a ballot.  A workgroup takes 32 rows of one head, a wave those
// that stand 4 and 4 in the order of the values' codes when the rows begin with a record: what it writes of them joins to whole runs.  Heads come first
// in the order of workgroups, so that (of a multiple of 8 heads) a record that two of them write stays in one XCD's L2: 8192 x 32 x 128
// fp16, keys and values, 45 us there (3.8 TB/s; rows first 58, 64 or 128 rows a workgroup 53 to 55, 8 rows the same, for few tokens too) and 30 us back (5.7 TB/s).
#include "mx4_cache.h"

namespace {

using namespace mx4;

constexpr int ST_THREADS = 256, ROWS = 32;
constexpr int QUAD_XOR1 = 0xB1, QUAD_XOR2 = 0x4E;

__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), QUAD_XOR1, 0xF, 0xF, false)));
    return max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), QUAD_XOR2, 0xF, 0xF, false)));
}

struct StoreArgs {
    const void* K;
    const void* V;
    int64_t tokens, ldk, ldv;
    const int32_t* slots;
    uint8_t* cache;
    int64_t slots_all;                            // pages * page
    int log_page, heads, dim;
};

// The row that group `at` of a workgroup takes: in runs of 4, those 16 apart next to each other.
__device__ __forceinline__ int row_in_turn(int at) { return 16 * ((at >> 2) & 1) + 4 * (at >> 3) + (at & 3); }

template <class T, int D>
__global__ __launch_bounds__(ST_THREADS) void mx4_cache_store_rows(StoreArgs a) {
    constexpr int LANES = D / 8, AT_ONCE = ST_THREADS / LANES, ITER = ROWS / AT_ONCE;
    typedef Record<D> R;
    const int x = threadIdx.x % LANES, d = 8 * x, have = min(8, a.dim - d), head = blockIdx.x % a.heads;
    const int64_t row0 = int64_t(blockIdx.x / a.heads) * ROWS;
    int64_t row[ITER];
    int32_t slot[ITER];
    typename Chunk<T, 8>::vec k[ITER], v[ITER];
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int at = threadIdx.x / LANES + AT_ONCE * i;
        row[i] = row0 + row_in_turn(at);
        slot[i] = row[i] < a.tokens ? a.slots[row[i]] : -1;
        if (slot[i] >= a.slots_all) slot[i] = -1;
        k[i] = typename Chunk<T, 8>::vec{};
        v[i] = typename Chunk<T, 8>::vec{};
        if (slot[i] >= 0 && have > 0) {
            k[i] = Chunk<T, 8>::load(static_cast<const T*>(a.K) + row[i] * a.ldk + int64_t(head) * a.dim + d, have);
            v[i] = Chunk<T, 8>::load(static_cast<const T*>(a.V) + row[i] * a.ldv + int64_t(head) * a.dim + d, have);
        }
    }
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        uint32_t word[2], byte[2];
        bool bad = false;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            float f[8];
            uint32_t big = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                f[j] = static_cast<float>(kv ? v[i][j] : k[i][j]);
                big = max(big, __float_as_uint(f[j]) & 0x7fffffffu);
            }
            big = quad_max(big);
            bad = bad || (big >> 23) == 255u;
            byte[kv] = big == 0 ? 127u : min(max(big >> 23, CACHE_LEAST + 2) - 2, CACHE_MOST);
            const float s = scale_operand(byte[kv]);
            uint32_t w = 0;
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], s, 0);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], s, 1);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], s, 2);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], s, 3);
            word[kv] = w;
        }
        const int lane = threadIdx.x & 63;
        const uint64_t mine = (LANES == 64 ? ~uint64_t(0) : ((uint64_t(1) << LANES) - 1)) << (lane / LANES * LANES);
        if (__ballot(bad) & mine) {
            word[0] = word[1] = 0;
            byte[0] = 255u;
            byte[1] = 127u;
        }
        if (slot[i] < 0) continue;
        const int at = slot[i] & ((1 << a.log_page) - 1), t = at & 31, g = R::quarter(t), place = R::place(t);
        uint8_t* const r = a.cache + record_of(slot[i] >> a.log_page, a.heads, head, a.log_page, at, R::BYTES);
        *reinterpret_cast<uint32_t*>(r + t * (D / 2) + 4 * x) = word[0];
        if constexpr (D == 64) {                                              // 4 elements a unit
            uint8_t* const p = r + R::VALUES + ((g * 16 + 2 * x) * 8 + place) * 2;
            *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(word[1]);
            *reinterpret_cast<uint16_t*>(p + 16) = static_cast<uint16_t>(word[1] >> 16);
        } else                                                                // 8, or half of 16
            *reinterpret_cast<uint32_t*>(r + R::VALUES + ((g * 16 + d / (D / 16)) * 8 + place) * R::UNIT + (D == 256 ? 4 * (x & 1) : 0)) = word[1];
        if ((x & 3) == 0) {
            r[R::KEY_SCALES + t * (D / 32) + x / 4] = static_cast<uint8_t>(byte[0]);
            r[R::VALUE_SCALES + (g * (D / 32) + x / 4) * 8 + place] = static_cast<uint8_t>(byte[1]);
        }
    }
}

struct LoadArgs {
    const int32_t* slots;
    int64_t tokens;
    const uint8_t* cache;
    int64_t slots_all;
    int log_page, heads, dim;
    void* K;
    void* V;
    int64_t ldk, ldv;
};

template <class T, int D>
__global__ __launch_bounds__(ST_THREADS) void mx4_cache_load_rows(LoadArgs a) {
    constexpr int LANES = D / 8, AT_ONCE = ST_THREADS / LANES, ITER = ROWS / AT_ONCE;
    typedef Record<D> R;
    const int x = threadIdx.x % LANES, d = 8 * x, have = min(8, a.dim - d), head = blockIdx.x % a.heads;
    const int64_t row0 = int64_t(blockIdx.x / a.heads) * ROWS;
    if (have <= 0) return;
    int64_t row[ITER];
    uint32_t word[ITER][2], byte[ITER][2];
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int n = threadIdx.x / LANES + AT_ONCE * i;
        row[i] = row0 + row_in_turn(n);
        if (row[i] >= a.tokens) row[i] = -1;
        const int32_t slot = row[i] >= 0 ? a.slots[row[i]] : -1;
        word[i][0] = word[i][1] = 0;
        byte[i][0] = byte[i][1] = 127u;
        if (slot < 0 || slot >= a.slots_all) continue;
        const int at = slot & ((1 << a.log_page) - 1), t = at & 31, g = R::quarter(t), place = R::place(t);
        const uint8_t* const r = a.cache + record_of(slot >> a.log_page, a.heads, head, a.log_page, at, R::BYTES);
        word[i][0] = *reinterpret_cast<const uint32_t*>(r + t * (D / 2) + 4 * x);
        if constexpr (D == 64) {
            const uint8_t* const p = r + R::VALUES + ((g * 16 + 2 * x) * 8 + place) * 2;
            word[i][1] = *reinterpret_cast<const uint16_t*>(p) | uint32_t(*reinterpret_cast<const uint16_t*>(p + 16)) << 16;
        } else
            word[i][1] = *reinterpret_cast<const uint32_t*>(r + R::VALUES + ((g * 16 + d / (D / 16)) * 8 + place) * R::UNIT + (D == 256 ? 4 * (x & 1) : 0));
        byte[i][0] = r[R::KEY_SCALES + t * (D / 32) + x / 4];
        byte[i][1] = r[R::VALUE_SCALES + (g * (D / 32) + x / 4) * 8 + place];
    }
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        if (row[i] < 0) continue;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            float f[8];
            values8(word[i][kv], scale_operand(byte[i][kv]), f);
            typename Chunk<T, 8>::vec o;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = static_cast<T>(f[j]);
            T* const y = static_cast<T*>(kv ? a.V : a.K) + row[i] * (kv ? a.ldv : a.ldk) + int64_t(head) * a.dim + d;
            Chunk<T, 8>::store(y, have, o);
        }
    }
}

}  // namespace

int launch_mx4_cache_store(adadim_ctx* ctx, const void* K, const void* V, int type, int64_t tokens, int64_t ldk, int64_t ldv,
                           const int32_t* slots, uint8_t* cache, int64_t pages, int log_page, int heads, int dim) {
    const StoreArgs a{K, V, tokens, ldk, ldv, slots, cache, pages << log_page, log_page, heads, dim};
    const dim3 grid(static_cast<unsigned>((tokens + ROWS - 1) / ROWS * heads)), block(ST_THREADS);
    ProfScope prof(ctx, "mx4_cache_store_rows");
#define CACHE_S(T, D) hipLaunchKernelGGL((mx4_cache_store_rows<T, D>), grid, block, 0, ctx->stream, a)
#define CACHE_ST(T)                                                                                          \
    do {                                                                                                     \
        switch (filled_head(dim)) {                                                                          \
            case 64: CACHE_S(T, 64); break;                                                                  \
            case 128: CACHE_S(T, 128); break;                                                                \
            default: CACHE_S(T, 256);                                                                        \
        }                                                                                                    \
    } while (0)
    if (type == ADADIM_TYPE_F16) CACHE_ST(_Float16);
    else if (type == ADADIM_TYPE_BF16) CACHE_ST(__bf16);
    else CACHE_ST(float);
#undef CACHE_ST
#undef CACHE_S
    ADADIM_LAUNCH_CHECK(ctx, "mx4_cache_store_rows");
    return ADADIM_OK;
}

int launch_mx4_cache_load(adadim_ctx* ctx, const int32_t* slots, int64_t tokens, const uint8_t* cache, int64_t pages, int log_page,
                          int heads, int dim, void* K, void* V, int type, int64_t ldk, int64_t ldv) {
    const LoadArgs a{slots, tokens, cache, pages << log_page, log_page, heads, dim, K, V, ldk, ldv};
    const dim3 grid(static_cast<unsigned>((tokens + ROWS - 1) / ROWS * heads)), block(ST_THREADS);
    ProfScope prof(ctx, "mx4_cache_load_rows");
#define CACHE_L(T, D) hipLaunchKernelGGL((mx4_cache_load_rows<T, D>), grid, block, 0, ctx->stream, a)
#define CACHE_LT(T)                                                                                          \
    do {                                                                                                     \
        switch (filled_head(dim)) {                                                                          \
            case 64: CACHE_L(T, 64); break;                                                                  \
            case 128: CACHE_L(T, 128); break;                                                                \
            default: CACHE_L(T, 256);                                                                        \
        }                                                                                                    \
    } while (0)
    if (type == ADADIM_TYPE_F16) CACHE_LT(_Float16);
    else if (type == ADADIM_TYPE_BF16) CACHE_LT(__bf16);
    else CACHE_LT(float);
#undef CACHE_LT
#undef CACHE_L
    ADADIM_LAUNCH_CHECK(ctx, "mx4_cache_load_rows");
    return ADADIM_OK;
}
