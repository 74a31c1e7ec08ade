// C-ABI entry points of the paged cache in mx4 and of the attention over it: argument validation, before the first HIP call.
#include "mx4_cache.h"

int launch_cache_reserve(adadim_ctx* ctx, const int32_t* held, const int32_t* added, int n, int log_page, int32_t* table, int64_t width,
                         const int32_t* free, int64_t pool, const int32_t* count, int32_t* lengths, int32_t* offsets, int32_t* slots,
                         int32_t* positions, int64_t tokens, int32_t* left, int32_t* lacking);
int launch_cache_trim(adadim_ctx* ctx, const int32_t* held, const int32_t* kept, int n, int log_page, const int32_t* table, int64_t width,
                      int32_t* free, int64_t pool, const int32_t* count, int32_t* lengths, int32_t* left);
int launch_mx4_cache_store(adadim_ctx* ctx, const void* K, const void* V, int type, int64_t tokens, int64_t ldk, int64_t ldv,
                           const int32_t* slots, uint8_t* cache, int64_t pages, int log_page, int heads, int dim);
int launch_mx4_cache_load(adadim_ctx* ctx, const int32_t* slots, int64_t tokens, const uint8_t* cache, int64_t pages, int log_page,
                          int heads, int dim, void* K, void* V, int type, int64_t ldk, int64_t ldv);
int launch_mx4_attention(adadim_ctx* ctx, const mx4::Attention& a, int q_type);

static bool is_float_type(int t) { return t == ADADIM_TYPE_F16 || t == ADADIM_TYPE_BF16 || t == ADADIM_TYPE_F32; }
static int type_size(int t) { return t == ADADIM_TYPE_F32 ? 4 : 2; }
static bool aligned_to(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// log2 of a page's positions; 0: not a page
static int log_of_page(int page) {
    for (int l = 5; l <= 16; ++l)
        if (page == 1 << l) return l;
    return 0;
}

constexpr int64_t MOST_TOKENS = int64_t(1) << 20;
constexpr int MOST_SEQUENCES = 4096, MOST_HEADS = 1024, MOST_GROUP = 1024;

// Positions are numbered in 32 bits, over a sequence's pages and over the pool's.
static bool pages_ok(int64_t pages, int page) { return pages >= 1 && pages <= INT32_MAX / page; }

extern "C" {

int64_t adadim_mx4_cache_bytes(int64_t pages, int page, int heads, int dim) {
    if (log_of_page(page) == 0 || !pages_ok(pages, page) || heads <= 0 || heads > MOST_HEADS || dim <= 0 || dim > 256) return 0;
    return pages * heads * (page / mx4::RECORD) * (34 * mx4::filled_head(dim));
}

static int pages_checked(adadim_ctx* ctx, const char* me, const void* held, const void* change, int sequences, int page, const void* table,
                         int64_t width, const void* free, int64_t pool, const void* count, const void* lengths, const void* left) {
    if (sequences <= 0 || sequences > MOST_SEQUENCES)
        return adadim_fail(ctx, ADADIM_EINVAL, "%s: sequences must be in [1,%d], got %d", me, MOST_SEQUENCES, sequences);
    if (log_of_page(page) == 0) return adadim_fail(ctx, ADADIM_EINVAL, "%s: page must be a power of two in [32,65536], got %d", me, page);
    // (sums of pages over the sequences are 32-bit numbers)
    if (!pages_ok(width, page) || !pages_ok(pool, page) || sequences * width > INT32_MAX)
        return adadim_fail(ctx, ADADIM_EINVAL,
                           "%s: need 1 <= width, pool, less than 2^31 positions in them and entries in the table (sequences=%d width=%lld pool=%lld page=%d)", me,
                           sequences, (long long)width, (long long)pool, page);
    if (!held || !change || !table || !free || !count || !lengths || !left)
        return adadim_fail(ctx, ADADIM_ENULL, "%s: a required pointer is NULL", me);
    if (!aligned_to(held, 4) || !aligned_to(change, 4) || !aligned_to(table, 4) || !aligned_to(free, 4) || !aligned_to(count, 4) ||
        !aligned_to(lengths, 4) || !aligned_to(left, 4))
        return adadim_fail(ctx, ADADIM_EALIGN, "%s: arrays must be 4-byte aligned", me);
    return ADADIM_OK;
}

int adadim_cache_reserve(adadim_ctx* ctx, const int32_t* held, const int32_t* added, int sequences, int page, int32_t* table, int64_t width,
                         const int32_t* free, int64_t pool, const int32_t* count, int32_t* lengths, int32_t* offsets, int32_t* slots,
                         int32_t* positions, int64_t tokens, int32_t* left, int32_t* lacking) {
    if (!ctx) return ADADIM_ENULL;
    const char* me = "adadim_cache_reserve";
    if (tokens < 0 || tokens > MOST_TOKENS) return adadim_fail(ctx, ADADIM_EINVAL, "%s: tokens must be in [0,2^20], got %lld", me, (long long)tokens);
    const int rc = pages_checked(ctx, me, held, added, sequences, page, table, width, free, pool, count, lengths, left);
    if (rc != ADADIM_OK) return rc;
    if (!offsets || !lacking || (tokens > 0 && (!slots || !positions))) return adadim_fail(ctx, ADADIM_ENULL, "%s: a required pointer is NULL", me);
    if (!aligned_to(offsets, 4) || !aligned_to(slots, 4) || !aligned_to(positions, 4) || !aligned_to(lacking, 4))
        return adadim_fail(ctx, ADADIM_EALIGN, "%s: arrays must be 4-byte aligned", me);
    return launch_cache_reserve(ctx, held, added, sequences, log_of_page(page), table, width, free, pool, count, lengths, offsets, slots,
                                positions, tokens, left, lacking);
}

int adadim_cache_trim(adadim_ctx* ctx, const int32_t* held, const int32_t* kept, int sequences, int page, const int32_t* table, int64_t width,
                      int32_t* free, int64_t pool, const int32_t* count, int32_t* lengths, int32_t* left) {
    if (!ctx) return ADADIM_ENULL;
    const int rc = pages_checked(ctx, "adadim_cache_trim", held, kept, sequences, page, table, width, free, pool, count, lengths, left);
    if (rc != ADADIM_OK) return rc;
    return launch_cache_trim(ctx, held, kept, sequences, log_of_page(page), table, width, free, pool, count, lengths, left);
}

static int cache_checked(adadim_ctx* ctx, const char* me, int64_t pages, int page, int heads, int dim) {
    if (log_of_page(page) == 0) return adadim_fail(ctx, ADADIM_EINVAL, "%s: page must be a power of two in [32,65536], got %d", me, page);
    if (!pages_ok(pages, page) || heads <= 0 || heads > MOST_HEADS || dim <= 0 || dim > 256)
        return adadim_fail(ctx, ADADIM_EINVAL, "%s: need 1 <= pages and less than 2^31 positions, 1..%d heads, dim 1..256 (pages=%lld page=%d heads=%d dim=%d)",
                           me, MOST_HEADS, (long long)pages, page, heads, dim);
    return ADADIM_OK;
}

int adadim_mx4_cache_store(adadim_ctx* ctx, const void* K, const void* V, int type, int64_t tokens, int64_t ldk, int64_t ldv,
                           const int32_t* slots, uint8_t* cache, int64_t pages, int page, int heads, int dim) {
    if (!ctx) return ADADIM_ENULL;
    const char* me = "adadim_mx4_cache_store";
    if (!is_float_type(type)) return adadim_fail(ctx, ADADIM_EINVAL, "%s: type must be F16, BF16 or F32, got %d", me, type);
    const int rc = cache_checked(ctx, me, pages, page, heads, dim);
    if (rc != ADADIM_OK) return rc;
    if (tokens < 0 || tokens > MOST_TOKENS || ldk < int64_t(heads) * dim || ldv < int64_t(heads) * dim || !launchable((tokens + 31) / 32 * heads, 256))
        return adadim_fail(ctx, ADADIM_EINVAL,
                           "%s: need tokens in [0,2^20], ldk, ldv >= heads * dim, fewer than 2^24 runs of 32 rows of a head (tokens=%lld heads=%d ldk=%lld ldv=%lld)",
                           me, (long long)tokens, heads, (long long)ldk, (long long)ldv);
    if (tokens == 0) return ADADIM_OK;
    if (!K || !V || !slots || !cache) return adadim_fail(ctx, ADADIM_ENULL, "%s: K, V, slots or cache is NULL", me);
    if (!aligned16(cache) || !aligned_to(slots, 4) || !aligned_to(K, type_size(type)) || !aligned_to(V, type_size(type)))
        return adadim_fail(ctx, ADADIM_EALIGN, "%s: cache must be 16-byte, slots 4-byte, K and V element aligned", me);
    return launch_mx4_cache_store(ctx, K, V, type, tokens, ldk, ldv, slots, cache, pages, log_of_page(page), heads, dim);
}

int adadim_mx4_cache_load(adadim_ctx* ctx, const int32_t* slots, int64_t tokens, const uint8_t* cache, int64_t pages, int page, int heads,
                          int dim, void* K, void* V, int type, int64_t ldk, int64_t ldv) {
    if (!ctx) return ADADIM_ENULL;
    const char* me = "adadim_mx4_cache_load";
    if (!is_float_type(type)) return adadim_fail(ctx, ADADIM_EINVAL, "%s: type must be F16, BF16 or F32, got %d", me, type);
    const int rc = cache_checked(ctx, me, pages, page, heads, dim);
    if (rc != ADADIM_OK) return rc;
    if (tokens < 0 || tokens > MOST_TOKENS || ldk < int64_t(heads) * dim || ldv < int64_t(heads) * dim || !launchable((tokens + 31) / 32 * heads, 256))
        return adadim_fail(ctx, ADADIM_EINVAL,
                           "%s: need tokens in [0,2^20], ldk, ldv >= heads * dim, fewer than 2^24 runs of 32 rows of a head (tokens=%lld heads=%d ldk=%lld ldv=%lld)",
                           me, (long long)tokens, heads, (long long)ldk, (long long)ldv);
    if (tokens == 0) return ADADIM_OK;
    if (!K || !V || !slots || !cache) return adadim_fail(ctx, ADADIM_ENULL, "%s: K, V, slots or cache is NULL", me);
    if (!aligned16(cache) || !aligned_to(slots, 4) || !aligned_to(K, type_size(type)) || !aligned_to(V, type_size(type)))
        return adadim_fail(ctx, ADADIM_EALIGN, "%s: cache must be 16-byte, slots 4-byte, K and V element aligned", me);
    return launch_mx4_cache_load(ctx, slots, tokens, cache, pages, log_of_page(page), heads, dim, K, V, type, ldk, ldv);
}

int adadim_mx4_attention(adadim_ctx* ctx, const void* Q, int q_type, int64_t tokens, int64_t ldq, int q_heads, const uint8_t* cache,
                         int64_t pages, int page, int heads, int dim, const int32_t* table, int64_t width, int sequences,
                         const int32_t* offsets, const int32_t* lengths, void* Y, int y_type, int64_t ldy, float scale, int causal,
                         int64_t window, int64_t max_new, int64_t max_length) {
    if (!ctx) return ADADIM_ENULL;
    const char* me = "adadim_mx4_attention";
    if (q_type != ADADIM_TYPE_F16 && q_type != ADADIM_TYPE_BF16)
        return adadim_fail(ctx, ADADIM_EINVAL, "%s: q_type must be F16 or BF16, got %d", me, q_type);
    if (!is_float_type(y_type)) return adadim_fail(ctx, ADADIM_EINVAL, "%s: y_type must be F16, BF16 or F32, got %d", me, y_type);
    const int rc = cache_checked(ctx, me, pages, page, heads, dim);
    if (rc != ADADIM_OK) return rc;
    if (q_heads <= 0 || q_heads % heads != 0 || q_heads / heads > MOST_GROUP)
        return adadim_fail(ctx, ADADIM_EINVAL, "%s: q_heads must be 1 to %d times heads (q_heads=%d heads=%d)", me, MOST_GROUP, q_heads, heads);
    if (sequences <= 0 || sequences > MOST_SEQUENCES || !pages_ok(width, page))
        return adadim_fail(ctx, ADADIM_EINVAL, "%s: need 1..%d sequences, 1 <= width and less than 2^31 positions (sequences=%d width=%lld page=%d)", me,
                           MOST_SEQUENCES, sequences, (long long)width, page);
    const int group = q_heads / heads;
    if (tokens < 0 || tokens > MOST_TOKENS || ldq < int64_t(q_heads) * dim || ldy < int64_t(q_heads) * dim ||
        !launchable((tokens * group / 16 + sequences) * heads, 512))
        return adadim_fail(ctx, ADADIM_EINVAL,
                           "%s: need tokens in [0,2^20], ldq, ldy >= q_heads * dim, fewer than 2^23 tiles of 16 rows (tokens=%lld ldq=%lld ldy=%lld)", me,
                           (long long)tokens, (long long)ldq, (long long)ldy);
    if (!(scale > 0.0f && scale <= 2e38f) || (causal != 0 && causal != 1) || window < 0)
        return adadim_fail(ctx, ADADIM_EINVAL, "%s: need a scale in (0, 2e38], causal 0 or 1, window >= 0 (scale=%g causal=%d window=%lld)", me, scale,
                           causal, (long long)window);
    if (tokens == 0) return ADADIM_OK;
    if (!Q || !cache || !table || !offsets || !lengths || !Y) return adadim_fail(ctx, ADADIM_ENULL, "%s: a required pointer is NULL", me);
    if (!aligned16(cache) || !aligned_to(Q, 2) || !aligned_to(Y, type_size(y_type)) || !aligned_to(table, 4) || !aligned_to(offsets, 4) ||
        !aligned_to(lengths, 4))
        return adadim_fail(ctx, ADADIM_EALIGN, "%s: cache must be 16-byte, the others element aligned", me);
    const int64_t most = width * page;
    const mx4::Attention a{Q, tokens, ldq, cache, pages, log_of_page(page), heads, group, dim, table, width, sequences, offsets, lengths, Y, y_type, ldy,
                           scale, causal, window < most ? window : 0, max_new < 1 ? (tokens + sequences - 1) / sequences : max_new > tokens ? tokens : max_new,
                           max_length < 1 || max_length > most ? most : max_length};
    return launch_mx4_attention(ctx, a, q_type);
}

}  // extern "C"
