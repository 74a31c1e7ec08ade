// Pages of a cache, on the device: what a batch's new tokens take from the stack of free pages, and what goes back to it.
//
// A sequence of `held` tokens has ceil(held / page) pages.  reserve: the sum of the new pages of the sequences in front of it is where a
// sequence's own begin on the stack, the sum of their new tokens where its rows begin; a row's slot is its page times page plus its place in
// it.  The row that begins a page is the one that writes it into the table, so rows need no order among them.  trim: the pages
// behind the kept tokens go onto the stack, sequence by sequence.
//
// Bound by latency: 8 bytes a sequence and 8 a row.  Up to SMALL_ROWS rows (SMALL_ENTRIES entries of the table) one workgroup does all: sums by lanes,
// then each thread its rows, whose sequence it finds in LDS.  Beyond, a second launch over the rows, with what it needs left in scratch: lengths
// may be written over what was held, and the count over itself, because only the first launch reads them.  A call by one launch and by two, from
// Python: 4000 rows 7.7 and 10.7 us, 9000 9.4 and 10.6, 17000 16.2 and 10.8; 256 sequences of 512 pages of which 4 end 6.3 and 9.1, all 11.4 and 9.3.
#include "common.h"

#include <algorithm>

namespace {

constexpr int PG_THREADS = 1024, PG_WAVES = PG_THREADS / 64, PG_SEQUENCES = 4096;
constexpr int SMALL_ROWS = 8192, SMALL_ENTRIES = 65536;

struct ReserveArgs {
    const int32_t *held, *added;
    int n, log_page;
    int32_t* table;
    int64_t width;
    const int32_t* free;
    int64_t pool;
    const int32_t* count;
    int32_t *lengths, *offsets, *slots, *positions;
    int64_t tokens;
    int32_t *left, *lacking;
    int32_t* plan;                                // scratch: held [n], first new page [n], count; NULL: the same launch does the rows
};

__device__ __forceinline__ int32_t pages_of(int32_t tokens, int log_page) {
    return static_cast<int32_t>((int64_t(tokens) + (1 << log_page) - 1) >> log_page);
}

// The sums of a and b of the threads in front of each (32 bits hold a workgroup's), and of all; s_sum: 2 PG_WAVES words.
__device__ __forceinline__ void sums_before(int32_t& a, int32_t& b, int32_t& all_a, int32_t& all_b, int32_t* s_sum) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t x = a, y = b;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int32_t o = __shfl_up(x, d), p = __shfl_up(y, d);
        if (lane >= d) {
            x += o;
            y += p;
        }
    }
    __syncthreads();                              // (s_sum may still be read)
    if (lane == 63) {
        s_sum[wave] = x;
        s_sum[PG_WAVES + wave] = y;
    }
    __syncthreads();
    int32_t before_a = 0, before_b = 0;
    all_a = all_b = 0;
#pragma unroll
    for (int w = 0; w < PG_WAVES; ++w) {
        const int32_t o = s_sum[w], p = s_sum[PG_WAVES + w];
        if (w < wave) {
            before_a += o;
            before_b += p;
        }
        all_a += o;
        all_b += p;
    }
    a = before_a + x - a;
    b = before_b + y - b;
}

// The last of the n sequences that begins at or before row r (offsets do not decrease, offsets[0] = 0).
__device__ __forceinline__ int sequence_of(const int32_t* offsets, int n, int32_t r) {
    int lo = 0, hi = n;                           // offsets[lo] <= r < offsets[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (offsets[mid] <= r) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ void place_row(const ReserveArgs& a, int64_t r, int s, int32_t begin, int32_t held, int32_t first, int32_t count) {
    const int32_t pos = held + static_cast<int32_t>(r - begin), page = pos >> a.log_page, in_page = pos & ((1 << a.log_page) - 1);
    const int32_t had = pages_of(held, a.log_page);
    int32_t* const entry = a.table + s * a.width + page;
    const int32_t id = page < had ? *entry : a.free[count - 1 - (first + page - had)];
    if (in_page == 0) *entry = id;
    const int64_t slot = (int64_t(id) << a.log_page) + in_page;
    a.slots[r] = slot >= 0 && slot <= INT32_MAX ? static_cast<int32_t>(slot) : -1;
    a.positions[r] = pos;
}

__global__ __launch_bounds__(PG_THREADS) void cache_reserve_plan(ReserveArgs a) {
    __shared__ int32_t s_sum[2 * PG_WAVES], s_begin[PG_SEQUENCES + 1], s_first[PG_SEQUENCES], s_held[PG_SEQUENCES];
    __shared__ int32_t s_bad;
    const int32_t count = static_cast<int32_t>(min(max(int64_t(a.count[0]), int64_t(0)), a.pool));
    if (threadIdx.x == 0) s_bad = 0;
    int64_t rows = 0, pages = 0;
    for (int s0 = 0; s0 < a.n; s0 += PG_THREADS) {
        const int s = s0 + threadIdx.x;
        int32_t held = 0, added = 0;
        bool bad = false;
        if (s < a.n) {
            held = a.held[s];
            added = a.added[s];
            bad = held < 0 || added < 0 || added > a.tokens || int64_t(held) + added > a.width << a.log_page;
            s_held[s] = held;
        }
        int32_t x = bad ? 0 : added, y = bad ? 0 : pages_of(held + added, a.log_page) - pages_of(held, a.log_page), all_x, all_y;
        sums_before(x, y, all_x, all_y, s_sum);
        if (bad) s_bad = 1;
        if (s < a.n) {                            // (sums beyond 32 bits: refused below, and not read)
            s_begin[s] = static_cast<int32_t>(rows + x);
            s_first[s] = static_cast<int32_t>(pages + y);
        }
        rows += all_x;
        pages += all_y;
    }
    __syncthreads();
    const bool bad = s_bad != 0 || rows > a.tokens, ok = !bad && pages <= count;
    if (threadIdx.x == 0) {
        s_begin[a.n] = static_cast<int32_t>(rows);
        a.offsets[a.n] = ok ? static_cast<int32_t>(rows) : 0;
        a.left[0] = ok ? static_cast<int32_t>(count - pages) : count;
        a.lacking[0] = bad ? -1 : ok ? 0 : static_cast<int32_t>(pages - count);
        if (a.plan) a.plan[2 * a.n] = count;
    }
    __syncthreads();
    for (int s = threadIdx.x; s < a.n; s += PG_THREADS) {
        const int32_t added = ok ? s_begin[s + 1] - s_begin[s] : 0;
        a.offsets[s] = ok ? s_begin[s] : 0;
        a.lengths[s] = s_held[s] + added;
        if (a.plan) {
            a.plan[s] = s_held[s];
            a.plan[a.n + s] = s_first[s];
        }
    }
    if (a.plan) return;
    for (int64_t r = threadIdx.x; r < a.tokens; r += PG_THREADS) {
        if (!ok || r >= rows) {
            a.slots[r] = a.positions[r] = -1;
            continue;
        }
        const int s = sequence_of(s_begin, a.n, static_cast<int32_t>(r));
        place_row(a, r, s, s_begin[s], s_held[s], s_first[s], count);
    }
}

__global__ __launch_bounds__(256) void cache_reserve_rows(ReserveArgs a) {
    const int64_t r = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (r >= a.tokens) return;
    if (r >= a.offsets[a.n]) {
        a.slots[r] = a.positions[r] = -1;
        return;
    }
    const int s = sequence_of(a.offsets, a.n, static_cast<int32_t>(r));
    place_row(a, r, s, a.offsets[s], a.plan[s], a.plan[a.n + s], a.plan[2 * a.n]);
}

struct TrimArgs {
    const int32_t *held, *kept;
    int n, log_page;
    const int32_t* table;
    int64_t width;
    int32_t* free;
    int64_t pool;
    const int32_t* count;
    int32_t *lengths, *left;
    int32_t* plan;                                // scratch: first page that goes [n], place on the stack of the first [n + 1]; NULL: in the same launch
};

// The pages from..to of a sequence's row of the table to the stack, `threads` threads at it.
__device__ __forceinline__ void give_back(const TrimArgs& a, int s, int32_t from, int32_t n, int32_t at, int thread, int threads) {
    for (int32_t i = thread; i < n; i += threads)
        if (at + i < a.pool) a.free[at + i] = a.table[s * a.width + from + i];
}

__global__ __launch_bounds__(PG_THREADS) void cache_trim_plan(TrimArgs a) {
    __shared__ int32_t s_sum[2 * PG_WAVES], s_at[PG_SEQUENCES + 1], s_from[PG_SEQUENCES];
    const int32_t count = static_cast<int32_t>(min(max(int64_t(a.count[0]), int64_t(0)), a.pool));
    int64_t pages = count;
    for (int s0 = 0; s0 < a.n; s0 += PG_THREADS) {
        const int s = s0 + threadIdx.x;
        int32_t y = 0, from = 0, zero = 0, all, none;
        if (s < a.n) {
            const int32_t held = static_cast<int32_t>(min(max(int64_t(a.held[s]), int64_t(0)), a.width << a.log_page));
            const int32_t kept = min(max(a.kept[s], 0), held);
            from = pages_of(kept, a.log_page);
            y = pages_of(held, a.log_page) - from;
            a.lengths[s] = kept;
            s_from[s] = from;
        }
        sums_before(y, zero, all, none, s_sum);
        if (s < a.n) s_at[s] = static_cast<int32_t>(min(pages + y, a.pool));
        pages = min(pages + all, a.pool);
    }
    if (threadIdx.x == 0) {
        s_at[a.n] = static_cast<int32_t>(pages);
        a.left[0] = static_cast<int32_t>(pages);
    }
    __syncthreads();
    if (a.plan) {
        for (int s = threadIdx.x; s <= a.n; s += PG_THREADS) {
            if (s < a.n) a.plan[s] = s_from[s];
            a.plan[a.n + s] = s_at[s];
        }
        return;
    }
    for (int s = threadIdx.x >> 6; s < a.n; s += PG_WAVES) give_back(a, s, s_from[s], s_at[s + 1] - s_at[s], s_at[s], threadIdx.x & 63, 64);
}

__global__ __launch_bounds__(256) void cache_trim_pages(TrimArgs a) {
    const int s = blockIdx.x;
    const int32_t at = a.plan[a.n + s];
    give_back(a, s, a.plan[s], a.plan[a.n + s + 1] - at, at, threadIdx.x, 256);
}

}  // namespace

int launch_cache_reserve(adadim_ctx* ctx, const int32_t* held, const int32_t* added, int n, int log_page, int32_t* table, int64_t width,
                         const int32_t* free, int64_t pool, const int32_t* count, int32_t* lengths, int32_t* offsets, int32_t* slots,
                         int32_t* positions, int64_t tokens, int32_t* left, int32_t* lacking) {
    ReserveArgs a{held, added, n, log_page, table, width, free, pool, count, lengths, offsets, slots, positions, tokens, left, lacking, nullptr};
    if (tokens > SMALL_ROWS) {
        a.plan = static_cast<int32_t*>(adadim_workspace(ctx, WS_CACHE_PLAN, (2 * PG_SEQUENCES + 1) * 4));
        if (!a.plan) return ADADIM_EHIP;
    }
    {
        ProfScope prof(ctx, "cache_reserve_plan");
        hipLaunchKernelGGL(cache_reserve_plan, dim3(1), dim3(PG_THREADS), 0, ctx->stream, a);
        ADADIM_LAUNCH_CHECK(ctx, "cache_reserve_plan");
    }
    if (a.plan) {
        ProfScope prof(ctx, "cache_reserve_rows");
        hipLaunchKernelGGL(cache_reserve_rows, dim3(static_cast<unsigned>((tokens + 255) / 256)), dim3(256), 0, ctx->stream, a);
        ADADIM_LAUNCH_CHECK(ctx, "cache_reserve_rows");
    }
    return ADADIM_OK;
}

int launch_cache_trim(adadim_ctx* ctx, const int32_t* held, const int32_t* kept, int n, int log_page, const int32_t* table, int64_t width,
                      int32_t* free, int64_t pool, const int32_t* count, int32_t* lengths, int32_t* left) {
    TrimArgs a{held, kept, n, log_page, table, width, free, pool, count, lengths, left, nullptr};
    if (n * width > SMALL_ENTRIES) {
        a.plan = static_cast<int32_t*>(adadim_workspace(ctx, WS_CACHE_PLAN, (2 * PG_SEQUENCES + 1) * 4));
        if (!a.plan) return ADADIM_EHIP;
    }
    {
        ProfScope prof(ctx, "cache_trim_plan");
        hipLaunchKernelGGL(cache_trim_plan, dim3(1), dim3(PG_THREADS), 0, ctx->stream, a);
        ADADIM_LAUNCH_CHECK(ctx, "cache_trim_plan");
    }
    if (a.plan) {
        ProfScope prof(ctx, "cache_trim_pages");
        hipLaunchKernelGGL(cache_trim_pages, dim3(n), dim3(256), 0, ctx->stream, a);
        ADADIM_LAUNCH_CHECK(ctx, "cache_trim_pages");
    }
    return ADADIM_OK;
}
