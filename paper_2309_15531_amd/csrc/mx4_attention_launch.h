// The attention kernels of one type of queries, and the choice among them.
#pragma once

#include "mx4_attention_tiles.h"

int attention_shares(adadim_ctx* ctx, size_t bytes, void*& shared);

namespace mx4 {

// How many shares a tile's records are cut into (an upper bound; a tile with few takes fewer) and how many records one has at least.
// Few rows: two rounds of workgroups, for sequences of unlike lengths.  A share costs about 10 us beside its records (start, the waves' sums, the way
// to the join), a record of eight waves 0.15: cut below 64 records only while the shares are one round.  Many rows: one round (2 x 4000 positions, 1000
// new ones, 32 heads: 125 us, 138 with two); a record takes 0.5 us there.
struct Shares { int most, least; };
// Whether the shares of several sequences are made alike on the device (work_of): longer ones then have more of them than two rounds would give each.
// Up to 64 sequences, which are one to a lane there.  64 of 1 to 16384 positions 146 us, 65 of them 153; one of 50000 beside 63 of 500 107 us, beside
// 64 of 500, as many shares for each, 310.
inline bool alike(const Attention& a) { return a.sequences > 1 && a.sequences <= 64; }
inline Shares shares_of(const Attention& a, int64_t tiles, int rows, bool few) {
    const int64_t seen = a.window ? std::min(a.max_length, a.window + a.max_new) : a.max_length;
    const int64_t records = (seen + 31) / 32 + 1;
    // tiles that hold rows, as far as the host can tell
    const int64_t real = std::max<int64_t>(1, std::min(tiles, a.sequences * ((a.max_new * a.group + rows - 1) / rows)) * a.heads);
    const int64_t wanted = (few ? alike(a) ? 2048 : 1024 : 256) / real;
    const int least = !few ? 16 : real * ((records + 31) / 32) > 512 ? 64 : 32;
    // (and no more shares in all than that, where the host knows less of the sequences than there is: sums of 17, 34 or 68 MB with heads filled up
    // to 64, 128 or 256, of many rows 138, 273 or 541)
    const int64_t n = std::min({wanted, records / least, (few ? AT_TICKETS / 2 : 2048) / (tiles * a.heads)});
    return {static_cast<int>(std::min<int64_t>(std::max<int64_t>(n, 1), MOST_SHARES)), least};
}

// The launch's tiles, shares and scratch; R: rows of a tile.
template <int R, int D>
int laid_out(adadim_ctx* ctx, const Attention& a, bool few, AttentionArgs& args, dim3& grid) {
    const int64_t tiles = a.tokens * a.group / R + a.sequences;
    const Shares s = shares_of(a, tiles, R, few);
    const float c = a.scale * 1.44269504088896340736f, step = RAISE / c;
    args = AttentionArgs{a, static_cast<int>(tiles), s.least, s.most, few && s.most > 1 && alike(a) ? (D <= 128 ? 512 : 256) : 0, c,
                         step < INFINITY ? step : 0.0f, nullptr, nullptr};
    grid = dim3(static_cast<unsigned>(tiles * a.heads), s.most);
    if (s.most == 1) return ADADIM_OK;
    void* shared = nullptr;
    const int rc = attention_shares(ctx, size_t(tiles) * a.heads * s.most * R * PART<D> * 4, shared);
    if (rc != ADADIM_OK) return rc;
    args.tickets = static_cast<unsigned*>(shared);
    args.parts = static_cast<float*>(shared) + AT_TICKETS;
    return ADADIM_OK;
}

template <class T, int D>
int launch_few(adadim_ctx* ctx, const Attention& a) {
    AttentionArgs args;
    dim3 grid;
    const int rc = laid_out<16, D>(ctx, a, true, args, grid);
    if (rc != ADADIM_OK) return rc;
    ProfScope prof(ctx, "mx4_attend_few");
    hipLaunchKernelGGL((mx4_attend_few<T, D>), grid, dim3(64 * AT_WAVES), 0, ctx->stream, args);
    ADADIM_LAUNCH_CHECK(ctx, "mx4_attend_few");
    return ADADIM_OK;
}

template <class T, int D>
int launch_tiles(adadim_ctx* ctx, const Attention& a) {
    static PerDeviceOnce once;
    ADADIM_HIP_TRY(ctx, once.run([] {
        return hipFuncSetAttribute(reinterpret_cast<const void*>(&mx4_attend_tiles<T, D>), hipFuncAttributeMaxDynamicSharedMemorySize, Stage<D>::LDS);
    }));
    AttentionArgs args;
    dim3 grid;
    const int rc = laid_out<TL_WAVES * 32, D>(ctx, a, false, args, grid);
    if (rc != ADADIM_OK) return rc;
    {
        ProfScope prof(ctx, "mx4_attend_tiles");
        hipLaunchKernelGGL((mx4_attend_tiles<T, D>), grid, dim3(64 * TL_WAVES), Stage<D>::LDS, ctx->stream, args);
        ADADIM_LAUNCH_CHECK(ctx, "mx4_attend_tiles");
    }
    if (args.most == 1) return ADADIM_OK;
    ProfScope prof(ctx, "mx4_attend_join");
    hipLaunchKernelGGL((mx4_attend_join<D>), dim3(grid.x, TL_WAVES), dim3(512), 0, ctx->stream, args);
    ADADIM_LAUNCH_CHECK(ctx, "mx4_attend_join");
    return ADADIM_OK;
}

// One form for all sequences of a call.  Up to 256 rows a sequence and head by tiles of 16, which read a cache once for each 16 rows but leave no wave without rows and share it finely:
// 2 x 4000 positions, 256 rows, 32 heads 51 us by them, 54 to 60 by tiles of 256; 1000 rows 160 and 125; 20000 positions, 8 heads, 256 rows 54 and
// 83, 1024 rows 158 and 112.  A chunk of 2048 tokens over 6144 positions beside 63 decoding sequences of 1024 to 8192, 64 heads over 8: 780 us, apart 568 and 85.
template <class T, int D>
int launch_head(adadim_ctx* ctx, const Attention& a) {
    return a.max_new * a.group <= 256 ? launch_few<T, D>(ctx, a) : launch_tiles<T, D>(ctx, a);
}

template <class T>
int launch_attention(adadim_ctx* ctx, const Attention& a) {
    switch (filled_head(a.dim)) {
        case 64: return launch_head<T, 64>(ctx, a);
        case 128: return launch_head<T, 128>(ctx, a);
        default: return launch_head<T, 256>(ctx, a);
    }
}

}  // namespace mx4
