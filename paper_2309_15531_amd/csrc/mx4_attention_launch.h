// The attention kernels of one type of queries, and the choice among them.
#pragma once

#include "mx4_attention.h"

int attention_shares(adadim_ctx* ctx, size_t bytes, void*& shared);

namespace mx4 {

// How many shares a tile's records are cut into (an upper bound; a tile with few takes fewer) and how many records one has at least.
struct Shares { int most, least; };
inline Shares shares_of(const Attention& a, int64_t tiles, int rows, bool keys) {
    const int64_t items = tiles * a.heads;
    const int64_t seen = a.window ? std::min(a.max_length, a.window + a.max_new) : a.max_length;
    const int64_t records = (seen + 31) / 32 + 1;
    // tiles that hold rows, as far as the host can tell
    const int64_t real = std::min(tiles, a.sequences * ((a.max_new * a.group + rows - 1) / rows)) * a.heads;
    const int least = keys ? 4 * AT_WAVES : 32;
    const int64_t wanted = (keys ? 1024 : 512) / std::max<int64_t>(real, 1);
    int64_t n = std::min(wanted, records / least);
    if (items > AT_TICKETS || n < 1) n = 1;
    return {static_cast<int>(std::min<int64_t>(n, 256)), least};
}

template <class T, int D, int NT, bool KEYS>
int launch_form(adadim_ctx* ctx, const Attention& a) {
    constexpr int R = KEYS ? 16 * NT : AT_WAVES * 16 * NT;
    const int64_t tiles = a.tokens * a.group / R + a.sequences;
    const Shares s = shares_of(a, tiles, R, KEYS);
    AttentionArgs args{a, static_cast<int>(tiles), s.least, nullptr, nullptr};
    if (s.most > 1) {
        void* shared = nullptr;
        const int rc = attention_shares(ctx, size_t(tiles) * a.heads * s.most * R * (D + 2) * 4, shared);
        if (rc != ADADIM_OK) return rc;
        args.tickets = static_cast<unsigned*>(shared);
        args.parts = static_cast<float*>(shared) + AT_TICKETS;
    }
    ProfScope prof(ctx, "mx4_attend");
    hipLaunchKernelGGL((mx4_attend<T, D, NT, KEYS>), dim3(static_cast<unsigned>(tiles * a.heads), s.most), dim3(64 * AT_WAVES), 0, ctx->stream, args);
    ADADIM_LAUNCH_CHECK(ctx, "mx4_attend");
    return ADADIM_OK;
}

template <class T, int D>
int launch_head(adadim_ctx* ctx, const Attention& a) {
    const int64_t rows = a.max_new * a.group;
    if (rows <= 16) return launch_form<T, D, 1, true>(ctx, a);
    if (rows <= 32) return launch_form<T, D, 2, true>(ctx, a);
    if constexpr (D <= 128) {
        if (rows <= 64) return launch_form<T, D, 4, true>(ctx, a);
        return launch_form<T, D, 4, false>(ctx, a);
    } else
        return launch_form<T, D, 2, false>(ctx, a);
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
