// The plan of microscaled products on the host: reads lines "rows out in experts mx copy", prints "form shares out_tiles row_tiles".
// Checks on the way that a plan is one that the kernels can run.
#include "../../paper_2309_15531_amd/csrc/mx4_plan.h"

#include <cstdio>

int main() {
    long long rows, out, in;
    int experts, mx, copy;
    while (std::scanf("%lld %lld %lld %d %d %d", &rows, &out, &in, &experts, &mx, &copy) == 6) {
        const mx4::Plan p = mx4::mx4_plan(rows, out, in, experts, mx != 0, copy != 0);
        const long long np = (in + 127) / 128;
        bool ok = p.shares >= 1 && p.shares <= np && (p.shares == 1 || experts == 0);
        if (p.form == mx4::Form::rows) {
            ok = ok && (p.out_tiles == 1 || p.out_tiles == 2 || p.out_tiles == 4) && (p.row_tiles == 1 || p.row_tiles == 2 || p.row_tiles == 4);
            if (p.shares > 1) ok = ok && (out + 16 * p.out_tiles - 1) / (16 * p.out_tiles) <= mx4::MOST_SHARED && rows <= 16 * p.row_tiles;
        } else {
            int n = 0;
            auto look = [&](const mx4::TileForm& f) {
                if (f.form != p.form) return;
                ++n;
                const long long tiles = (rows + f.bm - 1) / f.bm * ((out + f.bn - 1) / f.bn);
                ok = ok && (p.shares == 1 || (f.shares && (tiles + 7) / 8 * 8 <= mx4::MOST_SHARED));
            };
            if (mx) for (const auto& f : mx4::TILE_FORMS_MX) look(f);
            else for (const auto& f : mx4::TILE_FORMS_16) look(f);
            ok = ok && n == 1;
        }
        std::printf("%d %d %d %d %s\n", static_cast<int>(p.form), p.shares, p.out_tiles, p.row_tiles, ok ? "ok" : "BAD");
    }
    return 0;
}
