// Which kernel a microscaled product takes, from its sizes and X's type.  Host code without HIP.
//
// The kernels differ in how much of Y a workgroup owns.  Large tiles read each operand less often; small ones are more, start sooner and
// leave fewer compute units idle, and where even they are few the contraction is shared.  Which is ahead depends on all of rows, outputs,
// contraction, X's type and the groups, so each form's time is estimated and the shortest taken.  The estimates are fits to the
// kernels' times over shapes drawn at random (1 to 8192 rows, 64 to 28672 outputs, 64 to 28672 deep; 4 to 128 experts): mean error 9 to 15 % a form, and
// the form chosen is 2 % (one weight) and 4 % (experts) slower in the geometric mean than the best of them all.  (How far that best one is from
// what the sizes need is another matter: 1.1 to 3.8 times at sizes looked at, most between a few dozen and a few thousand rows.)
#pragma once

#include <algorithm>
#include <cstdint>

namespace mx4 {

// rows: 16 out_tiles outputs, a wave a share of the pieces.  The others by their tile (rows x outputs): ring32 32 x 256 (mx4 X: 32 x 128), ring64
// 64 x 64, ring64w 64 x 128, mid 128 x 128, big 128 x 256 (mx4 X: 256 x 256).
enum class Form { rows, ring32, ring64, ring64w, mid, big };

struct Plan {
    Form form;
    int shares;                    // of the contraction
    int out_tiles, row_tiles;      // of 16, of a workgroup (rows)
};

constexpr int MOST_SHARED = 1024;  // output tiles that can be shared: each has a counter

struct TileForm {
    Form form;
    int bm, bn, pieces;            // the tile, pieces of a stage
    bool shares;
    float start, tile, stage;      // us: of the launch, of a tile, of a stage
    float fill;                    // workgroups that run at once, over 256
    float steps;                   // how far a last round that is not full counts as one: 1 wholly, 0 by its share
    float share;                   // us: of adding up
    float read;                    // MB/us: operands through the L2
};
constexpr TileForm TILE_FORMS_16[] = {
    {Form::ring32, 32, 256, 1, true, 1.50f, 3.39f, 0.598f, 1.00f, 1.00f, 2.0f, 8.1f},
    {Form::ring64, 64, 64, 1, true, 3.25f, 1.53f, 0.422f, 1.09f, 0.25f, 2.1f, 12.6f},
    {Form::ring64w, 64, 128, 1, true, 3.73f, 1.68f, 0.544f, 1.03f, 0.46f, 3.5f, 31.4f},
    {Form::mid, 128, 128, 1, true, 1.53f, 4.24f, 0.808f, 1.00f, 0.99f, 3.2f, 8.5f},
    {Form::big, 128, 256, 1, true, 1.50f, 4.66f, 1.367f, 1.01f, 1.00f, 4.0f, 8.6f}};
constexpr TileForm TILE_FORMS_MX[] = {
    {Form::ring32, 32, 128, 1, true, 3.33f, 1.32f, 0.206f, 1.01f, 0.80f, 1.7f, 10.7f},
    {Form::ring64, 64, 64, 1, true, 3.67f, 0.68f, 0.188f, 1.19f, 0.60f, 1.9f, 29.4f},
    {Form::ring64w, 64, 128, 1, true, 4.34f, 0.60f, 0.234f, 1.01f, 0.65f, 3.4f, 20.7f},
    {Form::mid, 128, 128, 2, false, 3.50f, 1.88f, 0.602f, 1.03f, 0.41f, 0.0f, 34.9f},
    {Form::big, 256, 256, 2, false, 1.50f, 4.94f, 1.471f, 1.01f, 1.00f, 0.0f, 8.5f}};
struct RowForm {
    int out_tiles;
    float start, pass, piece, rows;   // us: of the launch, of a pass over the contraction, of a wave's piece, and of 16 rows of X with it
    float fill, steps;                // as above
    float share, more;                // us: of adding up for 16 rows, and for each 16 more
    float read;                       // MB/us: of W, most of it from memory
};
constexpr RowForm ROW_FORMS_16[] = {
    {1, 3.22f, 0.45f, 0.26f, 0.87f, 1.02f, 0.72f, 1.05f, 0.49f, 4.3f},
    {2, 3.10f, 0.71f, 0.46f, 0.94f, 0.96f, 0.52f, 0.96f, 0.80f, 4.6f},
    {4, 3.25f, 0.94f, 0.76f, 1.24f, 0.99f, 0.87f, 1.07f, 0.0f, 5.2f}};
constexpr RowForm ROW_FORMS_MX[] = {
    {1, 2.50f, 0.29f, 0.25f, 0.25f, 1.02f, 0.79f, 1.31f, 0.18f, 7.0f},
    {2, 2.70f, 0.26f, 0.39f, 0.36f, 1.05f, 0.94f, 1.01f, 0.63f, 6.5f},
    {4, 2.19f, 0.78f, 0.84f, 0.61f, 0.99f, 0.81f, 1.42f, 0.0f, 5.0f}};

// experts 0: one weight.  copy: X has to be copied for all forms but rows (a launch more).
inline Plan mx4_plan(int64_t n_rows, int64_t out, int64_t in, int experts, bool mx, bool copy) {
    const double np = double((in + 127) / 128);
    const double active = experts ? double(std::min<int64_t>(experts, n_rows)) : 1.0;         // groups that may have rows
    const double weight = active * double(out) * np * 68.0;                                   // bytes of W
    const double avg = double(n_rows) / active;
    const double part = double(n_rows) * double(out) * 8.0;                                   // bytes of a share's sums, out and back
    auto up = [](double v) { return double(int64_t(v) + (double(int64_t(v)) < v)); };
    Plan best{Form::ring64, 1, 0, 0};
    double least = 1e30;
    auto take = [&](double t, Plan p) {
        if (t < least) {
            least = t;
            best = p;
        }
    };
    // few rows, in passes over the contraction.  Beyond 32 a group the groups' lengths, which the host does not know, differ too much for
    // the estimate: with tiles there the chosen form was 5 % slower than the best, with these 7 %.
    const int64_t per_group = experts ? (n_rows + experts - 1) / experts : n_rows;
    if (per_group <= (experts ? 32 : 96)) {
        const int rt = per_group <= 16 ? 1 : per_group <= 32 ? 2 : 4;
        const double loops = std::max(1.0, (experts ? 3.0 : 1.0) * avg / (16 * rt));          // of the longest group
        for (const RowForm& f : mx ? ROW_FORMS_MX : ROW_FORMS_16) {
            if (f.out_tiles == 4 && rt > 1) break;             // (the estimates rarely had it ahead)
            const double tiles = up(double(out) / (16 * f.out_tiles));
            for (int s = 1; s <= 8; s *= 2) {
                if (s > 1 && (experts || n_rows > 64 || s > np || tiles > MOST_SHARED)) break;
                const double full = std::max(1.0, active * tiles * s / (256 * f.fill)), rounds = f.steps * up(full - 1e-9) + (1.0 - f.steps) * full, rows = std::min(avg / loops, 16.0 * rt);
                double t = f.start + rounds * loops * (f.pass + up(np / (8 * s)) * (f.piece + f.rows * rows / 16.0));
                // (a workgroup of few reads 28 GB/s: 64 to 128 of four output tiles 1.9 to 3.1 TB/s)
                t = std::max(t, f.start + weight / std::min(f.read * 1e6, active * tiles * s * 28e3)) + (s > 1 ? f.share + f.more * (rt - 1) : 0.0);
                take(t, Plan{Form::rows, s, f.out_tiles, rt});
            }
        }
    }
    auto tile = [&](const TileForm& f) {
        if (!experts && n_rows * 4 <= f.bm && f.bm > 64) return;  // (24 rows of 8320 -> 27392 took 1.3 times as long by 128 as by 32)
        const double rt = experts ? std::max(active, double(n_rows) / f.bm + 0.5 * active) : up(double(n_rows) / f.bm);
        const double tiles = rt * up(double(out) / f.bn);
        for (int s = 1; s <= (f.shares && !experts ? 8 : 1); s *= 2) {
            if (s > 1 && (s > np || tiles * s > MOST_SHARED)) break;
            const double full = std::max(1.0, tiles * s / (256 * f.fill)), rounds = f.steps * up(full - 1e-9) + (1.0 - f.steps) * full;
            double t = f.start + rounds * (f.tile + up(np / (s * f.pieces)) * f.stage) + double(n_rows) * double(out) * 2.0 / 5.0e6;      // (Y's way out)
            t = std::max({t, f.start + weight / 4.6e6, f.start + tiles * np * (f.bm * (mx ? 64.0 : 256.0) + f.bn * 64.0) / (f.read * 1e6)}) + (s > 1 ? f.share + s * part / 6.0e6 : 0.0);
            take(t + (copy ? 4.0 + double(n_rows) * double(in) * 4.0 / 5.0e6 : 0.0), Plan{f.form, s, 0, 0});
        }
    };
    if (mx)
        for (const TileForm& f : TILE_FORMS_MX) tile(f);
    else
        for (const TileForm& f : TILE_FORMS_16) tile(f);
    return best;
}

}  // namespace mx4
