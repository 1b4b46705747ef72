// Which tile a product of gemm_nt.h takes (64, 128 or 256 rows of x, and as many of w or their like): the one of
// least estimated time, among those that one launch can hold.  Host code alone.
//
// A tile's time is a part for what the CUs take at once, its share of them included, and a part for each further
// lot; small tiles lie two to a CU, but they read more for each product.  Units: about a microsecond for 2,048
// terms, the length that everything below was measured at.  Measured (us, 64 / 128 / 256):
//   8 bits, 1,024^2 11 / 20 / 45, 2,048^2 28 / 24 / 48, 2,500^2 45 / 33 / 48, 3,000^2 55 / 47 / 50,
//     4,096^2 91 / 66 / 75, 6,000^2 190 / 131 / 153, 4,096 x 8,192 187 / 130 / 121;
//   bf16 (with the gradient's elementwise part), 1,024^2 19 / 32 / 55, 2,048^2 42 / 35 / 58, 4,096 x 2,048
//     73 / 49 / 62, 3,000^2 81 / 71 / 57, 4,096^2 121 / 83 / 72;
//   gated (rows of x x outputs), 512 x 1,024 17 / 27 / 42, 2,048 x 1,024 28 / 28 / 43, 2,048^2 37 / 33 / 45,
//     3,000 x 1,500 57 / 58 / 47, 4,096 x 2,560 91 / 87 / 92, 4,096^2 134 / 126 / 109.
#pragma once

#include <cstdint>

namespace spingtp {

constexpr int64_t kMostTiles = int64_t{1} << 22;  // of a launch: below 2^32 threads

struct TileCost {
    int at_once;               // workgroups, those that share a CU included
    double first, share, more;  // up to that many tiles: first + share (their part of it); each further lot: more
};
struct TileCosts {
    TileCost of64, of128, of256;
};
inline double tile_time(const TileCost& c, int64_t tiles) {
    const int64_t full = (tiles - 1) / c.at_once;
    return c.more * static_cast<double>(full) + c.first + c.share * static_cast<double>(tiles - c.at_once * full) / c.at_once;
}
// The numbers of tiles of each size; too many of the largest are the caller's to refuse.
inline int pick_tile(const TileCosts& c, int64_t t64, int64_t t128, int64_t t256) {
    const double a = tile_time(c.of64, t64), b = tile_time(c.of128, t128), d = tile_time(c.of256, t256);
    if (t64 <= kMostTiles && a <= b && a <= d) return 64;
    return t128 <= kMostTiles && b <= d ? 128 : 256;
}
constexpr TileCosts kPlain8 = {{512, 5, 11.5, 11.5}, {512, 12, 24, 28}, {256, 38, 34, 46}};
constexpr TileCosts kPlain16 = {{512, 6, 14, 14}, {512, 23, 20, 36}, {256, 48, 16, 56}};
constexpr TileCosts kGated = {{256, 16, 11, 17}, {256, 25, 8, 33}, {256, 40, 15, 55}};

// tiles of outputs [rows][columns]; the gated block's have 128 columns each
inline int64_t tiles_of(int64_t rows, int64_t columns, int64_t tile_rows, int64_t tile_columns) {
    return ((rows + tile_rows - 1) / tile_rows) * ((columns + tile_columns - 1) / tile_columns);
}
inline int product_tile(const TileCosts& c, int64_t M, int64_t N) {
    return pick_tile(c, tiles_of(M, N, 64, 64), tiles_of(M, N, 128, 128), tiles_of(M, N, 256, 256));
}
inline int gated_tile(int64_t M, int64_t F) {
    return pick_tile(kGated, tiles_of(M, F, 64, 128), tiles_of(M, F, 128, 128), tiles_of(M, F, 256, 128));
}
// The linear layer's products have sums of any length.  A sum may be cut into slices, a workgroup to each, or a tile's
// workgroup may have twice the waves, each half of them half of the sum (64 and 128 alone: two tiles' worth of LDS).  A tile
// takes `fixed` for its start and end, and each step of its sum (128 bytes a row; two of them where two halves go) `step`, up
// to `more` longer with the part of the CUs that is busy; slices are written in fp32 and joined by a second launch.
// us, fitted to (64 / 64 by halves / 128 / 128 by halves / 256):
//   bf16 (rows x columns of w x sum), 8,192 x 2,048 x 8,192 409 / - / 240 / - / 211, 8,192 x 8,192 x 2,048 412 / - / 255 / - /
//     250, 100,000 x 512 x 128 60 / - / 33 / - / 63, 5,001 x 4,096 x 1,024 76 / - / 49 / - / 70, 3,000^3 114 / - / 97 / - / 80,
//     2,048^3 29 / 33 / 24 / 22 / 43, 3,000 x 1,500 x 1,024 21 / 26 / 16 / 22 / 30, 999 x 1,000 x 2,736 14 / 15 / 35 / 33 / 63,
//     700 x 700 x 2,048 11 / 8 / 16 / 14 / 45, 24 x 8,192 x 4,096 16 / 13 / 39 / 30 / 73; 300 x 300 x 8,192 30 / 22 / 74 / 59 /
//     144, in 8 slices 12 / 11 / 15 / 15 / 31;
//   8 bits, 24 x 2,048 x 8,192 29 / 20 / 57 / 44 / 141, in 8 slices 10 / 10 / 15 / 14 / 27, 2,048^3 26 / 32 / 21 / 18 / 44.
struct SliceCost {
    int tile, parts, at_once;
    double fixed, step, more;
};
struct SliceCosts {
    SliceCost of[5];
};
constexpr SliceCosts kSlices16 = {{{64, 1, 512, 1.7, 0.22, 0.17},
                                   {64, 2, 256, 1.8, 0.25, 0.27},
                                   {128, 1, 512, 3.6, 0.57, 0.35},
                                   {128, 2, 256, 3.6, 0.82, 0.18},
                                   {256, 1, 256, 12, 1.19, 0.42}}};
constexpr SliceCosts kSlices8 = {{{64, 1, 512, 1.7, 0.42, 0.34},
                                  {64, 2, 256, 1.8, 0.5, 0.15},
                                  {128, 1, 512, 3.6, 0.83, 0.85},
                                  {128, 2, 256, 3.6, 1.25, 0.35},
                                  {256, 1, 256, 12, 2.0, 1.2}}};
inline double slice_time(const SliceCost& c, int64_t workgroups, int64_t steps) {
    const int64_t full = workgroups / c.at_once, rest = workgroups - full * c.at_once;
    const double n = static_cast<double>((steps + c.parts - 1) / c.parts);
    double t = static_cast<double>(full) * (c.fixed + n * (c.step + c.more));
    if (rest > 0) t += c.fixed + n * (c.step + c.more * static_cast<double>(rest) / c.at_once);
    return t;
}
// The tile of a product of [M][N] outputs, the parts that its waves go by, and how many steps of `steps` a slice of its sum
// takes (all: one slice; 4 or more).  Slices and halves start at multiples of `grain` steps.
struct SumShape {
    int tile, parts;
    int64_t slices, per;
};
inline SumShape sum_shape(const SliceCosts& costs, int64_t M, int64_t N, int64_t steps, int64_t grain) {
    SumShape best{256, 1, 1, steps};
    double least = 1e300;
    for (const SliceCost& c : costs.of) {
        const int64_t tiles = ((M + c.tile - 1) / c.tile) * ((N + c.tile - 1) / c.tile);
        if (tiles > kMostTiles) continue;
        if (c.parts > 1 && (steps < 8 || (grain > 1 && steps % (c.parts * grain) != 0))) continue;
        const int64_t g = grain > 1 ? c.parts * grain : 1;
        for (int64_t want = 1; want <= 256; want = want < 4 ? want + 1 : want + want / 2) {
            if (want > 1 && (steps < 4 * c.parts * want || tiles * want > 1024)) break;
            const int64_t per = ((steps + want - 1) / want + g - 1) / g * g, slices = (steps + per - 1) / per;
            double t = slice_time(c, tiles * slices, slices > 1 ? per : steps);
            if (slices > 1)  // both ways through memory, and a launch
                t += 4.5 + 8.0 * static_cast<double>(slices) * static_cast<double>(M) * static_cast<double>(N) / 3.8e6;
            if (t < least) {
                least = t;
                best = SumShape{c.tile, c.parts, slices, slices > 1 ? per : steps};
            }
        }
    }
    return best;
}
// whether a launch can hold them in the largest tiles
inline bool product_fits(int64_t M, int64_t N) { return tiles_of(M, N, 256, 256) <= kMostTiles; }
inline bool gated_fits(int64_t M, int64_t F) { return tiles_of(M, F, 256, 128) <= kMostTiles; }

}  // namespace spingtp
