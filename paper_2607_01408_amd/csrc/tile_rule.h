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
// whether a launch can hold them in the largest tiles
inline bool product_fits(int64_t M, int64_t N) { return tiles_of(M, N, 256, 256) <= kMostTiles; }
inline bool gated_fits(int64_t M, int64_t F) { return tiles_of(M, F, 256, 128) <= kMostTiles; }

}  // namespace spingtp
