// Which way a 4-bit product takes.  Plain C++: nothing here needs HIP.
#pragma once
#include <cstdint>

// Tile shapes and their times: what a call and what a round of tiles over 256 compute units cost beside their steps, a step (128 numbers of the
// sum), and the work-groups that share a unit.  Those of the first four are fitted to 20 products (64 to 8192 rows, 1000 to 25088 columns, sums of 500 to 25088)
// each measured with every shape.  They read the scales of four steps at once; sums of fewer take the last one, 64 x 64 with scales step by
// step, fitted to 60 products (4 to 9000 rows, 3 to 25088 columns, sums of 100 to 384) measured that way and both ways without LDS: what is picked is the
// fastest or at most 6 % (0.2 us) behind it.
struct MxShape {
    int bm, bn;
    double call_us, start_us, step_us;
    int per_cu;
};
static const MxShape mx_shapes[5] = {
    {256, 256, 0.0, 8.0, 0.95, 1}, {256, 128, 0.0, 2.5, 0.67, 1}, {128, 128, 0.0, 1.0, 0.39, 1}, {64, 64, 0.0, 2.0, 0.255, 2}, {64, 64, 0.7, 1.3, 0.25, 2}};
constexpr int MX_NARROW = 4, MX_WIDE_STEPS = 4;

inline double mx_tile_time(const MxShape& s, int64_t m, int64_t n, int64_t steps)
{
    const int64_t tiles = ((m + s.bm - 1) / s.bm) * ((n + s.bn - 1) / s.bn);
    return s.call_us + (double)((tiles + 256 * s.per_cu - 1) / (256 * s.per_cu)) * (s.start_us + s.step_us * steps);
}

// The kernels without LDS (gvq_mx_few.hip), `tiles` times 16 rows of A and 16 of B a work-group: rounds over 256 compute units again.  Fitted to
// 120 products of 17 to 500 rows, 512 to 4096 columns and sums of 256 to 25088, where the better of the two is up to four times faster than any tile
// (77 x 1000 x 4096 5.9 us and 11.5, 48 x 512 x 25088 14.4 and 56) and up to four times slower where work-groups are many.
inline double mx_few_time(int64_t m, int64_t n, int64_t steps, int tiles)
{
    const int64_t groups = ((m + 16 * tiles - 1) / (16 * tiles)) * ((n + 15) / 16);
    return 1.5 + (double)((groups + 255) / 256) * (tiles == 1 ? 0.45 + 0.06 * steps : 0.3 + 0.096 * steps);
}

struct MxWay {
    int few;     // times 16 rows of A a work-group without LDS, 0: tiles
    int shape;   // of the tiles
    double us;   // about how long it takes
};
// The fastest tiles of those that a sum of `steps` steps can take.
inline MxWay mx_tiles(int64_t m, int64_t n, int64_t steps)
{
    const int first = steps < MX_WIDE_STEPS ? MX_NARROW : 0, last = steps < MX_WIDE_STEPS ? MX_NARROW : MX_NARROW - 1;
    MxWay best{0, first, mx_tile_time(mx_shapes[first], m, n, steps)};
    for (int k = first + 1; k <= last; ++k) {
        const double t = mx_tile_time(mx_shapes[k], m, n, steps);
        if (t < best.us) best = MxWay{0, k, t};
    }
    return best;
}
// The fastest way.
inline MxWay mx_way(int64_t m, int64_t n, int64_t steps)
{
    const MxWay tiles = mx_tiles(m, n, steps);
    const double one = mx_few_time(m, n, steps, 1), two = mx_few_time(m, n, steps, 2);
    if (one <= two && one < tiles.us) return {1, 0, one};
    return two < tiles.us ? MxWay{2, 0, two} : tiles;
}
