// Which way an 8-bit product takes.  Plain C++: nothing here needs HIP.
#pragma once
#include <cstdint>

// A way's time: rounds over 256 compute units, of up to `share` work-groups a unit; each round has a start and so much a step (128 numbers
// of the sum), more for every work-group that shares the unit.  Fitted to 263 products (17 to 4096 rows, 256 to 25088 columns, sums of 384 to
// 16384) that were each measured in all ways: what is picked is 1.2 % behind the fastest of them on average, four in a hundred more than 10 %, one 44 %.
// How far the fastest of them is from what the card could do is another matter: none shares a sum among work-groups, and 46 of the 263, those of few
// results and long sums, take more than three times the time of their bytes, their operations or a launch (500 x 256 x 16384 24 to 33 us of 3.5, 64 x
// 64 x 131072, beyond what was fitted, 114 of 3.5).
// Without the tiles whose sums two or four teams share the fastest of the others is 9 % behind on average; 64 x 64 with more stages, 128 x 128 with two
// teams and 128 x 64 with three would add 0.4 % and are not built.
struct I8Way {
    int rows, cols;   // of the result a work-group takes
    double call_us, start_us, step_us, more_us;
    int share;
};
enum { I8_FEW_16, I8_FEW_32, I8_TILE_64, I8_TILE_64_TWO, I8_TILE_64_FOUR, I8_TILE_128, I8_TILE_256, I8_WAYS };
static const I8Way i8_ways[I8_WAYS] = {
    {16, 16, 2.45, 0.96, 0.107, 0.110, 2},   // straight from memory, 16 rows of the first operand, and 32
    {32, 16, 2.42, 1.02, 0.149, 0.169, 2},
    {64, 64, 1.16, 2.77, 0.346, 0.152, 5},   // one team, two, four
    {64, 64, 1.83, 2.68, 0.246, 0.133, 2},
    {64, 64, 1.30, 3.84, 0.207, 0.0, 1},
    {128, 128, 1.73, 4.47, 0.580, 0.369, 2},
    {256, 256, 0.00, 9.49, 1.105, 0.0, 1},
};

// `groups` work-groups over `steps` steps each (on average).
inline double i8_rounds(const I8Way& w, int64_t groups, double steps)
{
    const int64_t per = (groups + 255) / 256, full = per / w.share, rest = per % w.share;
    double t = w.call_us + (double)full * (w.start_us + (w.step_us + w.more_us * (w.share - 1)) * steps);
    if (rest > 0) t += w.start_us + (w.step_us + w.more_us * (rest - 1)) * steps;
    return t;
}
// m x n results, each of `sums` sums (2: a gate's and another projection's): a tile has so many columns of sums, and without tiles a work-group takes
// both sums of its columns.
inline int64_t i8_groups(const I8Way& w, int64_t m, int64_t n, int sums)
{
    return (m + w.rows - 1) / w.rows * (w.cols == 16 ? (n + 15) / 16 : (n * sums + w.cols - 1) / w.cols);
}
inline double i8_way_time(const I8Way& w, int64_t m, int64_t n, int sums, int64_t steps)
{
    return i8_rounds(w, i8_groups(w, m, n, sums), (double)steps * (w.cols == 16 ? sums : 1));
}

inline int i8_pick(int64_t m, int64_t n, int sums, int64_t steps)
{
    int best = I8_TILE_64;
    double us = i8_way_time(i8_ways[best], m, n, sums, steps);
    for (int k = 0; k < I8_WAYS; ++k) {
        if (steps == 0 && i8_ways[k].cols == 16) continue;   // (a sum over nothing)
        const double t = i8_way_time(i8_ways[k], m, n, sums, steps);
        if (t < us) { us = t; best = k; }
    }
    return best;
}

// Two plain products: the tiles that take both in one launch, or -1 if a launch each, in its own way, is faster.  A launch of its own is 2 us.
inline int i8_pick_pair(int64_t m0, int64_t n0, int64_t steps0, int64_t m1, int64_t n1, int64_t steps1)
{
    int best = -1;
    double us = i8_way_time(i8_ways[i8_pick(m0, n0, 1, steps0)], m0, n0, 1, steps0) + i8_way_time(i8_ways[i8_pick(m1, n1, 1, steps1)], m1, n1, 1, steps1) + 2.0;
    for (int k = I8_TILE_64; k < I8_WAYS; ++k) {
        const int64_t g0 = i8_groups(i8_ways[k], m0, n0, 1), g1 = i8_groups(i8_ways[k], m1, n1, 1);
        const double t = i8_rounds(i8_ways[k], g0 + g1, ((double)g0 * steps0 + (double)g1 * steps1) / (double)(g0 + g1));
        if (t < us) { us = t; best = k; }
    }
    return best;
}
