// How products of 8-bit integers choose their kernels: plain arithmetic without a device in it.
#pragma once
#include <stdint.h>

namespace anr {
namespace i8 {

// ---- few rows

constexpr int kRowsChunk = 128;                 // k of a wave at a time: a line of a row
constexpr int most_waves(int TB) { return TB == 1 ? 16 : TB == 2 ? 8 : 4; }      // of a work-group: their buffers fit LDS

// Waves of a work-group: as far as there are chunks for them, eight for each CU over all work-groups, or long rows. us, 4 / 8 / 16 waves: 1 token 2048 -> 11264
// 6.0 / 6.9 / 9.7, 5632 -> 2048 4.8 / 4.0 / 4.3, 1024 -> 1024 2.74 / 2.68 / 3.1, 16384 -> 16384 54.1 / 50.6 / 52.2, 8 tokens 4096 -> 4096 5.9 / 5.6 / 5.4.
inline int waves_of(int64_t N, int64_t K, int most)
{
    const int64_t groups = (N + 15) / 16, chunks = (K + kRowsChunk - 1) / kRowsChunk;
    int waves = 4;
    while (waves < most && chunks >= 4 * waves && (groups * waves <= 2048 || chunks >= 16 * waves)) waves *= 2;
    return waves;
}

// ---- tiles

constexpr int64_t kChunk = 128;                  // k of a chunk
constexpr int kCus = 256;

// A tile, how many of its work-groups a CU takes at a time, and its estimated time in us: a chunk's where a work-group is alone on its CU and where that is full, and that
// of both ends.  The deep ones have a chunk more on their way, for products of few tiles: 64 tokens 4096 -> 11264 in tiles of 64 with two, three and four buffers 17.7 / 11.3 / 10.4 us, 777 tokens 640 -> 1363
// 5.2 / 5.4 / 5.7; 256 tokens 4096 -> 11264 in tiles of 128 with two and three 24.1 / 16.9 and 512 tokens 27.9 / 32.1.
struct Shape {
    int m, n, on_cu;
    double alone, full, ends;
};
enum { TILE_256, TILE_128, TILE_128_DEEP, TILE_64_128, TILE_64, TILE_64_DEEP, TILES, ROWS = TILES };
constexpr Shape kShapes[TILES] = {
    {256, 256, 1, 1.18, 1.18, 4.5}, {128, 128, 2, 0.59, 0.69, 3.3}, {128, 128, 1, 0.35, 0.35, 4.6}, {64, 128, 2, 0.30, 0.50, 3.1}, {64, 64, 3, 0.22, 0.69, 2.9}, {64, 64, 2, 0.175, 0.46, 3.4}};

inline int64_t tiles_of(int64_t M, int64_t N, const Shape& s) { return ((M + s.m - 1) / s.m) * ((N + s.n - 1) / s.n); }

inline double estimate(const Shape& s, int64_t tiles, int64_t chunks)
{
    const int64_t at_once = (int64_t)s.on_cu * kCus, rounds = tiles / at_once, rest = tiles % at_once, beside = (rest + kCus - 1) / kCus;
    double us = (double)rounds * (s.full * (double)chunks + s.ends);
    if (rest > 0) us += (s.on_cu > 1 ? s.alone + (s.full - s.alone) * (double)(beside - 1) / (double)(s.on_cu - 1) : s.full) * (double)chunks + s.ends;
    return us;
}

// The kernels for few rows: reading W, and X for every sixteen of W's rows, and a round of the waves' chunks.
inline double estimate_rows(int64_t M, int64_t N, int64_t K)
{
    const int64_t groups = (N + 15) / 16, blocks = (M + 15) / 16, chunks = (K + kChunk - 1) / kChunk, waves = waves_of(N, K, most_waves((int)blocks));
    return 3.0 + (double)N * (double)K / 11.1e6 + (double)(groups * blocks * 16) * (double)K / 71e6 + 0.078 * (double)((1 + blocks) * ((chunks + waves - 1) / waves));
}

// The tile, or the kernels for few rows, and the work-groups that share a tile's k where there are few, with the shortest estimated time, that of the launch that joins their
// sums among it.  A function of the extents alone.  The estimates' numbers are fitted to 272 products of 1 to 2048 rows, 256 -> 4096 to 4096 -> 16384, each by every tile and 1 to 8
// parts of k: what is chosen took 1 % longer than the fastest on average, 14 to 34 % for 20 to 48 rows 11264 -> 4096 (13.0 to 13.6 us in parts of k, 9.8 to 11.9 by the kernels for few rows).
struct Choice {
    int tile, splits;
};
constexpr int64_t kMostRows = 64;
inline Choice choose(int64_t M, int64_t N, int64_t K)
{
    const int64_t chunks = (K + kChunk - 1) / kChunk;
    Choice best{ROWS, 1};
    double least = M <= kMostRows ? estimate_rows(M, N, K) : 1e30;
    for (int t = 0; t < TILES; ++t)
        for (int s = 1; s <= 16 && (s == 1 || chunks / s >= 4); ++s) {
            const double us = estimate(kShapes[t], s * tiles_of(M, N, kShapes[t]), (chunks + s - 1) / s) + (s > 1 ? 3.45 + 2.0 * s * (double)M * (double)N * 4.0 / 4.6e6 : 0.0);
            if (us < least) {
                least = us;
                best = {t, s};
            }
        }
    return best;
}

}  // namespace i8
}  // namespace anr
