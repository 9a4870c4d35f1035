// cf_wgrad_plan.h -- which tile and how many splits of the rows a weight
// gradient (cf_wgrad.h) takes, in plain C++ so that a test can ask without a GPU.
#pragma once

#include <cmath>
#include <stddef.h>
#include <stdint.h>

namespace cf {
namespace wgrad {

// The tiles: m x n of dW; waves; bytes of a checkpoint's row a load; workgroups
// that run on a CU together; and what the choice among them estimates with, in
// microseconds.
struct Tile {
    int m, n, waves, qb, per_cu;
    double alone, full, fixed;
};
constexpr int TILE_COUNT = 7;
constexpr Tile TILES[TILE_COUNT] = {
    {64, 64, 4, 16, 3, 0.50, 0.386, 4.5},   // 0
    {128, 128, 4, 16, 3, 1.15, 0.72, 8.0},  // 1
    {256, 256, 8, 16, 1, 1.45, 2.00, 12.0}, // 2
    {256, 64, 8, 8, 1, 0.90, 0.92, 6.5},    // 3
    {64, 256, 8, 16, 1, 0.90, 0.88, 6.5},   // 4
    {128, 128, 8, 16, 1, 0.73, 0.80, 8.0},  // 5: two groups of four waves
    {64, 64, 16, 8, 1, 0.40, 0.362, 6.0},   // 6: four groups of four waves
};

struct Plan {
    int tile;  // index into TILES
    int splits;
    int64_t chunk;
};

inline int64_t tiles_of(const Tile &t, int K, int C) { return (int64_t)((K + t.m - 1) / t.m) * ((C + t.n - 1) / t.n); }

// Room for partial sums.
constexpr double PART_BYTES = 128 << 20;

// The tile and number of splits that take the least time by this estimate, in
// microseconds, fitted to runs of every tile over 24 shapes (K and C from 21
// to 8192, 27 to 401408 rows), where it picks the best or one within 15% of it:
//   - a workgroup's start and end (`fixed`);
//   - its rows, by 64 (whatever a step of the tile stages), each as long as for a
//     workgroup alone on its CU (`alone`) or as its share of a full one (`full`
//     times the workgroups of the CU), whichever is longer;
//   - partial sums written and read, at 6 TB/s, and a second launch.
// Large dW fill the chip with large tiles; small ones over many rows split the
// rows over workgroups whose wave groups share a tile (fewer partial sums);
// small ones over few rows take small tiles.
inline double time_of(const Tile &t, int64_t rows, int K, int C, int64_t splits, int64_t cus) {
    const int64_t each = (rows + splits - 1) / splits;
    // no rows still take a workgroup a tile: as many as one row
    const double work = (double)tiles_of(t, K, C) * splits, steps = each < 1 ? 1 : (each + 63) / 64;
    const double rounds = std::ceil(work / (cus * t.per_cu)), load = std::ceil(work / cus);
    const double step = t.alone * rounds > t.full * load ? t.alone * rounds : t.full * load;
    return t.fixed + steps * step + (splits > 1 ? 4.0 + splits * 8.0 * K * C / 6.0e6 : 0.0);
}

inline Plan plan_of(int64_t rows, int K, int C, int64_t cus) {
    Plan best = {0, 1, 0};
    double least = 1e300;
    for (int i = 0; i < TILE_COUNT; i++) {
        const Tile &t = TILES[i];
        const int64_t tiles = tiles_of(t, K, C);
        for (int r = 0; r <= t.per_cu; r++) {  // whole, or the splits that give r workgroups a CU
            int64_t splits = r ? r * cus / tiles : 1;
            const int64_t most = (rows + 63) / 64, room = (int64_t)(PART_BYTES / (4.0 * K * (C + 1.0)));
            splits = splits < most ? splits : most;
            splits = splits < room ? splits : room;
            if (splits < 1)
                splits = 1;
            const double time = time_of(t, rows, K, C, splits, cus);
            if (time < least) {
                least = time;
                best.tile = i;
                best.splits = (int)splits;
            }
        }
    }
    // rows of a split: whole steps
    const int64_t each = (rows + best.splits - 1) / best.splits;
    best.chunk = each < 1 ? 64 : (each + 63) / 64 * 64;
    best.splits = rows < 1 ? 1 : (int)((rows + best.chunk - 1) / best.chunk);
    return best;
}

}  // namespace wgrad
}  // namespace cf
