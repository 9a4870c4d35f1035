// cf_mm_plan.h -- which tile a matrix product (cf_mm.h) takes and over how many
// workgroups its sums are split, in plain C++ so that a test can ask without a
// GPU.
#pragma once

#include <cmath>
#include <stddef.h>
#include <stdint.h>

namespace cf {
namespace mm {

constexpr int STEP = 64;  // k's of a step

// The tiles, workgroups that run on a CU together, and what the choice among them
// estimates with, in microseconds.
struct Tile {
    int m, n, per_cu;
    double alone, ends;       // a step for a workgroup alone on its CU, and its start and end
    double full, full_ends;   // its share of a full CU
    double gate;              // a tile whose results are joined with 8 bytes and leave as 6, beyond the rest
};
constexpr int TILE_COUNT = 2;
constexpr Tile TILES[TILE_COUNT] = {
    {256, 256, 1, 0.56, 7.6, 1.505, 10.0, 47.5},
    {128, 128, 2, 0.751, 6.15, 0.616, 2.46, 8.5},
};

struct Plan {
    int tile, splits, per;  // per: steps of a split
};

inline int64_t steps_of(int64_t k) { return (k + STEP - 1) / STEP; }
inline int64_t tiles_of(const Tile &t, int64_t M, int64_t N) {
    return ((M + t.m - 1) / t.m) * ((N + t.n - 1) / t.n);
}

constexpr double PART_BYTES = 128 << 20;  // room for partial sums

// The tile and number of splits that take the least time by this estimate, fitted to
// runs of either tile, whole and split, over 35 shapes (16 to 131072 rows and
// columns, 16 to 50024 k's, with each kind of epilogue), where it picks the best
// or one within 4% of it: rounds of workgroups, each its steps and its ends, or a
// CU's share of all, whichever is longer; partial sums written and read, at 8
// TB/s.  Large tiles move least and win where they fill the chip; small
// ones start and end while their neighbour's products run.  GATE: what follows a
// tile of the gate's gradients, 14 bytes a result, which small tiles hide in part
// (25088 x 1024 x 256 94 us with small tiles, 120 with large ones; 4096 x 4096 x 8192
// 340 and 312).  Where more follows than a store, split sums are joined by a
// launch that does it, a little later and slower (3 us and 4 TB/s: a block of 32
// x 8192 with 2048 channels takes 38 us with split sums, 95 with whole ones, but one of
// 256 x 1024 with 2816 38 and 32).
enum After { STORE, MORE, GATE };
inline double time_of(const Tile &t, int64_t M, int64_t N, int64_t steps, int64_t batch, int64_t splits, int64_t cus,
                      After what) {
    const double work = (double)tiles_of(t, M, N) * batch * splits;
    const int64_t each = (steps + splits - 1) / splits;
    const double rounds = std::ceil(work / (cus * t.per_cu)), load = std::ceil(work / cus);
    const double after = what == GATE && splits == 1 ? t.gate : 0.0;
    const double one = rounds * (t.ends + after + each * t.alone), all = load * (t.full_ends + after + each * t.full);
    const double whole = one > all ? one : all, parts = splits * 8.0 * batch * M * N;
    return splits == 1 ? whole : what == STORE ? whole + parts / 8.0e6 : whole + parts / 4.0e6 + 3.0;
}

inline Plan plan_of(int64_t M, int64_t N, int64_t steps, int64_t batch, bool may_split, int64_t cus,
                    After what = STORE) {
    Plan best = {0, 1, (int)(steps < 1 ? 1 : steps)};
    if (M < 1 || N < 1)  // nothing to make
        return best;
    double least = 1e300;
    for (int i = 0; i < TILE_COUNT; i++) {
        const Tile &t = TILES[i];
        const int64_t tiles = tiles_of(t, M, N) * batch;
        for (int r = 0; r <= (may_split ? 2 * t.per_cu : 0); r++) {  // whole, or r / 2 workgroups a CU
            int64_t splits = r ? r * cus / (2 * tiles) : 1;
            const int64_t most = steps / 2, room = (int64_t)(PART_BYTES / (4.0 * batch * M * N + 1.0));
            splits = splits < most ? splits : most;
            splits = splits < room ? splits : room;
            if (splits < 1)
                splits = 1;
            const double time = time_of(t, M, N, steps, batch, splits, cus, what);
            if (time < least) {
                least = time;
                best.tile = i;
                best.splits = (int)splits;
            }
        }
    }
    if (steps >= 1) {
        best.per = (int)((steps + best.splits - 1) / best.splits);
        best.splits = (int)((steps + best.per - 1) / best.per);
    }
    return best;
}
inline size_t part_bytes(const Plan &p, int64_t M, int64_t N, int64_t batch) {
    return p.splits > 1 ? (size_t)p.splits * batch * M * N * 4 : 0;
}

}  // namespace mm
}  // namespace cf
