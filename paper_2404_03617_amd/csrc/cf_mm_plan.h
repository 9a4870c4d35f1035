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

struct Tile {
    int m, n, per_cu;
    double alone, full, fixed;  // microseconds: a step for a workgroup alone on its CU, its share of a full one, its ends
};
constexpr int TILE_COUNT = 2;
constexpr Tile TILES[TILE_COUNT] = {
    {256, 256, 1, 0.62, 0.62, 5.0},
    {128, 128, 2, 0.28, 0.21, 3.5},
};

struct Plan {
    int tile, splits, per;  // per: steps of a split
};

inline int64_t steps_of(int64_t k) { return (k + STEP - 1) / STEP; }
inline int64_t tiles_of(const Tile &t, int64_t M, int64_t N) {
    return ((M + t.m - 1) / t.m) * ((N + t.n - 1) / t.n);
}

constexpr double PART_BYTES = 128 << 20;  // room for partial sums

// The least time by an estimate, as for weight gradients: rounds of
// workgroups, each its steps and its ends; split sums are written, read and
// added by a second launch.
inline double time_of(const Tile &t, int64_t M, int64_t N, int64_t steps, int64_t batch, int64_t splits, int64_t cus) {
    const double work = (double)tiles_of(t, M, N) * batch * splits;
    const int64_t each = (steps + splits - 1) / splits;
    const double rounds = std::ceil(work / (cus * t.per_cu)), load = std::ceil(work / cus);
    const double step = t.alone * rounds > t.full * load ? t.alone * rounds : t.full * load;
    return t.fixed * rounds + each * step + (splits > 1 ? 4.0 + splits * 8.0 * batch * M * N / 5.0e6 : 0.0);
}

inline Plan plan_of(int64_t M, int64_t N, int64_t steps, int64_t batch, bool may_split, int64_t cus) {
    Plan best = {0, 1, (int)(steps < 1 ? 1 : steps)};
    if (M < 1 || N < 1)  // nothing to make
        return best;
    double least = 1e300;
    for (int i = 0; i < TILE_COUNT; i++) {
        const Tile &t = TILES[i];
        const int64_t tiles = tiles_of(t, M, N) * batch;
        for (int r = 0; r <= (may_split ? t.per_cu : 0); r++) {
            int64_t splits = r ? r * cus / tiles : 1;
            const int64_t most = steps / 4, room = (int64_t)(PART_BYTES / (4.0 * batch * M * N + 1.0));
            splits = splits < most ? splits : most;
            splits = splits < room ? splits : room;
            if (splits < 1)
                splits = 1;
            const double time = time_of(t, M, N, steps, batch, splits, cus);
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
