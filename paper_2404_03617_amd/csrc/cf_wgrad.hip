// cf_wgrad.hip -- which tile and how many splits of the rows a weight gradient
// (cf_wgrad.h) takes, and its launch.
#include "cf_wgrad.h"

#include <math.h>

namespace cf {

namespace {

struct Plan {
    int tile;  // index into TILES
    int splits;
    int64_t chunk;
};

int64_t tiles_of(const Tile &t, int K, int C) { return (int64_t)((K + t.m - 1) / t.m) * ((C + t.n - 1) / t.n); }

// Room for partial sums.
constexpr double PART_BYTES = 128 << 20;

// The tile and number of splits that take the least time by this estimate, in
// microseconds, fitted to runs of every tile over 24 shapes (K and C from 21
// to 8192, 27 to 401408 rows), where it picks the best or one within 15% of it:
//   - a workgroup's start and end (`fixed`);
//   - its steps of 64 rows, each as long as for a workgroup alone on its CU
//     (`alone`) or as its share of a full one (`full` times the workgroups of
//     the CU), whichever is longer;
//   - partial sums written and read, at 6 TB/s, and a second launch.
// Large dW fill the chip with large tiles; small ones over many rows split the
// rows over workgroups whose wave groups share a tile (fewer partial sums);
// small ones over few rows take small tiles.
double time_of(const Tile &t, int64_t rows, int K, int C, int64_t splits, int64_t cus) {
    const double work = (double)tiles_of(t, K, C) * splits, steps = ((rows + splits - 1) / splits + 63) / 64;
    const double rounds = ceil(work / (cus * t.per_cu)), load = ceil(work / cus);
    const double step = t.alone * rounds > t.full * load ? t.alone * rounds : t.full * load;
    return t.fixed + steps * step + (splits > 1 ? 4.0 + splits * 8.0 * K * C / 6.0e6 : 0.0);
}

Plan plan_of(int64_t rows, int K, int C) {
    const int64_t cus = device_cu_count();
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

}  // namespace

size_t wgrad_workspace_bytes(int64_t rows, int K, int C) {
    const Plan p = plan_of(rows, K, C);
    return p.splits > 1 ? (size_t)p.splits * K * ((size_t)C + 1) * sizeof(float) : 0;
}

hipError_t launch_wgrad(const WGrad &g, int64_t rows, int K, int C, int bf16, void *ws, hipStream_t st) {
    const Plan p = plan_of(rows, K, C);
    WGradArgs a;
    a.dy = (const uint16_t *)g.dy;
    a.q = g.x.q;
    a.scale = g.x.scale;
    a.stats = (const float2 *)g.stats;
    a.w = g.weight;
    a.b = g.bias;
    a.dw = (uint16_t *)g.dw;
    a.db = g.db;
    a.part = p.splits > 1 ? (float *)ws : nullptr;
    a.part_db = p.splits > 1 ? (float *)ws + (size_t)p.splits * K * C : nullptr;
    a.lddy = g.lddy;
    a.rows = rows;
    a.chunk = p.chunk;
    a.K = K;
    a.C = C;
    a.blocks = blocks_of(C);
    a.tiles_k = (K + TILES[p.tile].m - 1) / TILES[p.tile].m;
    a.tiles_c = (C + TILES[p.tile].n - 1) / TILES[p.tile].n;
    a.splits = p.splits;
    if (g.stats)
        return bf16 ? launch_wgrad_norm_bf16(a, p.tile, st) : launch_wgrad_norm_f16(a, p.tile, st);
    return bf16 ? launch_wgrad_bf16(a, p.tile, st) : launch_wgrad_f16(a, p.tile, st);
}

}  // namespace cf
