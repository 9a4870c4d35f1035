// cf_mm_plan.h -- which tile a matrix product (cf_mm.h) takes, over how many
// workgroups its sums are split, what its kernel is given of that, and the pieces
// that a vocabulary goes by, in plain C++ so that a test can ask without a GPU.
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

// A matrix as the tiles read it: 16-byte aligned rows that hold `ext` columns,
// a multiple of 8.
struct Matrix {
    const uint16_t *p;
    int64_t ld;
    int ext;
};

// A product as its kernel is given it.
struct Args {
    const uint16_t *a[2], *b[2];
    int64_t lda, ldb;     // of both
    int M, N, K;          // K of one segment
    int ext_a, ext_b;     // rows of a (KC), or the columns that its rows hold (RC); the same of b
    int seg;              // steps of the first segment of k (behind it a[1], b[1]), or all
    int steps;            // of both
    int per;              // steps a split
    int tiles_m, tiles_n, splits;
    unsigned items;       // tiles * splits * batch
    int batch;            // 2: a[1], b[1] and out[1] are a second problem
};

// A plan's product, or one with fewer k's than it was made for (the last piece of a
// vocabulary): as many splits as those fill, since the kernel reads the first steps of
// every split before it asks whether there are any.
inline Args args_of(const Plan &p, int M, int N, int K, const Matrix &a, int ext_a, const Matrix &b, int ext_b,
                    bool two_segments = false, int batch = 1) {
    Args r;
    r.a[0] = r.a[1] = a.p;
    r.b[0] = r.b[1] = b.p;
    r.lda = a.ld;
    r.ldb = b.ld;
    r.M = M;
    r.N = N;
    r.K = K;
    r.ext_a = ext_a;
    r.ext_b = ext_b;
    r.seg = (int)steps_of(K);
    r.steps = two_segments ? 2 * r.seg : r.seg;
    if (!two_segments)
        r.seg = 1 << 30;
    r.per = p.per;
    r.tiles_m = (M + TILES[p.tile].m - 1) / TILES[p.tile].m;
    r.tiles_n = (N + TILES[p.tile].n - 1) / TILES[p.tile].n;
    r.splits = r.steps > p.per ? (r.steps + p.per - 1) / p.per : 1;
    r.batch = batch;
    r.items = (unsigned)r.tiles_m * (unsigned)r.tiles_n * (unsigned)r.splits * (unsigned)batch;
    return r;
}

// Up to PART_ROWS rows, what a product rounds for the next one is kept with what the
// rounding takes, as rows of their own: a single row's rounding is not evened out by
// others (dW of one row in bf16 was up to twice as far off as a rounded exact one), and a
// tile is one high with them too.  A gated block of 1 x 4096 x 12288 takes 60 us, without
// them 59, backward 201 and 182; of 64 rows it would be 97 and 83, 221 and 192.
constexpr int PART_ROWS = 16;
inline bool in_parts(int64_t rows) { return rows > 0 && rows <= PART_ROWS; }

// The vocabulary of a gradient (cf_linear_lp.hip) goes by pieces, whose dz is in the
// workspace: PIECE_BYTES of it (two numbers of few rows: PART_BYTES), or 4096 columns if
// that is more, rounded up so that all but the last are multiples of 256.  The last
// may be shorter.
constexpr double PIECE_BYTES = 256 << 20;
struct Pieces {
    int columns, count;
};
inline Pieces pieces_of(int64_t rows, int V) {
    const double most = (in_parts(rows) ? PART_BYTES / 2 : PIECE_BYTES) / (2.0 * (rows > 0 ? rows : 1));
    const int64_t at_most = most < 4096 ? 4096 : most > (1 << 30) ? 1 << 30 : (int64_t)most;
    Pieces p;
    p.count = (int)((V + at_most - 1) / at_most);
    p.columns = p.count == 1 ? V : ((V + p.count - 1) / p.count + 255) / 256 * 256;
    p.count = (V + p.columns - 1) / p.columns;
    return p;
}

}  // namespace mm
}  // namespace cf
