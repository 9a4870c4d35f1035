// cf_wgrad.hip -- launch of a weight gradient (cf_wgrad.h) with the tile and
// splits of cf_wgrad_plan.h.
#include "cf_wgrad.h"

namespace cf {

namespace {

wgrad::Plan plan_of(int64_t rows, int K, int C) { return wgrad::plan_of(rows, K, C, device_cu_count()); }

}  // namespace

size_t wgrad_workspace_bytes(int64_t rows, int K, int C) {
    const wgrad::Plan p = plan_of(rows, K, C);
    return p.splits > 1 ? (size_t)p.splits * K * ((size_t)C + 1) * sizeof(float) : 0;
}

hipError_t launch_wgrad(const WGrad &g, int64_t rows, int K, int C, int bf16, void *ws, hipStream_t st) {
    const wgrad::Plan p = plan_of(rows, K, C);
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
    a.tiles_k = (K + wgrad::TILES[p.tile].m - 1) / wgrad::TILES[p.tile].m;
    a.tiles_c = (C + wgrad::TILES[p.tile].n - 1) / wgrad::TILES[p.tile].n;
    a.splits = p.splits;
    if (g.stats)
        return bf16 ? launch_wgrad_norm_bf16(a, p.tile, st) : launch_wgrad_norm_f16(a, p.tile, st);
    return bf16 ? launch_wgrad_bf16(a, p.tile, st) : launch_wgrad_f16(a, p.tile, st);
}

}  // namespace cf
