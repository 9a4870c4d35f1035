// cf_gnorm.hip -- host side of group norm (cf_gnorm.h), and the sums of its
// parameters' gradients.
#include "cf_gnorm.h"
#include "cf_head.h"

namespace cf {

using namespace gnorm;

namespace {

// dweight and dbias: L lanes a channel add the images' parts, then each other
template <int L>
__global__ __launch_bounds__(16 * L) void params_kernel(const float2 *part, int64_t parts, int C, float *dw, float *db) {
    __shared__ float2 s[L][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), l = threadIdx.x >> 4;
    float2 v = make_float2(0.0f, 0.0f);
    if (c < C)
#pragma unroll 4
        for (int64_t i = l; i < parts; i += L) {
            const float2 p = part[i * C + c];
            v.x += p.x;
            v.y += p.y;
        }
    s[l][threadIdx.x & 15] = v;
    __syncthreads();
    if (threadIdx.x < 16 && c < C) {
        float2 r = s[0][threadIdx.x];
        for (int i = 1; i < L; i++) {
            r.x += s[i][threadIdx.x].x;
            r.y += s[i][threadIdx.x].y;
        }
        db[c] = r.x;
        dw[c] = r.y;
    }
}

Plan forward_plan(int64_t N, int64_t P, int C, int G) { return gnorm::plan_of(N, P, C, G, FORWARD_NV, device_cu_count()); }
Plan backward_plan(int64_t N, int64_t P, int C, int G) { return gnorm::plan_of(N, P, C, G, BACKWARD_NV, device_cu_count()); }

Args args_of(const GroupNorm &g, const Plan &p) {
    Args a = {};
    a.x = (const uint16_t *)g.x;
    a.ldx = g.ldx;
    a.w = g.weight;
    a.b = g.bias;
    a.P = g.P;
    a.px = p.px;
    a.C = g.C;
    a.G = g.G;
    a.D = g.C / g.G;
    a.per_block = p.per_block;
    a.blocks = p.blocks;
    a.chunks = p.chunks;
    a.V = p.V;
    a.rows = p.rows;
    a.whole = p.chunks == 1;
    a.by_V = make_fastdiv((uint32_t)p.V);
    a.by_W = make_fastdiv((uint32_t)p.V * 8);
    a.by_D = make_fastdiv((uint32_t)a.D);
    return a;
}

}  // namespace

bool group_norm_fits(int64_t N, int64_t P, int C, int G) {
    for (int back = 0; back < 2; back++) {
        const Plan p = back ? backward_plan(N, P, C, G) : forward_plan(N, P, C, G);
        if (p.rows < 1 || (double)N * p.blocks * p.chunks * p.threads >= 4294967296.0 ||
            lds_bytes(p, 2) > 160 * 1024)
            return false;
    }
    return true;
}

size_t group_norm_workspace_bytes(int64_t N, int64_t P, int C, int G) {
    const Plan p = forward_plan(N, P, C, G);
    return p.chunks > 1 ? (size_t)N * p.chunks * G * sizeof(float2) : 0;
}

size_t group_norm_backward_workspace_bytes(int64_t N, int64_t P, int C, int G) {
    const Plan p = backward_plan(N, P, C, G);
    return (size_t)N * p.chunks * C * sizeof(float2);
}

hipError_t launch_group_norm(const GroupNorm &g, void *y, int64_t ldy, float *stats, float eps, int bf16, void *ws,
                             hipStream_t st) {
    const Plan p = forward_plan(g.N, g.P, g.C, g.G);
    Args a = args_of(g, p);
    a.out = (uint16_t *)y;
    a.ldo = ldy;
    a.stats = (float2 *)stats;
    a.part = (float2 *)ws;
    a.eps = eps;
    return bf16 ? forward_bf16(a, p, g.N, g.act, st) : forward_f16(a, p, g.N, g.act, st);
}

hipError_t launch_group_norm_backward(const GroupNorm &g, const void *dy, int64_t lddy, const float *stats, void *dx,
                                      int64_t lddx, float *dweight, float *dbias, int bf16, void *ws, hipStream_t st) {
    Plan p = {};
    const bool some = g.N > 0 && g.P > 0;
    if (some) {
        p = backward_plan(g.N, g.P, g.C, g.G);
        Args a = args_of(g, p);
        a.dy = (const uint16_t *)dy;
        a.lddy = lddy;
        a.out = (uint16_t *)dx;
        a.ldo = lddx;
        a.stats = (float2 *)stats;
        a.part = dweight || !a.whole ? (float2 *)ws : nullptr;
        const hipError_t e = bf16 ? backward_bf16(a, p, g.N, g.act, st) : backward_f16(a, p, g.N, g.act, st);
        if (e != hipSuccess)
            return e;
    }
    if (!dweight)
        return hipSuccess;
    const int64_t parts = some ? g.N * p.chunks : 0;
    const dim3 grid((unsigned)((g.C + 15) / 16));
    if (parts < 512)
        params_kernel<16><<<grid, 256, 0, st>>>((const float2 *)ws, parts, g.C, dweight, dbias);
    else  // (20000 images of 64 channels 36 us against 105)
        params_kernel<64><<<grid, 1024, 0, st>>>((const float2 *)ws, parts, g.C, dweight, dbias);
    return hipGetLastError();
}

}  // namespace cf
