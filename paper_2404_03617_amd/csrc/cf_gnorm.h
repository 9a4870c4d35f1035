// cf_gnorm.h -- group norm with an activation over NHWC feature maps:
//
//   y = act(w xh + b),  xh = (x - mean) * rstd over the P pixels and C / G channels
//   of a group;
//   du = dy act'(w xh + b),  g = w du:
//   dx = rstd (g - mean(g) - xh mean(g xh)),  dw = sum du xh,  db = sum du
//
// Bound by memory.  A workgroup takes a run of whole groups of one image, 64 or
// 128 bytes of every pixel, and holds it in registers between the sums and what
// needs them, so that x (and dy) are read once.  A thread keeps to its 8
// channels; sums meet in LDS by channel, then by group, always in the same
// order.  The variance is a second pass over registers.  Images that do not
// fit are cut into parts of their pixels: each part leaves its mean and its sum
// of squares around it (backward: its channels' sums), and a second launch
// joins them and reads x (and dy) again.
#pragma once

#include "cf_act.h"
#include "cf_gnorm_plan.h"
#include "cf_kernels.h"
#include "cf_rows.h"

namespace cf {
namespace gnorm {

struct Args {
    const uint16_t *x, *dy;
    uint16_t *out;  // y, or dx
    int64_t ldx, lddy, ldo;
    const float *w, *b;
    float2 *stats;  // [N][G] mean, rstd
    float2 *part;   // forward: [N][chunks][G] mean, squares; backward: [N][chunks][C] sums of du, du xh
    float eps;
    int64_t P, px;
    int C, G, D, per_block, blocks, chunks, V, rows;
    bool whole;  // one launch does everything
};

hipError_t forward_f16(const Args &a, const Plan &p, int64_t N, int act, hipStream_t st);
hipError_t forward_bf16(const Args &a, const Plan &p, int64_t N, int act, hipStream_t st);
hipError_t backward_f16(const Args &a, const Plan &p, int64_t N, int act, hipStream_t st);
hipError_t backward_bf16(const Args &a, const Plan &p, int64_t N, int act, hipStream_t st);

namespace {

struct Item {
    int64_t n, p0, p1;
    int chunk, g0, groups, c0, channels;
};
// The blocks of one image read the same cache lines and run behind one L2.
__device__ __forceinline__ Item item_of(const Args &a) {
    const unsigned n = gridDim.x, xcd = blockIdx.x & 7, q = n >> 3, rest = n & 7;
    unsigned i = xcd * q + (xcd < rest ? xcd : rest) + (blockIdx.x >> 3);
    Item t;
    const unsigned block = i % (unsigned)a.blocks;
    i /= (unsigned)a.blocks;
    t.chunk = (int)(i % (unsigned)a.chunks);
    t.n = i / (unsigned)a.chunks;
    t.p0 = t.chunk * a.px;
    t.p1 = t.p0 + a.px < a.P ? t.p0 + a.px : a.P;
    t.g0 = (int)block * a.per_block;
    t.groups = a.G - t.g0 < a.per_block ? a.G - t.g0 : a.per_block;
    t.c0 = t.g0 * a.D;
    t.channels = t.groups * a.D;
    return t;
}

// K sums of each of a thread's 8 channels over the threads that share them, in
// tot[k][channel of the workgroup].  red: threads * 8 * K floats.
template <int TH, int K>
__device__ __forceinline__ void channel_sums(const Args &a, const float (&s)[K][8], bool on, int row, int vec, float *red,
                                             float *tot) {
    const int W = a.V * 8;
    if (on) {
#pragma unroll
        for (int k = 0; k < K; k++)
#pragma unroll
            for (int e = 0; e < 8; e += 4)
                *reinterpret_cast<float4v *>(red + (k * a.rows + row) * W + vec * 8 + e) =
                    float4v{s[k][e], s[k][e + 1], s[k][e + 2], s[k][e + 3]};
    }
    __syncthreads();
    int parts = TH / W;
    parts = parts < 1 ? 1 : parts > a.rows ? a.rows : parts;
    // every sum of a part lies where its first row stood: no one else reads that
    for (int i = threadIdx.x; i < W * parts; i += TH) {
        const int c = i % W, p = i / W;
#pragma unroll
        for (int k = 0; k < K; k++) {
            float v = 0.0f;
            for (int r = p; r < a.rows; r += parts)
                v += red[(k * a.rows + r) * W + c];
            red[(k * a.rows + p) * W + c] = v;
        }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < W; c += TH)
#pragma unroll
        for (int k = 0; k < K; k++) {
            float v = 0.0f;
            for (int p = 0; p < parts; p++)
                v += red[(k * a.rows + p) * W + c];
            tot[k * W + c] = v;
        }
    __syncthreads();
}

// LDS: tot [2][V * 8], group values [2][per_block], red
__device__ __forceinline__ float *groups_at(const Args &a, float *lds) { return lds + 2 * a.V * 8; }
__device__ __forceinline__ float *red_at(const Args &a, float *lds) {
    return lds + 2 * a.V * 8 + ((2 * a.per_block + 3) & ~3);
}

// f(group) by one thread a group
template <typename F>
__device__ __forceinline__ void each_group(const Item &t, F &&f) {
    for (int g = threadIdx.x; g < t.groups; g += blockDim.x)
        f(g);
}

// f(group, K sums over its channels of what add(channel, sums) adds): by a thread
// a group or, for wide ones, a wave
template <int K, typename A, typename F>
__device__ __forceinline__ void group_sums(const Args &a, const Item &t, A &&add, F &&f) {
    if (a.D < 64) {
        each_group(t, [&](int g) {
            float s[K] = {};
            for (int c = g * a.D; c < (g + 1) * a.D; c++)
                add(c, s);
            f(g, s);
        });
        return;
    }
    for (int g = threadIdx.x >> 6; g < t.groups; g += blockDim.x >> 6) {
        float s[K] = {};
        for (int c = g * a.D + (threadIdx.x & 63); c < (g + 1) * a.D; c += 64)
            add(c, s);
#pragma unroll
        for (int k = 0; k < K; k++)
            s[k] = lanes<Add, 64>(s[k]);
        if ((threadIdx.x & 63) == 0)
            f(g, s);
    }
}

// mean and rstd of the groups of this item from the parts of the image
__device__ __forceinline__ void join_parts(const Args &a, const Item &t, float *gm, float *gr) {
    each_group(t, [&](int g) {
        const float2 *const p = a.part + t.n * a.chunks * a.G + t.g0 + g;
        const float all = (float)a.P;
        float mean = 0.0f;
        for (int i = 0; i < a.chunks; i++) {
            const int64_t left = a.P - i * a.px;
            mean += p[(int64_t)i * a.G].x * ((float)(left < a.px ? left : a.px) / all);
        }
        float m2 = 0.0f;
        for (int i = 0; i < a.chunks; i++) {
            const int64_t left = a.P - i * a.px;
            const float2 v = p[(int64_t)i * a.G];
            const float d = v.x - mean, count = (float)(left < a.px ? left : a.px) * (float)a.D;
            m2 += fmaf(d * d, count, v.y);
        }
        gm[g] = mean;
        gr[g] = 1.0f / sqrtf(m2 / (all * (float)a.D) + a.eps);
        if (t.chunk == 0 && a.stats)
            a.stats[t.n * a.G + t.g0 + g] = make_float2(gm[g], gr[g]);
    });
    __syncthreads();
}

// What a thread knows of its 8 channels.
struct Channels {
    float mean[8], rstd[8], w[8], b[8];
    int group[8];
    int c, left;  // first channel in the row, how many of the workgroup's there are from it
};
__device__ __forceinline__ void channels_of(const Args &a, const Item &t, int vec, Channels &h) {
    h.c = t.c0 + vec * 8;
    h.left = t.channels - vec * 8;
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const int c = e < h.left ? vec * 8 + e : t.channels - 1;
        h.group[e] = c / a.D;
    }
    load8f(a.w ? a.w + h.c : nullptr, h.left, 1.0f, h.w);
    load8f(a.b ? a.b + h.c : nullptr, h.left, 0.0f, h.b);
}
__device__ __forceinline__ void set_stats(Channels &h, const float *gm, const float *gr) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
        h.mean[e] = gm[h.group[e]];
        h.rstd[e] = gr[h.group[e]];
    }
}

template <typename T>
__device__ __forceinline__ void store_channels(uint16_t *row, const Channels &h, const float *v) {
    store8(row, h.c, h.c + (h.left < 8 ? h.left : 8), pack8<T>(v));
}

template <typename T, int ACT>
__device__ __forceinline__ void apply(const Channels &h, const u32x4 &raw, uint16_t *row) {
    float x[8];
    unpack8<T>(raw, x);
#pragma unroll
    for (int e = 0; e < 8; e++)
        x[e] = act_pair<ACT>(fmaf((x[e] - h.mean[e]) * h.rstd[e], h.w[e], h.b[e])).f;
    store_channels<T>(row, h, x);
}

template <typename T, int ACT, int TH, int NV>
__global__ __launch_bounds__(TH) void forward_kernel(Args a) {
    extern __shared__ __align__(16) float lds[];
    const Item t = item_of(a);
    float *const tot = lds, *const gm = groups_at(a, lds), *const gr = gm + a.per_block, *const red = red_at(a, lds);
    const int row = threadIdx.x / a.V, vec = threadIdx.x - row * a.V;
    Channels h;
    channels_of(a, t, vec, h);
    const bool on = row < a.rows && h.left > 0;
    const uint16_t *const x = a.x + t.n * a.P * a.ldx;

    u32x4 v[NV];
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int64_t p = t.p0 + row + i * a.rows;
        v[i] = on && p < t.p1 ? load8(x + p * a.ldx, h.c, a.C) : u32x4{0u, 0u, 0u, 0u};
    }
    float s[1][8] = {{0.0f}};
#pragma unroll
    for (int i = 0; i < NV; i++) {  // what is not there is 0
        float f[8];
        unpack8<T>(v[i], f);
#pragma unroll
        for (int e = 0; e < 8; e++)
            s[0][e] += f[e];
    }
    channel_sums<TH, 1>(a, s, row < a.rows, row, vec, red, tot);
    const float count = (float)(t.p1 - t.p0) * (float)a.D;
    auto add = [&](int c, float(&sum)[1]) { sum[0] += tot[c]; };
    group_sums<1>(a, t, add, [&](int g, const float(&sum)[1]) { gm[g] = sum[0] / count; });
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; e++) {
        h.mean[e] = gm[h.group[e]];
        s[0][e] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < NV; i++) {
        float f[8];
        unpack8<T>(v[i], f);
        const bool here = t.p0 + row + i * a.rows < t.p1;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float d = here ? f[e] - h.mean[e] : 0.0f;
            s[0][e] = fmaf(d, d, s[0][e]);
        }
    }
    channel_sums<TH, 1>(a, s, row < a.rows, row, vec, red, tot);
    if (!a.whole) {
        group_sums<1>(a, t, add, [&](int g, const float(&sum)[1]) {
            a.part[(t.n * a.chunks + t.chunk) * a.G + t.g0 + g] = make_float2(gm[g], sum[0]);
        });
        return;
    }
    group_sums<1>(a, t, add, [&](int g, const float(&sum)[1]) {
        gr[g] = 1.0f / sqrtf(sum[0] / count + a.eps);
        if (a.stats)
            a.stats[t.n * a.G + t.g0 + g] = make_float2(gm[g], gr[g]);
    });
    __syncthreads();
    set_stats(h, gm, gr);
    uint16_t *const y = a.out + t.n * a.P * a.ldo;
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int64_t p = t.p0 + row + i * a.rows;
        if (on && p < t.p1)
            apply<T, ACT>(h, v[i], y + p * a.ldo);
    }
}

// the second launch of images in parts
template <typename T, int ACT, int TH>
__global__ __launch_bounds__(TH) void forward_apply_kernel(Args a) {
    extern __shared__ __align__(16) float lds[];
    const Item t = item_of(a);
    float *const gm = groups_at(a, lds), *const gr = gm + a.per_block;
    const int row = threadIdx.x / a.V, vec = threadIdx.x - row * a.V;
    Channels h;
    channels_of(a, t, vec, h);
    join_parts(a, t, gm, gr);
    set_stats(h, gm, gr);
    if (row >= a.rows || h.left <= 0)
        return;
    const uint16_t *const x = a.x + t.n * a.P * a.ldx;
    uint16_t *const y = a.out + t.n * a.P * a.ldo;
#pragma unroll 4
    for (int64_t p = t.p0 + row; p < t.p1; p += a.rows)
        apply<T, ACT>(h, load8(x + p * a.ldx, h.c, a.C), y + p * a.ldo);
}

// du and xh of a vector
template <typename T, int ACT>
__device__ __forceinline__ void grads(const Channels &h, const u32x4 &xr, const u32x4 &dr, float *du,
                                      float *xh) {
    unpack8<T>(xr, xh);
    unpack8<T>(dr, du);
#pragma unroll
    for (int e = 0; e < 8; e++) {
        xh[e] = (xh[e] - h.mean[e]) * h.rstd[e];
        du[e] *= act_pair<ACT>(fmaf(xh[e], h.w[e], h.b[e])).d;
    }
}

// From the channels' totals of an image the groups' means of g and g xh.
__device__ __forceinline__ void group_means(const Args &a, const Item &t, const float *tot, float *ga, float *gb) {
    const float count = (float)a.P * (float)a.D;
    group_sums<2>(
        a, t,
        [&](int c, float(&s)[2]) {
            const float w = a.w ? a.w[t.c0 + c] : 1.0f;
            s[0] = fmaf(w, tot[c], s[0]);
            s[1] = fmaf(w, tot[a.V * 8 + c], s[1]);
        },
        [&](int g, const float(&s)[2]) {
            ga[g] = s[0] / count;
            gb[g] = s[1] / count;
        });
    __syncthreads();
}

template <typename T>
__device__ __forceinline__ void store_dx(const Channels &h, const float *du, const float *xh, const float *ga,
                                         const float *gb, uint16_t *row) {
    float d[8];
#pragma unroll
    for (int e = 0; e < 8; e++)
        d[e] = h.rstd[e] * (fmaf(h.w[e], du[e], -ga[h.group[e]]) - xh[e] * gb[h.group[e]]);
    store_channels<T>(row, h, d);
}

__device__ __forceinline__ void read_stats(const Args &a, const Item &t, Channels &h) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const float2 s = a.stats[t.n * a.G + t.g0 + h.group[e]];
        h.mean[e] = s.x;
        h.rstd[e] = s.y;
    }
}

template <typename T, int ACT, int TH, int NV>
__global__ __launch_bounds__(TH) void backward_kernel(Args a) {
    extern __shared__ __align__(16) float lds[];
    const Item t = item_of(a);
    float *const tot = lds, *const ga = groups_at(a, lds), *const gb = ga + a.per_block, *const red = red_at(a, lds);
    const int row = threadIdx.x / a.V, vec = threadIdx.x - row * a.V;
    Channels h;
    channels_of(a, t, vec, h);
    const bool on = row < a.rows && h.left > 0;
    const uint16_t *const x = a.x + t.n * a.P * a.ldx, *const dy = a.dy + t.n * a.P * a.lddy;

    u32x4 v[NV], d[NV];
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int64_t p = t.p0 + row + i * a.rows;
        const bool here = on && p < t.p1;
        v[i] = here ? load8(x + p * a.ldx, h.c, a.C) : u32x4{0u, 0u, 0u, 0u};
        d[i] = here ? load8(dy + p * a.lddy, h.c, a.C) : u32x4{0u, 0u, 0u, 0u};
    }
    read_stats(a, t, h);
    float s[2][8] = {{0.0f}, {0.0f}};
#pragma unroll
    for (int i = 0; i < NV; i++) {
        if (on && t.p0 + row + i * a.rows < t.p1) {
            float du[8], xh[8];
            grads<T, ACT>(h, v[i], d[i], du, xh);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                s[0][e] += du[e];
                s[1][e] = fmaf(du[e], xh[e], s[1][e]);
            }
        }
    }
    channel_sums<TH, 2>(a, s, row < a.rows, row, vec, red, tot);
    if (a.part)
        for (int c = threadIdx.x; c < t.channels; c += TH)
            a.part[(t.n * a.chunks + t.chunk) * a.C + t.c0 + c] = make_float2(tot[c], tot[a.V * 8 + c]);
    if (!a.whole)
        return;
    group_means(a, t, tot, ga, gb);
    uint16_t *const dx = a.out + t.n * a.P * a.ldo;
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int64_t p = t.p0 + row + i * a.rows;
        if (on && p < t.p1) {
            float du[8], xh[8];
            grads<T, ACT>(h, v[i], d[i], du, xh);
            store_dx<T>(h, du, xh, ga, gb, dx + p * a.ldo);
        }
    }
}

template <typename T, int ACT, int TH>
__global__ __launch_bounds__(TH) void backward_apply_kernel(Args a) {
    extern __shared__ __align__(16) float lds[];
    const Item t = item_of(a);
    float *const tot = lds, *const ga = groups_at(a, lds), *const gb = ga + a.per_block;
    const int row = threadIdx.x / a.V, vec = threadIdx.x - row * a.V;
    Channels h;
    channels_of(a, t, vec, h);
    for (int c = threadIdx.x; c < t.channels; c += TH) {
        float s1 = 0.0f, s2 = 0.0f;
        for (int i = 0; i < a.chunks; i++) {
            const float2 v = a.part[(t.n * a.chunks + i) * a.C + t.c0 + c];
            s1 += v.x;
            s2 += v.y;
        }
        tot[c] = s1;
        tot[a.V * 8 + c] = s2;
    }
    __syncthreads();
    group_means(a, t, tot, ga, gb);
    if (row >= a.rows || h.left <= 0)
        return;
    read_stats(a, t, h);
    const uint16_t *const x = a.x + t.n * a.P * a.ldx, *const dy = a.dy + t.n * a.P * a.lddy;
    uint16_t *const dx = a.out + t.n * a.P * a.ldo;
#pragma unroll 2
    for (int64_t p = t.p0 + row; p < t.p1; p += a.rows) {
        float du[8], xh[8];
        grads<T, ACT>(h, load8(x + p * a.ldx, h.c, a.C), load8(dy + p * a.lddy, h.c, a.C), du, xh);
        store_dx<T>(h, du, xh, ga, gb, dx + p * a.ldo);
    }
}

inline size_t lds_bytes(const Plan &p, int sums) {
    return ((size_t)2 * p.V * 8 + ((2 * p.per_block + 3) & ~3) + (size_t)sums * p.rows * p.V * 8) * 4;
}

hipError_t launch(void (*f)(Args), const Args &a, const Plan &p, int64_t N, int sums, hipStream_t st) {
    const size_t lds = lds_bytes(p, sums);
    if (lds > 64 * 1024) {
        const hipError_t e = allow_full_lds((const void *)f);
        if (e != hipSuccess)
            return e;
    }
    f<<<dim3((unsigned)(N * p.blocks * p.chunks)), dim3(p.threads), lds, st>>>(a);
    return hipGetLastError();
}

// A workgroup of 256 threads holds at most 4 vectors each, one of 512 up to
// FORWARD_NV or BACKWARD_NV.
template <typename T, int ACT>
hipError_t forward_act(const Args &a, const Plan &p, int64_t N, hipStream_t st) {
    const bool big = p.threads == 512;
    void (*const f)(Args) = !big ? (p.nv <= 1 ? forward_kernel<T, ACT, 256, 1> : forward_kernel<T, ACT, 256, 4>)
                            : p.nv <= 4  ? forward_kernel<T, ACT, 512, 4>
                            : p.nv <= 8  ? forward_kernel<T, ACT, 512, 8>
                            : p.nv <= 16 ? forward_kernel<T, ACT, 512, 16>
                                         : forward_kernel<T, ACT, 512, 32>;
    const hipError_t e = launch(f, a, p, N, 1, st);
    if (e != hipSuccess || a.whole)
        return e;
    return launch(big ? forward_apply_kernel<T, ACT, 512> : forward_apply_kernel<T, ACT, 256>, a, p, N, 0, st);
}

template <typename T, int ACT>
hipError_t backward_act(const Args &a, const Plan &p, int64_t N, hipStream_t st) {
    const bool big = p.threads == 512;
    void (*const f)(Args) = !big ? (p.nv <= 1 ? backward_kernel<T, ACT, 256, 1> : backward_kernel<T, ACT, 256, 4>)
                            : p.nv <= 4 ? backward_kernel<T, ACT, 512, 4>
                            : p.nv <= 8 ? backward_kernel<T, ACT, 512, 8>
                                        : backward_kernel<T, ACT, 512, 16>;
    const hipError_t e = launch(f, a, p, N, 2, st);
    if (e != hipSuccess || a.whole)
        return e;
    return launch(big ? backward_apply_kernel<T, ACT, 512> : backward_apply_kernel<T, ACT, 256>, a, p, N, 0, st);
}

template <typename T>
hipError_t forward(const Args &a, const Plan &p, int64_t N, int act, hipStream_t st) {
    return act == ACT_SILU   ? forward_act<T, ACT_SILU>(a, p, N, st)
           : act == ACT_GELU ? forward_act<T, ACT_GELU>(a, p, N, st)
           : act == ACT_RELU ? forward_act<T, ACT_RELU>(a, p, N, st)
                             : forward_act<T, ACT_NONE>(a, p, N, st);
}
template <typename T>
hipError_t backward(const Args &a, const Plan &p, int64_t N, int act, hipStream_t st) {
    return act == ACT_SILU   ? backward_act<T, ACT_SILU>(a, p, N, st)
           : act == ACT_GELU ? backward_act<T, ACT_GELU>(a, p, N, st)
           : act == ACT_RELU ? backward_act<T, ACT_RELU>(a, p, N, st)
                             : backward_act<T, ACT_NONE>(a, p, N, st);
}

}  // namespace

}  // namespace gnorm
}  // namespace cf
