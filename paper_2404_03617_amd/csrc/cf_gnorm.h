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
//
// 128 x 56 x 56 x 64 in 16 groups, ReLU, takes 24 us forward (4.3 TB/s); 128 x 28 x 28
// x 128 in 32 groups, GELU, 20.5 forward and 31 backward, whose vector units are 84%
// busy (du is made twice: keeping it takes a second workgroup off the CU); rows that
// start at any 2 bytes and groups of 11 channels cost twice that a byte.
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
    FastDiv by_V, by_W, by_D;  // vectors of a workgroup's row, their channels, channels of a group
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

// What a thread knows of its 8 channels, from c of a row on.  EVEN and FAST: they are
// all the workgroup's.  ODD: the last of a row may begin before the ones that
// nobody else has, and the last of a workgroup end behind its own: its channels
// are lo to hi.  A row of fewer than 8 channels is read one by one.
// FAST (forward): besides, the vectors of a pixel and the channels of a group are
// powers of two, the latter at least 8: a thread has one sum, and a wave's stay in
// registers (1 x 7 x 7 x 512 5.0 us against 6.5 through LDS by channel; with two
// sums a thread, or the backward pass's sixteen, it costs more than it saves).
enum { ODD = 0, EVEN = 1, FAST = 2 };
struct Channels {
    float mean[8], rstd[8], w[8], b[8];
    int group[8];
    int c, lo, hi;
    bool on;  // has pixels and channels
};
template <int MODE>
__device__ __forceinline__ void channels_of(const Args &a, const Item &t, int row, int vec, Channels &h) {
    const int from = t.c0 + vec * 8, end = t.c0 + t.channels;
    h.on = row < a.rows && from < end;
    h.c = MODE != ODD || from <= a.C - 8 ? from : a.C >= 8 ? a.C - 8 : 0;
    h.c = h.on || MODE != ODD ? h.c : a.C >= 8 && t.c0 > a.C - 8 ? a.C - 8 : a.C >= 8 ? t.c0 : 0;
    if (MODE != ODD && !h.on)
        h.c = t.c0;
    h.lo = MODE != ODD || !h.on ? 0 : from - h.c;
    h.hi = MODE != ODD || end - h.c >= 8 ? 8 : end - h.c;
#pragma unroll
    for (int e = 0; e < 8; e++) {
        int c = h.c + e;
        if (MODE == ODD)
            c = c < t.c0 ? t.c0 : c >= end ? end - 1 : c;
        h.group[e] = (int)fdiv((uint32_t)(c - t.c0), a.by_D);
        if (MODE == ODD && a.C < 8) {
            h.w[e] = a.w ? a.w[c] : 1.0f;
            h.b[e] = a.b ? a.b[c] : 0.0f;
        }
    }
    if (MODE != ODD || a.C >= 8) {
        load8f(a.w ? a.w + h.c : nullptr, 8, 1.0f, h.w);
        load8f(a.b ? a.b + h.c : nullptr, 8, 0.0f, h.b);
    }
}
__device__ __forceinline__ void set_stats(Channels &h, const float *gm, const float *gr) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
        h.mean[e] = gm[h.group[e]];
        h.rstd[e] = gr[h.group[e]];
    }
}

template <int MODE>
__device__ __forceinline__ u32x4 load_channels(const uint16_t *base, uint32_t off, int C) {
    const char *const p = (const char *)base + off;
    if (MODE != ODD || C >= 8)
        return reinterpret_cast<const Any16 *>(p)->v;
    u32x4 r = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 7; i++)
        if (i < C)
            r[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[i] << (16 * (i & 1));
    return r;
}
template <typename T, int MODE>
__device__ __forceinline__ void store_channels(uint16_t *base, uint32_t off, const Channels &h, const float *v) {
    const u32x4 r = pack8<T>(v);
    uint16_t *const p = reinterpret_cast<uint16_t *>((char *)base + off);
    if (MODE != ODD || (h.lo == 0 && h.hi == 8)) {
        reinterpret_cast<Any16 *>(p)->v = r;
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; e++)
        if (e >= h.lo && e < h.hi)
            p[e] = (uint16_t)(r[e / 2] >> (16 * (e & 1)));
}

// Sums over a wave's lanes that hold the same vector, V (a power of two up to 64)
// vectors beside each other: rotations within 16 lanes, then swaps of halves.
__device__ __forceinline__ float row_sum(float v, int V) {
    if (V <= 8)
        v += dpp<0x128>(v);
    if (V <= 4)
        v += dpp<0x124>(v);
    if (V <= 2)
        v += dpp<0x122>(v);
    if (V <= 1)
        v += dpp<0x121>(v);
    if (V <= 16) {
        const Two t = swap16(v);
        v = t.a + t.b;
    }
    if (V <= 32) {
        const Two t = swap32(v);
        v = t.a + t.b;
    }
    return v;
}
// over n (a power of two up to 64) lanes beside each other
__device__ __forceinline__ float next_sum(float v, int n) {
    if (n >= 2)
        v += dpp<DPP_XOR1>(v);
    if (n >= 4)
        v += dpp<DPP_XOR2>(v);
    if (n >= 8)
        v += dpp<DPP_MIRROR8>(v);
    if (n >= 16)
        v += dpp<DPP_MIRROR16>(v);
    if (n >= 32) {
        const Two t = swap16(v);
        v = t.a + t.b;
    }
    if (n >= 64) {
        const Two t = swap32(v);
        v = t.a + t.b;
    }
    return v;
}

// FAST: the sums of the workgroup's groups, f(group, sum) by one thread each.  red:
// TH / 64 floats a group; whoever calls twice alternates between two.
template <int TH, typename F>
__device__ __forceinline__ void fast_group_sums(const Args &a, const Item &t, const float (&s)[8], float *red, F &&f) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per = a.D / 8;  // vectors of a group
    const float v = row_sum(((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])), a.V);
    const float all = next_sum(v, per);
    if (lane < a.V && (lane & (per - 1)) == 0)
        red[(int)fdiv((uint32_t)lane * 8, a.by_D) * (TH / 64) + wave] = all;
    __syncthreads();
    for (int g = threadIdx.x; g < t.groups; g += TH) {
        float r = 0.0f;
#pragma unroll
        for (int w = 0; w < TH / 64; w++)
            r += red[g * (TH / 64) + w];
        f(g, r);
    }
    __syncthreads();
}

// K sums of each of a thread's 8 channels over the threads that share them, in
// tot[k][channel of the workgroup].  red: threads * 8 * K floats.
template <int TH, int K, int MODE>
__device__ __forceinline__ void channel_sums(const Args &a, const Item &t, const float (&s)[K][8], const Channels &h,
                                             int row, float *red, float *tot) {
    const int W = a.V * 8;
    if (h.on) {
#pragma unroll
        for (int k = 0; k < K; k++) {
            float *const p = red + (k * a.rows + row) * W + (h.c - t.c0);
            if (MODE != ODD || h.lo == 0) {
#pragma unroll
                for (int e = 0; e < 8; e += 4)
                    *reinterpret_cast<float4v *>(p + e) = float4v{s[k][e], s[k][e + 1], s[k][e + 2], s[k][e + 3]};
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (e >= h.lo)
                        p[e] = s[k][e];
            }
        }
    }
    __syncthreads();
    int parts = TH / W;
    parts = parts < 1 ? 1 : parts > a.rows ? a.rows : parts;
    // every sum of a part lies where its first row stood: no one else reads that
    for (int i = threadIdx.x; i < W * parts; i += TH) {
        const int p = (int)fdiv((uint32_t)i, a.by_W), c = i - p * W;
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

// mean and rstd of the groups of this item from the parts of the image: a wave a
// group, lanes beside each other take parts (1 x 256 x 256 x 64 in 128 parts,
// forward 14.3 us against 50.5 by a thread a group)
template <int TH>
__device__ __forceinline__ void join_parts(const Args &a, const Item &t, float *gm, float *gr) {
    const int lane = threadIdx.x & 63;
    for (int g = threadIdx.x >> 6; g < t.groups; g += TH / 64) {
        const float2 *const p = a.part + t.n * a.chunks * a.G + t.g0 + g;
        const float all = (float)a.P;
        auto pixels = [&](int i) {
            const int64_t left = a.P - i * a.px;
            return (float)(left < a.px ? left : a.px);
        };
        float mean = 0.0f;
        for (int i = lane; i < a.chunks; i += 64)
            mean = fmaf(p[(int64_t)i * a.G].x, pixels(i) / all, mean);
        mean = lanes<Add, 64>(mean);
        float m2 = 0.0f;
        for (int i = lane; i < a.chunks; i += 64) {
            const float2 v = p[(int64_t)i * a.G];
            const float d = v.x - mean;
            m2 += fmaf(d * d, pixels(i) * (float)a.D, v.y);
        }
        m2 = lanes<Add, 64>(m2);
        if (lane == 0) {
            gm[g] = mean;
            gr[g] = 1.0f / sqrtf(m2 / (all * (float)a.D) + a.eps);
            if (t.chunk == 0 && a.stats)
                a.stats[t.n * a.G + t.g0 + g] = make_float2(gm[g], gr[g]);
        }
    }
    __syncthreads();
}

template <typename T, int ACT, int MODE>
__device__ __forceinline__ void apply(const Channels &h, const u32x4 &raw, uint16_t *base, uint32_t off) {
    float x[8];
    unpack8<T>(raw, x);
#pragma unroll
    for (int e = 0; e < 8; e++)
        x[e] = act_value<ACT>(fmaf((x[e] - h.mean[e]) * h.rstd[e], h.w[e], h.b[e]));
    store_channels<T, MODE>(base, off, h, x);
}

// A thread's pixels are row, row + rows, ..; `here(i)` whether the i-th is in the
// item.  Its place is a uniform base, which moves from pixel to pixel, and 32 bits.
#define CF_GN_PLACES                                                                                                   \
    const Item t = item_of(a);                                                                                         \
    const int row = (int)fdiv(threadIdx.x, a.by_V), vec = (int)threadIdx.x - row * a.V;                                \
    Channels h;                                                                                                        \
    channels_of<MODE>(a, t, row, vec, h);                                                                              \
    const int left = h.on ? (int)(t.p1 - t.p0) - row : 0;                                                              \
    const int64_t first = t.n * a.P + t.p0;                                                                            \
    const uint32_t at_x = (uint32_t)row * (uint32_t)a.ldx * 2 + (uint32_t)h.c * 2,                                     \
                   at_o = (uint32_t)row * (uint32_t)a.ldo * 2 + (uint32_t)h.c * 2;                                     \
    const uint16_t *const x = a.x + first * a.ldx;                                                                     \
    uint16_t *const out = a.out + first * a.ldo;                                                                       \
    const int64_t step_x = a.rows * a.ldx, step_o = a.rows * a.ldo;                                                    \
    (void)at_o, (void)out, (void)step_o;

template <typename T, int ACT, int TH, int NV, int MODE>
__global__ __launch_bounds__(TH) void forward_kernel(Args a) {
    extern __shared__ __align__(16) float lds[];
    CF_GN_PLACES
    float *const tot = lds, *const gm = groups_at(a, lds), *const gr = gm + a.per_block, *const red = red_at(a, lds);

    u32x4 v[NV];
#pragma unroll
    for (int i = 0; i < NV; i++)
        if (i * a.rows < left)
            v[i] = load_channels<MODE>(x + i * step_x, at_x, a.C);
    float s[1][8] = {{0.0f}};
#pragma unroll
    for (int i = 0; i < NV; i++)
        if (i * a.rows < left) {
            float f[8];
            unpack8<T>(v[i], f);
#pragma unroll
            for (int e = 0; e < 8; e++)
                s[0][e] += f[e];
        }
    const float count = (float)(t.p1 - t.p0) * (float)a.D;
    // f(group, sum over its channels of s); the n-th call
    auto sums = [&](int n, auto &&f) {
        if constexpr (MODE == FAST) {
            fast_group_sums<TH>(a, t, s[0], red + n * (TH / 64) * a.V, f);
        } else {
            channel_sums<TH, 1, MODE>(a, t, s, h, row, red, tot);
            group_sums<1>(
                a, t, [&](int c, float(&sum)[1]) { sum[0] += tot[c]; }, [&](int g, const float(&sum)[1]) { f(g, sum[0]); });
            __syncthreads();
        }
    };
    sums(0, [&](int g, float sum) { gm[g] = sum / count; });
#pragma unroll
    for (int e = 0; e < 8; e++) {
        h.mean[e] = gm[h.group[e]];
        s[0][e] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < NV; i++)
        if (i * a.rows < left) {
            float f[8];
            unpack8<T>(v[i], f);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float d = f[e] - h.mean[e];
                s[0][e] = fmaf(d, d, s[0][e]);
            }
        }
    sums(1, [&](int g, float sum) {
        if (!a.whole) {
            a.part[(t.n * a.chunks + t.chunk) * a.G + t.g0 + g] = make_float2(gm[g], sum);
        } else {
            gr[g] = 1.0f / sqrtf(sum / count + a.eps);
            if (a.stats)
                a.stats[t.n * a.G + t.g0 + g] = make_float2(gm[g], gr[g]);
        }
    });
    if (!a.whole)
        return;
    set_stats(h, gm, gr);
#pragma unroll
    for (int i = 0; i < NV; i++)
        if (i * a.rows < left)
            apply<T, ACT, MODE>(h, v[i], out + i * step_o, at_o);
}

// the second launch of images in parts
template <typename T, int ACT, int TH, int MODE>
__global__ __launch_bounds__(TH) void forward_apply_kernel(Args a) {
    extern __shared__ __align__(16) float lds[];
    CF_GN_PLACES
    float *const gm = groups_at(a, lds), *const gr = gm + a.per_block;
    join_parts<TH>(a, t, gm, gr);
    set_stats(h, gm, gr);
#pragma unroll 4
    for (int i = 0; i * a.rows < left; i++)
        apply<T, ACT, MODE>(h, load_channels<MODE>(x + i * step_x, at_x, a.C), out + i * step_o, at_o);
}

// du and xh of a vector
template <typename T, int ACT>
__device__ __forceinline__ void grads(const Channels &h, const u32x4 &xr, const u32x4 &dr, float *du, float *xh) {
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

struct Means {
    float a[8], b[8];
};
__device__ __forceinline__ void set_means(const Channels &h, const float *ga, const float *gb, Means &m) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
        m.a[e] = ga[h.group[e]];
        m.b[e] = gb[h.group[e]];
    }
}
template <typename T, int MODE>
__device__ __forceinline__ void store_dx(const Channels &h, const Means &m, const float *du, const float *xh,
                                         uint16_t *base, uint32_t off) {
    float d[8];
#pragma unroll
    for (int e = 0; e < 8; e++)
        d[e] = h.rstd[e] * (fmaf(h.w[e], du[e], -m.a[e]) - xh[e] * m.b[e]);
    store_channels<T, MODE>(base, off, h, d);
}

__device__ __forceinline__ void read_stats(const Args &a, const Item &t, Channels &h) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const float2 s = a.stats[t.n * a.G + t.g0 + h.group[e]];
        h.mean[e] = s.x;
        h.rstd[e] = s.y;
    }
}

// Up to KEEP vectors a thread du stays in registers in fp32; more are made twice.
constexpr int KEEP = 8;

template <typename T, int ACT, int TH, int NV, int MODE>
__global__ __launch_bounds__(TH) void backward_kernel(Args a) {
    extern __shared__ __align__(16) float lds[];
    CF_GN_PLACES
    float *const tot = lds, *const ga = groups_at(a, lds), *const gb = ga + a.per_block, *const red = red_at(a, lds);
    const uint16_t *const dy = a.dy + first * a.lddy;
    const uint32_t at_d = (uint32_t)row * (uint32_t)a.lddy * 2 + (uint32_t)h.c * 2;
    const int64_t step_d = a.rows * a.lddy;

    u32x4 v[NV], d[NV];
    float kept[NV <= KEEP ? NV : 1][8];
#pragma unroll
    for (int i = 0; i < NV; i++)
        if (i * a.rows < left) {
            v[i] = load_channels<MODE>(x + i * step_x, at_x, a.C);
            d[i] = load_channels<MODE>(dy + i * step_d, at_d, a.C);
        }
    read_stats(a, t, h);
    float s[2][8] = {{0.0f}, {0.0f}};
#pragma unroll
    for (int i = 0; i < NV; i++)
        if (i * a.rows < left) {
            float du[8], xh[8];
            grads<T, ACT>(h, v[i], d[i], du, xh);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                s[0][e] += du[e];
                s[1][e] = fmaf(du[e], xh[e], s[1][e]);
                if constexpr (NV <= KEEP)
                    kept[i][e] = du[e];
            }
        }
    channel_sums<TH, 2, MODE>(a, t, s, h, row, red, tot);
    if (a.part)
        for (int c = threadIdx.x; c < t.channels; c += TH)
            a.part[(t.n * a.chunks + t.chunk) * a.C + t.c0 + c] = make_float2(tot[c], tot[a.V * 8 + c]);
    if (!a.whole)
        return;
    group_means(a, t, tot, ga, gb);
    Means m;
    set_means(h, ga, gb, m);
#pragma unroll
    for (int i = 0; i < NV; i++)
        if (i * a.rows < left) {
            float du[8], xh[8];
            if constexpr (NV <= KEEP) {
                unpack8<T>(v[i], xh);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    du[e] = kept[i][e];
                    xh[e] = (xh[e] - h.mean[e]) * h.rstd[e];
                }
            } else {
                grads<T, ACT>(h, v[i], d[i], du, xh);
            }
            store_dx<T, MODE>(h, m, du, xh, out + i * step_o, at_o);
        }
}

template <typename T, int ACT, int TH, int MODE>
__global__ __launch_bounds__(TH) void backward_apply_kernel(Args a) {
    extern __shared__ __align__(16) float lds[];
    CF_GN_PLACES
    float *const tot = lds, *const ga = groups_at(a, lds), *const gb = ga + a.per_block;
    const uint16_t *const dy = a.dy + first * a.lddy;
    const uint32_t at_d = (uint32_t)row * (uint32_t)a.lddy * 2 + (uint32_t)h.c * 2;
    const int64_t step_d = a.rows * a.lddy;
    int share = 1;  // lanes of a channel, which add its parts together
    while (share < 64 && share < a.chunks && 2 * share * t.channels <= TH)
        share *= 2;
    for (int i = threadIdx.x; i < t.channels * share; i += TH) {
        const int c = i / share;
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll 4
        for (int k = i % share; k < a.chunks; k += share) {
            const float2 v = a.part[(t.n * a.chunks + k) * a.C + t.c0 + c];
            s.x += v.x;
            s.y += v.y;
        }
        for (int d = 1; d < share; d *= 2) {
            s.x += __shfl_xor(s.x, d);
            s.y += __shfl_xor(s.y, d);
        }
        if (i % share == 0) {
            tot[c] = s.x;
            tot[a.V * 8 + c] = s.y;
        }
    }
    __syncthreads();
    group_means(a, t, tot, ga, gb);
    read_stats(a, t, h);
    Means m;
    set_means(h, ga, gb, m);
#pragma unroll 2
    for (int i = 0; i * a.rows < left; i++) {
        float du[8], xh[8];
        grads<T, ACT>(h, load_channels<MODE>(x + i * step_x, at_x, a.C), load_channels<MODE>(dy + i * step_d, at_d, a.C),
                      du, xh);
        store_dx<T, MODE>(h, m, du, xh, out + i * step_o, at_o);
    }
}
#undef CF_GN_PLACES

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

// The kernel that holds p.nv vectors a thread, as the plan counts on (`held`).
template <typename T, int ACT, int MODE>
hipError_t forward_act(const Args &a, const Plan &p, int64_t N, hipStream_t st) {
    const bool big = p.threads == 512;
    const int nv = held(p, FORWARD_NV);
    void (*const f)(Args) = big ? (nv == 16 ? forward_kernel<T, ACT, 512, 16, MODE> : forward_kernel<T, ACT, 512, FORWARD_NV, MODE>)
                            : nv == 1 ? forward_kernel<T, ACT, 256, 1, MODE>
                            : nv == 4 ? forward_kernel<T, ACT, 256, 4, MODE>
                            : nv == 8 ? forward_kernel<T, ACT, 256, 8, MODE>
                                      : forward_kernel<T, ACT, 256, SMALL_NV, MODE>;
    const hipError_t e = launch(f, a, p, N, 1, st);
    if (e != hipSuccess || a.whole)
        return e;
    return launch(big ? forward_apply_kernel<T, ACT, 512, MODE> : forward_apply_kernel<T, ACT, 256, MODE>, a, p, N, 0, st);
}

template <typename T, int ACT, int MODE>
hipError_t backward_act(const Args &a, const Plan &p, int64_t N, hipStream_t st) {
    const bool big = p.threads == 512;
    const int nv = held(p, BACKWARD_NV);
    void (*const f)(Args) = big ? backward_kernel<T, ACT, 512, BACKWARD_NV, MODE>
                            : nv == 1 ? backward_kernel<T, ACT, 256, 1, MODE>
                            : nv == 4 ? backward_kernel<T, ACT, 256, 4, MODE>
                            : nv == 8 ? backward_kernel<T, ACT, 256, 8, MODE>
                                      : backward_kernel<T, ACT, 256, SMALL_NV, MODE>;
    const hipError_t e = launch(f, a, p, N, 2, st);
    if (e != hipSuccess || a.whole)
        return e;
    return launch(big ? backward_apply_kernel<T, ACT, 512, MODE> : backward_apply_kernel<T, ACT, 256, MODE>, a, p, N, 0,
                  st);
}

// Whether every vector of 8 channels is one workgroup's alone, and the sizes are
// powers of two.
inline int mode_of(const Args &a) {
    if (a.C % 8 || (a.per_block * a.D % 8 && a.blocks > 1))
        return ODD;
    return a.V <= 64 && (a.V & (a.V - 1)) == 0 && (a.D & (a.D - 1)) == 0 && a.D >= 8 && a.V * 8 % a.D == 0 ? FAST : EVEN;
}

template <typename T, int ACT>
hipError_t forward_act(const Args &a, const Plan &p, int64_t N, hipStream_t st) {
    const int mode = mode_of(a);
    return mode == FAST   ? forward_act<T, ACT, FAST>(a, p, N, st)
           : mode == EVEN ? forward_act<T, ACT, EVEN>(a, p, N, st)
                          : forward_act<T, ACT, ODD>(a, p, N, st);
}
template <typename T, int ACT>
hipError_t backward_act(const Args &a, const Plan &p, int64_t N, hipStream_t st) {
    return mode_of(a) == ODD ? backward_act<T, ACT, ODD>(a, p, N, st) : backward_act<T, ACT, EVEN>(a, p, N, st);
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
