// cf_norm.hip -- layer norm over the channels of each row (an NHWC pixel, a
// token), forward and backward, with the 8-bit checkpoint of the input.
//
//   mean = 1/C sum_c x,  var = 1/C sum_c (x - mean)^2,  rstd = 1 / sqrt(var + eps)
//   xh = (x - mean) rstd,  y = w xh + b
//   g = w dy,  dx = rstd (g - 1/C sum_c g - xh 1/C sum_c g xh)
//   dw = sum_r dy xh,  db = sum_r dy
//
// Both passes are bound by memory: a row is read once, held in registers as
// fp32 (so the variance is a second pass over registers, without the
// cancellation of E[x^2] - mean^2) and written once.  G lanes share a row,
// 8 V channels each, in vectors of 8 that alternate between the lanes so that
// a group's loads are contiguous: narrow rows of 64 channels take 8 lanes, a
// wave then holds 8 rows, rows above 512 channels take several waves.
//
// Measured on MI355X, where a copy of 2 GiB moves 4.9 TB/s (kernel times):
//   forward   401408 x 64 fp16 with statistics and checkpoint 25.4 us, 5.2 TB/s;
//             25088 x 256 bf16 7.7 us; 2999 x 4095 bf16 13 us, 3.8 TB/s (rows
//             that start at any 2 bytes); one row of 512 1.8 us, a launch
//   backward  401408 x 64 from the checkpoint 25.0 us, 5.3 TB/s, and 4.8 us for
//             the second launch; 2999 x 4095 22 us, 3.4 TB/s, and 4 us: six turns
//             of 512 rows, whose first loads and last stores nothing hides
#include "cf_rows.h"
#include "cf_kernels.h"
#include "cf_train.h"

namespace cf {

namespace {

// Sums over the G lanes of a row.  Groups of up to a wave exchange registers;
// larger ones go through LDS, slot `buf` of `red`, with one barrier that every
// thread of the workgroup passes.  The slot may be used again after one more
// such barrier.
template <int G, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*red)[16][N], int buf) {
#pragma unroll
    for (int i = 0; i < N; i++)
        v[i] = lanes<Add, (G < 64 ? G : 64)>(v[i]);
    if constexpr (G > 64) {
        const int wave = threadIdx.x >> 6, w0 = wave / (G / 64) * (G / 64);
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; i++)
                red[buf][wave][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; i++) {
            float s = red[buf][w0][i];
#pragma unroll
            for (int k = 1; k < G / 64; k++)
                s += red[buf][w0 + k][i];
            v[i] = s;
        }
    }
}

// s / C, rounded like a division: with 1 / C alone the mean of a row of large
// equal values is off by a rounding that its spread of 0 does not hide.
__device__ __forceinline__ float mean_of(float s, float c, float inv_c) {
    const float m = s * inv_c;
    return fmaf(fmaf(-m, c, s), inv_c, m);
}

// Rows of more than 8 lanes hold a whole vector: the loads then need no way for
// shorter ones.
template <int G>
__device__ __forceinline__ void more_than_a_vector(int C) {
    if constexpr (G > 8)
        __builtin_assume(C > 8);
}

struct NormArgs {
    const uint16_t *x;
    uint16_t *y;
    const float *w, *b;
    float2 *stats;
    int8_t *q;
    float *scale;
    int64_t ldx, ldy, rows;
    int C, blocks;
    float eps;
};

// U rows a group: their loads are issued together.
template <typename T, int G, int V, int U>
__global__ __launch_bounds__(G > 256 ? G : 256) void norm_forward_kernel(NormArgs a) {
    constexpr int TH = G > 256 ? G : 256, NG = TH / G;
    __shared__ float red[2][16][U];
    more_than_a_vector<G>(a.C);
    const int grp = threadIdx.x / G, gl = threadIdx.x % G;
    const int64_t r0 = (int64_t)blockIdx.x * (NG * U) + grp;
    const float fc = (float)a.C, inv_c = 1.0f / fc;
    u32x4 raw[U][V];
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
        for (int v = 0; v < V; v++) {
            const int64_t r = r0 + u * NG;
            const int c = (gl + v * G) * 8;
            raw[u][v] = r < a.rows ? load8(a.x + r * a.ldx, c, a.C) : u32x4{0u, 0u, 0u, 0u};
        }
    float x[U][V * 8], s[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
        s[u] = 0.0f;
#pragma unroll
        for (int v = 0; v < V; v++) {
            unpack8<T>(raw[u][v], &x[u][8 * v]);
#pragma unroll
            for (int i = 0; i < 8; i++)
                s[u] += x[u][8 * v + i];
        }
    }
    if (a.q) {
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int v = 0; v < V; v++) {
                const int64_t r = r0 + u * NG;
                const int c = (gl + v * G) * 8;
                const Quant z = quant_of(lanes<Max, 8>(amax8(&x[u][8 * v])));
                if (r < a.rows && c < a.C) {
                    store8b(a.q + r * a.C, c, a.C, quant8(&x[u][8 * v], z.inv));
                    if ((threadIdx.x & 7) == 0)
                        a.scale[r * a.blocks + c / CKPT_BLOCK] = z.scale;
                }
            }
    }
    row_sums<G>(s, red, 0);
    float mean[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
        mean[u] = mean_of(s[u], fc, inv_c);
        s[u] = 0.0f;
#pragma unroll
        for (int v = 0; v < V; v++) {
            const int n = a.C - (gl + v * G) * 8;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                float &d = x[u][8 * v + i];
                d -= mean[u];
                s[u] = i < n ? fmaf(d, d, s[u]) : s[u];
            }
        }
    }
    row_sums<G>(s, red, 1);
    float rstd[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
        rstd[u] = 1.0f / sqrtf(fmaf(s[u], inv_c, a.eps));
        const int64_t r = r0 + u * NG;
        if (a.stats && gl == 0 && r < a.rows)
            a.stats[r] = make_float2(mean[u], rstd[u]);
    }
#pragma unroll
    for (int v = 0; v < V; v++) {
        const int c = (gl + v * G) * 8, n = a.C - c;
        float w[8], b[8];
        load8f(a.w ? a.w + c : nullptr, n, 1.0f, w);
        load8f(a.b ? a.b + c : nullptr, n, 0.0f, b);
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int64_t r = r0 + u * NG;
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; i++)
                y[i] = fmaf(x[u][8 * v + i] * rstd[u], w[i], b[i]);
            if (r < a.rows && n > 0)
                store8(a.y + r * a.ldy, c, a.C, pack8<T>(y));
        }
    }
}

struct NormBackArgs {
    const uint16_t *dy, *x;
    const int8_t *q;
    const float *scale;
    const float2 *stats;
    const float *w;
    uint16_t *dx;
    float *dw, *db;  // the gradients, or [workgroup][2][C] partial sums from dw on (db null)
    int64_t lddy, ldx, lddx, rows;
    int C, blocks;
};

// Threads of a workgroup of the backward kernel.  A workgroup's groups add
// their sums of dw and db before they are written: above 2048 channels, where
// those are many, one workgroup a CU writes half of what two would (norm and
// gradient of 2999 rows of 4095 41.9 -> 38.8 us, 560 of 2304 17.9 -> 15.7).
constexpr int back_threads(int G) { return G >= 512 ? 1024 : 512; }

constexpr int RED_BYTES = 2 * 16 * 2 * sizeof(float);

// CK: x from its checkpoint. Persistent: a group takes rows a grid apart, the
// next row's loads in flight while the current one is worked on (V = 1). The
// sums over rows stay in registers until the end and are added in a fixed
// order, within a workgroup through LDS, across workgroups by
// norm_reduce_kernel: no atomics, so the same input gives the same gradients,
// and one rounding of fp32 sums of a few rows each.
template <typename T, bool CK, int G, int V>
__global__ __launch_bounds__(back_threads(G), 4) void norm_backward_kernel(NormBackArgs a) {
    constexpr int TH = back_threads(G), NG = TH / G, WAVES = TH / 64;
    // the waves' sums of a row, then the weight while rows are worked on and
    // what the waves add up after that
    extern __shared__ float4 dynamic[];
    float(*const red)[16][2] = reinterpret_cast<float(*)[16][2]>(dynamic);
    float4 *const space = dynamic + RED_BYTES / 16;
    more_than_a_vector<G>(a.C);
    const int grp = threadIdx.x / G, gl = threadIdx.x % G, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float fc = (float)a.C, inv_c = 1.0f / fc;
    float w[8], dw[V * 8], db[V * 8];
#pragma unroll
    for (int v = 0; v < V; v++) {
        const int c = (gl + v * G) * 8;
        load8f(a.w ? a.w + c : nullptr, a.C - c, 1.0f, w);
        if (V > 1 && grp == 0) {
            space[(2 * v) * G + gl] = make_float4(w[0], w[1], w[2], w[3]);
            space[(2 * v + 1) * G + gl] = make_float4(w[4], w[5], w[6], w[7]);
        }
#pragma unroll
        for (int i = 0; i < 8; i++)
            dw[8 * v + i] = db[8 * v + i] = 0.0f;
    }
    if (V > 1)
        __syncthreads();
    // the weight of a lane's vector: from its registers, or (two vectors) from
    // LDS, as the registers hold the sums of both
    auto weight = [&](int v, float *f) {
        if constexpr (V > 1) {
            const float4 lo = space[(2 * v) * G + gl], hi = space[(2 * v + 1) * G + gl];
            f[0] = lo.x, f[1] = lo.y, f[2] = lo.z, f[3] = lo.w;
            f[4] = hi.x, f[5] = hi.y, f[6] = hi.z, f[7] = hi.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                f[i] = w[i];
        }
    };
    struct Row {
        u32x4 dy[V], x[V];
        float scale[V];
        float2 st;
    };
    auto fetch = [&](int64_t r) {
        // Past C dy is 0, but x is another of the row's values (a lane with
        // nothing of the row: its mean is 0): (0 - mean) * rstd may be infinite where
        // no channel's is, and 0 times that would make the row's sum NaN.
        Row t;
        t.st = make_float2(0.0f, 0.0f);
        if (r < a.rows && gl * 8 < a.C)
            t.st = a.stats[r];
#pragma unroll
        for (int v = 0; v < V; v++) {
            const int c = (gl + v * G) * 8;
            t.dy[v] = u32x4{0u, 0u, 0u, 0u};
            t.x[v] = v ? t.x[0] : u32x4{0u, 0u, 0u, 0u};
            t.scale[v] = v ? t.scale[0] : 0.0f;
            if (r < a.rows && c < a.C) {
                t.dy[v] = load8(a.dy + r * a.lddy, c, a.C);
                if constexpr (CK) {
                    const u32x2 q = load8b<true>(a.q + r * a.C, c, a.C);
                    t.x[v].x = q.x;
                    t.x[v].y = q.y;
                    t.scale[v] = a.scale[r * a.blocks + c / CKPT_BLOCK];
                } else {
                    t.x[v] = load8<true>(a.x + r * a.ldx, c, a.C);
                }
            }
        }
        return t;
    };
    const int64_t step = (int64_t)gridDim.x * NG;
    int64_t base = (int64_t)blockIdx.x * NG;
    // two vectors a lane leave no registers for the next row: norm and gradient
    // of 4096 rows of 16384 fp16 173 us with it, 163 without, from the checkpoint
    // 208 and 170
    Row next;
    if constexpr (V == 1)
        next = fetch(base + grp);
    for (int it = 0; base < a.rows; base += step, it ^= 1) {
        const int64_t r = base + grp;
        if constexpr (V > 1)
            next = fetch(r);
        const Row t = next;
        if constexpr (V == 1)
            next = fetch(r + step);
        // the row's values, from the registers they were loaded into: held as
        // 16 (or 8) bits and converted again after the sums, they leave room
        // for the next row
        auto values = [&](int v, float *dy, float *x) {
            unpack8<T>(t.dy[v], dy);
            if constexpr (CK)
                dequant8(u32x2{t.x[v].x, t.x[v].y}, t.scale[v], x);
            else
                unpack8<T>(t.x[v], x);
        };
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < V; v++) {
            float dy[8], x[8], f[8];
            values(v, dy, x);
            weight(v, f);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const int j = 8 * v + i;
                const float xh = (x[i] - t.st.x) * t.st.y, g = dy[i] * f[i];
                dw[j] = fmaf(dy[i], xh, dw[j]);
                db[j] += dy[i];
                s[0] += g;
                s[1] = fmaf(g, xh, s[1]);
            }
        }
        row_sums<G>(s, red, it);
        const float m0 = mean_of(s[0], fc, inv_c), m1 = mean_of(s[1], fc, inv_c);
#pragma unroll
        for (int v = 0; v < V; v++) {
            const int c = (gl + v * G) * 8;
            float dy[8], x[8], dx[8], f[8];
            values(v, dy, x);
            weight(v, f);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float xh = (x[i] - t.st.x) * t.st.y;
                dx[i] = t.st.y * (fmaf(dy[i], f[i], -m0) - xh * m1);
            }
            if (r < a.rows && c < a.C)
                store8(a.dx + r * a.lddx, c, a.C, pack8<T>(dx));
        }
    }
    if (!a.dw)
        return;
    // Lanes of a wave that hold the same channels, then the waves through LDS.
    float *const pw = a.db ? a.dw : a.dw + (int64_t)blockIdx.x * 2 * a.C;
    float *const pb = a.db ? a.db : pw + a.C;
    float4(*const part)[WAVES][64] = reinterpret_cast<float4(*)[WAVES][64]>(space);  // [dw, db][4 channels]
    constexpr int SUB = G > 64 ? G / 64 : 1;                                         // waves that share a row
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; k++)
#pragma unroll
        for (int j = 0; j < V * 2; j++) {
            float4 t;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                float f = k ? db[4 * j + i] : dw[4 * j + i];
                if constexpr (G <= 8)
                    f += dpp<0x128>(f);  // 8 lanes further in the row of 16
                if constexpr (G <= 16) {
                    const Two h = swap16(f);
                    f = h.a + h.b;
                }
                if constexpr (G <= 32) {
                    const Two h = swap32(f);
                    f = h.a + h.b;
                }
                (&t.x)[i] = f;
            }
            part[k * V * 2 + j][wave][lane] = t;
        }
    __syncthreads();
    constexpr int LANES = G < 64 ? G : 64, OUT = 4 * V * SUB * LANES;
    for (int o = threadIdx.x; o < OUT; o += TH) {
        const int l = o % LANES, sub = o / LANES % SUB, kj = o / (LANES * SUB), j = kj % (2 * V);
        float4 f = part[kj][sub][l];
        for (int n = 1; n < WAVES / SUB; n++) {
            const float4 g = part[kj][n * SUB + sub][l];
            f.x += g.x, f.y += g.y, f.z += g.z, f.w += g.w;
        }
        const int c = (sub * 64 + l + j / 2 * G) * 8 + (j & 1) * 4;
        float *const to = (kj < 2 * V ? pw : pb) + c;
        if (c + 4 <= a.C) {
            reinterpret_cast<AnyF4 *>(to)->v = float4v{f.x, f.y, f.z, f.w};
        } else {
#pragma unroll
            for (int i = 0; i < 3; i++)
                if (c + i < a.C)
                    to[i] = (&f.x)[i];
        }
    }
}

// Sum of `n` partials [n][2][C] into dw [C] and db [C]: 32 columns a
// workgroup (a cache line), 32 threads share a column and add every 32nd
// partial, eight loads at a time.  512 partials of 64 channels 4.7 us, 256 of
// 4095 (8.4 MB) 4.0 us: little more than a launch and two loads one after the
// other.
__global__ __launch_bounds__(1024) void norm_reduce_kernel(const float *part, float *dw, float *db, int n, int C) {
    __shared__ float s[32][33];
    const int col = threadIdx.x & 31, at = threadIdx.x >> 5;
    const int64_t i = (int64_t)blockIdx.x * 32 + col, pitch = 2 * (int64_t)C;
    float f = 0.0f;
    if (i < pitch) {
        int k = at;
        for (; k + 7 * 32 < n; k += 8 * 32) {
            float t[8];
#pragma unroll
            for (int u = 0; u < 8; u++)
                t[u] = part[(k + u * 32) * pitch + i];
            f += ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
        }
        for (; k < n; k += 32)
            f += part[k * pitch + i];
    }
    s[at][col] = f;
    __syncthreads();
    f = lanes<Add, 32>(s[col][at]);  // transposed: 32 lanes hold one column
    const int64_t o = (int64_t)blockIdx.x * 32 + at;
    if (col == 0 && o < pitch)
        (o < C ? dw[o] : db[o - C]) = f;
}

// Lanes and vectors of a row of C channels: one vector a lane where a workgroup
// can hold the row.  In the backward pass two (for which the registers do not
// suffice: some of them go to memory) take longer, norm and gradient of 25088
// rows of 1024 73 us against 58, of 2000 of 8192 51 against 41, of 37 of 986 14
// against 10.4.
#define CF_NORM_SHAPES(F)                                                                                              \
    if (C <= 64) return F(8, 1);                                                                                       \
    if (C <= 128) return F(16, 1);                                                                                     \
    if (C <= 256) return F(32, 1);                                                                                     \
    if (C <= 512) return F(64, 1);                                                                                     \
    if (C <= 1024) return F(128, 1);                                                                                   \
    if (C <= 2048) return F(256, 1);                                                                                   \
    if (C <= 4096) return F(512, 1);                                                                                   \
    if (C <= 8192) return F(1024, 1);                                                                                  \
    return F(1024, 2);

// U rows a group; false where that leaves fewer than `least` waves.
template <typename T, int G, int V, int U>
bool forward_rows(const NormArgs &a, int64_t least, hipStream_t st) {
    constexpr int TH = G > 256 ? G : 256, ROWS = TH / G * U;
    const int64_t grid = (a.rows + ROWS - 1) / ROWS;
    if (grid * (TH / 64) < least)
        return false;
    norm_forward_kernel<T, G, V, U><<<dim3((unsigned)grid), dim3(TH), 0, st>>>(a);
    return true;
}

template <typename T, int G, int V>
hipError_t forward_shape(const NormArgs &a, hipStream_t st) {
    // Four vectors a lane where that leaves 16 waves a CU: four rows, or
    // of rows above 512 channels two in half the lanes (2999 rows of 4095 with
    // one row 15.3 us, with four in all the lanes 15.9, with two in half 13.5).
    // Fewer rows take one at a time: 25088 of 256 7.6 us (with four 8.8), 512 of
    // 768 3.7 us a call (with two vectors a lane 4.0).
    constexpr int HALF = V == 1 && G > 64 ? G / 2 : G, VECS = V == 2 || G > 64 ? 2 : 1;
    if (!forward_rows<T, HALF, VECS, 4 / VECS>(a, 16 * (int64_t)device_cu_count(), st))
        forward_rows<T, G, V, 1>(a, 0, st);
    return hipGetLastError();
}

template <typename T>
hipError_t forward_type(const NormArgs &a, hipStream_t st) {
    const int C = a.C;
#define F(G, V) (forward_shape<T, G, V>(a, st))
    CF_NORM_SHAPES(F)
#undef F
}

// Workgroups of the backward pass: as many as run at once; and the groups of
// one.
int back_groups_of(int C) {
#define F(G, V) (back_threads(G) / G)
    CF_NORM_SHAPES(F)
#undef F
}
int64_t back_grid(int64_t rows, int C) {
    const int64_t ng = back_groups_of(C), need = (rows + ng - 1) / ng;
    const int64_t most = (int64_t)device_cu_count() * (C <= 2048 ? 2 : 1);  // 16 waves a CU
    return need <= 2 ? 1 : need < most ? need : most;  // two turns of one workgroup, and no second launch
}

int lanes_of(int C) {
#define F(G, V) (G)
    CF_NORM_SHAPES(F)
#undef F
}

template <typename T, bool CK, int G, int V>
hipError_t backward_shape(const NormBackArgs &a, unsigned grid, hipStream_t st) {
    constexpr int SUMS = back_threads(G) * V * 64, WEIGHT = V > 1 ? G * V * 32 : 0;
    constexpr int LDS = RED_BYTES + (SUMS > WEIGHT ? SUMS : WEIGHT);
    if (LDS > 64 * 1024) {
        const hipError_t e = allow_full_lds((const void *)norm_backward_kernel<T, CK, G, V>);
        if (e != hipSuccess)
            return e;
    }
    norm_backward_kernel<T, CK, G, V><<<dim3(grid), dim3(back_threads(G)), LDS, st>>>(a);
    return hipGetLastError();
}

template <typename T, bool CK>
hipError_t backward_type(const NormBackArgs &a, unsigned grid, hipStream_t st) {
    const int C = a.C;
#define F(G, V) (backward_shape<T, CK, G, V>(a, grid, st))
    CF_NORM_SHAPES(F)
#undef F
}

}  // namespace

// The forward grid stays below 2^32 threads.
bool norm_fits(int64_t rows, int C) { return C <= NORM_MAX_C && ((double)rows + 256) * lanes_of(C) < 4294967296.0; }

hipError_t launch_norm_forward(const void *x, int64_t ldx, void *y, int64_t ldy, const float *weight,
                               const float *bias, float *stats, const Ckpt &ckpt, int64_t rows, int C, float eps,
                               int bf16, hipStream_t st) {
    NormArgs a;
    a.x = (const uint16_t *)x;
    a.y = (uint16_t *)y;
    a.w = weight;
    a.b = bias;
    a.stats = (float2 *)stats;
    a.q = ckpt.q;
    a.scale = ckpt.scale;
    a.ldx = ldx;
    a.ldy = ldy;
    a.rows = rows;
    a.C = C;
    a.blocks = blocks_of(C);
    a.eps = eps;
    return bf16 ? forward_type<BF16>(a, st) : forward_type<F16>(a, st);
}

size_t norm_backward_workspace_bytes(int64_t rows, int C) {
    const int64_t grid = back_grid(rows, C);
    return grid > 1 ? (size_t)grid * 2 * C * sizeof(float) : 0;
}

hipError_t launch_norm_backward(const NormBackward &n, int64_t rows, int C, int bf16, void *ws, hipStream_t st) {
    const unsigned grid = (unsigned)back_grid(rows, C);
    NormBackArgs a;
    a.dy = (const uint16_t *)n.dy;
    a.x = (const uint16_t *)n.x;
    a.q = n.ckpt.q;
    a.scale = n.ckpt.scale;
    a.stats = (const float2 *)n.stats;
    a.w = n.weight;
    a.dx = (uint16_t *)n.dx;
    a.dw = !n.dweight || grid == 1 ? n.dweight : (float *)ws;
    a.db = grid == 1 ? n.dbias : nullptr;
    a.lddy = n.lddy;
    a.ldx = n.ldx;
    a.lddx = n.lddx;
    a.rows = rows;
    a.C = C;
    a.blocks = blocks_of(C);
    hipError_t e;
    if (n.ckpt.q)
        e = bf16 ? backward_type<BF16, true>(a, grid, st) : backward_type<F16, true>(a, grid, st);
    else
        e = bf16 ? backward_type<BF16, false>(a, grid, st) : backward_type<F16, false>(a, grid, st);
    if (e != hipSuccess || !n.dweight || grid == 1)
        return e;
    norm_reduce_kernel<<<dim3((2 * C + 31) / 32), dim3(1024), 0, st>>>((const float *)ws, n.dweight, n.dbias,
                                                                       (int)grid, C);
    return hipGetLastError();
}

}  // namespace cf
