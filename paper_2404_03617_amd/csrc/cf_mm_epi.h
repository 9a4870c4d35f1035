// cf_mm_epi.h -- what follows a product of cf_mm.h, on the sums that a lane
// holds: for the wave's 16 x 16 tiles (i, j), row m = m0 + 16 i + lane % 16 and
// columns n0 + 16 j + 4 (lane / 16) ... + 3.
#pragma once

#include "cf_act.h"
#include "cf_mm.h"

namespace cf {
namespace mm {

struct __attribute__((packed, aligned(2))) Any8 {
    u32x2 v;
};
struct __attribute__((packed, aligned(4))) Any16f {
    float4v v;
};

// four values from p on, `left` of which are in the row
template <typename T>
__device__ __forceinline__ void store4(uint16_t *p, const float4v &v, int left) {
    const u32x2 w = {T::pack2(v[0], v[1]), T::pack2(v[2], v[3])};
    if (left >= 4) {
        reinterpret_cast<Any8 *>(p)->v = w;
    } else {
#pragma unroll
        for (int i = 0; i < 3; i++)
            if (i < left)
                p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
}
__device__ __forceinline__ void store4f(float *p, const float4v &v, int left) {
    if (left >= 4) {
        reinterpret_cast<Any16f *>(p)->v = v;
    } else {
#pragma unroll
        for (int i = 0; i < 3; i++)
            if (i < left)
                p[i] = v[i];
    }
}
__device__ __forceinline__ float4v load4f(const float *p, int left) {
    if (left >= 4)
        return reinterpret_cast<const Any16f *>(p)->v;
    float4v v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 3; i++)
        if (i < left)
            v[i] = p[i];
    return v;
}

// --- the product itself, rounded once -------------------------------------
struct StoreArgs {
    uint16_t *out[2];
    int64_t ldo;
    const float *row_scale;  // [M], or null
    const float *scale;      // one number, or null
    float *acc;              // [M][N] running sums of several products
    int acc_in, acc_out;     // whether to add them, and to leave them there instead of a result
    float *part;             // [splits][batch][M][N] for split sums
};

template <typename T>
__device__ __forceinline__ void finish4(const StoreArgs &e, float4v v, int m, int n, int M, int N, int batch) {
    const int left = N - n;
    float *const acc = e.acc + (e.acc ? (int64_t)m * N + n : 0);
    if (e.acc_in)
        v += load4f(acc, left);
    if (e.acc_out) {
        store4f(acc, v, left);
        return;
    }
    if (e.row_scale)
        v *= e.row_scale[m];
    if (e.scale)
        v *= *e.scale;
    store4<T>(e.out[batch] + (int64_t)m * e.ldo + n, v, left);
}

struct Store {
    static constexpr bool DUAL = false;
    using Args = StoreArgs;
    template <typename T, typename S>
    static __device__ __forceinline__ void run(const StoreArgs &e, float4v (&acc)[S::FM][S::FN], const Work &at,
                                               const mm::Args &a, int m0, int n0, int lane, uint8_t *) {
        float *const part = a.splits > 1 ? e.part + ((int64_t)at.split * a.batch + at.batch) * a.M * a.N : nullptr;
#pragma unroll
        for (int i = 0; i < S::FM; i++) {
            const int m = m0 + 16 * i + (lane & 15);
            if (m >= a.M)
                continue;
#pragma unroll
            for (int j = 0; j < S::FN; j++) {
                const int n = n0 + 16 * j + 4 * (lane >> 4);
                if (n >= a.N)
                    continue;
                if (part)
                    store4f(part + (int64_t)m * a.N + n, acc[i][j], a.N - n);
                else
                    finish4<T>(e, acc[i][j], m, n, a.M, a.N, at.batch);
            }
        }
    }
};

// --- gate and up channels: h = act(g) u ------------------------------------
// The tile's groups of 16 columns are of the gate and of the up projection in
// turn.  h has `pad` columns, those past H zero; g and u are kept in fp32 for the
// backward pass where it is wanted (16 bits there would add two roundings to
// each gradient).
struct GatedArgs {
    uint16_t *h;
    int64_t ldh;
    float *saved;  // [M][2 H], g then u, or null
    int H, pad, act;
};

struct Gated {
    static constexpr bool DUAL = true;
    using Args = GatedArgs;
    template <typename T, typename S>
    static __device__ __forceinline__ void run(const GatedArgs &e, float4v (&acc)[S::FM][S::FN], const Work &,
                                               const mm::Args &a, int m0, int n0, int lane, uint8_t *) {
        with_act(e.act, [&](auto tag) {
            constexpr int ACT = decltype(tag)::value;
#pragma unroll
            for (int i = 0; i < S::FM; i++) {
                const int m = m0 + 16 * i + (lane & 15);
                if (m >= a.M)
                    continue;
#pragma unroll
                for (int j = 0; j < S::FN; j += 2) {
                    const int n = n0 / 2 + 8 * j + 4 * (lane >> 4);
                    if (n >= e.pad)
                        continue;
                    const int left = e.H - n;
                    float4v h;
#pragma unroll
                    for (int k = 0; k < 4; k++)
                        h[k] = k < left ? act_pair<ACT>(acc[i][j][k]).f * acc[i][j + 1][k] : 0.0f;
                    store4<T>(e.h + m * e.ldh + n, h, e.pad - n);
                    if (e.saved && left > 0) {
                        float *const s = e.saved + (int64_t)m * 2 * e.H + n;
                        store4f(s, acc[i][j], left);
                        store4f(s + e.H, acc[i][j + 1], left);
                    }
                }
            }
        });
    }
};

// --- their gradients from dh: dg = dh u act'(g), du = dh act(g), and h again ---
struct GatedBackArgs {
    const float *saved;
    uint16_t *d;  // [M][2 pad]: dg, du
    uint16_t *h;  // [M][pad]
    int H, pad, act;
};

struct GatedBack {
    static constexpr bool DUAL = false;
    using Args = GatedBackArgs;
    template <typename T, typename S>
    static __device__ __forceinline__ void run(const GatedBackArgs &e, float4v (&acc)[S::FM][S::FN], const Work &,
                                               const mm::Args &a, int m0, int n0, int lane, uint8_t *) {
        with_act(e.act, [&](auto tag) {
            constexpr int ACT = decltype(tag)::value;
#pragma unroll
            for (int i = 0; i < S::FM; i++) {
                const int m = m0 + 16 * i + (lane & 15);
                if (m >= a.M)
                    continue;
#pragma unroll
                for (int j = 0; j < S::FN; j++) {
                    const int n = n0 + 16 * j + 4 * (lane >> 4), left = e.H - n;
                    if (n >= e.pad)
                        continue;
                    const float *const s = e.saved + (int64_t)m * 2 * e.H + n;
                    const float4v g = load4f(s, left), u = load4f(s + e.H, left);
                    float4v dg, du, h;
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        const ActPair p = act_pair<ACT>(g[k]);
                        const float dh = acc[i][j][k];
                        dg[k] = k < left ? dh * u[k] * p.d : 0.0f;
                        du[k] = k < left ? dh * p.f : 0.0f;
                        h[k] = k < left ? p.f * u[k] : 0.0f;
                    }
                    uint16_t *const d = e.d + (int64_t)m * 2 * e.pad + n;
                    store4<T>(d, dg, e.pad - n);
                    store4<T>(d + e.pad, du, e.pad - n);
                    store4<T>(e.h + (int64_t)m * e.pad + n, h, e.pad - n);
                }
            }
        });
    }
};

// --- logits: largest and sum of exp(z - largest) of each row in the tile -------
struct LseArgs {
    float2 *part;  // [tiles_n][M]
    float *picked;  // [M]: the logit of the row's token
    const int64_t *tokens;  // or null
};

constexpr float LOG2E = 1.44269504088896f;

__device__ __forceinline__ float2 join_lse(float2 a, float2 b) {
    const float m = fmaxf(a.x, b.x), base = m == -INFINITY ? 0.0f : m;
    return make_float2(m, a.y * __builtin_amdgcn_exp2f((a.x - base) * LOG2E) +
                              b.y * __builtin_amdgcn_exp2f((b.x - base) * LOG2E));
}

struct Lse {
    static constexpr bool DUAL = false;
    using Args = LseArgs;
    template <typename T, typename S>
    static __device__ __forceinline__ void run(const LseArgs &e, float4v (&acc)[S::FM][S::FN], const Work &at,
                                               const mm::Args &a, int m0, int n0, int lane, uint8_t *lds) {
        float2 *const row = reinterpret_cast<float2 *>(lds);  // [WN][TM]
        const int wn = n0 % S::TN / (S::TN / S::WN), local = m0 % S::TM;
#pragma unroll
        for (int i = 0; i < S::FM; i++) {
            const int m = m0 + 16 * i + (lane & 15);
            const int64_t want = e.tokens && m < a.M ? e.tokens[m] : -1;
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < S::FN; j++) {
                const int n = n0 + 16 * j + 4 * (lane >> 4);
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    if (n + k >= a.N)
                        acc[i][j][k] = -INFINITY;
                    else if (n + k == want)
                        e.picked[m] = acc[i][j][k];
                    top = fmaxf(top, acc[i][j][k]);
                }
            }
            const float base = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < S::FN; j++)
#pragma unroll
                for (int k = 0; k < 4; k++)
                    sum += __builtin_amdgcn_exp2f((acc[i][j][k] - base) * LOG2E);
            float2 r = make_float2(top, sum);
            r = join_lse(r, make_float2(__shfl_xor(r.x, 16), __shfl_xor(r.y, 16)));
            r = join_lse(r, make_float2(__shfl_xor(r.x, 32), __shfl_xor(r.y, 32)));
            if (lane < 16)
                row[wn * S::TM + local + 16 * i + lane] = r;
        }
        __syncthreads();
        for (int t = threadIdx.x; t < S::TM; t += S::TH) {
            float2 r = row[t];
#pragma unroll
            for (int w = 1; w < S::WN; w++)
                r = join_lse(r, row[w * S::TM + t]);
            const int m = at.m * S::TM + t;
            if (m < a.M)
                e.part[(int64_t)at.n * a.M + m] = r;
        }
    }
};

// --- logits again: their gradients, c p + g 1[token], times a power of two ----
struct RowGrad {
    float c, g, lse;  // all 0 (and what multiplies them skipped) for a row without a gradient
    int token;
};
struct DzArgs {
    const RowGrad *rows;
    uint16_t *dz;  // [M][pad]
    int pad, v0;   // the piece's first token
};

struct Dz {
    static constexpr bool DUAL = false;
    using Args = DzArgs;
    template <typename T, typename S>
    static __device__ __forceinline__ void run(const DzArgs &e, float4v (&acc)[S::FM][S::FN], const Work &,
                                               const mm::Args &a, int m0, int n0, int lane, uint8_t *) {
#pragma unroll
        for (int i = 0; i < S::FM; i++) {
            const int m = m0 + 16 * i + (lane & 15);
            if (m >= a.M)
                continue;
            const RowGrad r = e.rows[m];
            const int want = r.token - e.v0;
            const bool any = !(r.c == 0.0f && r.g == 0.0f);
#pragma unroll
            for (int j = 0; j < S::FN; j++) {
                const int n = n0 + 16 * j + 4 * (lane >> 4);
                if (n >= e.pad)
                    continue;
                float4v d;
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const float p = __builtin_amdgcn_exp2f((acc[i][j][k] - r.lse) * LOG2E);
                    d[k] = any && n + k < a.N ? fmaf(r.c, p, n + k == want ? r.g : 0.0f) : 0.0f;
                }
                store4<T>(e.dz + (int64_t)m * e.pad + n, d, e.pad - n);
            }
        }
    }
};

}  // namespace mm
}  // namespace cf
