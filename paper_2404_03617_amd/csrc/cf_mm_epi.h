// cf_mm_epi.h -- what follows a product of cf_mm.h, on the sums that a lane
// holds (Results): rows m0 + 16 i + lane % 16, columns from n0 on.
#pragma once

#include "cf_act.h"
#include "cf_mm.h"
#include "cf_rows.h"

namespace cf {
namespace mm {

struct __attribute__((packed, aligned(4))) Any16f {
    float4v v;
};
struct __attribute__((packed, aligned(2))) Any8h {
    u32x2 v;
};

// N values (4, or a multiple of 8) from p on, `left` of which are in the row
template <typename T, int N, typename V>
__device__ __forceinline__ void store_row(uint16_t *p, const V &v, int left) {
    if constexpr (N == 4) {
        const u32x2 w = {T::pack2(v[0], v[1]), T::pack2(v[2], v[3])};
        if (left >= 4) {
            reinterpret_cast<Any8h *>(p)->v = w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (i < left)
                    p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        }
        return;
    }
#pragma unroll
    for (int c = 0; c + 8 <= N; c += 8) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; i++)
            w[i] = T::pack2(v[c + 2 * i], v[c + 2 * i + 1]);
        if (left >= c + 8) {
            reinterpret_cast<Any16 *>(p + c)->v = w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (c + i < left)
                    p[c + i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        }
    }
}
template <int N, typename V>
__device__ __forceinline__ void store_rowf(float *p, const V &v, int left) {
#pragma unroll
    for (int c = 0; c < N; c += 4) {
        if (left >= c + 4) {
            reinterpret_cast<Any16f *>(p + c)->v = float4v{v[c], v[c + 1], v[c + 2], v[c + 3]};
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (c + i < left)
                    p[c + i] = v[c + i];
        }
    }
}
template <int N, typename V>
__device__ __forceinline__ void load_rowf(const float *p, V &v, int left) {
#pragma unroll
    for (int c = 0; c < N; c += 4) {
        float4v w = {0.0f, 0.0f, 0.0f, 0.0f};
        if (left >= c + 4) {
            w = reinterpret_cast<const Any16f *>(p + c)->v;
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (c + i < left)
                    w[i] = p[c + i];
        }
#pragma unroll
        for (int i = 0; i < 4; i++)
            v[c + i] = w[i];
    }
}

// 8 values from p on, and with LO what rounding took from them `lo` elements further
// on: where there are few rows, one rounding counts, and a product of twice the
// rows costs nothing.
template <typename T, bool LO>
__device__ __forceinline__ void store_parts(uint16_t *p, int64_t lo, const float (&v)[8]) {
    const u32x4 r = pack8<T>(v);
    reinterpret_cast<Any16 *>(p)->v = r;
    if constexpr (LO) {
        float f[8];
        unpack8<T>(r, f);
#pragma unroll
        for (int k = 0; k < 8; k++)
            f[k] = fabsf(f[k]) < INFINITY ? v[k] - f[k] : 0.0f;
        reinterpret_cast<Any16 *>(p + lo)->v = pack8<T>(f);
    }
}

// --- the product itself, rounded once -------------------------------------
struct StoreArgs {
    uint16_t *out[2];
    int64_t ldo;
    const float *row_scale;  // [M], or null
    const float *scale;      // one number, or null
    float *acc;              // [M][N] running sums of several products
    int acc_in, acc_out;     // whether to add them, and to leave them there instead of a result
    float *part;             // [splits][batch][M][N] for sums that a launch of their own joins, or null
    int fold;                // there: the rows of the result, each the sum of rows m and m + fold; 0: of one each
};

// N sums of row m from column n on
template <typename T, int N, typename V>
__device__ __forceinline__ void finish(const StoreArgs &e, V &v, int m, int n, int M, int cols, int batch) {
    const int left = cols - n;
    float *const acc = e.acc + (e.acc ? (int64_t)m * cols + n : 0);
    if (e.acc_in) {
        float more[N];
        load_rowf<N>(acc, more, left);
#pragma unroll
        for (int i = 0; i < N; i++)
            v[i] += more[i];
    }
    if (e.acc_out) {
        store_rowf<N>(acc, v, left);
        return;
    }
    if (e.row_scale || e.scale) {
        const float f = (e.row_scale ? e.row_scale[m] : 1.0f) * (e.scale ? *e.scale : 1.0f);
#pragma unroll
        for (int i = 0; i < N; i++)
            v[i] *= f;
    }
    store_row<T, N>(e.out[batch] + (int64_t)m * e.ldo + n, v, left);
}

struct Store {
    static constexpr bool DUAL = false;
    template <typename S>
    static constexpr int lds_bytes() {
        return 0;
    }
    using Args = StoreArgs;
    template <typename T, typename S, bool G>
    static __device__ __forceinline__ void run(const StoreArgs &e, const Results<S, G> &t, const Work &at,
                                               const mm::Args &a, int m0, int n0, int lane, uint8_t *) {
        constexpr int W = Results<S, G>::W, PIECES = Results<S, G>::PIECES;
        float *const part = e.part ? e.part + ((int64_t)at.split * a.batch + at.batch) * a.M * a.N : nullptr;
#pragma unroll
        for (int i = 0; i < S::FM; i++) {
            const int m = m0 + 16 * i + (lane & 15);
            if (m >= a.M)
                continue;
#pragma unroll
            for (int p = 0; p < PIECES; p++) {
                const int n = n0 + t.column(p, lane);
                if (n >= a.N)
                    continue;
                float v[W];
#pragma unroll
                for (int k = 0; k < W; k++)
                    v[k] = t.get(i, p, k);
                if (part)
                    store_rowf<W>(part + (int64_t)m * a.N + n, v, a.N - n);
                else
                    finish<T, W>(e, v, m, n, a.M, a.N, at.batch);
            }
        }
    }
};

// --- gate and up channels: h = act(g) u ------------------------------------
// The tile's groups of 32 columns are of the gate and of the up projection in
// turn.  h has `pad` columns, those past H zero; g and u are kept in fp32 for the
// backward pass where it is wanted (16 bits there would add two roundings to
// each gradient).
struct GatedArgs {
    uint16_t *h;
    int64_t ldh, lo;  // lo: to what rounding h takes (few rows, cf_few.h)
    float *saved;  // [M][2 H], g then u, or null
    int H, pad, act;
};

struct Gated {
    static constexpr bool DUAL = true;
    template <typename S>
    static constexpr int lds_bytes() {
        return 0;
    }
    using Args = GatedArgs;
    // 8 channels of row m from n on; ends: H may be among them
    template <typename T, int ACT>
    static __device__ __forceinline__ void piece(const GatedArgs &e, const float (&g)[8], const float (&u)[8], int m, int n,
                                                 bool ends) {
        const int left = e.H - n;
        float h[8];
#pragma unroll
        for (int k = 0; k < 8; k++)
            h[k] = act_value<ACT>(g[k]) * u[k];
        if (ends)
#pragma unroll
            for (int k = 0; k < 8; k++)
                h[k] = k < left ? h[k] : 0.0f;
        store_parts<T, false>(e.h + m * e.ldh + n, 0, h);
        if (e.saved) {
            float *const s = e.saved + (int64_t)m * 2 * e.H + n;
            store_rowf<8>(s, g, left);
            store_rowf<8>(s + e.H, u, left);
        }
    }
    template <typename T, typename S, bool G>
    static __device__ __forceinline__ void run(const GatedArgs &e, const Results<S, G> &t, const Work &,
                                               const mm::Args &a, int m0, int n0, int lane, uint8_t *) {
        constexpr int PIECES = Results<S, G>::PIECES;
        with_act(e.act, [&](auto tag) {
#pragma unroll
            for (int i = 0; i < S::FM; i++) {
                const int m = m0 + 16 * i + (lane & 15);
                if (m >= a.M)
                    continue;
#pragma unroll
                for (int p = 0; p < PIECES; p += 2) {
                    const int n = n0 / 2 + t.column(p / 2, lane);
                    if (n >= e.pad)
                        continue;
                    float g[8], u[8];
#pragma unroll
                    for (int k = 0; k < 8; k++) {
                        g[k] = t.get(i, p, k);
                        u[k] = t.get(i, p + 1, k);
                    }
                    piece<T, decltype(tag)::value>(e, g, u, m, n, n0 / 2 + 8 * S::FN > e.H);
                }
            }
        });
    }
};

// --- their gradients from dh: dg = dh u act'(g), du = dh act(g), and h again ---
// 14 bytes a result pass here, which bound the launch where k is short: 25088 x 1024
// x 256 in 93 us, 3.9 TB/s (143 with stores of 4 columns a lane and without a read
// ahead, in large tiles).
struct GatedBackArgs {
    const float *saved;
    uint16_t *d;  // [M][2 ld]: dg, du
    uint16_t *h;  // [M][ld]
    int64_t ld, lo;  // lo: to what rounding h takes (d: twice that), or 0
    int H, pad, act;
};

struct GatedBack {
    static constexpr bool DUAL = false;
    template <typename S>
    static constexpr int lds_bytes() {
        return 0;
    }
    using Args = GatedBackArgs;
    static __device__ __forceinline__ void read(const GatedBackArgs &e, int m, int n, int left, float (&g)[8],
                                                float (&u)[8]) {
        const float *const s = e.saved + (int64_t)m * 2 * e.H + n;
        load_rowf<8>(s, g, left);
        load_rowf<8>(s + e.H, u, left);
    }
    template <typename T, int ACT, bool LO = false>
    static __device__ __forceinline__ void piece(const GatedBackArgs &e, const float (&dh)[8], const float (&g)[8],
                                                 const float (&u)[8], int m, int n) {
        const int left = e.H - n;
        float dg[8], du[8], h[8];
#pragma unroll
        for (int k = 0; k < 8; k++) {
            const ActPair q = act_pair<ACT>(g[k]);
            dg[k] = k < left ? dh[k] * u[k] * q.d : 0.0f;
            du[k] = k < left ? dh[k] * q.f : 0.0f;
            h[k] = k < left ? q.f * u[k] : 0.0f;
        }
        uint16_t *const d = e.d + m * 2 * e.ld + n;
        store_parts<T, LO>(d, 2 * e.lo, dg);
        store_parts<T, LO>(d + e.ld, 2 * e.lo, du);
        store_parts<T, LO>(e.h + m * e.ld + n, e.lo, h);
    }
    template <typename T, typename S, bool G>
    static __device__ __forceinline__ void run(const GatedBackArgs &e, const Results<S, G> &t, const Work &,
                                               const mm::Args &a, int m0, int n0, int lane, uint8_t *) {
        constexpr int PIECES = Results<S, G>::PIECES;
        with_act(e.act, [&](auto tag) {
            constexpr int COUNT = S::FM * PIECES;
            float g[2][8], u[2][8];
            // piece j of the wave's, whose g and u are read while the one before is worked on, but
            // for large tiles, whose registers spill then (8192 x 4096 x 1024 175 us, ahead 183)
            constexpr bool AHEAD = S::TM < 256;
            auto ask = [&](int j) {
                const int m = m0 + 16 * (j / PIECES) + (lane & 15), n = n0 + t.column(j % PIECES, lane);
                read(e, m, n, m < a.M ? e.H - n : 0, g[j % 2], u[j % 2]);
            };
            if (AHEAD)
                ask(0);
#pragma unroll
            for (int j = 0; j < COUNT; j++) {
                if (!AHEAD)
                    ask(j);
                else if (j + 1 < COUNT)
                    ask(j + 1);
                const int m = m0 + 16 * (j / PIECES) + (lane & 15), n = n0 + t.column(j % PIECES, lane);
                if (m >= a.M || n >= e.pad)
                    continue;
                float dh[8];
#pragma unroll
                for (int k = 0; k < 8; k++)
                    dh[k] = t.get(j / PIECES, j % PIECES, k);
                piece<T, decltype(tag)::value>(e, dh, g[j % 2], u[j % 2], m, n);
                if (!AHEAD)
                    __builtin_amdgcn_sched_barrier(0);
            }
        });
    }
};

// --- logits: largest and sum of exp(z - largest) of each row in the tile -------
// A sum is kept without the 1 of its largest term (-1: without any term), which
// would hide what is left where a class is nearly certain.
struct LseArgs {
    float2 *part;  // [tiles_n][M]
    float *picked;  // [M]: the logit of the row's token
    const int64_t *tokens;  // or null
};

constexpr float LOG2E = 1.44269504088896f;

__device__ __forceinline__ float2 join_lse(float2 a, float2 b) {
    const bool first = a.x >= b.x;  // NaN: either way it stays
    const float2 hi = first ? a : b, lo = first ? b : a;
    const float base = hi.x == -INFINITY ? 0.0f : hi.x;
    return make_float2(hi.x, fmaf(1.0f + lo.y, __builtin_amdgcn_exp2f((lo.x - base) * LOG2E), hi.y));
}
// of N logits, exactly
template <int N>
__device__ __forceinline__ float2 sum_exp(const float (&z)[N]) {
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < N; k++)
        top = fmaxf(top, z[k]);
    const float base = top == -INFINITY ? 0.0f : top;
    float rest = 0.0f, ones = 0.0f;
#pragma unroll
    for (int k = 0; k < N; k++) {
        const float e = __builtin_amdgcn_exp2f((z[k] - base) * LOG2E);
        const bool one = z[k] == base;
        rest += one ? e - 1.0f : e;  // NaN at +inf
        ones += one ? 1.0f : 0.0f;
    }
    return make_float2(top, rest + (top == -INFINITY ? -1.0f : ones - 1.0f));
}

struct Lse {
    static constexpr bool DUAL = false;
    template <typename S>
    static constexpr int lds_bytes() {
        return S::WN * S::TM * (int)sizeof(float2);
    }
    using Args = LseArgs;
    template <typename T, typename S, bool G>
    static __device__ __forceinline__ void run(const LseArgs &e, const Results<S, G> &t, const Work &at,
                                               const mm::Args &a, int m0, int n0, int lane, uint8_t *lds) {
        constexpr int W = Results<S, G>::W, PIECES = Results<S, G>::PIECES;
        float2 *const row = reinterpret_cast<float2 *>(lds);  // [WN][TM]
        const int wn = n0 % S::TN / (S::TN / S::WN), local = m0 % S::TM;
        constexpr int COLUMNS = 16 * S::FN;  // of a wave
#pragma unroll
        for (int i = 0; i < S::FM; i++) {
            const int m = m0 + 16 * i + (lane & 15);
            const int64_t want = e.tokens && m < a.M ? e.tokens[m] : -1;
            const bool here = want >= n0 && want < n0 + COLUMNS && want < a.N;
            constexpr int N = PIECES * W;
            float z[N];
#pragma unroll
            for (int k = 0; k < N; k++)
                z[k] = t.get(i, k / W, k % W);
            auto at_column = [&](int k) { return n0 + t.column(k / W, lane) + k % W; };
            // Both seldom, and the same for a wave: two comparisons a logit less.
            if (n0 + COLUMNS > a.N)
#pragma unroll
                for (int k = 0; k < N; k++)
                    if (at_column(k) >= a.N)
                        z[k] = -INFINITY;
            if (__any(here))
#pragma unroll
                for (int k = 0; k < N; k++)
                    if (here && at_column(k) == want)
                        e.picked[m] = z[k];
            float top = -INFINITY;
#pragma unroll
            for (int k = 0; k < N; k++)
                top = fmaxf(top, z[k]);
            const float base = top == -INFINITY ? 0.0f : top;
            float sum = -1.0f;
#pragma unroll
            for (int k = 0; k < N; k++)
                sum += __builtin_amdgcn_exp2f((z[k] - base) * LOG2E);
            auto over_lanes = [&](float2 r) {
                r = join_lse(r, make_float2(__shfl_xor(r.x, 16), __shfl_xor(r.y, 16)));
                return join_lse(r, make_float2(__shfl_xor(r.x, 32), __shfl_xor(r.y, 32)));
            };
            float2 r = over_lanes(make_float2(top, sum));
            if (__any(r.y < 0x1p-8f))  // a row with one large logit, the same for a wave: as exactly as it goes
                r = over_lanes(sum_exp(z));
            if (lane < 16)
                row[wn * S::TM + local + 16 * i + lane] = r;
        }
        __syncthreads();
        for (int l = threadIdx.x; l < S::TM; l += S::TH) {
            float2 r = row[l];
#pragma unroll
            for (int w = 1; w < S::WN; w++)
                r = join_lse(r, row[w * S::TM + l]);
            const int m = at.m * S::TM + l;
            if (m < a.M)
                e.part[(int64_t)at.n * a.M + m] = r;
        }
        __syncthreads();  // before the next item's
    }
};

// --- logits again: their gradients, c p and another at the token, times a power of two
struct RowGrad {
    float c, at, lse;  // c and at are 0 (and what multiplies them skipped) for a row without a gradient
    int token;         // or -1
};
struct DzArgs {
    const RowGrad *rows;
    uint16_t *dz;  // [M][ld], `pad` columns
    int64_t ld, lo;  // lo: to what rounding dz takes, or 0
    int pad, v0;  // the piece's first token
};

struct Dz {
    static constexpr bool DUAL = false;
    template <typename S>
    static constexpr int lds_bytes() {
        return 0;
    }
    using Args = DzArgs;
    // 8 classes of row m from n on; mine: the row's token may be among them, ends: the last class
    template <typename T, bool LO = false>
    static __device__ __forceinline__ void piece(const DzArgs &e, const RowGrad &r, const float (&z)[8], int m, int n, int N,
                                                 bool mine, bool ends) {
        const int want = r.token - e.v0;
        const bool any = !(r.c == 0.0f && r.at == 0.0f);
        float d[8];
#pragma unroll
        for (int k = 0; k < 8; k++) {
            const float q = r.c * __builtin_amdgcn_exp2f((z[k] - r.lse) * LOG2E);
            d[k] = any ? q : 0.0f;
        }
        if (mine)
#pragma unroll
            for (int k = 0; k < 8; k++)
                d[k] = any && n + k == want ? r.at : d[k];
        if (ends)
#pragma unroll
            for (int k = 0; k < 8; k++)
                d[k] = n + k < N ? d[k] : 0.0f;
        store_parts<T, LO>(e.dz + m * e.ld + n, e.lo, d);
    }
    template <typename T, typename S, bool G>
    static __device__ __forceinline__ void run(const DzArgs &e, const Results<S, G> &t, const Work &,
                                               const mm::Args &a, int m0, int n0, int lane, uint8_t *) {
        constexpr int PIECES = Results<S, G>::PIECES;
#pragma unroll
        for (int i = 0; i < S::FM; i++) {
            const int m = m0 + 16 * i + (lane & 15);
            if (m >= a.M)
                continue;
            const RowGrad r = e.rows[m];
            const int want = r.token - e.v0;
            // both seldom, and the same for a wave
            const bool mine = __any(want >= n0 && want < n0 + 16 * S::FN), ends = n0 + 16 * S::FN > a.N;
#pragma unroll
            for (int p = 0; p < PIECES; p++) {
                const int n = n0 + t.column(p, lane);
                if (n >= e.pad)
                    continue;
                float z[8];
#pragma unroll
                for (int k = 0; k < 8; k++)
                    z[k] = t.get(i, p, k);
                piece<T>(e, r, z, m, n, a.N, mine, ends);
            }
        }
    }
};

}  // namespace mm
}  // namespace cf
