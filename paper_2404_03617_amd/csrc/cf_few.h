// cf_few.h -- products x W^T of a few rows (up to 16: decoded tokens, a handful of
// features), bound by reading W once.  A workgroup takes 16 or 32 rows of W, its
// waves share k: each takes 256 k's of 16 rows at a time, or 128 of 32, straight from
// memory into MFMA fragments, eight loads in flight a wave.  A row's loads are issued
// one after the other, so that both halves of a cache line are asked for together: 16
// rows x 131072 x 4096 take 200 us, with the matrices' loads among each other 247.
// The rows of x come from the caches.  Rows may start anywhere and have any length:
// what is left of k goes element by element.  The waves' sums meet in LDS in a fixed order,
// and the first wave does what follows.  1 x 131072 x 4096 takes 182 us, 5.9 TB/s; a
// gated block of 1 x 4096 x 12288 60 us, 5.0 TB/s (59 without the second number of h).
#pragma once

#include "cf_mm_epi.h"

namespace cf {
namespace few {

constexpr int ROWS = 16;  // rows of x at most

struct Args {
    const uint16_t *x, *w[2];
    int64_t ldx, ldw[2], lo;  // lo: from x to what rounding it took, where a kernel has that
    int M, N, K;
};

// 8 k's of a row that has `left` of them from here on
__device__ __forceinline__ u32x4 load_k(const uint16_t *p, int left) {
    if (left >= 8)
        return reinterpret_cast<const Any16 *>(p)->v;
    u32x4 r = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 7; i++)
        if (i < left)
            r[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
    return r;
}

// What follows gets `sum(f)`, the four results of fragment f in row lane % 16 of x:
// rows n0 + 16 f + 4 (lane / 16) .. + 3 of W (DUAL: of either matrix, n0 alone).
struct Gated {
    static constexpr bool DUAL = true, LO = false, FOLD = false;
    using Extra = mm::GatedArgs;
    template <typename T, int FN>
    static __device__ __forceinline__ void run(const Extra &e, const float4v (&sum)[FN], const Args &a, int n0, int lane) {
        const int m = lane & 15, n = n0 + 4 * (lane >> 4), left = e.H - n;
        if (m >= a.M || n >= e.pad)
            return;
        mm::store_rowf<4>(e.saved ? e.saved + (int64_t)m * 2 * e.H + n : nullptr, sum[0], e.saved ? left : 0);
        mm::store_rowf<4>(e.saved ? e.saved + (int64_t)m * 2 * e.H + e.H + n : nullptr, sum[1], e.saved ? left : 0);
        with_act(e.act, [&](auto tag) {
            float4v h;
#pragma unroll
            for (int k = 0; k < 4; k++)
                h[k] = k < left ? act_value<decltype(tag)::value>(sum[0][k]) * sum[1][k] : 0.0f;
            mm::store_row<T, 4>(e.h + m * e.ldh + n, h, 4);
            const u32x4 r = {T::pack2(h[0], h[1]), T::pack2(h[2], h[3]), 0u, 0u};
            float f[8];
            unpack8<T>(r, f);
#pragma unroll
            for (int k = 0; k < 4; k++)
                f[k] = fabsf(f[k]) < INFINITY ? h[k] - f[k] : 0.0f;
            mm::store_row<T, 4>(e.h + e.lo + m * e.ldh + n, f, 4);
        });
    }
};

// x in two numbers: the second ones' rows in a fragment of their own, or FOLDED, for up
// to 8 rows, beside the first ones in the same (1 x 12288 in 4096 rows of W 25 us in
// two fragments, 23 in one).
template <bool FOLDED>
struct Store {
    static constexpr bool DUAL = false, LO = !FOLDED, FOLD = FOLDED;
    using Extra = mm::StoreArgs;
    template <typename T, int FN>
    static __device__ __forceinline__ void run(const Extra &e, const float4v (&sum)[FN], const Args &a, int n0, int lane) {
        const int m = lane & 15;
#pragma unroll
        for (int f = 0; f < FN; f++) {
            const int n = n0 + 16 * f + 4 * (lane >> 4);
            if (m < a.M && n < a.N)
                mm::store_row<T, 4>(e.out[0] + (int64_t)m * e.ldo + n, sum[f], a.N - n);
        }
    }
};

struct Lse {
    static constexpr bool DUAL = false, LO = false, FOLD = false;
    using Extra = mm::LseArgs;
    template <typename T, int FN>
    static __device__ __forceinline__ void run(const Extra &e, const float4v (&sum)[FN], const Args &a, int n0, int lane) {
        const int m = lane & 15;
        const int64_t want = e.tokens && m < a.M ? e.tokens[m] : -1;
        float z[4 * FN];
#pragma unroll
        for (int k = 0; k < 4 * FN; k++) {
            const int n = n0 + 16 * (k / 4) + 4 * (lane >> 4) + k % 4;
            z[k] = n < a.N ? sum[k / 4][k % 4] : -INFINITY;
            if (n == want)
                e.picked[m] = z[k];
        }
        float2 r = mm::sum_exp(z);
        r = mm::join_lse(r, make_float2(__shfl_xor(r.x, 16), __shfl_xor(r.y, 16)));
        r = mm::join_lse(r, make_float2(__shfl_xor(r.x, 32), __shfl_xor(r.y, 32)));
        if (lane < a.M && lane < 16)
            e.part[(int64_t)blockIdx.x * a.M + lane] = r;
    }
};

template <typename T, int WAVES, int FN, typename E>
__global__ __launch_bounds__(WAVES * 64) void kernel(Args a, typename E::Extra e) {
    __shared__ float4v red[WAVES][FN][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int n0 = blockIdx.x * (E::DUAL ? 16 : 16 * FN);
    const uint16_t *w[FN];
#pragma unroll
    for (int f = 0; f < FN; f++) {
        const int row = n0 + (E::DUAL ? 0 : 16 * f) + r;
        w[f] = (E::DUAL && f ? a.w[1] : a.w[0]) + (row < a.N ? row : a.N - 1) * (E::DUAL && f ? a.ldw[1] : a.ldw[0]) + q * 8;
    }
    const int row_x = E::FOLD ? r & 7 : r;
    const uint16_t *const x =
        a.x + (int64_t)(row_x < a.M ? row_x : a.M - 1) * a.ldx + q * 8 + (E::FOLD && r >= 8 ? a.lo : 0);
    float4v acc[FN];
#pragma unroll
    for (int f = 0; f < FN; f++)
        acc[f] = float4v{0.0f, 0.0f, 0.0f, 0.0f};

    constexpr int U = 8 / FN, SHARE = U * 32;
    int k0 = wave * SHARE;
    for (; k0 + SHARE <= a.K; k0 += WAVES * SHARE) {
        u32x4 fw[FN][U], fx[U], fl[E::LO ? U : 1];
#pragma unroll
        for (int f = 0; f < FN; f++)
#pragma unroll
            for (int u = 0; u < U; u++)
                fw[f][u] = reinterpret_cast<const Any16 *>(w[f] + k0 + 32 * u)->v;
#pragma unroll
        for (int u = 0; u < U; u++)
            fx[u] = reinterpret_cast<const Any16 *>(x + k0 + 32 * u)->v;
        if constexpr (E::LO)
#pragma unroll
            for (int u = 0; u < U; u++)
                fl[u] = reinterpret_cast<const Any16 *>(x + a.lo + k0 + 32 * u)->v;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int f = 0; f < FN; f++) {
                acc[f] = T::mfma(fw[f][u], fx[u], acc[f]);
                if constexpr (E::LO)
                    acc[f] = T::mfma(fw[f][u], fl[u], acc[f]);
            }
    }
    for (; k0 < a.K; k0 += 32) {  // the wave that has the last share of k, where it is not whole
        const int left = a.K - k0 - q * 8;
        const u32x4 fx = load_k(x + k0, left);
#pragma unroll
        for (int f = 0; f < FN; f++) {
            const u32x4 fw = load_k(w[f] + k0, left);
            acc[f] = T::mfma(fw, fx, acc[f]);
            if constexpr (E::LO)
                acc[f] = T::mfma(fw, load_k(x + a.lo + k0, left), acc[f]);
        }
    }
#pragma unroll
    for (int f = 0; f < FN; f++)
        red[wave][f][lane] = acc[f];
    __syncthreads();
    if (wave)
        return;
#pragma unroll
    for (int f = 0; f < FN; f++)
#pragma unroll
        for (int v = 1; v < WAVES; v++)
            acc[f] += red[v][f][lane];
    if constexpr (E::FOLD)
#pragma unroll
        for (int f = 0; f < FN; f++)
#pragma unroll
            for (int k = 0; k < 4; k++)
                acc[f][k] += __shfl_xor(acc[f][k], 8);
    E::template run<T, FN>(e, acc, a, n0, lane);
}

// Waves that share k: enough that each has one to four shares of it.
inline int waves_of(int K) { return K > 6144 ? 16 : K > 1536 ? 8 : 4; }

template <typename T, int FN, typename E>
hipError_t launch(const Args &a, const typename E::Extra &e, hipStream_t st) {
    const int per = E::DUAL ? 16 : 16 * FN, waves = waves_of(a.K);
    void (*const f)(Args, typename E::Extra) = waves == 16  ? kernel<T, 16, FN, E>
                                               : waves == 8 ? kernel<T, 8, FN, E>
                                                            : kernel<T, 4, FN, E>;
    f<<<dim3((unsigned)((a.N + per - 1) / per)), dim3(waves * 64), 0, st>>>(a, e);
    return hipGetLastError();
}

}  // namespace few
}  // namespace cf
