// cf_wgrad.hip -- the weight gradient of a linear (point-wise) layer from the
// 8-bit checkpoint of its input:
//
//   dW[k][c] = sum_r dy[r][k] x[r][c],   db[k] = sum_r dy[r][k]
//
// with x = q * scale, or, where the input was a layer norm of the
// checkpointed rows, x = w xh + b with xh = (q * scale - mean) * rstd.  There
//   dW[k][c] = w[c] sum_r dy[r][k] xh[r][c] + b[c] db[k],
// so that the main loop sees one factor and one offset for 64 channels of a
// row, and w and b meet the sums in the epilogue.
//
// A workgroup makes a TM x TN tile of dW: 64 rows of dy and q at a time go
// through registers into LDS, the bytes converted to the 16-bit type of dy on
// the way (one rounding of q * scale or xh, 2^-9 in bf16 against the 2^-8 of
// its block's largest value that 8 bits keep), two buffers, one barrier a
// step.  Both operands have the summed index r outermost, so MFMA fragments
// are read with the transposing LDS loads.  A row of LDS is padded by 64
// bytes: the 4 rows that 32 lanes read together then lie in different banks.
// Few tiles over many rows: the rows are split over workgroups that write fp32
// partial sums, and a second launch adds them in a fixed order.
#include "cf_rows.h"
#include "cf_kernels.h"
#include "cf_train.h"

namespace cf {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int BK = 64;   // rows of a step
constexpr int PAD = 32;  // elements behind each row of LDS

struct WGradArgs {
    const uint16_t *dy;
    const int8_t *q;
    const float *scale;
    const float2 *stats;
    const float *w, *b;
    uint16_t *dw;
    float *db;
    float *part;     // [splits][K][C] partial sums, null for one split
    float *part_db;  // [splits][K]
    int64_t lddy, rows, chunk;  // rows of a split, a multiple of BK
    int K, C, blocks;
};

// 4 rows x 16 columns of a 16-bit LDS tile, given as 4 columns of row lane / 4
// by each of 16 lanes; the lane gets its column's 4 rows.
__device__ __forceinline__ u32x2 read_tr(const uint16_t *p) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p));
}

template <typename T>
__device__ __forceinline__ f32x16 mfma32(const u32x4 &a, const u32x4 &b, const f32x16 &c) {
    Pack8 pa, pb;
    pa.u = a;
    pb.u = b;
    if constexpr (T::is_bf16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(pa.b, pb.b, c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(pa.h, pb.h, c, 0, 0, 0);
}

// 16 bytes of a checkpoint's row of C, from byte c on, zeros past its end
__device__ __forceinline__ u32x4 load16b(const int8_t *row, int c, int C) {
    struct __attribute__((packed, aligned(1))) Any {
        u32x4 v;
    };
    if (C - c >= 16)
        return reinterpret_cast<const Any *>(row + c)->v;
    const u32x2 lo = load8b(row, c, C), hi = load8b(row, c + 8, C);
    return u32x4{lo.x, lo.y, hi.x, hi.y};
}

template <typename T, int TM, int TN, int WM, int WN, bool NORM>
__global__ __launch_bounds__(64 * WM *WN) void wgrad_kernel(WGradArgs a) {
    constexpr int TH = 64 * WM * WN, SA = TM + PAD, SB = TN + PAD;
    constexpr int FM = TM / WM / 32, FN = TN / WN / 32;      // MFMA tiles of a wave
    constexpr int VA = BK * TM / 8 / TH, VB = BK * TN / 16 / TH;  // vectors of a thread and step
    static_assert(TH % (TM / 8) == 0 && VA >= 1 && VB >= 1, "a thread's dy vectors share their columns");
    extern __shared__ __align__(16) uint16_t lds[];
    uint16_t *const la = lds, *const lb = lds + 2 * BK * SA;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int k0 = blockIdx.y * TM, c0 = blockIdx.x * TN;
    const int64_t first = (int64_t)blockIdx.z * a.chunk;
    const int64_t last = first + a.chunk < a.rows ? first + a.chunk : a.rows;
    const bool affine = NORM && a.b;
    const bool sums = blockIdx.x == 0 || (affine && !a.part);

    const int ca = k0 + tid % (TM / 8) * 8, ra = tid / (TM / 8);
    const int cb = c0 + tid % (TN / 16) * 16, rb = tid / (TN / 16);
    constexpr int DA = TH / (TM / 8), DB = TH / (TN / 16);  // rows between a thread's vectors
    float db[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};

    struct Step {
        u32x4 a[VA], b[VB];
        float f[VB], o[VB];  // factor and offset of the biased bytes
    } st;
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int j = 0; j < VA; j++) {
            const int64_t row = r + ra + j * DA;
            st.a[j] = row < last && ca < a.K ? load8(a.dy + row * a.lddy, ca, a.K) : u32x4{0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int j = 0; j < VB; j++) {
            const int64_t row = r + rb + j * DB;
            st.b[j] = u32x4{0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};
            st.f[j] = st.o[j] = 0.0f;
            if (row < last && cb < a.C) {
                st.b[j] = load16b(a.q + row * a.C, cb, a.C);
                float f = a.scale[row * a.blocks + cb / CKPT_BLOCK], o = 0.0f;
                if constexpr (NORM) {
                    const float2 s = a.stats[row];
                    f *= s.y;
                    o = -s.x * s.y;
                }
                st.f[j] = f;
                st.o[j] = fmaf(-128.0f, f, o);
            }
        }
    };
    auto store = [&](int buf) {
        uint16_t *const pa = la + buf * (BK * SA), *const pb = lb + buf * (BK * SB);
#pragma unroll
        for (int j = 0; j < VA; j++)
            *reinterpret_cast<u32x4 *>(pa + (ra + j * DA) * SA + (ca - k0)) = st.a[j];
#pragma unroll
        for (int j = 0; j < VB; j++) {
            u32x4 v[2];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t w = st.b[j][i] ^ 0x80808080u;
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; e++)
                    x[e] = fmaf(biased(w, e), st.f[j], st.o[j]);
                v[i / 2][2 * (i & 1)] = T::pack2(x[0], x[1]);
                v[i / 2][2 * (i & 1) + 1] = T::pack2(x[2], x[3]);
            }
            uint16_t *const p = pb + (rb + j * DB) * SB + (cb - c0);
            *reinterpret_cast<u32x4 *>(p) = v[0];
            *reinterpret_cast<u32x4 *>(p + 8) = v[1];
        }
        if (sums)
#pragma unroll
            for (int j = 0; j < VA; j++) {
                float x[8];
                unpack8<T>(st.a[j], x);
#pragma unroll
                for (int i = 0; i < 8; i++)
                    db[i] += x[i];
            }
    };

    f32x16 acc[FM][FN];
#pragma unroll
    for (int m = 0; m < FM; m++)
#pragma unroll
        for (int n = 0; n < FN; n++)
#pragma unroll
            for (int i = 0; i < 16; i++)
                acc[m][n][i] = 0.0f;

    // this lane's share of a transposed read: row 8 (lane / 32) + lane % 16 / 4,
    // columns 16 (lane / 16 % 2) + 4 (lane % 4)
    const int tr_row = 8 * (lane >> 5) + ((lane & 15) >> 2), tr_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const int wm = wave / WN * (TM / WM), wn = wave % WN * (TN / WN);

    fetch(first);
    store(0);
    __syncthreads();
    int buf = 0;
    for (int64_t r = first; r < last; r += BK, buf ^= 1) {
        const bool more = r + BK < last;
        if (more)
            fetch(r + BK);
        const uint16_t *const pa = la + buf * (BK * SA) + tr_row * SA + wm + tr_col;
        const uint16_t *const pb = lb + buf * (BK * SB) + tr_row * SB + wn + tr_col;
#pragma unroll
        for (int k = 0; k < BK; k += 16) {
            u32x4 fa[FM], fb[FN];
#pragma unroll
            for (int m = 0; m < FM; m++) {
                const u32x2 lo = read_tr(pa + k * SA + 32 * m), hi = read_tr(pa + (k + 4) * SA + 32 * m);
                fa[m] = u32x4{lo.x, lo.y, hi.x, hi.y};
            }
#pragma unroll
            for (int n = 0; n < FN; n++) {
                const u32x2 lo = read_tr(pb + k * SB + 32 * n), hi = read_tr(pb + (k + 4) * SB + 32 * n);
                fb[n] = u32x4{lo.x, lo.y, hi.x, hi.y};
            }
#pragma unroll
            for (int m = 0; m < FM; m++)
#pragma unroll
                for (int n = 0; n < FN; n++)
                    acc[m][n] = mfma32<T>(fa[m], fb[n], acc[m][n]);
        }
        if (more)
            store(buf ^ 1);
        __syncthreads();
    }

    // column sums of dy: the threads that hold the same columns
    float *const lsum = reinterpret_cast<float *>(lds);  // [DA][TM], then the totals in its first row
    if (sums) {
#pragma unroll
        for (int i = 0; i < 8; i++)
            lsum[ra * TM + (ca - k0) + i] = db[i];
        __syncthreads();
        for (int k = tid; k < TM; k += TH) {
            float f = 0.0f;
#pragma unroll
            for (int j = 0; j < DA; j++)
                f += lsum[j * TM + k];
            lsum[k] = f;
            if (blockIdx.x == 0 && k0 + k < a.K)
                (a.part ? a.part_db + (int64_t)blockIdx.z * a.K : a.db)[k0 + k] = f;
        }
        __syncthreads();
    }
#pragma unroll
    for (int n = 0; n < FN; n++) {
        const int c = c0 + wn + 32 * n + (lane & 31);
        if (c >= a.C)
            continue;
        const float w = NORM && a.w ? a.w[c] : 1.0f, b = affine ? a.b[c] : 0.0f;
#pragma unroll
        for (int m = 0; m < FM; m++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int kl = wm + 32 * m + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3), k = k0 + kl;
                if (k >= a.K)
                    continue;
                float f = acc[m][n][i];
                if (a.part) {
                    a.part[((int64_t)blockIdx.z * a.K + k) * a.C + c] = f;
                } else {
                    if constexpr (NORM) {
                        f *= w;
                        if (affine)
                            f = fmaf(b, lsum[kl], f);
                    }
                    a.dw[(int64_t)k * a.C + c] = (uint16_t)T::pack2(f, 0.0f);
                }
            }
    }
}

// The sum of the splits: 64 columns of one row k a workgroup, S threads share
// a column.
template <typename T, int S>
__global__ __launch_bounds__(64 * S) void wgrad_reduce_kernel(WGradArgs a, int splits, int norm) {
    __shared__ float sum[S][64], sum_db[S];
    const int col = threadIdx.x & 63, s = threadIdx.x >> 6;
    const int k = blockIdx.x, c = blockIdx.y * 64 + col;
    float f = 0.0f;
    if (c < a.C)
        for (int z = s; z < splits; z += S)
            f += a.part[((int64_t)z * a.K + k) * a.C + c];
    const bool affine = norm && a.b;
    float d = 0.0f;
    if (blockIdx.y == 0 || affine) {  // one wave's lanes share each S-th part of the splits
        for (int z = s + S * col; z < splits; z += 64 * S)
            d += a.part_db[(int64_t)z * a.K + k];
        d = lanes<Add, 64>(d);
    }
    if constexpr (S > 1) {
        sum[s][col] = f;
        if (col == 0)
            sum_db[s] = d;
        __syncthreads();
        if (s > 0)
            return;
        f = sum[0][col];
        d = sum_db[0];
#pragma unroll
        for (int i = 1; i < S; i++) {
            f += sum[i][col];
            d += sum_db[i];
        }
    }
    if (blockIdx.y == 0 && col == 0)
        a.db[k] = d;
    if (c >= a.C)
        return;
    if (norm) {
        f *= a.w ? a.w[c] : 1.0f;
        if (affine)
            f = fmaf(a.b[c], d, f);
    }
    a.dw[(int64_t)k * a.C + c] = (uint16_t)T::pack2(f, 0.0f);
}

struct Plan {
    int tile;  // index into the tiles below
    int splits;
    int64_t chunk;
};

struct Tile {
    int m, n;
};
constexpr Tile TILES[] = {{64, 64}, {128, 128}, {256, 256}};

int64_t tiles_of(int t, int K, int C) {
    return (int64_t)((K + TILES[t].m - 1) / TILES[t].m) * ((C + TILES[t].n - 1) / TILES[t].n);
}

constexpr size_t PART_BYTES = (size_t)64 << 20;

Plan plan_of(int64_t rows, int K, int C) {
    const int64_t cus = device_cu_count();
    Plan p;
    p.tile = K >= 256 && C >= 256 && tiles_of(2, K, C) >= cus / 2 ? 2 : K > 64 && C > 64 && tiles_of(1, K, C) * (rows / 512 + 1) >= cus ? 1 : 0;
    const int64_t tiles = tiles_of(p.tile, K, C);
    int64_t splits = (2 * cus + tiles - 1) / tiles;
    const int64_t most = (rows + 4 * BK - 1) / (4 * BK), room = (int64_t)(PART_BYTES / (4.0 * K * (C + 1.0)));
    splits = splits < most ? splits : most;
    splits = splits < room ? splits : room;
    if (tiles >= cus || splits < 1)
        splits = 1;
    p.chunk = rows < 1 ? BK : ((rows + splits - 1) / splits + BK - 1) / BK * BK;
    p.splits = rows < 1 ? 1 : (int)((rows + p.chunk - 1) / p.chunk);
    return p;
}

template <typename T, int TM, int TN, int WM, int WN, bool NORM>
hipError_t launch_tile(const WGradArgs &a, int splits, hipStream_t st) {
    constexpr int SUMS = 64 * WM * WN / (TM / 8) * TM * 4;
    constexpr int STEP = 2 * BK * (TM + PAD + TN + PAD) * 2;
    constexpr int LDS = STEP > SUMS ? STEP : SUMS;
    const void *const f = (const void *)wgrad_kernel<T, TM, TN, WM, WN, NORM>;
    if (LDS > 64 * 1024) {
        const hipError_t e = allow_full_lds(f);
        if (e != hipSuccess)
            return e;
    }
    const dim3 grid((a.C + TN - 1) / TN, (a.K + TM - 1) / TM, splits);
    wgrad_kernel<T, TM, TN, WM, WN, NORM><<<grid, dim3(64 * WM * WN), LDS, st>>>(a);
    return hipGetLastError();
}

template <typename T, bool NORM>
hipError_t launch_type(const WGradArgs &a, const Plan &p, hipStream_t st) {
    hipError_t e;
    if (p.tile == 2)
        e = launch_tile<T, 256, 256, 2, 4, NORM>(a, p.splits, st);
    else if (p.tile == 1)
        e = launch_tile<T, 128, 128, 2, 2, NORM>(a, p.splits, st);
    else
        e = launch_tile<T, 64, 64, 2, 2, NORM>(a, p.splits, st);
    if (e != hipSuccess || p.splits == 1)
        return e;
    const dim3 grid(a.K, (a.C + 63) / 64);
    if (p.splits >= 32)
        wgrad_reduce_kernel<T, 16><<<grid, dim3(1024), 0, st>>>(a, p.splits, NORM);
    else
        wgrad_reduce_kernel<T, 1><<<grid, dim3(64), 0, st>>>(a, p.splits, NORM);
    return hipGetLastError();
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
    if (g.stats)
        return bf16 ? launch_type<BF16, true>(a, p, st) : launch_type<F16, true>(a, p, st);
    return bf16 ? launch_type<BF16, false>(a, p, st) : launch_type<F16, false>(a, p, st);
}

}  // namespace cf
