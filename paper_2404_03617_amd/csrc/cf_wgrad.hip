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
    int64_t lddy, rows, chunk;  // rows of a split, a multiple of ROWS
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

struct __attribute__((packed, aligned(1))) Any16b {
    u32x4 v;
};

// What a tile needs to know at compile time: TM x TN of dW, WM x WN waves, BK
// rows a step, QB bytes of a checkpoint's row a load.  EVEN: vectors lie in
// their rows whole (K a multiple of 8, C of QB) and 32 bits hold a step's
// offsets.
template <int TM_, int TN_, int WM_, int WN_, int BK_, int QB_>
struct Shape2 {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, BK = BK_, QB = QB_;
    static constexpr int TH = 64 * WM * WN, SA = TM + PAD, SB = TN + PAD;
    static constexpr int FM = TM / WM / 32, FN = TN / WN / 32, KS = BK / 16;    // MFMA tiles of a wave, steps of 16
    static constexpr int VA = BK * TM / 8 / TH, VB = BK * TN / QB / TH;         // vectors of a thread and step
    static constexpr int DA = TH / (TM / 8), DB = TH / (TN / QB);               // rows between them
    static constexpr int SUMS = DA * TM * 4, STEP = 2 * BK * (SA + SB) * 2, LDS = STEP > SUMS ? STEP : SUMS;
    static_assert(TH % (TM / 8) == 0 && TH % (TN / QB) == 0 && VA >= 1 && VB >= 1, "a thread's vectors share columns");
    static_assert(CKPT_BLOCK % QB == 0 && TN % CKPT_BLOCK == 0, "a vector has one scale");
};

template <typename T, typename S, bool NORM, bool EVEN>
__global__ __launch_bounds__(S::TH) void wgrad_kernel(WGradArgs a) {
    constexpr int TM = S::TM, TN = S::TN, WM = S::WM, WN = S::WN, BK = S::BK, QB = S::QB, TH = S::TH, SA = S::SA,
                  SB = S::SB, FM = S::FM, FN = S::FN, KS = S::KS, VA = S::VA, VB = S::VB, DA = S::DA, DB = S::DB;
    extern __shared__ __align__(16) uint16_t lds[];
    uint16_t *const la = lds, *const lb = lds + 2 * BK * SA;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int k0 = blockIdx.y * TM, c0 = blockIdx.x * TN;
    const int64_t first = (int64_t)blockIdx.z * a.chunk;
    const int64_t last = first + a.chunk < a.rows ? first + a.chunk : a.rows;
    const bool affine = NORM && a.b;
    const bool sums = blockIdx.x == 0 || (affine && !a.part);

    const int ka = tid % (TM / 8) * 8, ra = tid / (TM / 8), ca = k0 + ka;
    const int kb = tid % (TN / QB) * QB, rb = tid / (TN / QB), cb = c0 + kb;
    float db[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};

    // A step's share of a thread, in registers from one step to the next.
    u32x4 va[VA];
    u32x2 vb[VB][QB / 8];
    float vs[VB];
    float2 vn[VB];

    // Vectors past K or C are loaded from its start instead: what they hold
    // only reaches sums that are not stored.  Rows past the end are loaded
    // from the step's first row and taken as zeros when they are stored.
    const uint32_t oa = (uint32_t)((ca < a.K ? ca : 0) * 2), ob = (uint32_t)(cb < a.C ? cb : 0);
    auto fetch_a = [&](int j, int64_t r) {
        if constexpr (EVEN) {
            const int left = (int)(last - r < BK ? last - r : BK);
            const char *const p = (const char *)(a.dy + r * a.lddy);
            const int row = ra + j * DA < left ? ra + j * DA : 0;
            va[j] = reinterpret_cast<const Any16 *>(p + ((uint32_t)row * (uint32_t)(a.lddy * 2) + oa))->v;
        } else {
            const int64_t row = r + ra + j * DA;
            va[j] = row < last ? load8(a.dy + row * a.lddy, ca, a.K) : u32x4{0u, 0u, 0u, 0u};
        }
    };
    auto fetch_b = [&](int j, int64_t r) {
        if constexpr (EVEN) {
            const int left = (int)(last - r < BK ? last - r : BK);
            const int row = rb + j * DB < left ? rb + j * DB : 0;
            const char *const p = (const char *)(a.q + r * a.C);
            const uint32_t at = (uint32_t)row * (uint32_t)a.C + ob;
            if constexpr (QB == 16) {
                const u32x4 t = reinterpret_cast<const Any16b *>(p + at)->v;
                vb[j][0] = u32x2{t[0], t[1]};
                vb[j][QB / 8 - 1] = u32x2{t[2], t[3]};
            } else {
                vb[j][0] = reinterpret_cast<const Any8 *>(p + at)->v;
            }
            vs[j] = (a.scale + r * a.blocks)[(uint32_t)row * (uint32_t)a.blocks + ob / CKPT_BLOCK];
            if constexpr (NORM)
                vn[j] = (a.stats + r)[row];
        } else {
            const int64_t row = r + rb + j * DB;
            vs[j] = 0.0f;
            vn[j] = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < QB / 8; i++)
                vb[j][i] = row < last ? load8b(a.q + row * a.C, cb + 8 * i, a.C) : u32x2{0u, 0u};
            if (row < last && cb < a.C) {
                vs[j] = a.scale[row * a.blocks + cb / CKPT_BLOCK];
                if constexpr (NORM)
                    vn[j] = a.stats[row];
            }
        }
    };
    // into buffer `buf`, `left` rows of which are in the split
    auto store_a = [&](int j, int buf, int64_t left) {
        if (ra + j * DA >= left)
            va[j] = u32x4{0u, 0u, 0u, 0u};
        *reinterpret_cast<u32x4 *>(la + buf * (BK * SA) + (ra + j * DA) * SA + ka) = va[j];
        if (sums) {
            float x[8];
            unpack8<T>(va[j], x);
#pragma unroll
            for (int i = 0; i < 8; i++)
                db[i] += x[i];
        }
    };
    auto store_b = [&](int j, int buf, int64_t left) {
        // x = (byte - 128) f + o
        const bool on = rb + j * DB < left;
        const float f = !on ? 0.0f : NORM ? vs[j] * vn[j].y : vs[j];
        const float o = !on ? 0.0f : fmaf(-128.0f, f, NORM ? -vn[j].x * vn[j].y : 0.0f);
        uint16_t *const p = lb + buf * (BK * SB) + (rb + j * DB) * SB + kb;
#pragma unroll
        for (int i = 0; i < QB / 8; i++) {
            u32x4 v;
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const uint32_t w = vb[j][i][h] ^ 0x80808080u;
                v[2 * h] = T::pack2(fmaf(biased(w, 0), f, o), fmaf(biased(w, 1), f, o));
                v[2 * h + 1] = T::pack2(fmaf(biased(w, 2), f, o), fmaf(biased(w, 3), f, o));
            }
            *reinterpret_cast<u32x4 *>(p + 8 * i) = v;
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

    if (first < last) {
#pragma unroll
        for (int j = 0; j < VA; j++)
            fetch_a(j, first);
#pragma unroll
        for (int j = 0; j < VB; j++)
            fetch_b(j, first);
        const int64_t second = first + BK < last ? first + BK : first;  // a row to load from; not used past the end
#pragma unroll
        for (int j = 0; j < VA; j++) {
            store_a(j, 0, last - first);
            fetch_a(j, second);
        }
#pragma unroll
        for (int j = 0; j < VB; j++) {
            store_b(j, 0, last - first);
            fetch_b(j, second);
        }
        __syncthreads();
    }
    // Step by step: products of the step in one buffer while the next step,
    // fetched into registers a step ago, is written to the other and the one
    // after it is fetched.
    int buf = 0;
    for (int64_t r = first; r < last; r += BK, buf ^= 1) {
        const int64_t left = last - (r + BK), third = left > BK ? r + 2 * BK : r;
        const uint16_t *const pa = la + buf * (BK * SA) + tr_row * SA + wm + tr_col;
        const uint16_t *const pb = lb + buf * (BK * SB) + tr_row * SB + wn + tr_col;
#pragma unroll
        for (int k = 0; k < KS; k++) {
            u32x4 fa[FM], fb[FN];
#pragma unroll
            for (int m = 0; m < FM; m++) {
                const u32x2 lo = read_tr(pa + 16 * k * SA + 32 * m), hi = read_tr(pa + (16 * k + 4) * SA + 32 * m);
                fa[m] = u32x4{lo.x, lo.y, hi.x, hi.y};
            }
#pragma unroll
            for (int n = 0; n < FN; n++) {
                const u32x2 lo = read_tr(pb + 16 * k * SB + 32 * n), hi = read_tr(pb + (16 * k + 4) * SB + 32 * n);
                fb[n] = u32x4{lo.x, lo.y, hi.x, hi.y};
            }
#pragma unroll
            for (int m = 0; m < FM; m++)
#pragma unroll
                for (int n = 0; n < FN; n++)
                    acc[m][n] = mfma32<T>(fa[m], fb[n], acc[m][n]);
#pragma unroll
            for (int j = VA * k / KS; j < VA * (k + 1) / KS; j++) {
                store_a(j, buf ^ 1, left);
                fetch_a(j, third);
            }
#pragma unroll
            for (int j = VB * k / KS; j < VB * (k + 1) / KS; j++) {
                store_b(j, buf ^ 1, left);
                fetch_b(j, third);
            }
        }
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
    int tile;  // index into TILES
    int splits;
    int64_t chunk;
};

// Tiles and their waves.
typedef Shape2<64, 64, 2, 2, 64, 16> Tile64;
typedef Shape2<128, 128, 2, 2, 64, 16> Tile128;
typedef Shape2<256, 256, 2, 4, 64, 16> Tile256;
typedef Shape2<256, 64, 4, 2, 64, 8> TileTall;
typedef Shape2<64, 256, 2, 4, 64, 16> TileWide;
struct Tile {
    int m, n;
};
constexpr Tile TILES[] = {{64, 64}, {128, 128}, {256, 256}, {256, 64}, {64, 256}};
constexpr int ROWS = 64;  // of a step

int64_t tiles_of(int t, int K, int C) {
    return (int64_t)((K + TILES[t].m - 1) / TILES[t].m) * ((C + TILES[t].n - 1) / TILES[t].n);
}

constexpr size_t PART_BYTES = (size_t)64 << 20;

Plan plan_of(int64_t rows, int K, int C) {
    const int64_t cus = device_cu_count();
    Plan p;
    if (K >= 256 && C >= 256 && tiles_of(2, K, C) >= cus / 2)
        p.tile = 2;
    else if (C <= 64 && K > 128 && tiles_of(3, K, C) * (rows / 512 + 1) >= cus)
        p.tile = 3;
    else if (K <= 64 && C > 128 && tiles_of(4, K, C) * (rows / 512 + 1) >= cus)
        p.tile = 4;
    else if (K > 64 && C > 64 && tiles_of(1, K, C) * (rows / 512 + 1) >= cus)
        p.tile = 1;
    else
        p.tile = 0;
    const int64_t tiles = tiles_of(p.tile, K, C);
    const int per_cu = p.tile == 0 ? 3 : p.tile == 1 ? 2 : 1;
    int64_t splits = per_cu * cus / tiles;
    const int64_t most = (rows + 4 * ROWS - 1) / (4 * ROWS), room = (int64_t)(PART_BYTES / (4.0 * K * (C + 1.0)));
    splits = splits < most ? splits : most;
    splits = splits < room ? splits : room;
    if (tiles >= cus || splits < 1)
        splits = 1;
    p.chunk = rows < 1 ? ROWS : ((rows + splits - 1) / splits + ROWS - 1) / ROWS * ROWS;
    p.splits = rows < 1 ? 1 : (int)((rows + p.chunk - 1) / p.chunk);
    return p;
}

template <typename T, typename S, bool NORM>
hipError_t launch_tile(const WGradArgs &a, int splits, hipStream_t st) {
    const bool even = a.K % 8 == 0 && a.C % S::QB == 0 && a.lddy * 2 * S::BK < (int64_t)1 << 31 &&
                      (int64_t)a.C * S::BK < (int64_t)1 << 31;
    void (*const f)(WGradArgs) = even ? wgrad_kernel<T, S, NORM, true> : wgrad_kernel<T, S, NORM, false>;
    if (S::LDS > 64 * 1024) {
        const hipError_t e = allow_full_lds((const void *)f);
        if (e != hipSuccess)
            return e;
    }
    const dim3 grid((a.C + S::TN - 1) / S::TN, (a.K + S::TM - 1) / S::TM, splits);
    f<<<grid, dim3(S::TH), S::LDS, st>>>(a);
    return hipGetLastError();
}

template <typename T, bool NORM>
hipError_t launch_type(const WGradArgs &a, const Plan &p, hipStream_t st) {
    hipError_t e;
    switch (p.tile) {
    case 0: e = launch_tile<T, Tile64, NORM>(a, p.splits, st); break;
    case 1: e = launch_tile<T, Tile128, NORM>(a, p.splits, st); break;
    case 2: e = launch_tile<T, Tile256, NORM>(a, p.splits, st); break;
    case 3: e = launch_tile<T, TileTall, NORM>(a, p.splits, st); break;
    default: e = launch_tile<T, TileWide, NORM>(a, p.splits, st); break;
    }
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
