// cf_wgrad.h -- the weight gradient of a linear (point-wise) layer from the
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
// A workgroup makes a TM x TN tile of dW: 32 to 128 rows (by the tile) of dy and
// q at a time go through registers into LDS, the bytes converted to the 16-bit type
// of dy on the way (one rounding of q * scale or xh, 2^-9 in bf16 against the 2^-8
// of its block's largest value that 8 bits keep), two buffers, one barrier a
// step.  That rounding adds a third to the error of dW, most of which is the
// rounding of the result: 2.8e-4 of its norm instead of 2.1e-4 in fp16, 2.2e-3
// instead of 1.7e-3 in bf16.  Both operands have the summed index r outermost, so MFMA fragments
// are read with the transposing LDS loads.  A row of LDS is padded by 64
// bytes: the 4 rows that 32 lanes read together then lie in different banks.
// Few tiles over many rows: the rows are split over workgroups that write fp32
// partial sums, and a second launch adds them in a fixed order.
//
// Measured on MI355X (the library's product of two matrices of the largest size
// below, without bytes to convert, takes 466 us in bf16 and 485 in fp16; a copy
// moves 4.9 TB/s):
//   16384 rows, K = C = 4096: bf16 502 us, 1095 TFLOP/s, fp16 509; after a norm 539
//     and 567.  MFMA busy 65%, VALU 42%, LDS 49%: what stands beside the products, the
//     way of both operands through registers into LDS, bounds it, not memory.  The
//     sums of dy, in the tiles of the first columns alone, take 18 us of it in bf16
//     and none in fp16
//   401408 rows, K = 256, C = 64, fp16 after a norm: 45.8 us and 7.1 us for the
//     second launch, 5.0 TB/s: memory
//   49 rows, K = 2048, C = 512: 4.7 us, one step of 64 rows from load to store
#pragma once

#include "cf_rows.h"
#include "cf_kernels.h"
#include "cf_train.h"
#include "cf_wgrad_plan.h"

#include <type_traits>

namespace cf {

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
    int64_t lddy, rows, chunk;  // rows of a split, a multiple of 64
    int K, C, blocks, tiles_k, tiles_c, splits;
};

// One instance a dtype, with and without a norm before the layer (tile: index
// into wgrad::TILES).
hipError_t launch_wgrad_f16(const WGradArgs &a, int tile, hipStream_t st);
hipError_t launch_wgrad_bf16(const WGradArgs &a, int tile, hipStream_t st);
hipError_t launch_wgrad_norm_f16(const WGradArgs &a, int tile, hipStream_t st);
hipError_t launch_wgrad_norm_bf16(const WGradArgs &a, int tile, hipStream_t st);

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int PAD = 32;  // elements behind each row of LDS


// The tile and split of a workgroup.  Workgroups go to the eight XCDs in turn,
// each with an L2 of its own; here every XCD takes a run of the list of all
// tiles of the first split, of the second, and so on, so that the tiles that
// read the same rows of dy and q run next to each other behind one L2.  Within
// a split the list goes along c in bands of eight tiles of k: a part of a
// large dW is a block that shares rows of both operands.
struct Work {
    int k, c, split;
};
__device__ __forceinline__ Work work_of(int tiles_k, int tiles_c, int splits) {
    const unsigned n = gridDim.x, xcd = blockIdx.x & 7, q = n >> 3, rest = n & 7;
    unsigned i = xcd * q + (xcd < rest ? xcd : rest) + (blockIdx.x >> 3);
    const unsigned tiles = (unsigned)tiles_k * (unsigned)tiles_c, split = i / tiles;
    i -= split * tiles;
    const unsigned band = i / (8u * tiles_c), k0 = 8 * band, high = (unsigned)tiles_k - k0 < 8 ? tiles_k - k0 : 8;
    i -= band * 8 * tiles_c;
    return {(int)(k0 + i % high), (int)(i / high), (int)split};
}

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

// What a tile needs to know at compile time: TM x TN of dW, WM x WN waves for
// it and WK groups of them that share the rows of a step; BK rows a step, QB
// bytes of a checkpoint's row a load, DEPTH steps in registers on their way to
// LDS, OCC waves a SIMD.
template <int TM_, int TN_, int WM_, int WN_, int WK_, int BK_, int QB_, int DEPTH_, int OCC_>
struct Shape2 {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, WK = WK_, BK = BK_, QB = QB_, DEPTH = DEPTH_,
                         OCC = OCC_;
    static constexpr int TH = 64 * WM * WN * WK, SA = TM + PAD, SB = TN + PAD;
    static constexpr int FM = TM / WM / 32, FN = TN / WN / 32, KS = BK / WK / 16;  // MFMA tiles of a wave, its steps of 16
    static constexpr int VA = BK * TM / 8 / TH, VB = BK * TN / QB / TH;            // vectors of a thread and step
    static constexpr int DA = TH / (TM / 8), DB = TH / (TN / QB);                  // rows between them
    static constexpr int SUMS = DA * TM * 4, STEP = 2 * BK * (SA + SB) * 2;
    static constexpr int JOIN = WK > 1 ? TM * TN * 4 : 0;  // a group's results
    static constexpr int LDS = STEP > SUMS ? (STEP > JOIN ? STEP : JOIN) : (SUMS > JOIN ? SUMS : JOIN);
    static_assert(TH % (TM / 8) == 0 && TH % (TN / QB) == 0 && VA >= 1 && VB >= 1, "a thread's vectors share columns");
    static_assert(KS % 2 == 0, "fragments alternate between two sets of registers");
    static_assert(CKPT_BLOCK % QB == 0 && TN % CKPT_BLOCK == 0, "a vector has one scale");
};

// How vectors meet the ends of their rows.  EVEN: K is a multiple of 8 and C
// of QB, so that they do not.  SHIFT: the last vector of a row of q, or of dy
// where K is below the tile's, is loaded with what stands before it and moved
// down when it is stored.  ANY: element by element where it has to be, for rows
// shorter than a vector (and steps whose offsets pass 32 bits).
enum { EVEN = 0, SHIFT = 1, ANY = 2 };

template <typename T, typename S, bool NORM, int ENDS>
__global__ __launch_bounds__(S::TH, S::OCC) void wgrad_kernel(WGradArgs a) {
    constexpr int TM = S::TM, TN = S::TN, WM = S::WM, WN = S::WN, WK = S::WK, BK = S::BK, QB = S::QB, TH = S::TH, SA = S::SA,
                  SB = S::SB, DEPTH = S::DEPTH, FM = S::FM, FN = S::FN, KS = S::KS, VA = S::VA, VB = S::VB, DA = S::DA, DB = S::DB;
    extern __shared__ __align__(16) uint16_t lds[];
    uint16_t *const la = lds, *const lb = lds + 2 * BK * SA;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Work at = work_of(a.tiles_k, a.tiles_c, a.splits);
    // The last tile of K covers the last TM rows of dW, whole, and leaves those of
    // them that the tile before it writes: no vector of dy meets the end of its row
    // (16000 rows, K = 3001, C = 3008: 397 us in fp16 and 394 in bf16, with vectors
    // moved in that tile 660 and 508).
    const int own = at.k * TM, k0 = own + TM > a.K && a.K >= TM ? a.K - TM : own, c0 = at.c * TN;
    const int64_t first = (int64_t)at.split * a.chunk;
    const int64_t last = first + a.chunk < a.rows ? first + a.chunk : a.rows;
    const bool affine = NORM && a.b;
    const bool sums = at.c == 0 || (affine && !a.part);

    const int ka = tid % (TM / 8) * 8, ra = tid / (TM / 8), ca = k0 + ka;
    const int kb = tid % (TN / QB) * QB, rb = tid / (TN / QB), cb = c0 + kb;
    // Sums of fp16 as x * one + sum, which is one instruction with the conversion
    // and takes no registers for it: with a conversion before each sum the large
    // tiles ran out of them (16384 rows, K = C = 4096: 2535 us against 573).
    float db[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f}, one = 1.0f;
    asm("" : "+v"(one));

    // A step's share of a thread, in registers from its fetch to its store.
    struct Stage {
        u32x4 a[VA];
        u32x2 b[VB][QB / 8];
        float s[VB];
        float2 n[VB];
    } stage[DEPTH];

    // Vectors past K or C are loaded from its end instead: what they hold only
    // reaches sums that are not stored.  Rows past the end are loaded
    // from the step's first row and taken as zeros when they are stored.
    // Offsets of a thread's first vectors from the step's first row; those of
    // the others are uniform distances away.
    const uint32_t ld = (uint32_t)(a.lddy * 2), oa = (uint32_t)((ca + 8 <= a.K ? ca : a.K - 8) * 2),
                   ob = (uint32_t)(cb + QB <= a.C ? cb : a.C - QB),
                   os = (uint32_t)(cb < a.C ? cb : a.C - 1) / CKPT_BLOCK * 4;
    const int na = a.K - ca, nb = a.C - cb;  // elements of the thread's vectors in their rows
    const uint32_t ra_at = ra * ld + oa, rb_at = rb * (uint32_t)a.C + ob, rs_at = rb * (uint32_t)a.blocks * 4 + os;
    auto fetch_a = [&](Stage &t, int j, int64_t r) {
        if constexpr (ENDS != ANY) {
            const int left = (int)(last - r < BK ? last - r : BK);
            const uint32_t at = ra + j * DA < left ? ra_at + j * DA * ld : oa;
            t.a[j] = reinterpret_cast<const Any16 *>((const char *)(a.dy + r * a.lddy) + at)->v;
        } else {
            const int64_t row = r + ra + j * DA;
            t.a[j] = row < last ? load8(a.dy + row * a.lddy, ca, a.K) : u32x4{0u, 0u, 0u, 0u};
        }
    };
    auto fetch_b = [&](Stage &t, int j, int64_t r) {
        if constexpr (ENDS != ANY) {
            const int left = (int)(last - r < BK ? last - r : BK);
            const bool in = rb + j * DB < left;
            const char *const p = (const char *)(a.q + r * a.C) + (in ? rb_at + j * DB * (uint32_t)a.C : ob);
            if constexpr (QB == 16) {
                const u32x4 v = reinterpret_cast<const Any16b *>(p)->v;
                t.b[j][0] = u32x2{v[0], v[1]};
                t.b[j][QB / 8 - 1] = u32x2{v[2], v[3]};
            } else {
                t.b[j][0] = reinterpret_cast<const Any8 *>(p)->v;
            }
            t.s[j] = *reinterpret_cast<const float *>((const char *)(a.scale + r * a.blocks) +
                                                      (in ? rs_at + j * DB * (uint32_t)a.blocks * 4 : os));
            if constexpr (NORM)
                t.n[j] = (a.stats + r)[in ? (uint32_t)(rb + j * DB) : 0u];
        } else {
            const int64_t row = r + rb + j * DB;
            t.s[j] = 0.0f;
            t.n[j] = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < QB / 8; i++)
                t.b[j][i] = row < last ? load8b(a.q + row * a.C, cb + 8 * i, a.C) : u32x2{0u, 0u};
            if (row < last && cb < a.C) {
                t.s[j] = a.scale[row * a.blocks + cb / CKPT_BLOCK];
                if constexpr (NORM)
                    t.n[j] = a.stats[row];
            }
        }
    };
    // into buffer `buf`, `left` rows of which are in the split
    auto store_a = [&](auto with_sums, auto shift, Stage &t, int j, int buf, int left) {
        if constexpr (decltype(shift)::value == 2)
            t.a[j] = na > 0 && na < 8 ? from_end(t.a[j], na) : t.a[j];
        if (ra + j * DA >= left)
            t.a[j] = u32x4{0u, 0u, 0u, 0u};
        *reinterpret_cast<u32x4 *>(la + buf * (BK * SA) + (ra + j * DA) * SA + ka) = t.a[j];
        if constexpr (decltype(with_sums)::value) {
            float x[8];
            unpack8<T>(t.a[j], x);
#pragma unroll
            for (int i = 0; i < 8; i++)
                db[i] = T::is_bf16 ? db[i] + x[i] : fmaf(x[i], one, db[i]);
        }
    };
    auto store_b = [&](auto shift, Stage &t, int j, int buf, int left) {
        // The definition's operations in its order.  One step less, q + 128 with an
        // offset of -128 scales passes fp32 for blocks of bf16's largest values, and
        // q (scale rstd) - mean rstd for rows of large equal ones (16384 rows, K = C =
        // 4096 after a norm: fp16 530 us with the latter, 561 as it is, bf16 520 and 535).
        const bool on = rb + j * DB < left;
        const float f = on ? t.s[j] : 0.0f, m = NORM && on ? t.n[j].x : 0.0f, r = NORM && on ? t.n[j].y : 0.0f;
        auto value = [&](uint32_t w, int i) {
            const float q = signed_byte(w, i);
            return NORM ? fmaf(q, f, -m) * r : q * f;
        };
        uint16_t *const p = lb + buf * (BK * SB) + (rb + j * DB) * SB + kb;
        if (decltype(shift)::value != 0 && nb > 0 && nb < QB) {  // the last nb of QB bytes to the front
            uint64_t lo = __builtin_bit_cast(uint64_t, t.b[j][0]);
            uint64_t hi = QB == 16 ? __builtin_bit_cast(uint64_t, t.b[j][QB / 8 - 1]) : 0;
            const int s = 8 * (QB - nb);
            lo = s < 64 ? lo >> s | (QB == 16 ? hi << (64 - s) : 0) : hi >> (s - 64);
            hi = s < 64 ? hi >> s : 0;
            if (QB == 16)
                t.b[j][QB / 8 - 1] = __builtin_bit_cast(u32x2, hi);
            t.b[j][0] = __builtin_bit_cast(u32x2, lo);
        }
#pragma unroll
        for (int i = 0; i < QB / 8; i++) {
            u32x4 v;
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const uint32_t w = t.b[j][i][h];
                v[2 * h] = T::pack2(value(w, 0), value(w, 1));
                v[2 * h + 1] = T::pack2(value(w, 2), value(w, 3));
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
    const int group = wave / (WM * WN), wm = wave / WN % WM * (TM / WM), wn = wave % WN * (TN / WN);

    // Fragments of 16 rows from row 16 k of the group's share of a buffer.
    struct Frags {
        u32x4 a[FM], b[FN];
    };
    const uint16_t *const fa = la + (tr_row + group * KS * 16) * SA + wm + tr_col,
                         *const fb = lb + (tr_row + group * KS * 16) * SB + wn + tr_col;
    auto read = [&](Frags &f, int buf, int k) {
        const uint16_t *const pa = fa + buf * (BK * SA) + 16 * k * SA, *const pb = fb + buf * (BK * SB) + 16 * k * SB;
#pragma unroll
        for (int m = 0; m < FM; m++) {
            const u32x2 lo = read_tr(pa + 32 * m), hi = read_tr(pa + 4 * SA + 32 * m);
            f.a[m] = u32x4{lo.x, lo.y, hi.x, hi.y};
        }
#pragma unroll
        for (int n = 0; n < FN; n++) {
            const u32x2 lo = read_tr(pb + 32 * n), hi = read_tr(pb + 4 * SB + 32 * n);
            f.b[n] = u32x4{lo.x, lo.y, hi.x, hi.y};
        }
    };

    // Step by step.  While a step's products run from one buffer, its
    // fragments read 16 rows ahead, the next step is written from registers to
    // the other buffer, and the step DEPTH further is fetched into them.  The
    // barrier stands before the last 16 rows' products, whose fragments are in
    // registers by then, and behind it the next step's first fragments are
    // read.
    auto run = [&](auto with_sums, auto shift) {
        auto rows_of = [&](int64_t r) { return (int)(last - r < BK ? (last - r < 0 ? 0 : last - r) : BK); };
        auto from = [&](int64_t r) { return r < last ? r : first; };  // past the end: any row, stored as zeros
#pragma unroll
        for (int j = 0; j < VA; j++)
            fetch_a(stage[0], j, first);
#pragma unroll
        for (int j = 0; j < VB; j++)
            fetch_b(stage[0], j, first);
        if constexpr (DEPTH == 2) {
#pragma unroll
            for (int j = 0; j < VA; j++)
                fetch_a(stage[1], j, from(first + BK));
#pragma unroll
            for (int j = 0; j < VB; j++)
                fetch_b(stage[1], j, from(first + BK));
        }
#pragma unroll
        for (int j = 0; j < VA; j++) {
            store_a(with_sums, shift, stage[0], j, 0, rows_of(first));
            fetch_a(stage[0], j, from(first + DEPTH * BK));
        }
#pragma unroll
        for (int j = 0; j < VB; j++) {
            store_b(shift, stage[0], j, 0, rows_of(first));
            fetch_b(stage[0], j, from(first + DEPTH * BK));
        }
        __syncthreads();
        Frags f[2];
        read(f[0], 0, 0);
        // one step from buffer `buf`; t holds the next one
        auto step = [&](Stage &t, int buf, int64_t r) {
            const int left = rows_of(r + BK);
            const int64_t ahead = from(r + (DEPTH + 1) * BK);
#pragma unroll
            for (int k = 0; k < KS; k++) {
                if (k + 1 < KS) {
                    read(f[(k + 1) & 1], buf, k + 1);
#pragma unroll
                    for (int j = VA * k / (KS - 1); j < VA * (k + 1) / (KS - 1); j++) {
                        store_a(with_sums, shift, t, j, buf ^ 1, left);
                        fetch_a(t, j, ahead);
                    }
#pragma unroll
                    for (int j = VB * k / (KS - 1); j < VB * (k + 1) / (KS - 1); j++) {
                        store_b(shift, t, j, buf ^ 1, left);
                        fetch_b(t, j, ahead);
                    }
                } else {
                    __syncthreads();
                    read(f[0], buf ^ 1, 0);
                }
#pragma unroll
                for (int m = 0; m < FM; m++)
#pragma unroll
                    for (int n = 0; n < FN; n++)
                        acc[m][n] = mfma32<T>(f[k & 1].a[m], f[k & 1].b[n], acc[m][n]);
            }
        };
        for (int64_t r = first; r < last; r += 2 * BK) {
            step(stage[DEPTH - 1], 0, r);
            if (r + BK >= last)
                break;
            step(stage[0], 1, r + BK);
        }
        __syncthreads();
    };
    if (first < last) {
        auto choose = [&](auto with_sums) {
            // only the tiles at the end of C, or of a K below TM, have vectors to move
            if constexpr (ENDS == SHIFT) {
                if (k0 + TM > a.K)
                    return run(with_sums, std::integral_constant<int, 2>{});
                if (c0 + TN > a.C)
                    return run(with_sums, std::integral_constant<int, 1>{});
            }
            run(with_sums, std::integral_constant<int, 0>{});
        };
        if (sums)
            choose(std::true_type{});
        else
            choose(std::false_type{});
    }

    // the groups' results, added to the first's in their order
    if constexpr (WK > 1) {
        float *const join = reinterpret_cast<float *>(lds) + (tid % (64 * WM * WN));
#pragma unroll
        for (int g = 1; g < WK; g++) {
            if (group == g)
#pragma unroll
                for (int m = 0; m < FM; m++)
#pragma unroll
                    for (int n = 0; n < FN; n++)
#pragma unroll
                        for (int i = 0; i < 16; i++)
                            join[((m * FN + n) * 16 + i) * (64 * WM * WN)] = acc[m][n][i];
            __syncthreads();
            if (group == 0)
#pragma unroll
                for (int m = 0; m < FM; m++)
#pragma unroll
                    for (int n = 0; n < FN; n++)
#pragma unroll
                        for (int i = 0; i < 16; i++)
                            acc[m][n][i] += join[((m * FN + n) * 16 + i) * (64 * WM * WN)];
            __syncthreads();
        }
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
            if (at.c == 0 && k0 + k >= own && k0 + k < a.K)
                (a.part ? a.part_db + (int64_t)at.split * a.K : a.db)[k0 + k] = f;
        }
        __syncthreads();
    }
    // The results of a lane: column c, rows 8 (i / 4) + 4 (lane / 32) + i % 4 of
    // each MFMA tile.  Rows are a uniform distance apart, which leaves one
    // offset a lane; only the tiles at the end of K check theirs.
    if (group > 0)
        return;
    const int kl = wm + 4 * (lane >> 5), low = own - k0 - kl, lim = a.K - k0 - kl;
    const bool whole = own + TM <= a.K;
    char *const out = a.part ? (char *)(a.part + ((int64_t)at.split * a.K + k0) * a.C) : (char *)(a.dw + (int64_t)k0 * a.C);
    auto put = [&](auto check, auto partial) {
#pragma unroll
        for (int n = 0; n < FN; n++) {
            const int c = c0 + wn + 32 * n + (lane & 31);
            if (c >= a.C)
                continue;
            constexpr int64_t size = decltype(partial)::value ? 4 : 2;
            const uint64_t off = ((uint64_t)kl * (uint64_t)a.C + c) * size;
            const float w = NORM && a.w ? a.w[c] : 1.0f, b = affine ? a.b[c] : 0.0f;
#pragma unroll
            for (int m = 0; m < FM; m++)
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const int row = 32 * m + 8 * (i >> 2) + (i & 3);
                    if (decltype(check)::value && (row < low || row >= lim))
                        continue;
                    char *const o = out + (int64_t)row * a.C * size + off;
                    float f = acc[m][n][i];
                    if constexpr (decltype(partial)::value) {
                        *reinterpret_cast<float *>(o) = f;
                    } else {
                        if constexpr (NORM) {
                            f *= w;
                            if (affine)
                                f = fmaf(b, lsum[kl + row], f);
                        }
                        *reinterpret_cast<uint16_t *>(o) = (uint16_t)T::pack2(f, 0.0f);
                    }
                }
        }
    };
    auto put_as = [&](auto partial) {
        if (whole)
            put(std::false_type{}, partial);
        else
            put(std::true_type{}, partial);
    };
    if (a.part)
        put_as(std::true_type{});
    else
        put_as(std::false_type{});
}

// The sum of the splits: V neighbouring entries of a row of dW a thread, S
// threads of a workgroup share them and add every S-th split.
template <typename T, int V, int S>
__global__ __launch_bounds__(256) void wgrad_reduce_kernel(WGradArgs a, FastDiv per_row, int norm) {
    constexpr int N = 256 / S;
    const int t = threadIdx.x % N, s = threadIdx.x / N;
    const uint32_t i = blockIdx.x * N + t, k = fdiv(i, per_row), c = (i - k * per_row.d) * V;
    const bool on = (int)k < a.K, affine = norm && a.b;
    float f[V] = {}, d = 0.0f;
    if (on) {
        const int64_t pitch = (int64_t)a.K * a.C;
        const float *p = a.part + (int64_t)k * a.C + c, *const pd = a.part_db + k;
        const bool with_db = c == 0 || affine;
#pragma unroll 8
        for (int z = s; z < a.splits; z += S) {
            if constexpr (V == 4) {
                const float4v v = *reinterpret_cast<const float4v *>(p + z * pitch);
#pragma unroll
                for (int e = 0; e < V; e++)
                    f[e] += v[e];
            } else {
                f[0] += p[z * pitch];
            }
            d += with_db ? pd[(int64_t)z * a.K] : 0.0f;
        }
    }
    if constexpr (S > 1) {
        __shared__ float sum[V + 1][S][N];
#pragma unroll
        for (int e = 0; e < V; e++)
            sum[e][s][t] = f[e];
        sum[V][s][t] = d;
        __syncthreads();
        if (s > 0)
            return;
#pragma unroll
        for (int n = 1; n < S; n++) {
#pragma unroll
            for (int e = 0; e < V; e++)
                f[e] += sum[e][n][t];
            d += sum[V][n][t];
        }
    }
    if (!on)
        return;
    if (c == 0)
        a.db[k] = d;
    if (norm)
#pragma unroll
        for (int e = 0; e < V; e++)
            f[e] = fmaf(f[e], a.w ? a.w[c + e] : 1.0f, affine ? a.b[c + e] * d : 0.0f);
    uint16_t *const o = a.dw + (int64_t)k * a.C + c;
    if constexpr (V == 4)
        reinterpret_cast<Any8h *>(o)->v = u32x2{T::pack2(f[0], f[1]), T::pack2(f[2], f[3])};
    else
        *o = (uint16_t)T::pack2(f[0], 0.0f);
}

template <typename T, int V, int S>
hipError_t launch_reduce(const WGradArgs &a, bool norm, hipStream_t st) {
    const uint32_t per_row = (uint32_t)(a.C / V), n = per_row * (uint32_t)a.K;
    wgrad_reduce_kernel<T, V, S><<<dim3((n + 256 / S - 1) / (256 / S)), dim3(256), 0, st>>>(a, make_fastdiv(per_row),
                                                                                            norm);
    return hipGetLastError();
}

// Threads that share entries: enough for 64K threads, each with a few splits.
template <typename T, int V>
hipError_t launch_reduce(const WGradArgs &a, bool norm, hipStream_t st) {
    const int64_t n = (int64_t)a.K * a.C / V;
    if (n >= 65536 || a.splits < 8)
        return launch_reduce<T, V, 1>(a, norm, st);
    if (n >= 16384 || a.splits < 64)
        return launch_reduce<T, V, 4>(a, norm, st);
    return launch_reduce<T, V, 16>(a, norm, st);
}

// Tiles and their waves.
typedef Shape2<64, 64, 2, 2, 1, 64, 16, 2, 3> Tile64;
typedef Shape2<128, 128, 2, 2, 1, 32, 16, 2, 3> Tile128;
typedef Shape2<256, 256, 2, 4, 1, 64, 16, 1, 2> Tile256;
typedef Shape2<256, 64, 4, 2, 1, 64, 8, 2, 2> TileTall;
typedef Shape2<64, 256, 2, 4, 1, 64, 16, 2, 2> TileWide;
typedef Shape2<128, 128, 2, 2, 2, 64, 16, 2, 2> Deep128;
typedef Shape2<64, 64, 2, 2, 4, 128, 8, 2, 4> Deep64;

template <typename T, typename S, bool NORM, int TILE>
hipError_t launch_tile(const WGradArgs &a, hipStream_t st) {
    constexpr wgrad::Tile t = wgrad::TILES[TILE];
    static_assert(S::TM == t.m && S::TN == t.n && S::TH == 64 * t.waves && S::QB == t.qb, "what the plan counts with");
    const bool small = a.lddy * 2 * S::BK < (int64_t)1 << 31 && (int64_t)a.C * S::BK < (int64_t)1 << 31;
    const int ends = a.K < 8 || a.C < S::QB || !small ? ANY : a.K % 8 || a.C % S::QB ? SHIFT : EVEN;
    void (*const f)(WGradArgs) = ends == EVEN    ? wgrad_kernel<T, S, NORM, EVEN>
                                 : ends == SHIFT ? wgrad_kernel<T, S, NORM, SHIFT>
                                                 : wgrad_kernel<T, S, NORM, ANY>;
    if (S::LDS > 64 * 1024) {
        const hipError_t e = allow_full_lds((const void *)f);
        if (e != hipSuccess)
            return e;
    }
    const unsigned grid = (unsigned)a.tiles_k * a.tiles_c * a.splits;
    f<<<dim3(grid), dim3(S::TH), S::LDS, st>>>(a);
    return hipGetLastError();
}

template <typename T, bool NORM>
hipError_t launch_type(const WGradArgs &a, int tile, hipStream_t st) {
    hipError_t e;
    switch (tile) {
    case 0: e = launch_tile<T, Tile64, NORM, 0>(a, st); break;
    case 1: e = launch_tile<T, Tile128, NORM, 1>(a, st); break;
    case 2: e = launch_tile<T, Tile256, NORM, 2>(a, st); break;
    case 3: e = launch_tile<T, TileTall, NORM, 3>(a, st); break;
    case 4: e = launch_tile<T, TileWide, NORM, 4>(a, st); break;
    case 5: e = launch_tile<T, Deep128, NORM, 5>(a, st); break;
    default: e = launch_tile<T, Deep64, NORM, 6>(a, st); break;
    }
    if (e != hipSuccess || a.splits == 1)
        return e;
    return a.C % 4 ? launch_reduce<T, 1>(a, NORM, st) : launch_reduce<T, 4>(a, NORM, st);
}

}  // namespace

}  // namespace cf
