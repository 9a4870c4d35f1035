// cf_mm.h -- tiles of 16-bit matrix products out[m][n] = sum_k A(m, k) B(n, k)
// for the gated feed-forward block and the log probabilities from features,
// with what follows each product fused behind it.
//
// An operand is stored with k contiguous (KC: x W^T has both so) or with its
// other index contiguous (RC: gradients sum over rows or over outputs).  A
// workgroup makes a TM x TN tile.  Steps of 32 k go by LDS-DMA into a ring of
// STAGES buffers, as the instruction writes them: 16 bytes a lane, one after
// the other.  A lane chooses what it fetches, so that the tile stands there
// swizzled and the fragment reads meet no bank twice:
//   KC  rows of 64 bytes, their 16-byte pieces permuted by bits 1 and 2 of the row;
//       fragments by 16-byte loads
//   RC  rows of one k, their 32-byte pieces permuted by the lowest bits of k;
//       fragments by transposing loads, whose 16 lanes read 32 bytes of 4 rows.
//       Rows of 512 bytes: one bit, and 64 bytes between pairs of rows (two
//       bits, or three, took eight addresses a lane, and the tile spilled)
// While the products of a step run, the next step's fragments are read into a
// second set of registers and the step STAGES further is fetched: one barrier a
// step, and no wait but for copies issued STAGES - 1 steps before.
//
// MFMA 16x16x32 takes B's fragment first: a lane then holds four consecutive n
// of one m, which is what a store, a sum over n or a pair of gate and up
// channels wants.
//
// The ends: rows of A and B past the last are read from the last (they reach
// results that are not stored), k past the last from a page of zeros.  So an
// operand must have 16-byte aligned rows whose contiguous extent is a multiple
// of 8 (zeros behind the last k of KC); others are packed first (cf_mm.hip).
#pragma once

#include "cf_device.h"
#include "cf_kernels.h"
#include "cf_mm_plan.h"

namespace cf {
namespace mm {

enum { KC = 0, RC = 1 };

struct Args {
    const uint16_t *a[2], *b[2];
    int64_t lda, ldb;     // of both
    int M, N, K;          // K of one segment
    int ext_a, ext_b;     // rows of a (KC), or the columns that its rows hold (RC); the same of b
    int seg;              // steps of the first segment of k (behind it a[1], b[1]), or all
    int steps;            // of both
    int per;              // steps a split
    int tiles_m, tiles_n, splits;
    int batch;            // 2: a[1] and out[1] are a second problem with the same b[0]
};

struct Work {
    int m, n, split, batch;
};
// Workgroups go to the eight XCDs in turn, each with an L2 of its own; every XCD
// takes a run of the list of tiles, in bands eight tiles of m high, so that what
// runs together behind one L2 shares rows of both operands.
__device__ __forceinline__ Work work_of(const Args &a) {
    const unsigned n = gridDim.x, xcd = blockIdx.x & 7, q = n >> 3, rest = n & 7;
    unsigned i = xcd * q + (xcd < rest ? xcd : rest) + (blockIdx.x >> 3);
    const unsigned tiles = (unsigned)a.tiles_m * (unsigned)a.tiles_n, part = i / tiles;
    i -= part * tiles;
    const unsigned band = i / (8u * a.tiles_n), m0 = 8 * band,
                   high = (unsigned)a.tiles_m - m0 < 8 ? a.tiles_m - m0 : 8;
    i -= band * 8 * a.tiles_n;
    return {(int)(m0 + i % high), (int)(i / high), (int)(part / a.batch), (int)(part % a.batch)};
}

// the 1024 bytes of a copy instruction, and what is left free behind them
template <int L, int R>
constexpr int PITCH = L == RC && R == 256 ? 1088 : 1024;
template <int L, int R>
constexpr int BYTES = R * STEP * 2 / 1024 * PITCH<L, R>;

template <int TM_, int TN_, int WM_, int WN_, int OCC_>
struct Shape {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, OCC = OCC_;
    static constexpr int TH = 64 * WM * WN, FM = TM / WM / 16, FN = TN / WN / 16;
    static constexpr int COPIES = (TM + TN) * STEP * 2 / (TH * 16);  // LDS-DMA instructions of a wave and stage
    static_assert(TM * STEP * 2 % (TH * 16) == 0 && TN * STEP * 2 % (TH * 16) == 0, "whole copies");
};

static __device__ __attribute__((aligned(16))) const uint32_t zero_page[4] = {0, 0, 0, 0};

// 16 bytes a lane from base + voff to LDS address lds + 16 lane
__device__ __forceinline__ void copy16(const void *base, uint32_t voff, uint32_t lds) {
    asm volatile(
        "s_mov_b32 m0, %2\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %0, %1"
        :
        : "v"(voff), "s"(base), "s"(lds)
        : "memory", "m0");
}
// the same from an address a lane
__device__ __forceinline__ void copy16_any(const void *p, uint32_t lds) {
    asm volatile(
        "s_mov_b32 m0, %1\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %0, off"
        :
        : "v"((uint64_t)(uintptr_t)p), "s"(lds)
        : "memory", "m0");
}

// all but the last n copies of this wave have arrived
template <int N>
__device__ __forceinline__ void wait_copies() {
    static_assert(N < 64, "six bits");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

template <int R>
__device__ __forceinline__ int rc_swizzle(int k) {
    return R == 256 ? k & 1 : k & 3;
}

// 4 k x 16 columns of an RC tile, given as 4 columns of row lane / 4 by each of
// 16 lanes; the lane gets its column's 4 k
__device__ __forceinline__ u32x2 read_tr(const uint8_t *p) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p));
}

// One operand's copies: R rows (columns) of the tile from r0 on.  DUAL: groups of
// 16 rows come from two matrices in turn, r0 / 2 being the first row of either.
template <int L, int R, int TH, bool DUAL>
struct Copies {
    static constexpr int N = R * STEP * 2 / (TH * 16);
    uint32_t off[N];
    int k[N];  // the first k of this lane's 16 bytes within a step

    __device__ __forceinline__ void init(int tid, int r0, int ext, int64_t ld) {
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int s = i * TH + tid;
            if constexpr (L == KC) {
                const int row = s >> 3, c = (s & 7) ^ (row & 7);
                const int at = DUAL ? (row >> 5) * 16 + (row & 15) : row, first = DUAL ? r0 / 2 : r0;
                const int r = first + at < ext ? at : ext - 1 - first;
                off[i] = (uint32_t)r * (uint32_t)(ld * 2) + c * 16;
                k[i] = c * 8;
            } else {
                constexpr int PER = R / 8;
                const int kk = s / PER, p = s % PER;
                const int col = (((p >> 1) ^ rc_swizzle<R>(kk)) << 4) + (p & 1) * 8;
                const int c = r0 + col <= ext - 8 ? col : ext - 8 - r0;
                off[i] = (uint32_t)kk * (uint32_t)(ld * 2) + c * 2;
                k[i] = kk;
            }
        }
    }
    // The i-th copy of a step from the tile's first row of each matrix, `left` k's
    // of them.
    __device__ __forceinline__ void issue(int i, const uint16_t *p0, const uint16_t *p1, int left, uint32_t lds,
                                          int wave) const {
        const uint16_t *const p = DUAL && (((i * TH / 64 + wave) >> 1) & 1) ? p1 : p0;
        const uint32_t to = lds + (i * TH / 64 + wave) * PITCH<L, R>;
        if (left >= STEP)
            copy16(p, off[i], to);
        else
            copy16_any(k[i] < left ? (const uint8_t *)p + off[i] : (const uint8_t *)zero_page, to);
    }
};

template <int L, int R>
struct Reader {
    // this lane's places in a stage for rows (columns) w0 + 16 i .., k's from 32 h on
    static constexpr int N = L == KC ? 2 : R == 256 ? 2 : 4;
    static constexpr int ROW = R * 2, PER = 1024 / ROW;  // RC: bytes of a row, rows of a copy
    int at[N];
    __device__ __forceinline__ void init(int lane, int w0) {
        if constexpr (L == KC) {
            const int r = lane & 15;
            at[0] = (w0 + r) * 128 + (((lane >> 4) ^ (r & 7)) << 4);
            at[1] = at[0] ^ 64;
        } else {
            const int k = 8 * (lane >> 4) + ((lane & 15) >> 2);
#pragma unroll
            for (int i = 0; i < N; i++)  // w0 / 16 is a multiple of N
                at[i] = k / PER * PITCH<L, R> + k % PER * ROW + w0 * 2 + ((i ^ rc_swizzle<R>(k)) << 5) + 8 * (lane & 3);
        }
    }
    __device__ __forceinline__ u32x4 get(const uint8_t *stage, int h, int i) const {
        if constexpr (L == KC) {
            return *reinterpret_cast<const u32x4 *>(stage + at[h] + i * 2048);
        } else {
            const uint8_t *const p = stage + at[i % N] + i / N * (N * 32) + h * (32 / PER * PITCH<L, R>);
            const u32x2 lo = read_tr(p), hi = read_tr(p + 4 / PER * PITCH<L, R>);
            return u32x4{lo.x, lo.y, hi.x, hi.y};
        }
    }
};

// E: what follows the product.  E::DUAL as above; E::Args; run(args, acc, work,
// mm args, wave's first m and n, lane, LDS).
template <typename T, typename S, int LA, int LB, typename E>
__global__ __launch_bounds__(S::TH, S::OCC) void kernel(Args a, typename E::Args e) {
    constexpr int TM = S::TM, TN = S::TN, FM = S::FM, FN = S::FN;
    constexpr int BYTES_A = BYTES<LA, TM>, STAGE = BYTES_A + BYTES<LB, TN>;
    static_assert(FM % 4 == 0 && FN % 4 == 0, "a wave's first row and column");
    extern __shared__ __align__(1024) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Work at = work_of(a);
    const int m0 = at.m * TM, n0 = at.n * TN;
    const int wm = wave / S::WN * (TM / S::WM), wn = wave % S::WN * (TN / S::WN);

    const int first = at.split * a.per;
    int steps = a.steps - first < a.per ? a.steps - first : a.per;
    steps = steps < 0 ? 0 : steps;

    Copies<LA, TM, S::TH, false> ca;
    Copies<LB, TN, S::TH, E::DUAL> cb;
    ca.init(tid, m0, a.ext_a, a.lda);
    cb.init(tid, n0, a.ext_b, a.ldb);
    Reader<LA, TM> ra;
    Reader<LB, TN> rb;
    ra.init(lane, wm);
    rb.init(lane, wn);
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;

    // The next step to fetch: its place in its segment of k, its buffer and what is
    // left of k.  Everything here is uniform.
    const int64_t step_a = LA == KC ? STEP : STEP * a.lda,
                  step_b = LB == KC ? STEP : STEP * a.ldb;
    const int64_t row_a = LA == KC ? (int64_t)m0 * a.lda : m0,
                  row_b = LB == KC ? (int64_t)(E::DUAL ? n0 / 2 : n0) * a.ldb : n0;
    struct Next {
        const uint16_t *a, *b, *b1;
        int left, segment, buffer;
    } nx;
    {
        const int two = first >= a.seg, in = two ? first - a.seg : first;
        nx.a = a.a[two | at.batch] + row_a + in * step_a;
        nx.b = a.b[E::DUAL ? 0 : two] + row_b + in * step_b;
        nx.b1 = E::DUAL ? a.b[1] + row_b + in * step_b : nullptr;
        nx.left = a.K - in * STEP;
        nx.segment = two ? 1 << 30 : a.seg - first;  // steps to its end
        nx.buffer = 0;
    }
    constexpr int CA = Copies<LA, TM, S::TH, false>::N, CB = Copies<LB, TN, S::TH, E::DUAL>::N;
    auto copy = [&](int i) {  // the i-th of the step's copies
        const uint32_t to = lds_at + nx.buffer * STAGE;
        if (i < CA)
            ca.issue(i, nx.a, nullptr, nx.left, to, wave);
        else
            cb.issue(i - CA, nx.b, nx.b1, nx.left, to + BYTES_A, wave);
    };
    auto advance = [&] {
        nx.a += step_a;
        nx.b += step_b;
        nx.b1 += E::DUAL ? step_b : 0;
        nx.left -= STEP;
        nx.buffer ^= 1;
        if (--nx.segment == 0) {
            nx.a = a.a[1] + row_a;
            nx.b = a.b[1] + row_b;
            nx.left = a.K;
            nx.segment = 1 << 30;
        }
    };

    float4v acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < FN; j++)
            acc[i][j] = float4v{0.0f, 0.0f, 0.0f, 0.0f};

    struct Frags {
        u32x4 a[FM], b[FN];
    } f[2];
    auto read = [&](Frags &t, const uint8_t *stage, int h, int i) {  // the i-th fragment of 32 k's
        if (i < FN)
            t.b[i] = rb.get(stage + BYTES_A, h, i);
        else
            t.a[i - FN] = ra.get(stage, h, i - FN);
    };
    auto barrier = [&] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // The products of 32 k's in FM groups, each of which starts with a share of what
    // goes on beside them: the next fragments' reads and, in the second half of a
    // step, the copies of the step after the next.
    constexpr int READS = FM + FN, PER = (READS + FM - 2) / (FM - 1);  // no reads in the last group
    auto half = [&](const Frags &now, Frags &next, const uint8_t *from, int h, bool copies) {
#pragma unroll
        for (int i = 0; i < FM; i++) {
#pragma unroll
            for (int r = i * PER; r < (i + 1) * PER; r++)
                if (r < READS)
                    read(next, from, h, r);
            if (copies) {
#pragma unroll
                for (int c = 0; c < S::COPIES; c++)
                    if (c * FM / S::COPIES == i)
                        copy(c);
            }
#pragma unroll
            for (int j = 0; j < FN; j++)
                acc[i][j] = T::mfma(now.b[j], now.a[i], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    if (steps > 0) {
        for (int s = 0; s < 2 && s < steps; s++) {
#pragma unroll
            for (int c = 0; c < S::COPIES; c++)
                copy(c);
            advance();
        }
        if (steps > 1)
            wait_copies<S::COPIES>();
        else
            wait_copies<0>();
        barrier();
#pragma unroll
        for (int r = 0; r < READS; r++)
            read(f[0], lds, 0, r);
        const uint8_t *now = lds, *next = lds + STAGE;
        for (int s = 0; s < steps; s++) {
            half(f[0], f[1], now, 1, false);
            // This wave has read all of the step, and its share of the next one is there.
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            barrier();
            // (behind the last step: fragments that nobody uses)
            half(f[1], f[0], next, 0, s + 2 < steps);
            if (s + 2 < steps)
                advance();
            const uint8_t *const t = now;
            now = next;
            next = t;
        }
    }
    E::template run<T, S>(e, acc, at, a, m0 + wm, n0 + wn, lane, lds);
}

template <typename T, typename S, int LA, int LB, typename E>
hipError_t launch(const Args &a, const typename E::Args &e, hipStream_t st) {
    void (*const f)(Args, typename E::Args) = kernel<T, S, LA, LB, E>;
    constexpr int LDS = 2 * (BYTES<LA, S::TM> + BYTES<LB, S::TN>);
    if (LDS > 64 * 1024) {
        const hipError_t err = allow_full_lds((const void *)f);
        if (err != hipSuccess)
            return err;
    }
    const int64_t grid = (int64_t)a.tiles_m * a.tiles_n * a.splits * a.batch;
    f<<<dim3((unsigned)grid), dim3(S::TH), LDS, st>>>(a, e);
    return hipGetLastError();
}

// the plan's tiles
typedef Shape<256, 256, 2, 4, 2> Tile256;
typedef Shape<128, 128, 2, 2, 2> Tile128;

template <typename T, int LA, int LB, typename E>
hipError_t launch_tile(const Args &a, const typename E::Args &e, int tile, hipStream_t st) {
    static_assert(Tile256::TM == TILES[0].m && Tile256::TN == TILES[0].n && Tile128::TM == TILES[1].m &&
                      Tile128::TN == TILES[1].n, "what the plan counts with");
    return tile == 0 ? launch<T, Tile256, LA, LB, E>(a, e, st) : launch<T, Tile128, LA, LB, E>(a, e, st);
}

}  // namespace mm
}  // namespace cf
