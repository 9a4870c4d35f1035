// cf_mm.h -- tiles of 16-bit matrix products out[m][n] = sum_k A(m, k) B(n, k)
// for the gated feed-forward block and the log probabilities from features,
// with what follows each product fused behind it.
//
// An operand is stored with k contiguous (KC: x W^T has both so) or with its
// other index contiguous (RC: gradients sum over rows or over outputs).  A
// workgroup makes TM x TN tiles, one after the other.  Steps of 64 k go by LDS-DMA
// into two buffers, as the instruction writes them: 16 bytes a lane, one after the
// other.  A lane chooses what it fetches, so that the tile stands there permuted
// and fragment reads meet no bank twice:
//   KC  rows of 128 bytes, a cache line each (half a line a step costs a fifth of
//       the rate), in pieces of 16; fragments by 16-byte loads
//   RC  rows of one k, their 32-byte pieces permuted by the lowest bits of k;
//       fragments by transposing loads, whose 16 lanes read 32 bytes of 4 rows.
//       Rows of 512 bytes: one bit, and 32 bytes between pairs of rows (three
//       bits took eight addresses a lane, and the tile spilled)
// While the products of half a step run, the next half's fragments are read into
// a second set of registers; once everyone has read a step, its buffer receives
// the step after the next: one barrier a step.  The copies run on through the
// ends of tiles.
//
// MFMA 16x16x32 takes B's fragment first: a lane then holds columns beside each
// other of one row, which is what a store, a sum over columns or a pair of gate and up
// channels wants.  (32x32x16 keeps the matrix unit busier, 72% against 68, at a
// lower clock: 1287 TFLOP/s against 1350.)
//
// The ends: rows of A and B past the last are read from the last (they reach
// results that are not stored); k's past the last are read from the step's first
// and cleared in LDS.  So an operand must have 16-byte aligned rows whose
// contiguous extent is a multiple of 8 (zeros behind the last k of KC); others are
// packed first (cf_mm.hip).
//
// Bound by the matrix unit and the power it draws: 8192 x 8192 x 8192 in bf16 runs
// at 1360 TFLOP/s (KC, KC), 1361 (KC, RC) and 1332 (RC, RC), the unit 64 to 71% busy
// at 2.0 GHz; nobody waits for LDS (27% busy, no conflicts).
#pragma once

#include "cf_device.h"
#include "cf_kernels.h"
#include "cf_mm_plan.h"

namespace cf {
namespace mm {

enum { KC = 0, RC = 1 };

struct Work {
    int m, n, split, batch;
};
// The item that comes `turn`-th.  Workgroups, and with them their items, go to the
// eight XCDs in turn, each with an L2 of its own; every XCD takes a run of the list of
// tiles, in bands eight tiles of m high, so that what runs together behind one L2
// shares rows of both operands.
__device__ __forceinline__ Work work_of(const Args &a, unsigned turn) {
    const unsigned n = a.items, xcd = turn & 7, q = n >> 3, rest = n & 7;
    unsigned i = xcd * q + (xcd < rest ? xcd : rest) + (turn >> 3);
    const unsigned tiles = (unsigned)a.tiles_m * (unsigned)a.tiles_n, part = i / tiles;
    i -= part * tiles;
    const unsigned band = i / (8u * a.tiles_n), m0 = 8 * band,
                   high = (unsigned)a.tiles_m - m0 < 8 ? a.tiles_m - m0 : 8;
    i -= band * 8 * a.tiles_n;
    return {(int)(m0 + i % high), (int)(i / high), (int)(part / a.batch), (int)(part % a.batch)};
}

// the 1024 bytes of a copy instruction, and what is left free behind them
template <int L, int R>
constexpr int PITCH = L == KC ? 1024 : R == 256 ? 1056 : 1088;
template <int L, int R>
constexpr int BYTES = R * STEP * 2 / 1024 * PITCH<L, R>;

template <int TM_, int TN_, int WM_, int WN_, int OCC_>
struct Shape {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, OCC = OCC_;
    static constexpr int TH = 64 * WM * WN, FM = TM / WM / 16, FN = TN / WN / 16;
    static constexpr int COPIES = (TM + TN) * STEP * 2 / (TH * 16);  // LDS-DMA instructions of a wave and stage
    static_assert(TM * STEP * 2 % (TH * 16) == 0 && TN * STEP * 2 % (TH * 16) == 0, "whole copies");
};

// 16 bytes a lane from base + voff to LDS address lds + AT + 16 lane
template <int AT>
__device__ __forceinline__ void copy16(const void *base, uint32_t voff, uint32_t lds) {
    const uint64_t b = (uint64_t)(uintptr_t)base;
    const uint64_t uniform = ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)) << 32) |
                             (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b);
    asm volatile(
        "s_add_u32 m0, %2, %3\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %0, %1"
        :
        : "v"(voff), "s"(uniform), "s"(lds), "n"(AT)
        : "memory", "m0", "scc");
}

// all but the last n copies of this wave have arrived
template <int N>
__device__ __forceinline__ void wait_copies() {
    static_assert(N < 64, "six bits");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

// What the 16-byte pieces of a KC row are permuted by: 8 lanes beside each other
// read 8 rows in different banks.  B's rows of a fragment are 4 of every 8.
template <bool B>
__device__ __forceinline__ int kc_swizzle(int row) {
    return B ? (row & 3) | (row >> 1 & 4) : row & 7;
}
// By what the 32-byte pieces of row k of an RC tile are permuted: with what is free
// behind a copy, the 8 rows that 32 lanes read together (8 q to 8 q + 3 and 8
// further) lie in different banks.
template <int R>
__device__ __forceinline__ int rc_swizzle(int k) {
    return R == 256 ? (k & 1) << 1 : k & 3;
}

// 4 k x 16 columns of an RC tile, given as 4 columns of row lane / 4 by each of
// 16 lanes; the lane gets its column's 4 k
__device__ __forceinline__ u32x2 read_tr(const uint8_t *p) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p));
}

// One operand's copies: R rows (columns) of the tile from r0 on.  DUAL: groups of
// 32 rows come from two matrices in turn, r0 / 2 being the first row of either.
template <int L, int R, int TH, bool B, bool DUAL>
struct Copies {
    static constexpr int N = R * STEP * 2 / (TH * 16);
    static constexpr int ROWS = L == KC ? TH / 8 : TH / (R / 8);  // rows (k's) between a lane's copies
    static_assert(L == KC ? ROWS % 16 == 0 : ROWS % 4 == 0, "the same piece of each row");
    uint32_t off[L == KC ? N : 1], col;  // RC: of the first copy, of its columns alone
    int k;                          // the first k of this lane's 16 bytes (RC: of the first copy)

    __device__ __forceinline__ void init(int tid, int r0, int ext, int64_t ld) {
        if constexpr (L == KC) {
            const int c = (tid & 7) ^ kc_swizzle<B>(tid >> 3);
            k = c * 8;
#pragma unroll
            for (int i = 0; i < N; i++) {
                const int row = i * ROWS + (tid >> 3);
                const int at = DUAL ? (row >> 6) * 32 + (row & 31) : row, first = DUAL ? r0 / 2 : r0;
                const int r = first + at < ext ? at : ext - 1 - first;
                off[i] = (uint32_t)r * (uint32_t)(ld * 2) + c * 16;
            }
        } else {
            constexpr int PER = R / 8;
            const int p = tid % PER;
            k = tid / PER;
            const int at = (((p >> 1) ^ rc_swizzle<R>(k)) << 4) + (p & 1) * 8;
            const int c = r0 + at <= ext - 8 ? at : ext - 8 - r0;
            col = c * 2;
            off[0] = (uint32_t)k * (uint32_t)(ld * 2) + col;
        }
    }
    // The I-th copy of a step of which `left` k's are there, from the tile's first row
    // of each matrix, to `lds`, the wave's place.  k's past them are read from the
    // step's first, and cleared once they are in LDS.
    template <int I>
    __device__ __forceinline__ void issue(const uint16_t *p0, const uint16_t *p1, uint32_t row, int left, uint32_t lds,
                                          int wave) const {
        constexpr int AT = I * (TH / 64) * PITCH<L, R>;
        if constexpr (L == KC) {
            static_assert(!DUAL || TH / 64 % 4 == 0, "groups of 32 rows are 4 waves' copies");
            copy16<AT>(DUAL && ((wave / 4 + I * (TH / 256)) & 1) ? p1 : p0, off[I] - (k < left ? 0u : (uint32_t)k * 2), lds);
        } else {
            copy16<AT>(p0, k < left - I * ROWS ? off[0] + I * ROWS * row : col, lds);
        }
    }
    __device__ __forceinline__ void clear(int left, uint8_t *stage, int wave, int lane) const {
#pragma unroll
        for (int i = 0; i < N; i++)
            if (k + (L == RC ? i * ROWS : 0) >= left)
                *reinterpret_cast<u32x4 *>(stage + (i * TH / 64 + wave) * PITCH<L, R> + lane * 16) = u32x4{0u, 0u, 0u, 0u};
    }
};

// Fragments of 16 rows (columns) from w0 on.  A's are in order.  B's of a KC tile are
// ordered so that two beside each other give a lane 8 columns beside each other:
// row d of fragment i is row 32 (i / 2) + 8 (d / 4) + 4 (i % 2) + d % 4.
template <int L, int R, bool B>
struct Reader {
    // this lane's places in a stage for rows (columns) w0 + 16 i .., k's from 32 h on
    // (RC: of the i that differ in the bits that rows permute)
    static constexpr int N = L == KC ? 2 : R == 256 ? 2 : 4;
    static constexpr int ROW = R * 2, PER = 1024 / ROW;  // RC: bytes of a row, rows of a copy
    int at[N];
    static constexpr int which(int i) { return R == 256 ? i >> 1 & 1 : i & 3; }
    static constexpr int rest(int i) { return R == 256 ? i & ~2 : i & ~3; }
    __device__ __forceinline__ void init(int lane, int w0) {
        if constexpr (L == KC) {
            const int d = lane & 15, r = w0 + (B ? (d >> 2) * 8 + (d & 3) : d);
            at[0] = r * 128 + (((lane >> 4) ^ kc_swizzle<B>(r)) << 4);
            at[1] = at[0] ^ 64;
        } else {
            const int k = 8 * (lane >> 4) + ((lane & 15) >> 2);
#pragma unroll
            for (int i = 0; i < N; i++)  // w0 / 16 is a multiple of 4
                at[i] = k / PER * PITCH<L, R> + k % PER * ROW + w0 * 2 + 8 * (lane & 3) +
                        (((R == 256 ? 2 * i : i) ^ rc_swizzle<R>(k)) << 5);
        }
    }
    __device__ __forceinline__ u32x4 get(const uint8_t *stage, int h, int i) const {
        if constexpr (L == KC) {
            return *reinterpret_cast<const u32x4 *>(stage + at[h] + (B ? i / 2 * 32 + i % 2 * 4 : i * 16) * 128);
        } else {
            const uint8_t *const p = stage + at[which(i)] + rest(i) * 32 + h * (32 / PER * PITCH<L, R>);
            const u32x2 lo = read_tr(p), hi = read_tr(p + 4 / PER * PITCH<L, R>);
            return u32x4{lo.x, lo.y, hi.x, hi.y};
        }
    }
};

template <int V>
struct Number {
    static constexpr int value = V;
};
// f(Number<0>()) .. f(Number<N - 1>())
template <int N, int I = 0, typename F>
__device__ __forceinline__ void each(F &&f) {
    if constexpr (I < N) {
        f(Number<I>());
        each<N, I + 1>(f);
    }
}

// A wave's results: FM rows a lane (16 apart), in PIECES pieces of W = 8 columns
// beside each other.  With B in KC its fragments are read so that two of them make a
// piece; with B in RC every fragment has 16 columns that lie together, 4 a lane,
// and lanes 16 apart exchange halves of two (`gather`): 16 instructions for 64
// results, for stores of 16 bytes a lane in place of 8.
template <typename S, bool GATHERED>
struct Results {
    static constexpr int W = 8, PIECES = S::FN / 2;
    float4v (&acc)[S::FM][S::FN];
    __device__ __forceinline__ void gather() const {
        if constexpr (GATHERED) {
#pragma unroll
            for (int i = 0; i < S::FM; i++)
#pragma unroll
                for (int p = 0; p < S::FN; p += 2)
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[i][p][k]),
                                                                        __float_as_uint(acc[i][p + 1][k]), false, false);
                        acc[i][p][k] = __uint_as_float(r[0]);
                        acc[i][p + 1][k] = __uint_as_float(r[1]);
                    }
        }
    }
    static __device__ __forceinline__ int column(int piece, int lane) {
        const int q = lane >> 4;
        return 32 * piece + (GATHERED ? 16 * (q & 1) + 8 * (q >> 1) : 8 * q);
    }
    __device__ __forceinline__ float get(int i, int piece, int k) const { return acc[i][2 * piece + k / 4][k % 4]; }
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
    const int wm = wave / S::WN * (TM / S::WM), wn = wave % S::WN * (TN / S::WN);

    Copies<LA, TM, S::TH, false, false> ca;
    Copies<LB, TN, S::TH, true, E::DUAL> cb;
    Reader<LA, TM, false> ra;
    Reader<LB, TN, true> rb;
    ra.init(lane, wm);
    rb.init(lane, wn);
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;

    // The next step to fetch, which may be of the next item: where it is, which item
    // and how many more steps of it there are, its buffer and what is left of k.
    // Everything here is uniform.
    const int64_t step_a = LA == KC ? STEP : STEP * a.lda,
                  step_b = LB == KC ? STEP : STEP * a.ldb;
    struct Next {
        const uint16_t *a, *b, *b1;
        int64_t row_a, row_b;
        unsigned item;
        int left, segment, buffer, steps, first, batch;
    } nx;
    auto steps_of = [&](const Work &w) {
        const int left = a.steps - w.split * a.per;
        return left < a.per ? left : a.per;
    };
    auto restart = [&] {  // to the first step of the item that was entered last
        const int two = nx.first >= a.seg, in = two ? nx.first - a.seg : nx.first;
        nx.a = (two | nx.batch ? a.a[1] : a.a[0]) + nx.row_a + in * step_a;
        nx.b = (!E::DUAL && (two | nx.batch) ? a.b[1] : a.b[0]) + nx.row_b + in * step_b;
        nx.b1 = E::DUAL ? a.b[1] + nx.row_b + in * step_b : nullptr;
        nx.left = a.K - in * STEP;
        nx.segment = two ? 1 << 30 : a.seg - nx.first;  // steps to its end
    };
    auto enter = [&] {
        const Work w = work_of(a, nx.item);
        const int m0 = w.m * TM, n0 = w.n * TN;
        nx.first = w.split * a.per;
        nx.batch = w.batch;
        ca.init(tid, m0, a.ext_a, a.lda);
        cb.init(tid, n0, a.ext_b, a.ldb);
        nx.row_a = LA == KC ? (int64_t)m0 * a.lda : m0;
        nx.row_b = LB == KC ? (int64_t)(E::DUAL ? n0 / 2 : n0) * a.ldb : n0;
        nx.steps = steps_of(w);
        restart();
    };
    constexpr int CA = Copies<LA, TM, S::TH, false, false>::N, CB = Copies<LB, TN, S::TH, true, E::DUAL>::N;
    static_assert(CA + CB == S::COPIES, "");
    const uint32_t row_bytes_a = (uint32_t)(a.lda * 2), row_bytes_b = (uint32_t)(a.ldb * 2);
    const uint32_t to_a = lds_at + wave * PITCH<LA, TM>, to_b = lds_at + BYTES_A + wave * PITCH<LB, TN>;
    auto copy = [&](auto which) {  // one of the step's copies
        constexpr int I = decltype(which)::value;
        const uint32_t buffer = (uint32_t)__builtin_amdgcn_readfirstlane(nx.buffer) * STAGE;
        if constexpr (I < CA)
            ca.template issue<I>(nx.a, nullptr, row_bytes_a, nx.left, to_a + buffer, wave);
        else
            cb.template issue<I - CA>(nx.b, nx.b1, row_bytes_b, nx.left, to_b + buffer, wave);
    };
    auto advance = [&] {
        nx.a += step_a;
        nx.b += step_b;
        nx.b1 += E::DUAL ? step_b : 0;
        nx.left -= STEP;
        nx.buffer ^= 1;
        if (--nx.segment == 0) {
            nx.a = a.a[1] + nx.row_a;
            nx.b = a.b[1] + nx.row_b;
            nx.left = a.K;
            nx.segment = 1 << 30;
        }
        if (--nx.steps == 0) {
            nx.item += gridDim.x;
            if (nx.item < a.items)
                enter();
        }
    };

    float4v acc[FM][FN];
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
    // The products of 32 k's, and one after the other between them what goes on
    // beside them: the next fragments' reads and, with COPIES, the copies of the
    // step after the next.  A product keeps the matrix unit busy for four
    // instructions' time; what stands in that shadow costs nothing.  There is no
    // branch: with another version of the loop for the ends the registers spill.
    constexpr int READS = FM + FN, PRODUCTS = FM * FN;
    auto half = [&](const Frags &now, Frags &next, const uint8_t *from, int h, auto copies) {
        constexpr int COPIES = decltype(copies)::value, PIECES = READS + COPIES;
        each<PRODUCTS>([&](auto product) {
            constexpr int T0 = decltype(product)::value, I = T0 / FN, J = T0 % FN;
            acc[I][J] = T::mfma(now.b[J], now.a[I], acc[I][J]);
            // (products have no side effects: without this they are gathered behind
            // the copies, which are volatile)
            asm volatile("" ::"v"(acc[I][J]));
            // reads and copies in turn, over all products but the last few
            each<PIECES>([&](auto piece) {
                constexpr int P = decltype(piece)::value;
                if constexpr (P * (PRODUCTS - 2) / PIECES == T0) {
                    if constexpr (COPIES == 0)
                        read(next, from, h, P);
                    else if constexpr (P < 2 * COPIES && P % 2 == 1)
                        copy(Number<P / 2>());
                    else
                        read(next, from, h, P < 2 * COPIES ? P / 2 : P - COPIES);
                }
            });
            __builtin_amdgcn_sched_barrier(0);
        });
    };

    // what is left of k in the step that lies in a buffer, where that is not all of it
    auto clear = [&](uint8_t *stage, int left) {
        ca.clear(left, stage, wave, lane);
        cb.clear(left, stage + BYTES_A, wave, lane);
    };
    uint8_t *now = lds, *next = lds + STAGE;
    int left_now = STEP, left_next = STEP;
    // No k's at all: nothing to fetch.
    nx.item = a.steps > 0 ? blockIdx.x : a.items;
    nx.buffer = 0;
    if (nx.item < a.items) {
        enter();
        left_now = nx.left;
        each<S::COPIES>(copy);
        advance();
        if (nx.item < a.items) {
            left_next = nx.left;
            each<S::COPIES>(copy);
            advance();
        }
        wait_copies<0>();
        if (left_now < STEP)
            clear(now, left_now);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        barrier();
#pragma unroll
        for (int r = 0; r < READS; r++)
            read(f[0], lds, 0, r);
    }
    // Item by item.  The copies go on through the ends of items: while one's results
    // are stored, the first two steps of the next are on their way.
    for (unsigned item = blockIdx.x; item < a.items; item += gridDim.x) {
        const Work at = work_of(a, item);
        const int steps = a.steps > 0 ? steps_of(at) : 0;
#pragma unroll
        for (int i = 0; i < FM; i++)
#pragma unroll
            for (int j = 0; j < FN; j++)
                acc[i][j] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < steps; s++) {
            half(f[0], f[1], now, 1, Number<0>());
            // This wave has read all of the step, and its share of the next one is there.
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            if (left_next < STEP) {
                clear(next, left_next);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
            barrier();
            // Behind the last step of all: what nobody reads, from where the item that was
            // last entered began.
            const bool more = nx.item < a.items;
            if (!more)
                restart();
            left_now = nx.left;
            half(f[1], f[0], next, 0, Number<S::COPIES>());
            if (more)
                advance();
            uint8_t *const t = now;
            now = next;
            next = t;
            const int l = left_now;
            left_now = left_next;
            left_next = l;
        }
        const Results<S, LB == RC> results = {acc};
        results.gather();
        E::template run<T>(e, results, at, a, at.m * TM + wm, at.n * TN + wn, lane, lds + 2 * STAGE);
    }
    wait_copies<0>();  // nothing may arrive in LDS that is another workgroup's
}

template <typename T, typename S, int LA, int LB, typename E>
hipError_t launch(const Args &a, const typename E::Args &e, int per_cu, hipStream_t st) {
    void (*const f)(Args, typename E::Args) = kernel<T, S, LA, LB, E>;
    constexpr int LDS = 2 * (BYTES<LA, S::TM> + BYTES<LB, S::TN>) + E::template lds_bytes<S>();
    static_assert(LDS <= 160 * 1024, "a CU's");
    if (LDS > 64 * 1024) {
        const hipError_t err = allow_full_lds((const void *)f);
        if (err != hipSuccess)
            return err;
    }
    // as many workgroups as run together, a multiple of the XCDs
    const unsigned most = (unsigned)(device_cu_count() * per_cu) & ~7u, grid = a.items < most || most == 0 ? a.items : most;
    f<<<dim3(grid), dim3(S::TH), LDS, st>>>(a, e);
    return hipGetLastError();
}

// the plan's tiles
typedef Shape<256, 256, 2, 4, 2> Tile256;
typedef Shape<128, 128, 2, 2, 2> Tile128;

template <typename T, int LA, int LB, typename E>
hipError_t launch_tile(const Args &a, const typename E::Args &e, int tile, hipStream_t st) {
    static_assert(Tile256::TM == TILES[0].m && Tile256::TN == TILES[0].n && Tile128::TM == TILES[1].m &&
                      Tile128::TN == TILES[1].n, "what the plan counts with");
    return tile == 0 ? launch<T, Tile256, LA, LB, E>(a, e, TILES[0].per_cu, st)
                     : launch<T, Tile128, LA, LB, E>(a, e, TILES[1].per_cu, st);
}

}  // namespace mm
}  // namespace cf
