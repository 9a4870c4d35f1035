// cf_mm_run.h -- host side of the products of cf_mm.h: operands, plans and
// launches.  Each kernel is instantiated in one of the files cf_mm_*.hip.
#pragma once

#include "cf_mm_epi.h"

namespace cf {
namespace mm {

template <typename T, int LA, int LB>
hipError_t launch_store(const Args &a, const StoreArgs &e, int tile, hipStream_t st);
template <typename T>
hipError_t launch_gated(const Args &a, const GatedArgs &e, int tile, hipStream_t st);
template <typename T>
hipError_t launch_gated_back(const Args &a, const GatedBackArgs &e, int tile, hipStream_t st);
template <typename T>
hipError_t launch_lse(const Args &a, const LseArgs &e, int tile, hipStream_t st);
template <typename T>
hipError_t launch_dz(const Args &a, const DzArgs &e, int tile, hipStream_t st);

// Sums of split products, and what follows: a store, h of the gate (batch 0) and
// up channels (batch 1), their gradients, the largest logits and sums of
// JOIN_CLASSES classes each, the logits' gradients.
constexpr int JOIN_CLASSES = 2048;
hipError_t launch_join(const Args &a, const StoreArgs &e, int bf16, hipStream_t st);
hipError_t launch_join(const Args &a, const float *part, const GatedArgs &e, int bf16, hipStream_t st);
hipError_t launch_join(const Args &a, const float *part, const GatedBackArgs &e, int bf16, hipStream_t st);
hipError_t launch_join(const Args &a, const float *part, const LseArgs &e, int bf16, hipStream_t st);
hipError_t launch_join(const Args &a, const float *part, const DzArgs &e, int bf16, hipStream_t st);

inline int up8(int n) { return (n + 7) & ~7; }
// whether rows of `cols` can be read where they are
inline bool fits(const void *p, int64_t ld, int cols) {
    return cols % 8 == 0 && ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && ld < (int64_t)1 << 22;
}
// The row stride of what lies in the workspace: whole cache lines, for rows of at
// least one (8192 x 8192 x 4104 1132 TFLOP/s, with rows that start in the middle of
// a line, x 4160 1282).
inline int64_t stride_of(int cols) { return cols < 64 ? up8(cols) : ((int64_t)cols + 63) & ~(int64_t)63; }
// bytes of a packed copy, whose rows are filled up to a multiple of 8 with zeros
inline size_t packed_bytes(int64_t rows, int cols) { return (size_t)rows * stride_of(cols) * 2; }
// whether the copy's vectors can be numbered
inline bool pack_fits(int64_t rows, int cols) { return (double)rows * (up8(cols) / 8) < 2147483648.0; }
// row m times factor[m] (1 if null), rows of factor 0 as zeros
hipError_t launch_pack(const void *src, int64_t ld, int64_t rows, int cols, const float *factor, void *dst, int bf16,
                       hipStream_t st);

inline Plan plan(int64_t M, int64_t N, int64_t K, bool may_split, int batch = 1, int segments = 1,
                 After what = STORE) {
    return plan_of(M, N, steps_of(K) * segments, batch, may_split, device_cu_count(), what);
}
// a workgroup a tile: a launch holds 2^32 threads
inline bool grid_fits(int64_t M, int64_t N) { return (double)((M + 127) / 128) * (double)((N + 127) / 128) < 4.0e6; }

// Pieces of a workspace, one after the other; without one, their size.
struct Room {
    uint8_t *p;
    size_t used = 0;
    void *take(size_t n) {
        uint8_t *const r = p ? p + used : nullptr;
        used += (n + 255) & ~(size_t)255;
        return r;
    }
};

// An operand where it is, or room for a packed copy of it.
struct Operand {
    Matrix m;
    const void *from;
    int64_t ld, rows;
    int cols;
    void *copy;
};
inline Operand operand(const void *from, int64_t ld, int64_t rows, int cols, bool copied, Room &room) {
    Operand o = {Matrix{(const uint16_t *)from, ld, cols}, from, ld, rows, cols, nullptr};
    if (copied) {
        o.copy = room.take(packed_bytes(rows, cols));
        o.m = Matrix{(const uint16_t *)o.copy, stride_of(cols), up8(cols)};
    }
    return o;
}
inline hipError_t pack(const Operand &o, int bf16, hipStream_t st) {
    return o.copy ? launch_pack(o.from, o.ld, o.rows, o.cols, nullptr, o.copy, bf16, st) : hipSuccess;
}

// room for the sums of a product that a launch of its own joins
inline size_t joined_bytes(const Plan &p, int64_t M, int64_t N, int64_t batch, bool always) {
    return always ? (size_t)p.splits * batch * M * N * 4 : part_bytes(p, M, N, batch);
}

#define CF_HIP(call)                                                                                                   \
    do {                                                                                                               \
        const hipError_t e_ = (call);                                                                                  \
        if (e_ != hipSuccess)                                                                                          \
            return e_;                                                                                                 \
    } while (0)

template <int LA, int LB>
hipError_t run_store(const Args &a, StoreArgs e, const Plan &p, void *part, int bf16, hipStream_t st) {
    const bool join = a.splits > 1 || e.fold;
    e.part = join ? (float *)part : nullptr;
    const hipError_t r = bf16 ? launch_store<BF16, LA, LB>(a, e, p.tile, st) : launch_store<F16, LA, LB>(a, e, p.tile, st);
    return r != hipSuccess || !join ? r : launch_join(a, e, bf16, st);
}

// The parts alone of a split product, and what follows.
template <int LA, int LB, typename E>
hipError_t run_split(const Args &a, const E &e, const Plan &p, void *part, int bf16, hipStream_t st) {
    StoreArgs s = {};
    s.part = (float *)part;
    CF_HIP((bf16 ? launch_store<BF16, LA, LB>(a, s, p.tile, st) : launch_store<F16, LA, LB>(a, s, p.tile, st)));
    return launch_join(a, s.part, e, bf16, st);
}

}  // namespace mm
}  // namespace cf
