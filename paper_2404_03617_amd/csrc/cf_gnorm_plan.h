// cf_gnorm_plan.h -- how a group norm (cf_gnorm.hip) is cut into workgroups, in
// plain C++ so that a test can ask without a GPU.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace cf {
namespace gnorm {

// The most vectors that a thread's registers hold (backward: of x and of dy), and that the kernels
// of 256 threads have.
constexpr int FORWARD_NV = 28, BACKWARD_NV = 16, SMALL_NV = 16;

// A workgroup takes `per_block` groups of one image, or a part of its pixels,
// and holds them in registers: `nv` vectors of 8 channels a thread.
struct Plan {
    int per_block, blocks;  // groups of a workgroup, workgroups beside each other
    int chunks;             // parts of an image's pixels
    int64_t px;             // pixels of a part
    int V, rows;            // vectors beside each other, pixels at a time
    int threads, nv;
};

// The vectors of a thread that the kernel launched for a plan holds.
inline int held(const Plan &p, int most_nv) {
    if (p.threads == 256)
        return p.nv <= 1 ? 1 : p.nv <= 4 ? 4 : p.nv <= 8 ? 8 : SMALL_NV;
    return p.nv <= 16 ? 16 : most_nv;
}

// The channels of a workgroup are a run of whole groups, at least `want` bytes
// of each pixel.
inline Plan shape(int64_t N, int64_t P, int C, int G, int want, int most_nv, int64_t cus) {
    const int D = C / G;
    Plan p;
    p.per_block = (want + 2 * D - 1) / (2 * D);
    p.per_block = p.per_block > G ? G : p.per_block;
    p.blocks = (G + p.per_block - 1) / p.per_block;
    p.V = (p.per_block * D + 7) / 8;
    const int64_t vectors = P * p.V;
    // a workgroup that has its CU to itself is better large (32 x 28 x 28 x 192 in 6 groups, forward
    // 10.0 us against 12.5)
    p.threads = vectors > 4096 || (vectors > 2048 && N * p.blocks <= cus && N * p.blocks >= cus / 2) || p.V > 256 ? 512 : 256;
    // and where 256 threads, some of them without a vector, do not hold the image (128 x 14 x 14 x 1280
    // in 8 groups 36.5 us, in parts of 256 threads 41.3; 260 x 17 x 1032 in one 15.0 and 20.3)
    if (p.threads == 256 && most_nv > SMALL_NV && P > (int64_t)SMALL_NV * (256 / p.V))
        p.threads = 512;
    p.rows = p.threads / p.V;
    const int64_t hold = p.rows > 0 ? (int64_t)p.rows * most_nv : 0;  // pixels that fit
    p.chunks = hold ? (int)((P + hold - 1) / hold) : 0;
    p.px = p.chunks ? (P + p.chunks - 1) / p.chunks : 0;
    p.nv = p.rows ? (int)((p.px + p.rows - 1) / p.rows) : 0;
    return p;
}

// 64 bytes of a pixel: half a cache line, whose other half is read behind the
// same L2 at about the same time, makes twice the workgroups that 128 bytes do
// (128 x 14 x 14 x 256, forward 12.1 us against 13.7, backward 20.4 against 22.1).
inline Plan plan_of(int64_t N, int64_t P, int C, int G, int most_nv, int64_t cus) {
    Plan p = shape(N, P, C, G, 64, most_nv, cus);
    // Few workgroups with much to do each: parts of at least 4 vectors a thread, as many as make a
    // workgroup a CU.  What is in parts anyhow is cut further (8 x 64 x 64 x 320 in 32 groups, forward
    // 22.6 us against 31.4; a few workgroups more than CUs cost a second round).
    const int64_t now = N * p.blocks * p.chunks;
    if (p.nv > 4 && now < (p.chunks > 1 ? cus : cus / 2)) {
        int64_t chunks = cus / (N * p.blocks);
        const int64_t most = (P + 4 * p.rows - 1) / (4 * p.rows);
        chunks = chunks < most ? chunks : most;
        if (chunks > p.chunks) {
            p.px = (P + chunks - 1) / chunks;
            p.chunks = (int)((P + p.px - 1) / p.px);
            p.nv = (int)((p.px + p.rows - 1) / p.rows);
        }
    }
    return p;
}

}  // namespace gnorm
}  // namespace cf
