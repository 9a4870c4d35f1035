// cf_head.h -- launchers of the operators for heads over features: group norm
// with an activation, the gated feed-forward block, log probabilities from
// features.  Between the C ABI layer (cf_head_api.hip) and their kernels;
// internal, arguments have been checked.  Rows as in cf_train.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace cf {

// --- group norm: N images of P pixels, C channels in G groups ---------------
struct GroupNorm {
    const void *x;
    int64_t ldx;
    const float *weight, *bias;  // [C], may be null
    int64_t N, P;
    int C, G, act;
};
bool group_norm_fits(int64_t N, int64_t P, int C, int G);
size_t group_norm_workspace_bytes(int64_t N, int64_t P, int C, int G);
hipError_t launch_group_norm(const GroupNorm &a, void *y, int64_t ldy, float *stats, float eps, int bf16, void *ws,
                             hipStream_t st);
size_t group_norm_backward_workspace_bytes(int64_t N, int64_t P, int C, int G);
hipError_t launch_group_norm_backward(const GroupNorm &a, const void *dy, int64_t lddy, const float *stats, void *dx,
                                      int64_t lddx, float *dweight, float *dbias, int bf16, void *ws, hipStream_t st);

// --- gated feed-forward block ---------------------------------------------------
struct RowsIn {
    const void *p;
    int64_t ld;
};
struct GatedFfn {
    RowsIn x, w_gate, w_up, w_down;  // [rows][C], [H][C], [H][C], [C][H]
    int rows, C, H, act;
};
// whether rows of `cols` can be read by the products where they are
bool products_read(const void *p, int64_t ld, int cols);
// whether the grids hold these sizes
bool gated_fits(int64_t rows, int C, int H);
size_t gated_workspace_bytes(int64_t rows, int C, int H, bool aligned);
hipError_t launch_gated(const GatedFfn &a, void *y, int64_t ldy, float *saved, int bf16, void *ws, hipStream_t st);
size_t gated_backward_workspace_bytes(int64_t rows, int C, int H, bool aligned);
struct GatedGrads {
    void *dx;
    int64_t lddx;
    void *dw_gate, *dw_up, *dw_down;  // dense
};
hipError_t launch_gated_backward(const GatedFfn &a, RowsIn dy, const float *saved, const GatedGrads &g, int bf16,
                                 void *ws, hipStream_t st);

// --- log probabilities from features ----------------------------------------
struct LinearLogProbs {
    RowsIn x, w;  // [rows][C], [V][C]
    const int64_t *tokens;
    int rows, C, V;
};
bool linear_fits(int64_t rows, int C, int V);
size_t linear_workspace_bytes(int64_t rows, int C, int V, bool aligned);
hipError_t launch_linear_log_probs(const LinearLogProbs &a, float *logp, float *lse, int bf16, void *ws,
                                   hipStream_t st);
size_t linear_backward_workspace_bytes(int64_t rows, int C, int V, bool aligned);
struct LinearGrads {
    const float *logp, *lse, *d_logp, *d_lse;  // logp for d_logp; d_* may be null
    void *dx;
    int64_t lddx;
    void *dw;  // [V][C] dense
};
hipError_t launch_linear_log_probs_backward(const LinearLogProbs &a, const LinearGrads &g, int bf16, void *ws,
                                            hipStream_t st);

}  // namespace cf
