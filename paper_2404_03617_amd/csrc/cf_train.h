// cf_train.h -- launchers of the training and scoring operators, between the C
// ABI layer (cf_train_api.hip) and their kernels.  Internal; arguments have
// been checked when these are called.  Rows are [rows][C], channels fastest,
// with a row stride (ld*, in elements) for 16-bit tensors and logits;
// checkpoints (q [rows][C], scale [rows][ceil(C/64)]) and fp32 vectors are
// dense.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace cf {

struct Ckpt {
    int8_t *q;
    float *scale;
};
struct CkptIn {
    const int8_t *q;
    const float *scale;
};

// whether there is a kernel for rows of C channels, and a grid for as many
bool norm_fits(int64_t rows, int C);
// stats [rows][2] (mean, 1 / standard deviation); stats and the checkpoint of x may be null
hipError_t launch_norm_forward(const void *x, int64_t ldx, void *y, int64_t ldy, const float *weight,
                               const float *bias, float *stats, const Ckpt &ckpt, int64_t rows, int C, float eps,
                               int bf16, hipStream_t st);

// x or its checkpoint; dweight and dbias both or neither, with their workspace
struct NormBackward {
    const void *dy;
    int64_t lddy;
    const void *x;
    int64_t ldx;
    CkptIn ckpt;
    const float *stats, *weight;
    void *dx;
    int64_t lddx;
    float *dweight, *dbias;
};
size_t norm_backward_workspace_bytes(int64_t rows, int C);
hipError_t launch_norm_backward(const NormBackward &a, int64_t rows, int C, int bf16, void *ws, hipStream_t st);

// h = act(u) (h may be null), checkpoints of u and of the rounded h (q null: none)
hipError_t launch_act_forward(const void *u, int64_t ldu, void *h, int64_t ldh, const Ckpt &of_u, const Ckpt &of_h,
                              int64_t rows, int C, int act, int bf16, hipStream_t st);
// du = dh act'(u); dh null: the values of u themselves
hipError_t launch_act_backward(const void *dh, int64_t lddh, const CkptIn &u, void *du, int64_t lddu, int64_t rows,
                               int C, int act, int bf16, hipStream_t st);
// whether the vectors of these rows can be numbered in 31 bits
bool act_fits(int64_t rows, int C);

// dw [K][C] = dy^T x, db [K] = column sums of dy; with stats (and weight,
// bias) x is weight * (x - mean) * rstd + bias of the checkpointed rows
struct WGrad {
    const void *dy;
    int64_t lddy;
    CkptIn x;
    const float *stats, *weight, *bias;
    void *dw;
    float *db;
};
size_t wgrad_workspace_bytes(int64_t rows, int K, int C);
hipError_t launch_wgrad(const WGrad &a, int64_t rows, int K, int C, int bf16, void *ws, hipStream_t st);

enum { LOGITS_F16 = 0, LOGITS_BF16 = 1, LOGITS_F32 = 2 };
constexpr int TOP_MAX = 32;
struct LogProbs {  // tokens and logp may be null
    const void *z;
    int64_t ldz;
    const int64_t *tokens;
    float *logp, *entropy;
    float *stats;  // [rows][2]: largest logit, log of the sum of exp(z - largest); may be null
    float *top_logp;
    int64_t *top_ids;
};
size_t log_probs_workspace_bytes(int64_t rows, int V, int top);
hipError_t launch_log_probs(const LogProbs &a, int64_t rows, int V, int top, int dt, void *ws, hipStream_t st);

struct LogProbsBackward {
    const void *z;
    int64_t ldz;
    const int64_t *tokens;
    const float *stats, *entropy, *d_logp, *d_entropy;  // d_* may be null
    void *dz;
    int64_t lddz;
};
// whether the grids of the passes hold these rows
bool log_probs_fit(int64_t rows, int V);
bool log_probs_backward_fits(const LogProbsBackward &a, int64_t rows, int V, int dt);
hipError_t launch_log_probs_backward(const LogProbsBackward &a, int64_t rows, int V, int dt, hipStream_t st);

}  // namespace cf
