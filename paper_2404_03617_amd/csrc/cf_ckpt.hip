// cf_ckpt.hip -- activations kept in 8 bits from the forward to the backward
// pass: writing a checkpoint, alone or along with the activation function, and
// reading it back, as values or in the activation's gradient.
//
//   h = act(u);  checkpoint of u (and of h, the next layer's input)
//   du = dh act'(u'),  u' = q * scale of the checkpoint
//
// Elementwise and bound by memory: a lane takes 8 channels, 8 lanes the 64
// that share a scale (an exchange of registers finds their maximum).  Rows
// are cut into whole blocks of 64, so a row's last block may hold idle lanes.
//
// Measured on MI355X, where a copy of 2 GiB moves 4.9 TB/s (kernel times):
// 100352 x 128 bf16 written in 8.3 and read back in 7.9 us (39 MB each way, 4.7
// and 5.0 TB/s); 6272 x 2048 fp16 through GELU with its checkpoint 15.5 us (65 MB,
// 4.2 TB/s), with the result's too 18.6 (79 MB), and its gradient 13.4 us (65 MB, 4.8
// TB/s), with the VALU 99% busy: the erf polynomial costs as much as the memory.
#include "cf_rows.h"
#include "cf_kernels.h"
#include "cf_train.h"

namespace cf {

namespace {

// gelu'(u) = Phi(u) + u phi(u), with the tail 1 - Phi(|u|) = q(t) exp(-u^2/2)
// of gelu_f32, whose coefficients these are (1.5e-8): the exponential serves both
// terms.
__device__ __forceinline__ float gelu_slope(float u) {
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(u), 0.32f, 1.0f));
    float q = fmaf(-0.129858347f, t, 0.495794653f);
    q = fmaf(q, t, -0.265561934f);
    q = fmaf(q, t, 0.314940331f);
    q = fmaf(q, t, 0.079603797f);
    q = fmaf(q, t, 0.005081451f);
    const float e = __builtin_amdgcn_exp2f(u * u * -0.721347520f), tail = q * e;
    // |u| capped where the exponential is 0 anyway: no infinity times 0
    return fmaf(__builtin_amdgcn_fmed3f(u, -32.0f, 32.0f), e * 0.398942280f, u > 0.0f ? 1.0f - tail : tail);
}

// NaN stays NaN
template <int ACT>
__device__ __forceinline__ float act_of(float u) {
    if constexpr (ACT == ACT_GELU)
        return gelu_f32(u);
    else if constexpr (ACT == ACT_RELU)
        return u < 0.0f ? 0.0f : u;
    else
        return u;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float u) {
    if constexpr (ACT == ACT_GELU)
        return gelu_slope(u) + (u - u);
    else if constexpr (ACT == ACT_RELU)
        return u > 0.0f ? 1.0f : u <= 0.0f ? 0.0f : u;
    else
        return 1.0f;
}

struct ActArgs {
    const uint16_t *in;  // u, or dh
    uint16_t *out;       // h, or du
    Ckpt u, h;           // backward: u is read
    int64_t ldi, ldo;
    int C, blocks;
    uint32_t n;  // vectors: rows * blocks * 8
    FastDiv per_row;
};

struct At {
    int64_t r;
    int c, n;  // channel, and how many of the row are left
};
__device__ __forceinline__ At place(const ActArgs &a, uint32_t i) {
    const uint32_t r = fdiv(i, a.per_row);
    const int c = (int)(i - r * a.per_row.d) * 8;
    return {(int64_t)r, c, a.C - c};
}

__device__ __forceinline__ void keep(const Ckpt &k, const At &p, const ActArgs &a, const float *x) {
    const Quant z = quant_of(lanes<Max, 8>(amax8(x)));
    if (p.n <= 0)
        return;
    store8b(k.q + p.r * a.C, p.c, a.C, quant8(x, z.inv));
    if ((threadIdx.x & 7) == 0)
        k.scale[p.r * a.blocks + p.c / CKPT_BLOCK] = z.scale;
}

template <typename T, int ACT>
__global__ __launch_bounds__(256) void act_forward_kernel(ActArgs a) {
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i >= a.n)  // whole groups of 8 lanes
        return;
    const At p = place(a, i);
    const u32x4 raw = load8(a.in + p.r * a.ldi, p.c, a.C);
    float x[8];
    unpack8<T>(raw, x);
    if (a.u.q)
        keep(a.u, p, a, x);
    if (!a.out && !a.h.q)
        return;
#pragma unroll
    for (int e = 0; e < 8; e++)
        x[e] = act_of<ACT>(x[e]);
    const u32x4 y = pack8<T>(x);
    if (a.out && p.n > 0)
        store8(a.out + p.r * a.ldo, p.c, a.C, y);
    if (a.h.q) {
        unpack8<T>(y, x);  // the checkpoint is of the values the next layer reads
        keep(a.h, p, a, x);
    }
}

template <typename T, int ACT>
__global__ __launch_bounds__(256) void act_backward_kernel(ActArgs a) {
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i >= a.n)
        return;
    const At p = place(a, i);
    if (p.n <= 0)
        return;
    const u32x2 q = load8b(a.u.q + p.r * a.C, p.c, a.C);
    const float scale = a.u.scale[p.r * a.blocks + p.c / CKPT_BLOCK];
    float u[8];
    dequant8(q, scale, u);
    if (a.in) {
        float d[8];
        unpack8<T>(load8(a.in + p.r * a.ldi, p.c, a.C), d);
#pragma unroll
        for (int e = 0; e < 8; e++)
            u[e] = d[e] * act_slope<ACT>(u[e]);
    }
    store8(a.out + p.r * a.ldo, p.c, a.C, pack8<T>(u));
}

ActArgs args_of(const void *in, int64_t ldi, void *out, int64_t ldo, const Ckpt &u, const Ckpt &h, int64_t rows,
                int C) {
    ActArgs a;
    a.in = (const uint16_t *)in;
    a.out = (uint16_t *)out;
    a.u = u;
    a.h = h;
    a.ldi = ldi;
    a.ldo = ldo;
    a.C = C;
    a.blocks = blocks_of(C);
    a.n = (uint32_t)(rows * a.blocks * 8);
    a.per_row = make_fastdiv((uint32_t)a.blocks * 8);
    return a;
}

template <typename T>
hipError_t forward(const ActArgs &a, int act, hipStream_t st) {
    const dim3 grid((a.n + 255) / 256), wg(256);
    if (act == ACT_GELU)
        act_forward_kernel<T, ACT_GELU><<<grid, wg, 0, st>>>(a);
    else if (act == ACT_RELU)
        act_forward_kernel<T, ACT_RELU><<<grid, wg, 0, st>>>(a);
    else
        act_forward_kernel<T, ACT_NONE><<<grid, wg, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T>
hipError_t backward(const ActArgs &a, int act, hipStream_t st) {
    const dim3 grid((a.n + 255) / 256), wg(256);
    if (act == ACT_GELU)
        act_backward_kernel<T, ACT_GELU><<<grid, wg, 0, st>>>(a);
    else if (act == ACT_RELU)
        act_backward_kernel<T, ACT_RELU><<<grid, wg, 0, st>>>(a);
    else
        act_backward_kernel<T, ACT_NONE><<<grid, wg, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

bool act_fits(int64_t rows, int C) { return (double)rows * blocks_of(C) * 8 < 2147483648.0; }

hipError_t launch_act_forward(const void *u, int64_t ldu, void *h, int64_t ldh, const Ckpt &of_u, const Ckpt &of_h,
                              int64_t rows, int C, int act, int bf16, hipStream_t st) {
    const ActArgs a = args_of(u, ldu, h, ldh, of_u, of_h, rows, C);
    return bf16 ? forward<BF16>(a, act, st) : forward<F16>(a, act, st);
}

hipError_t launch_act_backward(const void *dh, int64_t lddh, const CkptIn &u, void *du, int64_t lddu, int64_t rows,
                               int C, int act, int bf16, hipStream_t st) {
    const ActArgs a = args_of(dh, lddh, du, lddu, Ckpt{(int8_t *)u.q, (float *)u.scale}, Ckpt{nullptr, nullptr}, rows,
                              C);
    return bf16 ? backward<BF16>(a, act, st) : backward<F16>(a, act, st);
}

}  // namespace cf
