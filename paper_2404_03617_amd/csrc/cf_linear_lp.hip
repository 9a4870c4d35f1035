// cf_linear_lp.hip -- log probabilities of classes or tokens from features and
// a weight matrix, z = x W^T with W [V][C], without keeping the logits:
//
//   lse = log sum exp z,  logp = z[token] - lse
//
// Forward: every tile of logits (cf_mm.h) leaves the largest and the sum of exp(z -
// largest) of its rows, and the token's logit where it has it; a second launch
// joins the tiles of a row.  Where there are few tiles and many features, their
// sums are split and the logits' parts joined before (64 x 7680 x 6864 32 us against
// 84).
//
// Backward, with c = d_lse - d_logp and p = exp(z - lse):
//
//   dz = c p + d_logp 1[token];  dx = dz W;  dW = dz^T x
//
// piece by piece of the vocabulary: the piece's logits are made again and become dz
// in 16 bits (pieces_of: PIECE_BYTES, or 4096 classes of many rows), which two
// products read.  dx runs over the pieces in fp32.
//
// A gradient in 16 bits: in bf16 its range is that of fp32.  In fp16 a row's
// values are scaled by a power of two, so that the largest of c and the token's value
// lies in [2^13, 2^14) and a probability of 4e-9 still has all bits; dx is scaled
// back by row, and the rows of x that dW sums are scaled against each other, so that
// the largest product of a row's gradient and one of its features becomes a number in
// [2^14, 2^15): products down to 2^-28 of it keep all bits, and what smaller ones lose
// is below 2^-38 of it, about as far as fp16's least number lies below its largest.
// The same copy of x leaves out rows without a gradient: what their features hold,
// NaN included, reaches nothing.
//
// Bound by the matrix unit: 8192 x 4096 x 131072 in bf16 6.5 ms forward (1350 TFLOP/s);
// backward 8 pieces of dz 0.88, dx 0.87 and dW 0.85 ms (1256, 1261, 1297).  Pieces of
// 128 MiB to 2 GiB make 1 to 4% either way there, and up to 12% with few features.
#include "cf_few.h"
#include "cf_head.h"
#include "cf_mm_run.h"
#include "cf_rows.h"

namespace cf {

using namespace mm;

namespace {

// Fragments of 16 classes a workgroup where there are few rows: one or two rows come
// from the caches at little cost (1 x 131072 x 4096 182 us with one, 197 with two),
// more rather once for two (8 rows 205 and 192, 16 rows 245 and 197).
constexpr int few_of(int64_t rows) { return rows <= 2 ? 1 : 2; }

// L lanes join the parts of a row.
template <int L>
__global__ __launch_bounds__(256) void join_lse_kernel(const float2 *part, const float *picked, const int64_t *tokens,
                                                       float *logp, float *lse, int rows, int V, int parts) {
    const int lane = threadIdx.x % L, r = blockIdx.x * (256 / L) + threadIdx.x / L;
    float2 v = make_float2(-INFINITY, -1.0f);
    if (r < rows)
#pragma unroll 4
        for (int i = lane; i < parts; i += L)
            v = join_lse(v, part[(int64_t)i * rows + r]);
#pragma unroll
    for (int d = 1; d < (L < 64 ? L : 64); d *= 2)
        v = join_lse(v, make_float2(__shfl_xor(v.x, d), __shfl_xor(v.y, d)));
    if constexpr (L == 256) {
        __shared__ float2 s[4];
        if ((lane & 63) == 0)
            s[lane >> 6] = v;
        __syncthreads();
        v = join_lse(join_lse(s[0], s[1]), join_lse(s[2], s[3]));
    }
    if (lane || r >= rows)
        return;
    const float ls = log1pf(v.y);
    lse[r] = v.x + ls;
    if (logp) {
        const int64_t t = tokens[r];
        float l = 0.0f;
        if (t >= V)
            l = NAN;
        else if (t >= 0)
            l = v.x == -INFINITY && !(v.y != v.y) ? -INFINITY : picked[r] - v.x - ls;
        logp[r] = l;
    }
}

// What a row's gradient is made of; none for c = at = 0.  At the token, c p + d_logp
// is d_lse p + d_logp (1 - p) with both factors from logp: where p is nearly 1, lse in
// fp32 has lost what is left of 1 - p (a row with lse = 15 and 1 - p = 5e-7: all of it).
// A weight of 0 takes nothing from a log probability that may be NaN.
__device__ __forceinline__ RowGrad grad_of(const LinearGrads &g, const int64_t *tokens, int V, int r) {
    const int64_t t = g.d_logp ? tokens[r] : -1;
    const float gl = t >= V ? NAN : t >= 0 ? g.d_logp[r] : 0.0f, gs = g.d_lse ? g.d_lse[r] : 0.0f, lse = g.lse[r];
    RowGrad w = {gs - gl, 0.0f, lse, t < V ? (int)t : -1};
    if (w.token >= 0)
        w.at = (gs != 0.0f ? gs * expf(g.logp[r]) : 0.0f) - (gl != 0.0f ? gl * expm1f(g.logp[r]) : 0.0f);
    if (lse == -INFINITY)
        w.c = w.at = 0.0f;
    return w;
}
// 2^e <= the larger of |c| and |at| < 2^(e+1), within what fp32 can be scaled by
constexpr int E_MIN = -100, E_MAX = 100;
__device__ __forceinline__ int exponent_of(const RowGrad &w) {
    const float a = fmaxf(fabsf(w.c), fabsf(w.at));
    const int e = (int)(__float_as_uint(a) >> 23) - 127;
    return e < E_MIN ? E_MIN : e > E_MAX ? E_MAX : e;
}
__device__ __forceinline__ float pow2(int e) { return e < -126 ? 0.0f : __uint_as_float((uint32_t)(e + 127) << 23); }

__device__ __forceinline__ int wave_max(int e) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int k = __shfl_xor(e, d);
        e = k > e ? k : e;
    }
    return e;
}

// The exponent of a magnitude in fp16, or less than any for 0; the largest finite one of 8.
constexpr int NO_EXPONENT = -1000;
__device__ __forceinline__ int feature_exponent(uint32_t bits) {
    return bits ? (int)(__float_as_uint(F16::lo(bits)) >> 23) - 127 : NO_EXPONENT;
}
__device__ __forceinline__ uint32_t largest_of(const u32x4 &v, uint32_t most) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const uint32_t h = v[i / 2] >> (16 * (i & 1)) & 0x7fffu;
        most = h < 0x7c00u && h > most ? h : most;
    }
    return most;
}

// fp16: the largest exponent of a gradient and a feature among each workgroup's rows
// (those without a gradient left out), EXPONENTS workgroups at most.  x as the products
// read it, `vectors` a row, which 2^log_lanes threads share.  1 to 2 us of a call's 113
// (64 x 7680 x 6864) or 69 (6272 x 512 x 1000) are for the features.
constexpr int EXPONENTS = 512;
__global__ __launch_bounds__(1024) void exponents_kernel(LinearGrads g, const int64_t *tokens, int V, int rows,
                                                         const uint16_t *x, int64_t ldx, int vectors, int log_lanes,
                                                         int *most) {
    __shared__ int s[16];
    const int lane = threadIdx.x & ((1 << log_lanes) - 1), beside = 1024 >> log_lanes;
    int e = E_MIN;
#pragma unroll 2
    for (int r = blockIdx.x * beside + (threadIdx.x >> log_lanes); r < rows; r += gridDim.x * beside) {
        const u32x4 *const p = reinterpret_cast<const u32x4 *>(x + r * ldx);
        uint32_t top = 0;
        for (int i = lane; i < vectors; i += 1 << log_lanes)
            top = largest_of(p[i], top);
        const RowGrad w = grad_of(g, tokens, V, r);
        const int k = w.c == 0.0f && w.at == 0.0f ? E_MIN : exponent_of(w) + feature_exponent(top);
        e = k > e ? k : e;
    }
    e = wave_max(e);
    if ((threadIdx.x & 63) == 0)
        s[threadIdx.x >> 6] = e;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 16; i++)
            e = s[i] > e ? s[i] : e;
        most[blockIdx.x] = e;
    }
}

// fp16: `counts` of those, and scale receives the factor of dW's sums.
__global__ __launch_bounds__(256) void row_grads_kernel(LinearGrads g, const int64_t *tokens, int V, int rows,
                                                        const int *exponents, int counts, RowGrad *out, float *factor,
                                                        float *row_scale, float *scale) {
    const int r = blockIdx.x * 256 + threadIdx.x;
    int most = E_MIN;
#pragma unroll 4
    for (int i = threadIdx.x & 63; i < counts; i += 64)
        most = exponents[i] > most ? exponents[i] : most;
    most = wave_max(most);
    if (r == 0 && counts)
        *scale = pow2(most - 13 - 14);
    if (r >= rows)
        return;
    RowGrad w = grad_of(g, tokens, V, r);
    const bool none = w.c == 0.0f && w.at == 0.0f;
    float f = none ? 0.0f : 1.0f;
    if (counts) {
        const int e = exponent_of(w);
        w.c *= pow2(13 - e);
        w.at *= pow2(13 - e);
        row_scale[r] = pow2(e - 13);
        const int up = e - most + 14;  // below -126 nothing of x is left but NaN; above 126 x is 0
        f = none ? 0.0f : pow2(up < -126 ? -126 : up > 126 ? 126 : up);
    }
    out[r] = w;
    factor[r] = f;
}

struct ForwardPlan {
    Room room;
    Operand x, w;
    Plan z;
    int parts;
    float2 *part;
    float *picked;
    void *sums;
};
ForwardPlan forward_plan(const LinearLogProbs &a, bool copy_x, bool copy_w, void *ws) {
    ForwardPlan p;
    copy_x &= a.rows > few::ROWS;  // fewer are read wherever they are
    copy_w &= a.rows > few::ROWS;
    p.room.p = (uint8_t *)ws;
    p.x = operand(a.x.p, a.x.ld, a.rows, a.C, copy_x, p.room);
    p.w = operand(a.w.p, a.w.ld, a.V, a.C, copy_w, p.room);
    p.z = plan(a.rows, a.V, a.C, true, 1, 1, MORE);
    const int n = a.rows <= few::ROWS ? 16 * few_of(a.rows) : p.z.splits > 1 ? JOIN_CLASSES : TILES[p.z.tile].n;
    p.parts = (a.V + n - 1) / n;
    p.part = (float2 *)p.room.take((size_t)p.parts * a.rows * sizeof(float2));
    p.picked = (float *)p.room.take((size_t)a.rows * 4);
    p.sums = a.rows <= few::ROWS ? nullptr : p.room.take(part_bytes(p.z, a.rows, a.V, 1));
    return p;
}

struct BackwardPlan {
    Room room;
    Operand x, w;
    uint16_t *xs, *dz;
    RowGrad *rows;
    float *factor, *row_scale, *scale, *acc;
    int *most;
    int piece, pieces;
    Plan z, dx, dw;
    void *part;
};
BackwardPlan backward_plan(const LinearLogProbs &a, bool copy_x, bool copy_w, void *ws) {
    BackwardPlan p;
    p.room.p = (uint8_t *)ws;
    p.x = operand(a.x.p, a.x.ld, a.rows, a.C, copy_x, p.room);
    p.w = operand(a.w.p, a.w.ld, a.V, a.C, copy_w, p.room);
    p.xs = (uint16_t *)p.room.take(packed_bytes(a.rows, a.C));
    p.rows = (RowGrad *)p.room.take((size_t)a.rows * sizeof(RowGrad));
    p.factor = (float *)p.room.take((size_t)a.rows * 4);
    p.row_scale = (float *)p.room.take((size_t)a.rows * 4);
    p.scale = (float *)p.room.take(4);
    p.most = (int *)p.room.take(EXPONENTS * 4);
    const bool lo = in_parts(a.rows);
    const int64_t rows = lo ? 2 * a.rows : a.rows;
    const Pieces cut = pieces_of(a.rows, a.V);
    p.piece = cut.columns;
    p.pieces = cut.count;
    p.dz = (uint16_t *)p.room.take((size_t)rows * stride_of(p.piece) * 2);
    p.acc = p.pieces > 1 ? (float *)p.room.take((size_t)a.rows * a.C * 4) : nullptr;
    p.z = plan(a.rows, p.piece, a.C, true, 1, 1, MORE);
    p.dx = plan(rows, a.C, p.piece, true);
    p.dw = plan(p.piece, a.C, a.rows, true, 1, lo ? 2 : 1);
    const size_t one = joined_bytes(p.dx, rows, a.C, 1, lo), two = part_bytes(p.dw, p.piece, a.C, 1);
    const size_t three = joined_bytes(p.z, a.rows, p.piece, 1, lo), most_of = one > two ? one : two;
    p.part = p.room.take(most_of > three ? most_of : three);
    return p;
}

template <typename T>
hipError_t forward(const LinearLogProbs &a, const ForwardPlan &p, float *logp, float *lse, int bf16, hipStream_t st) {
    CF_HIP(pack(p.x, bf16, st));
    CF_HIP(pack(p.w, bf16, st));
    const LseArgs e = {p.part, p.picked, logp ? a.tokens : nullptr};
    const few::Args f = {p.x.m.p, {p.w.m.p, p.w.m.p}, p.x.m.ld, {p.w.m.ld, p.w.m.ld}, 0, a.rows, a.V, a.C};
    if (a.rows <= few::ROWS) {
        CF_HIP((few_of(a.rows) == 1 ? few::launch<T, 1, few::Lse>(f, e, st) : few::launch<T, 2, few::Lse>(f, e, st)));
    } else {
        const Args z = args_of(p.z, a.rows, a.V, a.C, p.x.m, a.rows, p.w.m, a.V);
        if (p.z.splits > 1)
            CF_HIP((run_split<KC, KC>(z, e, p.z, p.sums, bf16, st)));
        else
            CF_HIP(launch_lse<T>(z, e, p.z.tile, st));
    }
    // few rows of many parts: a workgroup each
    if (a.rows <= 256 && p.parts > 64)
        join_lse_kernel<256><<<dim3((unsigned)a.rows), 256, 0, st>>>(p.part, p.picked, a.tokens, logp, lse, a.rows, a.V,
                                                                     p.parts);
    else
        join_lse_kernel<16><<<dim3((unsigned)((a.rows + 15) / 16)), 256, 0, st>>>(p.part, p.picked, a.tokens, logp, lse,
                                                                                  a.rows, a.V, p.parts);
    return hipGetLastError();
}

template <typename T>
hipError_t backward(const LinearLogProbs &a, const BackwardPlan &p, const LinearGrads &g, int bf16, hipStream_t st) {
    CF_HIP(pack(p.x, bf16, st));
    CF_HIP(pack(p.w, bf16, st));
    if (a.rows > 0) {
        int counts = 0;
        if (!bf16) {
            int log_lanes = 0;
            while (log_lanes < 10 && 8 << log_lanes < a.C)
                log_lanes++;
            const int beside = 1024 >> log_lanes, groups = (a.rows + beside - 1) / beside;
            counts = groups < EXPONENTS ? groups : EXPONENTS;
            exponents_kernel<<<counts, 1024, 0, st>>>(g, a.tokens, a.V, a.rows, p.x.m.p, p.x.m.ld, p.x.m.ext / 8, log_lanes,
                                                      p.most);
        }
        row_grads_kernel<<<dim3((unsigned)((a.rows + 255) / 256)), 256, 0, st>>>(
            g, a.tokens, a.V, a.rows, p.most, counts, p.rows, p.factor, p.row_scale, p.scale);
        CF_HIP(hipGetLastError());
        CF_HIP(launch_pack(a.x.p, a.x.ld, a.rows, a.C, p.factor, p.xs, bf16, st));
    }
    const Matrix xs = {p.xs, stride_of(a.C), up8(a.C)};
    for (int i = 0; i < p.pieces; i++) {
        const int v0 = i * p.piece, n = a.V - v0 < p.piece ? a.V - v0 : p.piece, pad = up8(n);
        const Matrix w = {p.w.m.p + (int64_t)v0 * p.w.m.ld, p.w.m.ld, p.w.m.ext}, dz = {p.dz, stride_of(n), pad};
        const int64_t lo = in_parts(a.rows) ? a.rows * dz.ld : 0;
        if (a.rows > 0) {
            const Args z = args_of(p.z, a.rows, n, a.C, p.x.m, a.rows, w, n);
            const DzArgs e = {p.rows, p.dz, dz.ld, lo, pad, v0};
            if (p.z.splits > 1 || lo)
                CF_HIP((run_split<KC, KC>(z, e, p.z, p.part, bf16, st)));
            else
                CF_HIP(launch_dz<T>(z, e, p.z.tile, st));
            StoreArgs s = {};
            s.out[0] = s.out[1] = (uint16_t *)g.dx;
            s.ldo = g.lddx;
            s.row_scale = bf16 ? nullptr : p.row_scale;
            s.fold = lo ? a.rows : 0;
            s.acc = p.acc;
            s.acc_in = i > 0;
            s.acc_out = i + 1 < p.pieces;
            const int rows = lo ? 2 * a.rows : a.rows;
            CF_HIP((run_store<KC, RC>(args_of(p.dx, rows, a.C, n, dz, rows, w, w.ext), s, p.dx, p.part, bf16, st)));
        }
        StoreArgs s = {};
        s.out[0] = s.out[1] = (uint16_t *)g.dw + (int64_t)v0 * a.C;
        s.ldo = a.C;
        s.scale = bf16 || a.rows == 0 ? nullptr : p.scale;
        Args dw = args_of(p.dw, n, a.C, a.rows, dz, pad, xs, xs.ext, lo != 0);
        dw.a[1] = p.dz + lo;
        CF_HIP((run_store<RC, RC>(dw, s, p.dw, p.part, bf16, st)));
    }
    return hipSuccess;
}

}  // namespace

bool linear_fits(int64_t rows, int C, int V) {
    // 16 lanes a row, and 256 threads for 16 classes of few rows: a launch holds 2^32
    return rows < (int64_t)1 << 28 && C <= 1 << 20 && V < 1 << 28 && grid_fits(rows, V) && grid_fits(V, C) &&
           grid_fits(rows, C) && pack_fits(rows, C) && pack_fits(V, C);
}

size_t linear_workspace_bytes(int64_t rows, int C, int V, bool aligned) {
    LinearLogProbs a = {};
    a.rows = (int)rows;
    a.C = C;
    a.V = V;
    const bool copy = C % 8 || !aligned;
    return forward_plan(a, copy, copy, nullptr).room.used;
}

size_t linear_backward_workspace_bytes(int64_t rows, int C, int V, bool aligned) {
    LinearLogProbs a = {};
    a.rows = (int)rows;
    a.C = C;
    a.V = V;
    const bool copy = C % 8 || !aligned;
    return backward_plan(a, copy, copy, nullptr).room.used;
}

hipError_t launch_linear_log_probs(const LinearLogProbs &a, float *logp, float *lse, int bf16, void *ws,
                                   hipStream_t st) {
    const ForwardPlan p = forward_plan(a, !fits(a.x.p, a.x.ld, a.C), !fits(a.w.p, a.w.ld, a.C), ws);
    return bf16 ? forward<BF16>(a, p, logp, lse, bf16, st) : forward<F16>(a, p, logp, lse, bf16, st);
}

hipError_t launch_linear_log_probs_backward(const LinearLogProbs &a, const LinearGrads &g, int bf16, void *ws,
                                            hipStream_t st) {
    const bool some = a.rows > 0;  // else nothing is read
    const BackwardPlan p = backward_plan(a, some && !fits(a.x.p, a.x.ld, a.C), some && !fits(a.w.p, a.w.ld, a.C), ws);
    return bf16 ? backward<BF16>(a, p, g, bf16, st) : backward<F16>(a, p, g, bf16, st);
}

}  // namespace cf
