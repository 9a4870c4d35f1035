// cf_mm.hip -- what stands around the products of cf_mm.h: packed copies of
// operands that the tiles cannot read where they are, and the joining of split
// sums, in a fixed order, with what follows them.  Both are bound by memory: 67 MB of
// features are copied in 21 us; the joins take 4 to 13 us.
#include "cf_mm_run.h"
#include "cf_rows.h"

namespace cf {
namespace mm {

namespace {

template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const uint16_t *src, int64_t ld, int cols, const float *factor,
                                                   u32x4 *dst, int64_t ldd, uint32_t n, FastDiv per_row) {
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i >= n)
        return;
    const uint32_t r = fdiv(i, per_row);
    const int c = (int)(i - r * per_row.d) * 8;
    u32x4 v = {0u, 0u, 0u, 0u};
    const float f = factor ? factor[r] : 1.0f;
    if (f != 0.0f) {
        v = load8(src + (int64_t)r * ld, c, cols);
        if (f != 1.0f) {
            float x[8];
            unpack8<T>(v, x);
#pragma unroll
            for (int k = 0; k < 8; k++)
                x[k] *= f;
            v = pack8<T>(x);
        }
    }
    dst[r * ldd + c / 8] = v;
}

// G lanes share four entries, each adding every G-th split; then they add
// theirs, always in the same order.
template <typename T, int G>
__global__ __launch_bounds__(256) void join_kernel(Args a, StoreArgs e, int per_row, int64_t n) {
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) / G;
    const int g = threadIdx.x % G;
    if (i >= n)  // whole groups of lanes
        return;
    const int64_t row = i / per_row;  // of the batch's
    const int rows = e.fold ? e.fold : a.M;
    const int batch = (int)(row / rows), m = (int)(row - (int64_t)batch * rows), c = (int)(i - row * per_row) * 4;
    const int64_t step = (int64_t)a.batch * a.M * a.N;
    const float *p = e.part + ((int64_t)batch * a.M + m) * a.N + c;
    float4v v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int s = g; s < a.splits; s += G) {
        float4v w;
        load_rowf<4>(p + s * step, w, a.N - c);
        v += w;
        if (e.fold) {
            load_rowf<4>(p + s * step + (int64_t)e.fold * a.N, w, a.N - c);
            v += w;
        }
    }
#pragma unroll
    for (int d = 1; d < G; d *= 2)
#pragma unroll
        for (int k = 0; k < 4; k++)
            v[k] += __shfl_xor(v[k], d);
    if (g == 0)
        finish<T, 4>(e, v, m, c, a.M, a.N, batch);
}

template <typename T>
hipError_t join(const Args &a, const StoreArgs &e, hipStream_t st) {
    const int per_row = (a.N + 3) / 4;
    const int64_t n = (int64_t)a.batch * (e.fold ? e.fold : a.M) * per_row;
    if (n >= 65536 || a.splits < 8)
        join_kernel<T, 1><<<dim3((unsigned)((n + 255) / 256)), 256, 0, st>>>(a, e, per_row, n);
    else
        join_kernel<T, 8><<<dim3((unsigned)((n * 8 + 255) / 256)), 256, 0, st>>>(a, e, per_row, n);
    return hipGetLastError();
}

// The sums of 8 columns of row m from n on, in the order of the splits; batch b.
__device__ __forceinline__ void sum_parts(const Args &a, const float *part, int b, int m, int n, float (&v)[8]) {
    const int64_t step = (int64_t)a.batch * a.M * a.N;
    const float *p = part + ((int64_t)b * a.M + m) * a.N + n;
#pragma unroll
    for (int k = 0; k < 8; k++)
        v[k] = 0.0f;
#pragma unroll 4
    for (int s = 0; s < a.splits; s++) {
        float w[8];
        load_rowf<8>(p + s * step, w, a.N - n);
#pragma unroll
        for (int k = 0; k < 8; k++)
            v[k] += w[k];
    }
}

// a thread 8 columns, `vectors` of them a row
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(Args a, const float *part, GatedArgs e, FastDiv vectors, uint32_t all) {
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i >= all)
        return;
    const int m = (int)fdiv(i, vectors), n = (int)(i - (uint32_t)m * vectors.d) * 8;
    float g[8], u[8];
    sum_parts(a, part, 0, m, n, g);
    sum_parts(a, part, 1, m, n, u);
    with_act(e.act, [&](auto tag) { Gated::piece<T, decltype(tag)::value>(e, g, u, m, n, true); });
}
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(Args a, const float *part, GatedBackArgs e, FastDiv vectors,
                                                   uint32_t all) {
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i >= all)
        return;
    const int m = (int)fdiv(i, vectors), n = (int)(i - (uint32_t)m * vectors.d) * 8;
    float g[8], u[8], dh[8];
    GatedBack::read(e, m, n, e.H - n, g, u);
    sum_parts(a, part, 0, m, n, dh);
    with_act(e.act, [&](auto tag) {
        if (e.lo)
            GatedBack::piece<T, decltype(tag)::value, true>(e, dh, g, u, m, n);
        else
            GatedBack::piece<T, decltype(tag)::value>(e, dh, g, u, m, n);
    });
}
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(Args a, const float *part, DzArgs e, FastDiv vectors, uint32_t all) {
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i >= all)
        return;
    const int m = (int)fdiv(i, vectors), n = (int)(i - (uint32_t)m * vectors.d) * 8;
    float z[8];
    sum_parts(a, part, 0, m, n, z);
    if (e.lo)
        Dz::piece<T, true>(e, e.rows[m], z, m, n, a.N, true, true);
    else
        Dz::piece<T>(e, e.rows[m], z, m, n, a.N, true, true);
}

// A workgroup JOIN_CLASSES classes of a row, a thread 8 of them.
__global__ __launch_bounds__(JOIN_CLASSES / 8) void join_kernel(Args a, const float *part, LseArgs e, int chunks) {
    constexpr int WAVES = JOIN_CLASSES / 8 / 64;
    __shared__ float2 s[WAVES];
    const int m = (int)(blockIdx.x / (unsigned)chunks), chunk = (int)(blockIdx.x - (unsigned)m * chunks),
              n = chunk * JOIN_CLASSES + threadIdx.x * 8;
    float2 r = make_float2(-INFINITY, -1.0f);
    if (n < a.N) {
        const int64_t want = e.tokens ? e.tokens[m] : -1;
        float z[8];
        sum_parts(a, part, 0, m, n, z);
#pragma unroll
        for (int k = 0; k < 8; k++) {
            if (n + k >= a.N)
                z[k] = -INFINITY;
            else if (n + k == want)
                e.picked[m] = z[k];
        }
        r = sum_exp(z);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
        r = join_lse(r, make_float2(__shfl_xor(r.x, d), __shfl_xor(r.y, d)));
    if ((threadIdx.x & 63) == 0)
        s[threadIdx.x >> 6] = r;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < WAVES; w++)
            r = join_lse(r, s[w]);
        e.part[(int64_t)chunk * a.M + m] = r;
    }
}

template <typename E>
hipError_t join_rows(const Args &a, const float *part, const E &e, int columns, int bf16, hipStream_t st) {
    const uint32_t vectors = (uint32_t)(columns + 7) / 8, all = (uint32_t)a.M * vectors;
    const dim3 grid((all + 255) / 256);
    if (bf16)
        join_kernel<BF16><<<grid, 256, 0, st>>>(a, part, e, make_fastdiv(vectors), all);
    else
        join_kernel<F16><<<grid, 256, 0, st>>>(a, part, e, make_fastdiv(vectors), all);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_join(const Args &a, const float *part, const GatedArgs &e, int bf16, hipStream_t st) {
    return join_rows(a, part, e, e.pad, bf16, st);
}
hipError_t launch_join(const Args &a, const float *part, const GatedBackArgs &e, int bf16, hipStream_t st) {
    return join_rows(a, part, e, e.pad, bf16, st);
}
hipError_t launch_join(const Args &a, const float *part, const DzArgs &e, int bf16, hipStream_t st) {
    return join_rows(a, part, e, e.pad, bf16, st);
}
hipError_t launch_join(const Args &a, const float *part, const LseArgs &e, int, hipStream_t st) {
    const int chunks = (a.N + JOIN_CLASSES - 1) / JOIN_CLASSES;
    join_kernel<<<dim3((unsigned)a.M * (unsigned)chunks), JOIN_CLASSES / 8, 0, st>>>(a, part, e, chunks);
    return hipGetLastError();
}

hipError_t launch_pack(const void *src, int64_t ld, int64_t rows, int cols, const float *factor, void *dst, int bf16,
                       hipStream_t st) {
    const uint32_t per_row = (uint32_t)up8(cols) / 8, n = (uint32_t)(rows * per_row);
    if (n == 0)
        return hipSuccess;
    const dim3 grid((n + 255) / 256);
    if (bf16)
        pack_kernel<BF16><<<grid, 256, 0, st>>>((const uint16_t *)src, ld, cols, factor, (u32x4 *)dst, stride_of(cols) / 8, n,
                                                make_fastdiv(per_row));
    else
        pack_kernel<F16><<<grid, 256, 0, st>>>((const uint16_t *)src, ld, cols, factor, (u32x4 *)dst, stride_of(cols) / 8, n,
                                               make_fastdiv(per_row));
    return hipGetLastError();
}

hipError_t launch_join(const Args &a, const StoreArgs &e, int bf16, hipStream_t st) {
    return bf16 ? join<BF16>(a, e, st) : join<F16>(a, e, st);
}

}  // namespace mm
}  // namespace cf
