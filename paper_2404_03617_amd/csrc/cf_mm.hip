// cf_mm.hip -- what stands around the products of cf_mm.h: packed copies of
// operands that the tiles cannot read where they are, and the joining of split
// sums.  Both are bound by memory.
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
    const int64_t row = i / per_row;  // of batch * M
    const int batch = (int)(row / a.M), m = (int)(row - (int64_t)batch * a.M), c = (int)(i - row * per_row) * 4;
    const int64_t step = (int64_t)a.batch * a.M * a.N;
    const float *p = e.part + ((int64_t)batch * a.M + m) * a.N + c;
    float4v v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int s = g; s < a.splits; s += G)
    {
        float4v w;
        load_rowf<4>(p + s * step, w, a.N - c);
        v += w;
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
    const int64_t n = (int64_t)a.batch * a.M * per_row;
    if (n >= 65536 || a.splits < 8)
        join_kernel<T, 1><<<dim3((unsigned)((n + 255) / 256)), 256, 0, st>>>(a, e, per_row, n);
    else
        join_kernel<T, 8><<<dim3((unsigned)((n * 8 + 255) / 256)), 256, 0, st>>>(a, e, per_row, n);
    return hipGetLastError();
}

}  // namespace

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
