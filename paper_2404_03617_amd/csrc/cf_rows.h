// cf_rows.h -- device helpers of the row operators (layer norm, activation
// checkpoints, log probabilities): vectors of a row at any alignment, sums
// and maxima over groups of lanes, and the 8-bit block format.  Internal
// header; not part of the C ABI.
#pragma once

#include "cf_device.h"

namespace cf {

// Largest row lengths with a kernel, and the channels that share one scale of
// a checkpoint.
constexpr int NORM_MAX_C = 16384;
constexpr int CKPT_BLOCK = 64;
// A block whose largest magnitude is below this is kept as zeros: 127 / a
// stays finite.
constexpr float CKPT_TINY = 0x1p-119f;

// 16 or 8 bytes that start at any element: rows of odd lengths and views of
// wider tensors start anywhere.  One (unaligned) load either way; the
// hardware splits those that cross a cache line.
struct __attribute__((packed, aligned(2))) Any16 {
    u32x4 v;
};
struct __attribute__((packed, aligned(1))) Any8 {
    u32x2 v;
};

struct __attribute__((packed, aligned(2))) Any4h {
    uint32_t v;
};
struct __attribute__((packed, aligned(2))) Any8h {
    u32x2 v;
};

// the last n of 16 (8) bytes' values, of 16 (8) bits each, moved to the front;
// behind them zeros or, with `around`, the values that stood before them
template <bool AROUND = false>
__device__ __forceinline__ u32x4 from_end(const u32x4 &r, int n) {
    const int s = 16 * (8 - n);  // 16 .. 112
    const uint64_t lo = __builtin_bit_cast(uint64_t, u32x2{r[0], r[1]}), hi = __builtin_bit_cast(uint64_t, u32x2{r[2], r[3]});
    uint64_t l = s < 64 ? lo >> s | hi << (64 - s) : hi >> (s - 64), h = s < 64 ? hi >> s : 0;
    if constexpr (AROUND) {
        l |= s > 64 ? lo << (128 - s) : 0;
        h |= s < 64 ? lo << (64 - s) : s == 64 ? lo : lo >> (s - 64) | hi << (128 - s);
    }
    return {(uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32)};
}

// An offset that is the same in all lanes, in a vector register: a uniform
// address would go to a scalar load, which needs 4-byte alignment.
__device__ __forceinline__ int per_lane(int i) {
    asm("" : "+v"(i));
    return i;
}

// 8 elements of a row of C, from element c on, zeros past its end (AROUND:
// other elements of the row, where c is in it).  The last ones of a row that is
// no multiple of 8 come with those before them.
template <bool AROUND = false>
__device__ __forceinline__ u32x4 load8(const uint16_t *row, int c, int C) {
    const int n = C - c;
    if (n >= 8)
        return reinterpret_cast<const Any16 *>(row + c)->v;
    if (n <= 0)
        return u32x4{0u, 0u, 0u, 0u};
    if (C >= 8)
        return from_end<AROUND>(reinterpret_cast<const Any16 *>(row + per_lane(C - 8))->v, n);
    u32x4 r = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < (AROUND ? 8 : 7); i++)
        if (AROUND || i < n)
            r[i / 2] |= (uint32_t)row[c + (i < n ? i : 0)] << (16 * (i & 1));
    return r;
}

__device__ __forceinline__ void store8(uint16_t *row, int c, int C, const u32x4 &r) {
    const int n = C - c;
    uint16_t *const p = row + c;
    if (n >= 8) {
        reinterpret_cast<Any16 *>(p)->v = r;
        return;
    }
    if (n <= 0)
        return;
    const uint32_t w2 = n & 4 ? r[2] : r[0], w3 = n & 4 ? r[3] : r[1];  // what follows the first 0 or 4
    if (n & 4)
        reinterpret_cast<Any8h *>(p)->v = u32x2{r[0], r[1]};
    if (n & 2)
        reinterpret_cast<Any4h *>(p + (n & 4))->v = w2;
    if (n & 1)
        p[n - 1] = (uint16_t)(n & 2 ? w3 : w2);
}

// 8 bytes of a checkpoint's row, the same way.
template <bool AROUND = false>
__device__ __forceinline__ u32x2 load8b(const int8_t *row, int c, int C) {
    const int n = C - c;
    if (n >= 8)
        return reinterpret_cast<const Any8 *>(row + c)->v;
    if (n <= 0)
        return u32x2{0u, 0u};
    if (C >= 8) {
        const uint64_t v = __builtin_bit_cast(uint64_t, reinterpret_cast<const Any8 *>(row + per_lane(C - 8))->v);
        return __builtin_bit_cast(u32x2, v >> (8 * (8 - n)) | (AROUND ? v << (8 * n) : 0));
    }
    u32x2 r = {0u, 0u};
#pragma unroll
    for (int i = 0; i < (AROUND ? 8 : 7); i++)
        if (AROUND || i < n)
            r[i / 4] |= (uint32_t)(uint8_t)row[c + (i < n ? i : 0)] << (8 * (i & 3));
    return r;
}

__device__ __forceinline__ void store8b(int8_t *row, int c, int C, const u32x2 &r) {
    const int n = C - c;
    if (n >= 8) {
        reinterpret_cast<Any8 *>(row + c)->v = r;
        return;
    }
#pragma unroll
    for (int i = 0; i < 7; i++)
        if (i < n)
            row[c + i] = (int8_t)(r[i / 4] >> (8 * (i & 3)));
}

// 8 floats of a vector (weight, bias) from p, `rest` from element n on or
// where there is no vector.
struct __attribute__((packed, aligned(4))) AnyF4 {
    float4v v;
};
__device__ __forceinline__ void load8f(const float *p, int n, float rest, float *f) {
    if (p && n >= 8) {
        const float4v a = reinterpret_cast<const AnyF4 *>(p)->v, b = reinterpret_cast<const AnyF4 *>(p + 4)->v;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            f[i] = a[i];
            f[4 + i] = b[i];
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++)
        f[i] = p && i < n ? p[i] : rest;
}

template <typename T>
__device__ __forceinline__ void unpack8(const u32x4 &r, float *f) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
        f[2 * i] = T::lo(r[i]);
        f[2 * i + 1] = T::hi(r[i]);
    }
}

template <typename T>
__device__ __forceinline__ u32x4 pack8(const float *f) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; i++)
        r[i] = T::pack2(f[2 * i], f[2 * i + 1]);
    return r;
}

// ---------------------------------------------------------------------------
// Sums over aligned groups of G lanes, the result in every lane: lanes 1 and 2
// apart by quad permutes, the two quads of 8 and the two halves of 16 by
// mirrors, rows of 16 and halves of the wave by the swap instructions.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    const int i = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, CTRL, 0xf, 0xf, true));
}
constexpr int DPP_XOR1 = 0xb1, DPP_XOR2 = 0x4e, DPP_MIRROR8 = 0x141, DPP_MIRROR16 = 0x140;

// both halves of the exchange, for the caller to combine
struct Two {
    float a, b;
};
__device__ __forceinline__ Two swap16(float v) {
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return {__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1])};
}
__device__ __forceinline__ Two swap32(float v) {
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return {__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1])};
}

struct Add {
    static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};
// a NaN on either side is the result (IEEE 754-2019 maximum)
struct Max {
    static __device__ __forceinline__ float of(float a, float b) { return __builtin_elementwise_maximum(a, b); }
};

template <typename Op, int G>
__device__ __forceinline__ float lanes(float v) {
    static_assert(G == 1 || G == 2 || G == 4 || G == 8 || G == 16 || G == 32 || G == 64, "a part of a wave");
    if constexpr (G >= 2)
        v = Op::of(v, dpp<DPP_XOR1>(v));
    if constexpr (G >= 4)
        v = Op::of(v, dpp<DPP_XOR2>(v));
    if constexpr (G >= 8)
        v = Op::of(v, dpp<DPP_MIRROR8>(v));
    if constexpr (G >= 16)
        v = Op::of(v, dpp<DPP_MIRROR16>(v));
    if constexpr (G >= 32) {
        const Two t = swap16(v);
        v = Op::of(t.a, t.b);
    }
    if constexpr (G >= 64) {
        const Two t = swap32(v);
        v = Op::of(t.a, t.b);
    }
    return v;
}

// ---------------------------------------------------------------------------
// The 8-bit format: for each block of 64 channels of a row, with a = max |x|,
//   q = rint(x * (127 / a)),  scale = a * (1 / 127),  x ~ q * scale,
// in fp32 with one rounding an operation, so that q depends on the 16-bit
// values alone.  a < 2^-119: zeros with scale 0; infinities or NaN: the scale
// is NaN and so is every value of the block.
struct Quant {
    float inv, scale;
};

__device__ __forceinline__ Quant quant_of(float a) {
    Quant z;
    z.inv = a >= CKPT_TINY && a < INFINITY ? 127.0f / a : 0.0f;
    z.scale = a < CKPT_TINY ? 0.0f : a < INFINITY ? a * (1.0f / 127.0f) : NAN;
    return z;
}

// largest magnitude of 8 values (NaN if any is)
__device__ __forceinline__ float amax8(const float *x) {
    float a = fabsf(x[0]);
#pragma unroll
    for (int i = 1; i < 8; i++)
        a = Max::of(a, fabsf(x[i]));
    return a;
}

// 8 values to 8 bytes.  The sum with 1.5 * 2^23 rounds the product to an
// integer in the low bits; product and sum are rounded one after the other.
// inv is 0 where the block is not finite: its bytes are zeros or whatever the
// low bits of NaN are, and its scale is NaN.
__device__ __forceinline__ u32x2 quant8(const float *x, float inv) {
#pragma clang fp contract(off)
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float p = x[i] * inv;
        b[i] = __builtin_bit_cast(uint32_t, p + 12582912.0f);
    }
    u32x2 r;
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const uint32_t lo = __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x0c0c0400u);
        r[i] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
    }
    return r;
}

// byte i of 4 as a float
__device__ __forceinline__ float signed_byte(uint32_t w, int i) { return (float)(int8_t)(w >> (8 * i)); }

// 8 bytes to values q * scale, each rounded to fp32 before anything else is done
// with it: most 16-bit values that were the largest of their block come back as
// they were, and so does a row of them, whose x - mean is 0.  (Fused with the
// subtraction of the mean the product keeps the rounding of the scale.)
__device__ __forceinline__ void dequant8(const u32x2 &q, float scale, float *x) {
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < 8; i++)
        x[i] = signed_byte(q[i / 4], i & 3) * scale;
}

inline int blocks_of(int C) { return (C + CKPT_BLOCK - 1) / CKPT_BLOCK; }

}  // namespace cf
