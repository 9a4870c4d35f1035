// cf_act.h -- activation functions with their slopes in fp32, for operators
// whose backward pass makes both from one argument.
#pragma once

#include "cf_device.h"

namespace cf {

enum { ACT_SILU = 3 };  // after ACT_GELU, ACT_RELU and ACT_NONE

struct ActPair {
    float f, d;  // act(u), act'(u)
};

// NaN stays NaN; infinities give the limits (0 and 0 at -inf, inf and 1 at inf;
// for ACT_NONE the identity).
//   GELU  Phi = 1 - tail or tail with the tail q(t) exp(-u^2/2) of gelu_f32, whose
//         coefficients these are (1.5e-8): f = max(u, 0) - |u| tail, d = Phi + u phi(u)
//   SiLU  s = 1 / (1 + exp(-u)): f = u s, d = s (1 + u (1 - s)), u taken as -128 below
//         it, where both are 0 in fp32
//   ReLU  d(0) = 0
template <int ACT>
__device__ __forceinline__ ActPair act_pair(float u) {
    if constexpr (ACT == ACT_GELU) {
        const float v = __builtin_amdgcn_fmed3f(u, -32.0f, 32.0f);  // where the exponential is 0
        const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(u), 0.32f, 1.0f));
        float q = fmaf(-0.129858347f, t, 0.495794653f);
        q = fmaf(q, t, -0.265561934f);
        q = fmaf(q, t, 0.314940331f);
        q = fmaf(q, t, 0.079603797f);
        q = fmaf(q, t, 0.005081451f);
        const float e = __builtin_amdgcn_exp2f(u * u * -0.721347520f), tail = q * e;  // NaN where u is
        return {fmaf(-fabsf(v), tail, fmaxf(u, 0.0f)), fmaf(v, e * 0.398942280f, v > 0.0f ? 1.0f - tail : tail)};
    } else if constexpr (ACT == ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u * -1.44269504f));  // NaN where u is
        const float f = fmaxf(u, -128.0f) * s;
        return {f, fmaf(fminf(f, 128.0f), 1.0f - s, s)};
    } else if constexpr (ACT == ACT_RELU) {
        return {u < 0.0f ? 0.0f : u, u > 0.0f ? 1.0f : u <= 0.0f ? 0.0f : u};
    } else {
        return {u, u != u ? u : 1.0f};
    }
}

// act(u) alone; GELU at -inf is 0 here too.
template <int ACT>
__device__ __forceinline__ float act_value(float u) {
    if constexpr (ACT == ACT_GELU)
        return gelu_f32(u);
    else
        return act_pair<ACT>(u).f;
}

template <int A>
struct ActTag {
    static constexpr int value = A;
};
// f(ActTag<act>()), one uniform branch for all that f does
template <typename F>
__device__ __forceinline__ void with_act(int act, F &&f) {
    if (act == ACT_SILU)
        f(ActTag<ACT_SILU>());
    else if (act == ACT_GELU)
        f(ActTag<ACT_GELU>());
    else if (act == ACT_RELU)
        f(ActTag<ACT_RELU>());
    else
        f(ActTag<ACT_NONE>());
}

}  // namespace cf
