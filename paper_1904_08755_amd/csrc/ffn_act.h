// Activations of the feed-forward block's gate and their derivatives (ffn.hip, ffn_res.hip).
#pragma once

#include "row_vec.h"

namespace gsc {

__device__ __forceinline__ float ffn_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896f); }
__device__ __forceinline__ float ffn_sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + ffn_exp(-x)); }

// act(g) and (D) its derivative.  The hardware's exponential and reciprocal: within about |g| + 2 units in
// the last place of float32, far inside what the products' sums lose.
template <int ACT, bool D>
__device__ __forceinline__ void ffn_act(float g, float& a, float& d) {
    if constexpr (ACT == GSC_GATE_RELU) {
        a = g < 0.f ? 0.f : g;   // NaN passes through
        if (D) d = g > 0.f ? 1.f : 0.f;
    } else if constexpr (ACT == GSC_GATE_SIGMOID) {
        a = ffn_sigmoid(g);
        if (D) d = a * (1.f - a);
    } else if constexpr (ACT == GSC_GATE_SILU) {
        const float p = ffn_sigmoid(g);
        a = g * p;
        if (D) d = fmaf(a, 1.f - p, p);
    } else if constexpr (ACT == GSC_GATE_GELU) {
        // the normal distribution function from Abramowitz & Stegun 7.1.26 (absolute error of erf 1.5e-7),
        // its density shared with the derivative
        const float z = fabsf(g) * 0.70710678118655f;
        const float e = ffn_exp(-0.5f * g * g);
        const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, z, 1.f));
        float q = fmaf(1.061405429f, t, -1.453152027f);
        q = fmaf(q, t, 1.421413741f);
        q = fmaf(q, t, -0.284496736f);
        q = fmaf(q, t, 0.254829592f);
        q = 0.5f * q * t * e;              // the upper tail at |g|
        const float p = g < 0.f ? q : 1.f - q;
        a = g * p;
        if (D) d = fmaf(g * 0.398942280401433f, e, p);
    } else {
        // 0.5 (1 + tanh(u)) = sigmoid(2 u)
        const float k = 0.797884560802865f, c = 0.044715f;
        const float g2 = g * g;
        const float p = ffn_sigmoid(2.f * k * g * fmaf(c, g2, 1.f));
        a = g * p;
        if (D) d = fmaf(2.f * a * (1.f - p), k * fmaf(3.f * c, g2, 1.f), p);
    }
}

// f(activation as a constant)
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
    switch (act) {
        case GSC_GATE_RELU: f(std::integral_constant<int, GSC_GATE_RELU>{}); break;
        case GSC_GATE_SIGMOID: f(std::integral_constant<int, GSC_GATE_SIGMOID>{}); break;
        case GSC_GATE_GELU: f(std::integral_constant<int, GSC_GATE_GELU>{}); break;
        case GSC_GATE_GELU_TANH: f(std::integral_constant<int, GSC_GATE_GELU_TANH>{}); break;
        default: f(std::integral_constant<int, GSC_GATE_SILU>{}); break;
    }
}

}  // namespace gsc
