// Activations of the feed-forward block's gate and their derivatives (ffn.hip, ffn_res.hip).
#pragma once

#include "row_vec.h"

namespace gsc {

__device__ __forceinline__ float ffn_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896f); }

// p = 1 / (1 + exp(-x)) and (D) q = 1 - p, without the difference, which at large x leaves q no digits.
template <bool D>
__device__ __forceinline__ void ffn_sigmoid(float x, float& p, float& q) {
    const float e = ffn_exp(-x);
    p = __builtin_amdgcn_rcpf(1.f + e);
    if (D) q = fminf(e * p, 1.f);   // (e = infinity, p = 0: the minimum of a NaN and 1 is 1)
}

// P(g) of the normal distribution function from e = exp(-g^2 / 2).  Up to |g| = 1 it is 1/2 + g S(g^2), beyond it q = P(-|g|)
// = e t T(t) with t = 1 / (1 + 0.39 |g|); either polynomial is the least-error fit of its degree, S within 7.4e-9 absolutely
// and T within 1.0e-7 of its value out to where q leaves float32's range.  SHORT: one such fit for all g, within 7.9e-7 of q,
// for values that are rounded to bfloat16 (300,000 rows, 256 channels, 1,024 hidden forward 583 us, 611 with both).
template <bool SHORT>
__device__ __forceinline__ float ffn_normal(float g, float e) {
    const float z = fabsf(g);
    if constexpr (SHORT) {
        const float t = __builtin_amdgcn_rcpf(fmaf(0.36f, z, 1.f));
        float q = fmaf(4.7344416e-02f, t, -1.8075161e-01f);
        q = fmaf(q, t, 1.8229754e-01f);
        q = fmaf(q, t, 2.5623852e-02f);
        q = fmaf(q, t, 1.4005741e-01f);
        q = fmaf(q, t, 1.4171067e-01f);
        q = fmaf(q, t, 1.4371744e-01f);
        q = q * t * e;
        return g < 0.f ? q : 1.f - q;
    }
    const float x = g * g;
    float s = fmaf(9.246837e-05f, x, -1.1653508e-03f);
    s = fmaf(s, x, 9.9641671e-03f);
    s = fmaf(s, x, -6.6488728e-02f);
    s = fmaf(s, x, 3.989422e-01f);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.39f, z, 1.f));
    float q = fmaf(6.2847801e-02f, t, -1.8644381e-01f);
    q = fmaf(q, t, 1.2459602e-01f);
    q = fmaf(q, t, 4.986674e-02f);
    q = fmaf(q, t, 1.3879442e-01f);
    q = fmaf(q, t, 1.5486196e-01f);
    q = fmaf(q, t, 1.556191e-01f);
    q = q * t * e;
    return z < 1.f ? fmaf(s, g, 0.5f) : (g < 0.f ? q : 1.f - q);
}

// act(g) and (D) its derivative.  The hardware's exponential and reciprocal, each within a step of float32; what counts in the
// tails is the rounding of the exponential's argument.  In units of 2^-24 of their values SILU and SIGMOID are within
// 1.5 |g| + 8, GELU within 1.25 g^2 + 16, GELU_TANH within 6 |u| + 10 with u = 2 sqrt(2 / pi) (g + 0.044715 g^3), and the
// derivatives, sums of two terms, within about twice as much of either term (32-bit erf and tanh forms are that far off in
// absolute terms, which leaves their negative tails few digits or none).  BF16: the value is rounded to bfloat16 (GELU
// within 1.25 g^2 + 32 units).
template <int ACT, bool D, bool BF16>
__device__ __forceinline__ void ffn_act(float g, float& a, float& d) {
    if constexpr (ACT == GSC_GATE_RELU) {
        a = g < 0.f ? 0.f : g;   // NaN passes through
        if (D) d = g > 0.f ? 1.f : 0.f;
    } else if constexpr (ACT == GSC_GATE_SIGMOID) {
        float q;
        ffn_sigmoid<D>(g, a, q);
        if (D) d = a * q;
    } else if constexpr (ACT == GSC_GATE_SILU) {
        float p, q;
        ffn_sigmoid<D>(g, p, q);
        a = g * p;
        if (D) d = fmaf(a, q, p);
    } else if constexpr (ACT == GSC_GATE_GELU) {
        const float e = ffn_exp(-0.5f * g * g);   // (the derivative takes the density from it)
        const float p = ffn_normal<BF16>(g, e);
        a = g * p;
        if (D) d = fmaf(g * 0.398942280401433f, e, p);
    } else {
        // 0.5 (1 + tanh(u / 2)) = sigmoid(u).  The square is held at 10^4, where the sigmoid is long 0 or 1: without it the
        // derivative is 0 times infinity from |g| = 1.9e19 on.
        const float k = 1.59576912160573f, c = 0.044715f;   // 2 sqrt(2 / pi)
        const float g2 = fminf(g * g, 1e4f);
        float p, q;
        ffn_sigmoid<D>(k * g * fmaf(c, g2, 1.f), p, q);
        a = g * p;
        if (D) d = fmaf(a * q, k * fmaf(3.f * c, g2, 1.f), p);
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
