// The activations of a gated feed-forward block and their slopes, in fp32.
//   silu      x s(x), s(x) = 1 / (1 + e^-x)                    slope  s (1 + x (1 - s))
//   gelu      x Phi(x), Phi(x) = (1 + erf(x / sqrt 2)) / 2     slope  Phi + x e^(-x^2 / 2) / sqrt(2 pi)
//   gelu_tanh x t(x), t(x) = s(2 k (x + 0.044715 x^3)), k = sqrt(2 / pi), since (1 + tanh z) / 2 = s(2 z)
//                                                              slope  t + x t (1 - t) 2 k (1 + 3 0.044715 x^2)
#pragma once

#include "windq_common.hpp"

namespace windq {

#ifdef __HIPCC__

// e^x as 2^h (1 + l ln 2) with x log2 e = h + l, h in fp32 and l what that leaves: two units in the last place, a third of the instructions of a
// library's exponential and quotient (64 results a lane wait for them at the end of a tile).  Below 2^-126 it is 0.
__device__ __forceinline__ float exponential(float x) {
    const float h = x * 1.44269504f, l = fmaf(x, 1.44269504f, -h) + x * 1.92596303e-8f;
    const float p = __builtin_amdgcn_exp2f(h);
    return h < 127.0f && h > -200.0f ? fmaf(p, l * 0.693147181f, p) : p;      // an infinite p or h has no use for l
}
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + exponential(-x)); }

// act(x), and its slope where SLOPE.
template <bool SLOPE>
__device__ __forceinline__ float activation(int act, float x, float& slope) {
    float y;
    if (act == WINDQ_SILU) {
        const float s = sigmoid(x);
        y = x * s;
        if (SLOPE) slope = s * (1.0f + x * (1.0f - s));
    } else if (act == WINDQ_GELU) {
        // erfc in the place of 1 + erf: Phi keeps its digits far to the left
        const float phi = 0.5f * erfcf(x * -0.70710678118654752f);
        y = x * phi;
        if (SLOPE) slope = phi + x * (exponential(-0.5f * x * x) * 0.39894228040143268f);
    } else {
        constexpr float K2 = 1.5957691216057308f;          // 2 sqrt(2 / pi)
        const float x2 = x * x, t = sigmoid(K2 * (x + 0.044715f * x2 * x));
        y = x * t;
        const float q = t * (1.0f - t);                    // 0 far from 0, where x^2 may be infinite
        if (SLOPE) slope = q > 0.0f ? t + x * q * (K2 * (1.0f + 0.134145f * x2)) : t;
    }
    return y;
}

#endif  // __HIPCC__

}  // namespace windq
