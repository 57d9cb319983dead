// Activations and their slopes, fp32.
//
//   gelu       x Phi(x), slope Phi(x) + x phi(x)          Phi, phi: the normal distribution function and its density
//   gelu_tanh  x s, s = sigmoid(2 sqrt(2 / pi) (x + 0.044715 x^3)) = (1 + tanh(..)) / 2, slope s + x s (1 - s) times the inner slope
//   silu       x sigmoid(x), slope s (1 + x (1 - s))
//
// Phi from its upper tail: with a = |x| and t = 1 / (1 + 0.3 a), 1 - Phi(a) = exp(-a^2 / 2) t P(t); P is a polynomial of degree 7
// fitted to erfc(a / sqrt 2) exp(a^2 / 2) / (2 t) over 0 <= a <= 13.5 so that its largest relative error is least (1.3e-7).  The
// exponential serves the density too: one reciprocal, one exponential and 15 other instructions for value and slope together.
// In fp32 the tail is within 1e-6 of its value (most of it the exponential's argument).  What the formula makes of an infinity is
// left as it is (0 times infinity is NaN).
#pragma once
#include <cuda_runtime.h>

namespace excp {

enum Activation { ACT_NONE = 0, ACT_GELU = 1, ACT_GELU_TANH = 2, ACT_SILU = 3 };

__device__ __forceinline__ float act_exp2(float x) {       // relative error 2^-22
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float act_rcp(float x) {        // relative error 2^-23; 0 of infinity
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float sigmoid_of_log2(float u) { return act_rcp(1.f + act_exp2(-u)); }      // u in powers of two

constexpr float ACT_LOG2E = 1.4426950408889634f;

// Phi(x), and e = exp(-x^2 / 2).
__device__ __forceinline__ float normal_cdf(float x, float& e) {
    const float a = fabsf(x);
    const float t = act_rcp(fmaf(0.3f, a, 1.f));
    e = act_exp2(a * a * (-0.5f * ACT_LOG2E));
    float p = 0.03593173727211247f;
    p = fmaf(p, t, -0.15827600776286366f);
    p = fmaf(p, t, 0.20820661648988342f);
    p = fmaf(p, t, -0.055393854726378096f);
    p = fmaf(p, t, 0.12946920384180685f);
    p = fmaf(p, t, 0.0996374922613058f);
    p = fmaf(p, t, 0.12079835853475632f);
    p = fmaf(p, t, 0.11962638971394199f);
    const float tail = e * t * p;
    return x > 0.f ? 1.f - tail : tail;
}

template <int ACT>
__device__ __forceinline__ float act_value(float x) {
    if constexpr (ACT == ACT_GELU) {
        float e;
        return x * normal_cdf(x, e);
    } else if constexpr (ACT == ACT_GELU_TANH) {
        constexpr float C = 2.f * 0.7978845608028654f * ACT_LOG2E;
        return x * sigmoid_of_log2(C * x * fmaf(0.044715f * x, x, 1.f));
    } else if constexpr (ACT == ACT_SILU) {
        return x * sigmoid_of_log2(ACT_LOG2E * x);
    }
    return x;
}

// The slope; `value` is the activation's value.
template <int ACT>
__device__ __forceinline__ float act_slope(float x, float& value) {
    if constexpr (ACT == ACT_GELU) {
        float e;
        const float cdf = normal_cdf(x, e);
        value = x * cdf;
        return fmaf(x * 0.3989422804014327f, e, cdf);
    } else if constexpr (ACT == ACT_GELU_TANH) {
        constexpr float K = 2.f * 0.7978845608028654f;
        const float s = sigmoid_of_log2(K * ACT_LOG2E * x * fmaf(0.044715f * x, x, 1.f));
        value = x * s;
        // the bound keeps 0 times infinity out: s (1 - s) is 0 long before it
        const float inner = K * fmaf(3.f * 0.044715f, fminf(x * x, 1e18f), 1.f);
        return fmaf(value * (1.f - s), inner, s);
    } else if constexpr (ACT == ACT_SILU) {
        const float s = sigmoid_of_log2(ACT_LOG2E * x);
        value = x * s;
        return fmaf(value, 1.f - s, s);
    }
    value = x;
    return 1.f;
}

}  // namespace excp
