// Activations and their slopes, fp32.
//
//   gelu       x Phi(x), slope Phi(x) + x phi(x)          Phi, phi: the normal distribution function and its density
//   gelu_tanh  x s, s = sigmoid(2 sqrt(2 / pi) (x + 0.044715 x^3)) = (1 + tanh(..)) / 2, slope s + x s (1 - s) times the inner slope
//   silu       x sigmoid(x), slope s (1 + x (1 - s))
//
// Phi from its upper tail: with a = |x| and t = 1 / (1 + 0.3 a), 1 - Phi(a) = exp(-a^2 / 2) t P(t); P is a polynomial of degree 7
// fitted to erfc(a / sqrt 2) exp(a^2 / 2) / (2 t) over 0 <= a <= 13.5 so that its largest relative error is least (1.3e-7).  The
// exponential serves the density too: two values and slopes take two reciprocals, two exponentials and 23 other instructions.
// In fp32 the tail is within about (4 + a^2) 2^-23 of its value (the rounding of the exponential's argument, a^2 / 2, and the approximate
// instructions): 5e-7 at 0, 2e-6 at 4, 2e-5 at 13, where it is 1e-38.  Of x Phi(x), and of the slope, it is a share that falls faster than that grows.
// What the formula makes of an infinity is left as it is (0 times infinity is NaN).
#pragma once
#include <cuda_runtime.h>

#include "packed.cuh"

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
constexpr float ACT_LOG2E = 1.4426950408889634f;

__device__ __forceinline__ f32x2 act_exp2(f32x2 x) { return pack_2(act_exp2(low_2(x)), act_exp2(high_2(x))); }
__device__ __forceinline__ f32x2 act_rcp(f32x2 x) { return pack_2(act_rcp(low_2(x)), act_rcp(high_2(x))); }

// Two values at a time.  Phi(x), and e = exp(-x^2 / 2).
__device__ __forceinline__ f32x2 normal_cdf(f32x2 x, f32x2& e) {
    const f32x2 a = x & 0x7fffffff7fffffffull;
    const f32x2 t = act_rcp(fma_2(both_2(0.3f), a, both_2(1.f)));
    e = act_exp2(mul_2(mul_2(a, a), both_2(-0.5f * ACT_LOG2E)));
    f32x2 p = both_2(0.03593173727211247f);
    p = fma_2(p, t, both_2(-0.15827600776286366f));
    p = fma_2(p, t, both_2(0.20820661648988342f));
    p = fma_2(p, t, both_2(-0.055393854726378096f));
    p = fma_2(p, t, both_2(0.12946920384180685f));
    p = fma_2(p, t, both_2(0.0996374922613058f));
    p = fma_2(p, t, both_2(0.12079835853475632f));
    p = fma_2(p, t, both_2(0.11962638971394199f));
    const f32x2 tail = mul_2(mul_2(e, t), p), rest = fma_2(tail, both_2(-1.f), both_2(1.f));
    return pack_2(low_2(x) > 0.f ? low_2(rest) : low_2(tail), high_2(x) > 0.f ? high_2(rest) : high_2(tail));
}
__device__ __forceinline__ f32x2 sigmoid_of_minus_log2(f32x2 u) { return act_rcp(add_2(both_2(1.f), act_exp2(u))); }   // 1 / (1 + 2^u)

// The activation's value, and with SLOPE its slope.
template <int ACT, bool SLOPE>
__device__ __forceinline__ f32x2 act_of(f32x2 x, f32x2& slope) {
    if constexpr (ACT == ACT_GELU) {
        f32x2 e;
        const f32x2 cdf = normal_cdf(x, e);
        if (SLOPE) slope = fma_2(mul_2(x, both_2(0.3989422804014327f)), e, cdf);
        return mul_2(x, cdf);
    } else if constexpr (ACT == ACT_GELU_TANH) {
        constexpr float K = 2.f * 0.7978845608028654f;
        const f32x2 square = mul_2(x, x);
        const f32x2 s = sigmoid_of_minus_log2(mul_2(mul_2(x, both_2(-K * ACT_LOG2E)), fma_2(both_2(0.044715f), square, both_2(1.f))));
        const f32x2 value = mul_2(x, s);
        if (SLOPE) {
            // the bound keeps 0 times infinity out: s (1 - s) is 0 long before it
            const f32x2 bounded = pack_2(fminf(low_2(square), 1e18f), fminf(high_2(square), 1e18f));
            const f32x2 inner = fma_2(both_2(3.f * 0.044715f * K), bounded, both_2(K));
            slope = fma_2(mul_2(value, fma_2(s, both_2(-1.f), both_2(1.f))), inner, s);
        }
        return value;
    } else if constexpr (ACT == ACT_SILU) {
        const f32x2 s = sigmoid_of_minus_log2(mul_2(x, both_2(-ACT_LOG2E))), value = mul_2(x, s);
        if (SLOPE) slope = fma_2(value, fma_2(s, both_2(-1.f), both_2(1.f)), s);
        return value;
    }
    slope = both_2(1.f);
    return x;
}
template <int ACT, int N>
__device__ __forceinline__ void act_values(float (&f)[N]) {
    static_assert(N % 2 == 0, "pairs");
#pragma unroll
    for (int e = 0; e < N; e += 2) {
        f32x2 none;
        const f32x2 v = act_of<ACT, false>(pack_2(f[e], f[e + 1]), none);
        f[e] = low_2(v);
        f[e + 1] = high_2(v);
    }
}

}  // namespace excp
