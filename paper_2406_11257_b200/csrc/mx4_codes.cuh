// From values to 4-bit codes and block scales (definitions: include/excp.h).
#pragma once
#include <cuda_fp8.h>

#include "score.cuh"

namespace excp {

constexpr u32 NONFINITE_BITS = 0x7f800000u;        // magnitudes at or above: infinity and NaN

// Eight values as eight 4-bit floats (nearest, ties to even, at most 6), the first in the low bits.
__device__ __forceinline__ u32 e2m1x8(const float* t) {
    u32 w;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(w)
        : "f"(t[0]), "f"(t[1]), "f"(t[2]), "f"(t[3]), "f"(t[4]), "f"(t[5]), "f"(t[6]), "f"(t[7]));
    return w;
}

// Two fp32 lanes per instruction.
__device__ __forceinline__ u64 f2_pack(float a, float b) { u64 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void f2_unpack(u64 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ u64 f2_mul(u64 a, u64 b) { u64 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ u64 f2_fma(u64 a, u64 b, u64 c) { u64 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }

// The block's scale byte, and N of its values divided by the scale (in place).  `m`: pattern of the block's largest
// magnitude.
template <int N>
__device__ __forceinline__ u32 scale_e8m0(float (&v)[N], u32 m) {
    if (m >= NONFINITE_BITS) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = 0.f;
        return 0xffu;
    }
    const int lg = (m >> 23) ? (int)(m >> 23) - 127 : (m ? -118 - __clz(m) : -1000);   // floor(log2): bit b of a subnormal is 2^(b - 149)
    const int e = max(lg - 2, -127);
    const float inv = __uint_as_float((u32)(127 - e) << 23);                            // 2^-e: exact, -e in [-125, 127]
    const u64 inv2 = f2_pack(inv, inv);
#pragma unroll
    for (int k = 0; k < N; k += 2) f2_unpack(f2_mul(f2_pack(v[k], v[k + 1]), inv2), v[k], v[k + 1]);
    return (u32)(e + 127);
}
// The same for blocks of 16, but the quotients come out with the other sign (codes_of puts it right): one step from a negative
// reciprocal keeps the sign of a zero, one from a positive reciprocal makes -0 a +0.
template <int N>
__device__ __forceinline__ u32 scale_e4m3(float (&v)[N], u32 m, float g, float six_g) {
    u32 byte = 0x7fu;
    float sg = 0.f;
    if (m < NONFINITE_BITS) {
        const __nv_fp8_storage_t s = __nv_cvt_float_to_fp8(m ? __fdiv_rn(__uint_as_float(m), six_g) : 0.f, __NV_SATFINITE, __NV_E4M3);
        byte = s;
        sg = __half2float(__half(__nv_cvt_fp8_to_halfraw(s, __NV_E4M3))) * g;
    }
    if (sg >= 0x1p-80f && sg <= 0x1p80f && __uint_as_float(m) < 0x1p20f * sg) {
        // The rounded quotient from the rounded reciprocal: one step with the exact remainder (Markstein 1990).  Without it a
        // value halfway between two codes could fall to the wrong side.
        const float r = -__frcp_rn(sg);
        const u64 r2 = f2_pack(r, r), d2 = f2_pack(sg, sg);
#pragma unroll
        for (int k = 0; k < N; k += 2) {
            const u64 x = f2_pack(v[k], v[k + 1]), q = f2_mul(x, r2);
            f2_unpack(f2_fma(f2_fma(q, d2, x), r2, q), v[k], v[k + 1]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = sg > 0.f ? __fdiv_rn(v[k], -sg) : -0.f;
    }
    return byte;
}

// Eight codes of what scale_e8m0 or scale_e4m3 left.
template <int FMT>
__device__ __forceinline__ u32 codes_of(const float* t) {
    return FMT == MX4_E4M3_16 ? e2m1x8(t) ^ 0x88888888u : e2m1x8(t);
}

// Four scale bytes of a row as one word: block k's byte is held by the lanes around 8-value group src + k * PER.
template <int FMT>
__device__ __forceinline__ u32 scale_word(u32 byte, u32 src) {
    constexpr int PER = mx4_block(FMT) / 8;        // lanes (8 values each) to a block
    u32 w = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) w |= __shfl_sync(0xffffffffu, byte, src + k * PER) << (8 * k);
    return w;
}

}  // namespace excp
