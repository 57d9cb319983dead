// What the two kernels of the 4-bit product share: bounded waits of whole warps, the ring of stages.
#pragma once
#include "score_launch.cuh"
#include "tcgen05.cuh"

namespace excp {

constexpr u64 DRAIN_NS = 100000000ull;             // a copy in flight lands within microseconds

// A whole warp waits for phase `parity` of `bar`; false when the limit has passed or another role gave up.
template <typename S>
__device__ __forceinline__ bool wait_long(S* sh, unsigned long long* bar, u32 parity, u64 limit_ns, u32* flag) {
    if (limit_ns) {
        const u64 t0 = global_ns();
        while (!__any_sync(0xffffffffu, sh->abort)) {
            if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
            if (__any_sync(0xffffffffu, global_ns() - t0 > limit_ns)) break;
        }
    }
    if (!__any_sync(0xffffffffu, sh->abort)) {
        sh->abort = 1;
        *reinterpret_cast<volatile u32*>(flag) = 1;
        __threadfence_system();
    }
    return false;
}
template <typename S>
__device__ __forceinline__ bool wait_warp(S* sh, unsigned long long* bar, u32 parity, u64 limit_ns, u32* flag) {
    if (limit_ns)
        for (int i = 0; i < 32; ++i)
            if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    return wait_long(sh, bar, parity, limit_ns, flag);
}
// The same without raising anything: for letting one's own work land before leaving.
__device__ __forceinline__ void drain_warp(unsigned long long* bar, u32 parity) {
    const u64 t0 = global_ns();
    while (!__all_sync(0xffffffffu, mbar_try_wait(bar, parity)) && !__any_sync(0xffffffffu, global_ns() - t0 > DRAIN_NS)) {}
}

// The two tensor scales (null = 1) as factors that a sum is multiplied with, one after the other.  Mostly their product and 1;
// where the product leaves fp32's normal numbers, what brings the sum back to the middle first goes first, so that
// neither a result that fits is lost nor 0 times infinity is formed.
struct TensorScales {
    float first, second;
};
__device__ __forceinline__ TensorScales tensor_scales(const float* a, const float* b) {
    const float x = a ? __ldg(a) : 1.f, y = b ? __ldg(b) : 1.f, both = x * y;
    if (both >= 0x1p-126f && both <= 0x1.fffffep127f) return TensorScales{both, 1.f};
    const float low = fminf(x, y), high = fmaxf(x, y);
    return both < 1.f ? TensorScales{high, low} : TensorScales{low, high};
}

// The place in the ring of stages, and the parity of its current turn.
template <int STAGES>
struct Ring {
    u32 s = 0, parity = 0;
    __device__ __forceinline__ void next() {
        if (++s == STAGES) { s = 0; parity ^= 1; }
    }
};

}  // namespace excp
