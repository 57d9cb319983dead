// How the scoring kernels are launched: each may be set up while the one before it in the stream still runs (programmatic
// dependent launch), waits for that one's end before it touches what others write, and only then lets the next be set up.  So
// a kernel that has begun knows that everything before its immediate predecessor has ended.
#pragma once
#include <atomic>

#include "score.cuh"

namespace excp {

// Every thread, first of all.  (Does nothing behind a kernel of another kind, which has ended by then.)
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// cluster: blocks per cluster, 0 where the kernel says so itself or has none.
template <typename... P, typename... A>
bool launch_chained(void (*kernel)(P...), u32 grid, u32 block, u32 smem, u32 cluster, cudaStream_t s, const A&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) == cudaSuccess;
}

// Lets `kernel` use up to `bytes` of dynamic shared memory; asked of the driver once per device (`done`: one bit each).
template <typename K>
bool allow_smem(K kernel, std::atomic<u64>& done, u32 bytes) {
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess) return false;
    const u64 bit = 1ull << (device & 63);
    if (done.load(std::memory_order_relaxed) & bit) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) return false;
    done.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

}  // namespace excp
