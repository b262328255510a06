// Launches of the 8-bit cache's kernels.
//
// They follow one another in short chains, so each is launched as a programmatic dependent of what is before it on the
// stream: its CTAs may be set up while that still runs, and wait (pdl_wait, before they touch memory) until it has ended
// and its writes are visible.  A kernel that calls pdl_open at its start lets what comes behind it be set up beside it.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

namespace bct {

__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_open() { asm volatile("griddepcontrol.launch_dependents;"); }

template <typename... P, typename... A>
cudaError_t pdl_launch(void (*kernel)(P...), unsigned grid, unsigned threads, size_t smem, cudaStream_t s, const A&... args) {
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(grid);
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    c.stream = s;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    c.attrs = &at;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, kernel, args...);
}

// The opt-in for more than 48 KiB of shared memory, once for each device; done: a kernel's own, a bit per device.
template <typename K>
cudaError_t allow_smem(K kernel, int bytes, std::atomic<uint64_t>* done) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < 64 && ((done->load(std::memory_order_relaxed) >> dev) & 1))) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev < 64) done->fetch_or(1ull << dev, std::memory_order_relaxed);
    return e;
}

}  // namespace bct
