// Asynchronous copies to shared memory, by a thread for itself.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

namespace mqg {

template <int BYTES> __device__ __forceinline__ void copy_async(void* to, const void* from)
{
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Lets `kernel` use `bytes` of dynamic shared memory on the current device.  `ready`: of this kernel, by device.
template <typename Kernel> cudaError_t allow_shared(Kernel kernel, size_t bytes, std::atomic<bool> (&ready)[64])
{
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev].load(std::memory_order_relaxed)) {
        err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (err != cudaSuccess) return err;
        ready[dev].store(true, std::memory_order_relaxed);
    }
    return cudaSuccess;
}

}  // namespace mqg
