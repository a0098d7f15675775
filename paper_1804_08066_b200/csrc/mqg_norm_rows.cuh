// What the layer norm's forward and backward kernels share.
#pragma once

#include <stdint.h>

#include "mqg_vector.cuh"

namespace mqg {

constexpr int kLongThreads = 512;

// Sum over a CTA of kLongThreads threads, in 64 bits, in a fixed order.
__device__ __forceinline__ double long_sum(double v)
{
    __shared__ double warp_sum[kLongThreads / 32];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    __syncthreads();                                    // the sums before these have been read
    if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = v;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int w = 0; w < kLongThreads / 32; ++w) t += warp_sum[w];
    return t;
}

__device__ __forceinline__ float reciprocal_deviation(float variance, float eps) { return __frcp_rn(__fsqrt_rn(variance + eps)); }

__device__ __forceinline__ float weight_at(const void* w, int dtype, uint64_t i)
{
    return dtype == kF32 ? static_cast<const float*>(w)[i] : widen(static_cast<const __nv_bfloat16*>(w)[i]);
}

}  // namespace mqg
