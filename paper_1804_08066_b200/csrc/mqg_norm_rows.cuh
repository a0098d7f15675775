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

// Sum over `lanes` neighbouring lanes, a power of two up to 32.
__device__ __forceinline__ float lanes_sum(float v, uint32_t lanes)
{
#pragma unroll
    for (uint32_t d = 16; d > 0; d >>= 1)
        if (d < lanes) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

__device__ __forceinline__ float reciprocal_deviation(float variance, float eps) { return __frcp_rn(__fsqrt_rn(variance + eps)); }

__device__ __forceinline__ float weight_at(const void* w, int dtype, uint64_t i)
{
    return dtype == kF32 ? static_cast<const float*>(w)[i] : widen(static_cast<const __nv_bfloat16*>(w)[i]);
}

// V weights from element i on, or V times `none`.  Every row reads them: they stay in L1.
template <int V> __device__ __forceinline__ void weights_at(const void* w, int dtype, uint32_t i, float none, float (&out)[V])
{
    if (w == nullptr) {
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = none;
    } else if (dtype == kF32) {
        constexpr int kWord = V < 4 ? V : 4;
        const auto* p = reinterpret_cast<const typename Word<4 * kWord>::type*>(static_cast<const float*>(w) + i);
        union { typename Word<4 * kWord>::type w[V / kWord]; float e[V]; } u;
#pragma unroll
        for (int k = 0; k < V / kWord; ++k) u.w[k] = __ldg(p + k);
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = u.e[e];
    } else {
        union { typename Word<2 * V>::type w; __nv_bfloat16 e[V]; } u;
        u.w = __ldg(reinterpret_cast<const typename Word<2 * V>::type*>(static_cast<const __nv_bfloat16*>(w) + i));
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = widen(u.e[e]);
    }
}

// The elements of a vector: 16 bytes where both types are bf16 or fp32 (x and y of a call), 4 elements of mixed ones.
template <int A, int B> constexpr int kVector = A == kBf16 && B == kBf16 ? 8 : 4;

// Whether vectors of v elements fit rows of `dim` elements that start at p.
inline bool vectors_fit(const void* p, int bytes, int v, uint64_t dim)
{
    const int word = v * bytes < 16 ? v * bytes : 16;
    return dim % v == 0 && (reinterpret_cast<uintptr_t>(p) & (word - 1)) == 0;
}

inline int element_bytes(int dtype) { return dtype == kF32 ? 4 : 2; }

}  // namespace mqg
