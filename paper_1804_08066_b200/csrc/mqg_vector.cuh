// Vectors of V consecutive fp32 or bf16 elements: loads widened to fp32, stores rounded once (to nearest even).
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "mqg_common.cuh"

namespace mqg {

constexpr int kF32 = 0, kBf16 = 1;                      // the values of mqg_dtype
template <int DTYPE> constexpr int kElemBytes = DTYPE == kF32 ? 4 : 2;

template <int DTYPE> struct Element { using type = float; };
template <> struct Element<kBf16> { using type = __nv_bfloat16; };

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void narrow(float x, float& y) { y = x; }
__device__ __forceinline__ void narrow(float x, __nv_bfloat16& y) { y = __float2bfloat16_rn(x); }

// The widest access of V elements: 16 bytes where they fill them, else all of them at once.
template <int BYTES> struct Word;
template <> struct Word<2> { using type = uint16_t; };
template <> struct Word<4> { using type = uint32_t; };
template <> struct Word<8> { using type = uint2; };
template <> struct Word<16> { using type = uint4; };

template <int DTYPE, int V> struct Packed {
    static constexpr int kBytes = V * kElemBytes<DTYPE>;
    static constexpr int kWordBytes = kBytes < 16 ? kBytes : 16;
    static constexpr int kWords = kBytes / kWordBytes;
    using word = typename Word<kWordBytes>::type;
    union {
        word w[kWords];
        typename Element<DTYPE>::type e[V];
    };
    // `p` is aligned to kWordBytes.  Read once: the lines need not stay in L1.
    __device__ __forceinline__ void load(const typename Element<DTYPE>::type* p)
    {
#pragma unroll
        for (int k = 0; k < kWords; ++k) w[k] = __ldcg(reinterpret_cast<const word*>(p) + k);
    }
    __device__ __forceinline__ void store(typename Element<DTYPE>::type* p) const
    {
#pragma unroll
        for (int k = 0; k < kWords; ++k) reinterpret_cast<word*>(p)[k] = w[k];
    }
    __device__ __forceinline__ float get(int i) const { return widen(e[i]); }
    __device__ __forceinline__ void set(int i, float x) { narrow(x, e[i]); }
};

// The V elements of `in` in fp32; a pair of bf16 by a shift and a mask.
template <int DTYPE, int V> __device__ __forceinline__ void widen_to(const Packed<DTYPE, V>& in, float* out)
{
    if constexpr (DTYPE == kBf16 && V > 1) {
        const auto* w = reinterpret_cast<const uint32_t*>(&in);
#pragma unroll
        for (int k = 0; k < V / 2; ++k) {
            out[2 * k] = __uint_as_float(w[k] << 16);
            out[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = in.get(e);
    }
}

// The longest vector of at most `most` elements that divides rows of `dim` elements and starts on its accesses' boundaries
// in both buffers (a null buffer fits all).
inline int row_vector(int most, uint64_t dim, const void* a, int a_bytes, const void* b, int b_bytes)
{
    const auto fits = [](const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & ((bytes < 16 ? bytes : 16) - 1)) == 0; };
    int v = most;
    while (v > 1 && (dim % v != 0 || !fits(a, v * a_bytes) || !fits(b, v * b_bytes))) v /= 2;
    return v;
}

}  // namespace mqg
