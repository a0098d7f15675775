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

// W elements from x on, put together from the aligned word that holds the first of them and the word behind it; `bytes` of the
// first word lie before x.  Words of 4 to 16 bytes.
template <int DTYPE, int W>
__device__ __forceinline__ Packed<DTYPE, W> load_across(const typename Element<DTYPE>::type* x, uint32_t bytes)
{
    constexpr int N = W * kElemBytes<DTYPE> / 4;         // 32-bit words of a word
    const auto* aligned = reinterpret_cast<const typename Packed<DTYPE, W>::word*>(reinterpret_cast<const char*>(x) - bytes);
    union { Packed<DTYPE, W> p[2]; uint32_t w[2 * N]; } in;
    union { Packed<DTYPE, W> p; uint32_t w[N]; } out;
    in.p[0].w[0] = aligned[0];
    in.p[1].w[0] = aligned[1];
    const uint32_t words = bytes / 4, bits = bytes % 4 * 8;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        uint32_t lo = in.w[k], hi = in.w[k + 1];
#pragma unroll
        for (int q = 1; q < N; ++q)
            if (words == (uint32_t)q) { lo = in.w[k + q]; hi = k + q + 1 < 2 * N ? in.w[k + q + 1] : 0; }
        out.w[k] = __funnelshift_r(lo, hi, bits);
    }
    return out.p;
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
