// What the layer norm's forward and backward kernels share.
#pragma once

#include <stdint.h>

#include "mqg_async.cuh"
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

// ---- rows by groups of threads ----------------------------------------------------------------------------------------------
// A row is E elements to a thread: a group of 1, 2, 4, 8 or 16 lanes, or of up to 16 whole warps (WIDE).  A CTA has as many groups as
// fit 16 warps.  A thread has K vectors of V elements, those of a group's threads side by side; single elements (V = 1) of a WIDE
// group, those of a warp's lanes, so that the distance between a thread's elements is a constant (10,007 rows of 515 in fp32: 14.7 us,
// 18.3 without; for vectors it makes no difference or, in long rows, costs up to a sixth).  Vectors come to shared memory by asynchronous
// copies, rows ahead; single elements straight to registers, one row ahead (copies of 4 bytes each: 14.7 us, so 11.9).

constexpr int kRowThreads = 512;

struct RowGroups {
    uint32_t threads;        // of a group
    uint32_t block;          // of a CTA
    uint32_t ctas;           // a grid that fills the device, where there are rows for it
};

// E * kRowThreads elements at most.  per_sm: threads that the kernel's registers leave room for; most_ctas: CTAs that its shared memory does.
inline RowGroups row_groups(uint64_t rows, uint64_t dim, uint32_t e, uint32_t per_sm, uint32_t most_ctas = 32)
{
    RowGroups g;
    const uint32_t need = (uint32_t)((dim + e - 1) / e);
    if (need <= 16) {
        for (g.threads = 1; g.threads < need;) g.threads *= 2;
        g.block = kRowThreads;
    } else {
        g.threads = (need + 31) / 32 * 32;
        g.block = kRowThreads / g.threads * g.threads;
    }
    const uint64_t per_cta = g.block / g.threads, wanted = (rows + per_cta - 1) / per_cta;
    const uint64_t most = 148ull * (per_sm / g.block < most_ctas ? per_sm / g.block : most_ctas);
    g.ctas = (uint32_t)(wanted < 1 ? 1 : wanted < most ? wanted : most);
    return g;
}

// A thread's vectors: their places in the row, which of them the row has (FULL: all, of every thread).
template <int V, int K, bool WIDE, bool FULL> struct RowPlace {
    static constexpr bool kByWarp = WIDE && V == 1;
    uint32_t start, threads, vectors, held;
    __device__ __forceinline__ RowPlace(uint64_t dim, uint32_t place, uint32_t group_threads)
        : start(kByWarp ? (place & ~31u) * K + (place & 31) : place), threads(group_threads), vectors((uint32_t)(dim / V)),
          held(vectors > start ? (vectors - start + 31) / 32 : 0) {}
    __device__ __forceinline__ uint32_t step() const { return kByWarp ? 32 : threads; }
    __device__ __forceinline__ bool has(int k) const { return FULL || (kByWarp ? (uint32_t)k < held : start + k * step() < vectors); }
    __device__ __forceinline__ uint32_t element(int k) const { return (start + k * step()) * V; }
    __device__ __forceinline__ uint32_t beyond(int k) const { return k * step() * V; }          // element(k) - element(0)
};

// Sum over `lanes` neighbouring lanes, a power of two up to 32.
__device__ __forceinline__ float lanes_sum(float v, uint32_t lanes)
{
#pragma unroll
    for (uint32_t d = 16; d > 0; d >>= 1)
        if (d < lanes) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

__device__ __forceinline__ void group_barrier(uint32_t group, uint32_t threads)
{
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(threads) : "memory");
}

// Sums over a group of one or two values of each thread, the same for all of its threads.  A group of several warps meets once for
// each sum; `turn` alternates, so that nothing is written that a slow warp has yet to read.
struct RowSums {
    float2 of_warp[2][kRowThreads / 32];

    __device__ __forceinline__ float one(float v, uint32_t threads, uint32_t group, int turn)
    {
        v = lanes_sum(v, threads);
        if (threads <= 32) return v;
        const uint32_t warps = threads / 32, lane = threadIdx.x & 31;
        if (lane == 0) of_warp[turn][threadIdx.x >> 5].x = v;
        group_barrier(group, threads);
        return lanes_sum((lane & 15) < warps ? of_warp[turn][group * warps + (lane & 15)].x : 0.0f, 16);
    }
    __device__ __forceinline__ float2 two(float2 v, uint32_t threads, uint32_t group, int turn)
    {
        if (threads < 32) return make_float2(lanes_sum(v.x, threads), lanes_sum(v.y, threads));
        // from here on lanes below 16 have the first value and the others the second: six steps for both instead of ten
        const uint32_t lane = threadIdx.x & 31;
        const bool low = lane < 16;
        float mine = (low ? v.x : v.y) + __shfl_xor_sync(0xFFFFFFFFu, low ? v.y : v.x, 16);
        mine = lanes_sum(mine, 16);
        if (threads > 32) {
            const uint32_t warps = threads / 32;
            float* sums = reinterpret_cast<float*>(of_warp[turn]);
            if ((lane & 15) == 0) sums[2 * (threadIdx.x >> 5) + (low ? 0 : 1)] = mine;
            group_barrier(group, threads);
            mine = lanes_sum((lane & 15) < warps ? sums[2 * (group * warps + (lane & 15)) + (low ? 0 : 1)] : 0.0f, 16);
        }
        const float other = __shfl_xor_sync(0xFFFFFFFFu, mine, 16);
        return low ? make_float2(mine, other) : make_float2(other, mine);
    }
};

// Rows that an SM has at once, where there are many: what rounding up to whole warps and whole CTAs leaves of its threads.
inline uint32_t rows_at_once(uint64_t dim, uint32_t e, uint32_t per_sm, uint32_t most_ctas = 32)
{
    const RowGroups g = row_groups(1ull << 40, dim, e, per_sm, most_ctas);
    return g.ctas / 148 * (g.block / g.threads);
}

// Whether rows x dim elements keep less than the threads of a device busy, 8 elements to a thread: then more elements to a thread
// take longer.
inline bool few_elements(uint64_t rows, uint64_t dim) { return rows * dim <= 148ull * 2 * kRowThreads * 8; }
// Whether they are enough for several turns, where the rows that an SM has at once count.
inline bool many_elements(uint64_t rows, uint64_t dim) { return rows * dim >= 4000000; }

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
