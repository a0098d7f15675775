// The global norm of many gradient tensors, and clipping by it.
//
//   N = sqrt(sum over all elements of x^2)        c = 1 where N <= max_norm, else max_norm / N
//   y = fl(c * x)
//
// The tensors are cut into tiles of 16 KB.  The measuring kernel's CTAs take the tiles in turn and leave one partial sum
// each; every CTA of the kernel that scales then adds up the partial sums itself (at most 1184 of them for each launch of
// the first kernel, from L2), so that there is no launch between the two, no atomic, and a fixed order of every sum.
// Squares are summed in fp32 inside a thread's share of a tile (at most 32 of them) and in 64 bits from there on.  A share
// whose sum of squares leaves the range where fp32 holds it is summed again in 64 bits: the norm is right for every finite
// gradient, also where single squares overflow or vanish in fp32.
#include <cmath>

#include "mqg_tma.cuh"
#include "mqg_training.h"
#include "mqg_vector.cuh"

namespace mqg {
namespace {

constexpr int kThreads = 256;
constexpr int kTileBytes = 16384;
constexpr int kMaxBlocks = 1184;                        // 8 CTAs for each of 148 SMs

// Tensors of one launch, passed by value: a kernel's parameters hold 32,764 bytes.
template <int CAP> struct TensorTable {
    int count;
    uint32_t tile_start[CAP + 1];
    uint64_t first[CAP + 1];                            // elements before the tensor in the whole list
    const void* ptr[CAP];
    uint8_t dtype[CAP];
};
constexpr int kSmallTable = 64, kLargeTable = 1024;

template <int CAP> __device__ __forceinline__ int find_tensor(const TensorTable<CAP>& tab, uint32_t tile)
{
    int lo = 0, hi = tab.count - 1;                     // the last tensor that starts at or before the tile
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.tile_start[mid] <= tile) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double warp_sum[kThreads / 32];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = v;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) t += warp_sum[w];
    return t;
}

// What fp32 holds a sum of at most 32 squares in without loss: none overflows, and what vanishes of the smallest is below
// 2^-40 of the sum.
__device__ __forceinline__ bool squares_in_range(float s) { return s >= 0x1p-100f && s <= 0x1p120f; }

// Sum of squares of m <= a tile's elements from p on, this thread's share.
template <int DTYPE>
__device__ __forceinline__ double tile_squares(const typename Element<DTYPE>::type* p, uint32_t m)
{
    constexpr int V = 16 / kElemBytes<DTYPE>, K = kTileBytes / 16 / kThreads;
    const uint32_t to_boundary = (uint32_t)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / kElemBytes<DTYPE>;
    const uint32_t head = to_boundary < m ? to_boundary : m;
    const uint32_t nvec = (m - head) / V, tail = m - head - nvec * V;
    Packed<DTYPE, V> x[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const uint32_t i = threadIdx.x + k * kThreads;
        if (i < nvec) x[k].load(p + head + i * V);
        else x[k].w[0] = make_uint4(0, 0, 0, 0);
    }
    float edge = 0.0f;                                  // the elements before the first and behind the last vector
    if (threadIdx.x < head) edge = widen(p[threadIdx.x]);
    else if (threadIdx.x < head + tail) edge = widen(p[m - tail + (threadIdx.x - head)]);
    float s[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        s[k] = x[k].get(0) * x[k].get(0);
#pragma unroll
        for (int e = 1; e < V; ++e) s[k] = __fmaf_rn(x[k].get(e), x[k].get(e), s[k]);
    }
    float t = edge * edge;
#pragma unroll
    for (int k = 0; k < K; ++k) t += s[k];
    if (squares_in_range(t)) return (double)t;
    double d = (double)edge * (double)edge;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) d = fma((double)x[k].get(e), (double)x[k].get(e), d);
    return d;
}

template <int CAP>
__global__ void __launch_bounds__(kThreads)
norm_kernel(const __grid_constant__ TensorTable<CAP> tab, double* __restrict__ partial)
{
    const uint32_t ntiles = tab.tile_start[tab.count];
    double sum = 0.0;
    grid_dependency_wait();
    for (uint32_t tile = blockIdx.x; tile < ntiles; tile += gridDim.x) {
        const int j = find_tensor(tab, tile);
        const uint64_t n = tab.first[j + 1] - tab.first[j];
        const uint32_t at = tile - tab.tile_start[j];
        if (tab.dtype[j] == kF32) {
            constexpr uint32_t E = kTileBytes / 4;
            const uint64_t e0 = (uint64_t)at * E;
            sum += tile_squares<kF32>(static_cast<const float*>(tab.ptr[j]) + e0, (uint32_t)min((uint64_t)E, n - e0));
        } else {
            constexpr uint32_t E = kTileBytes / 2;
            const uint64_t e0 = (uint64_t)at * E;
            sum += tile_squares<kBf16>(static_cast<const __nv_bfloat16*>(tab.ptr[j]) + e0, (uint32_t)min((uint64_t)E, n - e0));
        }
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

// The clipping factor from the partial sums, the same in every CTA.  The norm is compared and divided in 64 bits; a NaN
// among the elements makes the norm and the factor NaN, an infinity makes the factor 0.
__device__ __forceinline__ float factor_of(const double* partial, int npartial, float max_norm, float* norm)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < npartial; i += kThreads) s += __ldcg(partial + i);
    const double n = sqrt(block_sum(s));
    *norm = (float)n;
    return n <= (double)max_norm ? 1.0f : (float)((double)max_norm / n);
}

__device__ __forceinline__ void write_result(float* result, float norm, float factor)
{
    if (blockIdx.x == 0 && threadIdx.x == 0) { result[0] = norm; result[1] = factor; }
}

__global__ void __launch_bounds__(kThreads)
norm_result_kernel(const double* __restrict__ partial, int npartial, float max_norm, float* __restrict__ result)
{
    grid_dependency_wait();
    float norm;
    const float c = factor_of(partial, npartial, max_norm, &norm);
    write_result(result, norm, c);
}

// y[i] = c * x[i] for m <= a tile's elements, in place.
template <int DTYPE>
__device__ __forceinline__ void scale_tile(typename Element<DTYPE>::type* p, uint32_t m, float c)
{
    constexpr int V = 16 / kElemBytes<DTYPE>, K = kTileBytes / 16 / kThreads;
    const uint32_t to_boundary = (uint32_t)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / kElemBytes<DTYPE>;
    const uint32_t head = to_boundary < m ? to_boundary : m;
    const uint32_t nvec = (m - head) / V, tail = m - head - nvec * V;
    Packed<DTYPE, V> x[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const uint32_t i = threadIdx.x + k * kThreads;
        if (i < nvec) x[k].load(p + head + i * V);
    }
    if (threadIdx.x < head + tail) {
        const uint32_t i = threadIdx.x < head ? threadIdx.x : m - tail + (threadIdx.x - head);
        narrow(c * widen(p[i]), p[i]);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const uint32_t i = threadIdx.x + k * kThreads;
        if (i >= nvec) continue;
#pragma unroll
        for (int e = 0; e < V; ++e) x[k].set(e, c * x[k].get(e));
        x[k].store(p + head + i * V);
    }
}

// y[i] = c * x[i] for m elements, x and y of different buffers: vectors from y's first 16-byte boundary on; x is read by
// vectors where it is on a boundary there, else element by element.
template <int SRC, int DST>
__device__ __forceinline__ void copy_tile(const typename Element<SRC>::type* x, typename Element<DST>::type* y, uint32_t m, float c)
{
    constexpr int V = 16 / (kElemBytes<SRC> > kElemBytes<DST> ? kElemBytes<DST> : kElemBytes<SRC>);
    constexpr int W = Packed<SRC, V>::kWordBytes;
    const uint32_t to_boundary = (uint32_t)((16 - (reinterpret_cast<uintptr_t>(y) & 15)) & 15) / kElemBytes<DST>;
    const uint32_t head = to_boundary < m ? to_boundary : m;
    const uint32_t nvec = (m - head) / V, tail = m - head - nvec * V;
    const bool together = (reinterpret_cast<uintptr_t>(x + head) & (W - 1)) == 0;
    if (threadIdx.x < head + tail) {
        const uint32_t i = threadIdx.x < head ? threadIdx.x : m - tail + (threadIdx.x - head);
        narrow(c * widen(x[i]), y[i]);
    }
    for (uint32_t i = threadIdx.x; i < nvec; i += kThreads) {
        const uint32_t at = head + i * V;
        Packed<SRC, V> in;
        if (together) in.load(x + at);
        else {
#pragma unroll
            for (int e = 0; e < V; ++e) in.e[e] = x[at + e];
        }
        Packed<DST, V> out;
#pragma unroll
        for (int e = 0; e < V; ++e) out.set(e, c * in.get(e));
        out.store(y + at);
    }
}

// Scales the tiles of one table, the last first: what the measuring kernel read last is what L2 still holds.
// partial == nullptr: the factor is at `factor`.  DST < 0: in place.
template <int CAP, int DST>
__global__ void __launch_bounds__(kThreads)
scale_kernel(const __grid_constant__ TensorTable<CAP> tab, const double* __restrict__ partial, int npartial, float max_norm,
             const float* __restrict__ factor, void* __restrict__ flat, float* __restrict__ result)
{
    const uint32_t ntiles = tab.tile_start[tab.count];
    grid_dependency_wait();
    float c;
    if (partial != nullptr) {
        float norm;
        c = factor_of(partial, npartial, max_norm, &norm);
        if (result != nullptr) write_result(result, norm, c);
    } else {
        c = __ldcg(factor);
    }
    if (DST < 0 && c == 1.0f) return;                   // every product would be its own factor
    for (uint32_t i = blockIdx.x; i < ntiles; i += gridDim.x) {
        const uint32_t tile = ntiles - 1 - i;
        const int j = find_tensor(tab, tile);
        const uint64_t n = tab.first[j + 1] - tab.first[j];
        const uint32_t at = tile - tab.tile_start[j];
        const uint32_t E = tab.dtype[j] == kF32 ? kTileBytes / 4 : kTileBytes / 2;
        const uint64_t e0 = (uint64_t)at * E;
        const uint32_t m = (uint32_t)min((uint64_t)E, n - e0);
        if constexpr (DST < 0) {
            if (tab.dtype[j] == kF32) scale_tile<kF32>(static_cast<float*>(const_cast<void*>(tab.ptr[j])) + e0, m, c);
            else scale_tile<kBf16>(static_cast<__nv_bfloat16*>(const_cast<void*>(tab.ptr[j])) + e0, m, c);
        } else {
            auto* y = static_cast<typename Element<DST>::type*>(flat) + tab.first[j] + e0;
            if (tab.dtype[j] == kF32) copy_tile<kF32, DST>(static_cast<const float*>(tab.ptr[j]) + e0, y, m, c);
            else copy_tile<kBf16, DST>(static_cast<const __nv_bfloat16*>(tab.ptr[j]) + e0, y, m, c);
        }
    }
}

// params[i] <- fma(-lr, fl(c * acc[i]), params[i])
__global__ void __launch_bounds__(kThreads)
apply_clipped_kernel(float* __restrict__ params, const float* __restrict__ acc, float lr, const float* __restrict__ factor,
                     uint64_t n)
{
    const uint64_t n4 = n / 4, stride = (uint64_t)gridDim.x * blockDim.x;
    grid_dependency_wait();
    const float c = __ldcg(factor);
    for (uint64_t i = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n4; i += stride) {
        float4 p = __ldcg(reinterpret_cast<const float4*>(params) + i);
        const float4 g = __ldcg(reinterpret_cast<const float4*>(acc) + i);
        p.x = __fmaf_rn(-lr, __fmul_rn(c, g.x), p.x);
        p.y = __fmaf_rn(-lr, __fmul_rn(c, g.y), p.y);
        p.z = __fmaf_rn(-lr, __fmul_rn(c, g.z), p.z);
        p.w = __fmaf_rn(-lr, __fmul_rn(c, g.w), p.w);
        reinterpret_cast<float4*>(params)[i] = p;
    }
    if (blockIdx.x == 0 && threadIdx.x < (n & 3)) {
        const uint64_t i = n4 * 4 + threadIdx.x;
        params[i] = __fmaf_rn(-lr, __fmul_rn(c, __ldcg(acc + i)), __ldcg(params + i));
    }
}

// Fills `tab` with the tensors of the list from *next on, as many as fit; false if there are none left.
template <int CAP> void fill_table(const TensorList& list, int first, int last, uint64_t before, TensorTable<CAP>& tab)
{
    uint64_t tiles = 0;
    int k = 0;
    for (int j = first; j < last; ++j, ++k) {
        const uint64_t per_tile = list.dtype[j] == kF32 ? kTileBytes / 4 : kTileBytes / 2;
        tab.tile_start[k] = (uint32_t)tiles;
        tab.first[k] = before;
        tab.ptr[k] = list.ptr[j];
        tab.dtype[k] = (uint8_t)list.dtype[j];
        tiles += (list.size[j] + per_tile - 1) / per_tile;
        before += list.size[j];
    }
    tab.tile_start[k] = (uint32_t)tiles;
    tab.first[k] = before;
    tab.count = k;
}

// Calls fn(table, elements before it) for the list in tables of at most kLargeTable tensors.
template <typename Fn> cudaError_t for_each_table(const TensorList& list, Fn&& fn)
{
    uint64_t before = 0;
    for (int first = 0; first < list.count;) {
        const int last = list.count - first > kLargeTable ? first + kLargeTable : list.count;
        cudaError_t err;
        if (last - first <= kSmallTable) {
            TensorTable<kSmallTable> tab;
            fill_table(list, first, last, before, tab);
            before = tab.first[tab.count];
            err = fn(tab);
        } else {
            TensorTable<kLargeTable> tab;
            fill_table(list, first, last, before, tab);
            before = tab.first[tab.count];
            err = fn(tab);
        }
        if (err != cudaSuccess) return err;
        first = last;
    }
    return cudaSuccess;
}

template <int CAP> unsigned blocks_of(const TensorTable<CAP>& tab)
{
    const uint32_t tiles = tab.tile_start[tab.count];
    return tiles < (uint32_t)kMaxBlocks ? tiles : (unsigned)kMaxBlocks;
}

template <int DST, int CAP>
cudaError_t scale_table(const TensorTable<CAP>& tab, const double* partial, int npartial, float max_norm, const float* factor,
                        void* flat, float* result, cudaStream_t stream)
{
    const unsigned blocks = blocks_of(tab);
    if (blocks == 0) return cudaSuccess;
    return launch_pdl(scale_kernel<CAP, DST>, blocks, kThreads, stream, tab, partial, npartial, max_norm, factor, flat, result);
}

}  // namespace

size_t norm_workspace_floats(int count)
{
    const size_t tables = count <= 0 ? 1 : ((size_t)count + kLargeTable - 1) / kLargeTable;
    return tables * kMaxBlocks * 2;                     // a 64-bit sum for each CTA
}

cudaError_t launch_clip(const TensorList& list, float max_norm, ClipForm form, void* flat, int flat_dtype, float* result,
                        float* workspace, cudaStream_t stream)
{
    double* partial = reinterpret_cast<double*>(workspace);
    int npartial = 0;
    cudaError_t err = for_each_table(list, [&](const auto& tab) {
        const unsigned blocks = blocks_of(tab);
        if (blocks == 0) return cudaSuccess;
        using Tab = std::decay_t<decltype(tab)>;
        constexpr int CAP = sizeof(tab.dtype);
        static_assert(std::is_same_v<Tab, TensorTable<CAP>>, "one byte for each tensor");
        const cudaError_t e = launch_pdl(norm_kernel<CAP>, blocks, kThreads, stream, tab, partial + npartial);
        npartial += (int)blocks;
        return e;
    });
    if (err != cudaSuccess) return err;
    if (form == kMeasureOnly || npartial == 0)
        return launch_pdl(norm_result_kernel, 1, kThreads, stream, partial, npartial, max_norm, result);
    float* to = result;                                 // the first launch writes the result
    return for_each_table(list, [&](const auto& tab) {
        if (tab.tile_start[tab.count] == 0) return cudaSuccess;
        const cudaError_t e =
            form == kInPlace ? scale_table<-1>(tab, partial, npartial, max_norm, nullptr, nullptr, to, stream)
            : flat_dtype == kF32 ? scale_table<kF32>(tab, partial, npartial, max_norm, nullptr, flat, to, stream)
                                 : scale_table<kBf16>(tab, partial, npartial, max_norm, nullptr, flat, to, stream);
        to = nullptr;
        return e;
    });
}

cudaError_t launch_scale_tensors(const TensorList& list, const float* factor, cudaStream_t stream)
{
    return for_each_table(list, [&](const auto& tab) {
        return scale_table<-1>(tab, nullptr, 0, 0.0f, factor, nullptr, nullptr, stream);
    });
}

cudaError_t launch_apply_clipped(float* params, const float* acc, float lr, const float* factor, uint64_t n,
                                 cudaStream_t stream)
{
    uint64_t blocks = (n / 4 + kThreads - 1) / kThreads;
    if (blocks < 1) blocks = 1;
    if (blocks > 2 * kMaxBlocks) blocks = 2 * kMaxBlocks;
    return launch_pdl(apply_clipped_kernel, (unsigned)blocks, kThreads, stream, params, acc, lr, factor, n);
}

}  // namespace mqg
