// Layer norm over rows of `dim` elements:
//   mu = mean(x),  r = 1 / sqrt(mean((x - mu)^2) + eps),  y = (x - mu) * r * weight + bias
//
// Bound by memory: x is read and y written.  A row stays in the registers of the threads that read it, so that the squares are
// those of the differences from the mean (a difference of large sums would lose what rows far from zero have in common).
#include "mqg_norm_rows.cuh"
#include "mqg_tma.cuh"
#include "mqg_training.h"
#include "mqg_vector.cuh"

namespace mqg {
namespace {

struct NormArgs {
    const void* x;
    const void* weight;
    const void* bias;
    void* y;
    float* stats;
    uint64_t rows, dim;
    float eps;
    int w_dtype;
};

constexpr int kThreads = 256;                           // of a CTA with a row to at most a warp
constexpr int kMostThreads = 512;                       // of one with a row to the CTA

// Sum over the threads that have a row: `lanes` neighbours, or (WIDE) all of a CTA, the `turn`-th of a row.
template <bool WIDE> __device__ __forceinline__ float row_sum(float v, uint32_t lanes, int turn)
{
    v = lanes_sum(v, WIDE ? 32 : lanes);
    if (WIDE) {
        __shared__ float warp_sum[2][kMostThreads / 32];
        if ((threadIdx.x & 31) == 0) warp_sum[turn][threadIdx.x >> 5] = v;
        __syncthreads();
        const uint32_t lane = threadIdx.x & 31;
        v = lanes_sum(lane < blockDim.x / 32 ? warp_sum[turn][lane] : 0.0f, 32);
    }
    return v;
}

// K vectors of V elements to a thread.  WIDE: a CTA to a row, else `lanes` neighbouring lanes, a power of two.
template <int X, int Y, int V, int K, bool WIDE>
__global__ void __launch_bounds__(WIDE ? kMostThreads : kThreads) norm_kernel(const NormArgs a, uint32_t lanes)
{
    const uint32_t threads = WIDE ? blockDim.x : lanes, place = WIDE ? threadIdx.x : threadIdx.x & (lanes - 1);
    const uint64_t row = WIDE ? blockIdx.x : ((uint64_t)blockIdx.x * kThreads + threadIdx.x) / lanes;
    const uint32_t vectors = row < a.rows ? (uint32_t)(a.dim / V) : 0;
    grid_dependency_wait();
    const auto* x = static_cast<const typename Element<X>::type*>(a.x) + row * a.dim;
    float v[K][V];
    float sum = 0.0f;
    Packed<X, V> in[K];
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (place + k * threads < vectors) in[k].load(x + (place + k * threads) * V);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const bool has = place + k * threads < vectors;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            v[k][e] = has ? in[k].get(e) : 0.0f;
            sum += v[k][e];
        }
    }
    const float n = (float)a.dim, mean = __fdiv_rn(row_sum<WIDE>(sum, lanes, 0), n);
    float squares = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (place + k * threads >= vectors) continue;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            v[k][e] -= mean;
            squares = fmaf(v[k][e], v[k][e], squares);
        }
    }
    const float rstd = reciprocal_deviation(__fdiv_rn(row_sum<WIDE>(squares, lanes, 1), n), a.eps);
    if (row >= a.rows) return;
    if (place == 0 && a.stats != nullptr) { a.stats[2 * row] = mean; a.stats[2 * row + 1] = rstd; }
    auto* y = static_cast<typename Element<Y>::type*>(a.y) + row * a.dim;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const uint32_t i = (place + k * threads) * V;
        if (place + k * threads >= vectors) continue;
        float w[V], b[V];
        weights_at<V>(a.weight, a.w_dtype, i, 1.0f, w);
        weights_at<V>(a.bias, a.w_dtype, i, 0.0f, b);
        Packed<Y, V> out;
#pragma unroll
        for (int e = 0; e < V; ++e) out.set(e, fmaf(v[k][e] * rstd, w[e], b[e]));
        out.store(y + i);
    }
}

// Rows of any length: a CTA to a row, which it reads three times, sums in 64 bits.
template <int X, int Y> __global__ void __launch_bounds__(kLongThreads) norm_long_kernel(const NormArgs a)
{
    grid_dependency_wait();
    const uint64_t row = blockIdx.x;
    const auto* x = static_cast<const typename Element<X>::type*>(a.x) + row * a.dim;
    auto* y = static_cast<typename Element<Y>::type*>(a.y) + row * a.dim;
    double sum = 0.0;
    for (uint64_t i = threadIdx.x; i < a.dim; i += kLongThreads) sum += (double)widen(x[i]);
    const float mean = (float)(long_sum(sum) / (double)a.dim);
    double squares = 0.0;
    for (uint64_t i = threadIdx.x; i < a.dim; i += kLongThreads) {
        const float d = widen(x[i]) - mean;
        squares = fma((double)d, (double)d, squares);
    }
    const float rstd = reciprocal_deviation((float)(long_sum(squares) / (double)a.dim), a.eps);
    if (threadIdx.x == 0 && a.stats != nullptr) { a.stats[2 * row] = mean; a.stats[2 * row + 1] = rstd; }
    for (uint64_t i = threadIdx.x; i < a.dim; i += kLongThreads) {
        const float w = a.weight ? weight_at(a.weight, a.w_dtype, i) : 1.0f, b = a.bias ? weight_at(a.bias, a.w_dtype, i) : 0.0f;
        narrow(fmaf((widen(x[i]) - mean) * rstd, w, b), y[i]);
    }
}

template <int X, int Y, int V, int E> cudaError_t launch_elements(const NormArgs& a, cudaStream_t stream)
{
    constexpr int K = E / V;
    const uint32_t threads = (uint32_t)((a.dim + E - 1) / E);
    if (threads > 32)
        return launch_pdl(norm_kernel<X, Y, V, K, true>, (unsigned)a.rows, (threads + 31) / 32 * 32, stream, a, 32u);
    uint32_t lanes = 1;
    while (lanes < threads) lanes *= 2;
    const uint64_t per_cta = kThreads / lanes;
    return launch_pdl(norm_kernel<X, Y, V, K, false>, (unsigned)((a.rows + per_cta - 1) / per_cta), kThreads, stream, a, lanes);
}

template <int X, int Y, int V> cudaError_t launch_vectors(const NormArgs& a, cudaStream_t stream)
{
    // 32 elements to a thread where there are rows for all threads, 8 where there are not, or the row is short
    if (a.dim <= 8 * 32 || (a.dim <= 8 * kMostThreads && a.rows * a.dim <= 148ull * 2048 * 8)) return launch_elements<X, Y, V, 8>(a, stream);
    return launch_elements<X, Y, V, 32>(a, stream);
}

template <int X, int Y> cudaError_t launch(const NormArgs& a, cudaStream_t stream)
{
    if (a.dim > 32 * kMostThreads) return launch_pdl(norm_long_kernel<X, Y>, (unsigned)a.rows, kLongThreads, stream, a);
    constexpr int V = kVector<X, Y>;
    const int w = element_bytes(a.w_dtype);
    const bool fit = vectors_fit(a.x, kElemBytes<X>, V, a.dim) && vectors_fit(a.y, kElemBytes<Y>, V, a.dim) &&
                     vectors_fit(a.weight, w, V, a.dim) && vectors_fit(a.bias, w, V, a.dim);
    return fit ? launch_vectors<X, Y, V>(a, stream) : launch_vectors<X, Y, 1>(a, stream);
}

}  // namespace

cudaError_t launch_layer_norm(const NormRows& in, float eps, void* y, int y_dtype, float* stats, cudaStream_t stream)
{
    if (in.rows == 0 || in.dim == 0) return cudaSuccess;
    const NormArgs a = {in.x, in.weight, in.bias, y, stats, in.rows, in.dim, eps, in.w_dtype};
    return in.x_dtype == kF32 ? (y_dtype == kF32 ? launch<kF32, kF32>(a, stream) : launch<kF32, kBf16>(a, stream))
                              : (y_dtype == kF32 ? launch<kBf16, kF32>(a, stream) : launch<kBf16, kBf16>(a, stream));
}

}  // namespace mqg
