// Layer norm over rows of `dim` elements:
//   mu = mean(x),  r = 1 / sqrt(mean((x - mu)^2) + eps),  y = (x - mu) * r * weight + bias
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

template <int X, int Y> cudaError_t launch(const NormArgs& a, cudaStream_t stream)
{
    return launch_pdl(norm_long_kernel<X, Y>, (unsigned)a.rows, kLongThreads, stream, a);
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
