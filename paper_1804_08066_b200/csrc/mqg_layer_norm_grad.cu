// The gradient of the layer norm, from the rows' means mu and reciprocal deviations r:
//   h = (x - mu) * r,  a = weight * dy
//   dx = r * (a - mean(a) - h * mean(a * h)),  dweight = sum over rows of dy * h,  dbias = sum over rows of dy
#include "mqg_norm_rows.cuh"
#include "mqg_tma.cuh"
#include "mqg_training.h"
#include "mqg_vector.cuh"

namespace mqg {
namespace {

struct GradArgs {
    const void* x;
    const void* dy;
    const void* weight;
    const float* stats;
    void* dx;
    float* partial;          // [parts][2][dim]: sums for dweight and dbias
    uint64_t rows, dim;
    int w_dtype;
};

// Rows of any length: a CTA to a row, which it reads twice, sums in 64 bits.
template <int X, int Y> __global__ void __launch_bounds__(kLongThreads) grad_long_kernel(const GradArgs a)
{
    grid_dependency_wait();
    const uint64_t row = blockIdx.x;
    const auto* x = static_cast<const typename Element<X>::type*>(a.x) + row * a.dim;
    const auto* dy = static_cast<const typename Element<Y>::type*>(a.dy) + row * a.dim;
    auto* dx = static_cast<typename Element<X>::type*>(a.dx) + row * a.dim;
    const float mean = a.stats[2 * row], rstd = a.stats[2 * row + 1];
    double sum = 0.0, along = 0.0;
    for (uint64_t i = threadIdx.x; i < a.dim; i += kLongThreads) {
        const float g = widen(dy[i]) * (a.weight ? weight_at(a.weight, a.w_dtype, i) : 1.0f), h = (widen(x[i]) - mean) * rstd;
        sum += (double)g;
        along = fma((double)g, (double)h, along);
    }
    const float m1 = (float)(long_sum(sum) / (double)a.dim), m2 = (float)(long_sum(along) / (double)a.dim);
    for (uint64_t i = threadIdx.x; i < a.dim; i += kLongThreads) {
        const float g = widen(dy[i]) * (a.weight ? weight_at(a.weight, a.w_dtype, i) : 1.0f), h = (widen(x[i]) - mean) * rstd;
        narrow(rstd * (g - m1 - h * m2), dx[i]);
    }
}

// Sums over a part of the rows, a thread to a column.
constexpr int kColumns = 64, kStripes = 4;
template <int X, int Y> __global__ void __launch_bounds__(kColumns* kStripes) columns_kernel(const GradArgs a, uint64_t per_part)
{
    __shared__ float sums[kStripes][2][kColumns];
    const uint32_t at = threadIdx.x % kColumns, stripe = threadIdx.x / kColumns;
    grid_dependency_wait();
    const uint64_t col = (uint64_t)blockIdx.x * kColumns + at;
    const uint64_t first = blockIdx.y * per_part, last = min(first + per_part, a.rows);
    const auto* x = static_cast<const typename Element<X>::type*>(a.x) + col;
    const auto* dy = static_cast<const typename Element<Y>::type*>(a.dy) + col;
    float dw = 0.0f, db = 0.0f;
    if (col < a.dim)
        for (uint64_t row = first + stripe; row < last; row += kStripes) {
            const float g = widen(dy[row * a.dim]), h = (widen(x[row * a.dim]) - a.stats[2 * row]) * a.stats[2 * row + 1];
            dw = fmaf(g, h, dw);
            db += g;
        }
    sums[stripe][0][at] = dw;
    sums[stripe][1][at] = db;
    __syncthreads();
    if (stripe != 0 || col >= a.dim) return;
#pragma unroll
    for (int k = 1; k < kStripes; ++k) { dw += sums[k][0][at]; db += sums[k][1][at]; }
    a.partial[(blockIdx.y * 2 + 0) * a.dim + col] = dw;
    a.partial[(blockIdx.y * 2 + 1) * a.dim + col] = db;
}

// The parts' sums, in 64 bits, in order.
template <int W> __global__ void __launch_bounds__(256)
join_kernel(const float* __restrict__ partial, uint32_t parts, uint64_t dim, void* dweight, void* dbias, int add)
{
    grid_dependency_wait();
    const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= 2 * dim) return;
    auto* to = static_cast<typename Element<W>::type*>(i < dim ? dweight : dbias);
    if (to == nullptr) return;
    const uint64_t col = i < dim ? i : i - dim;
    double sum = 0.0;
    for (uint32_t k = 0; k < parts; ++k) sum += (double)__ldcg(partial + k * 2 * dim + i);
    if (add) sum += (double)widen(to[col]);
    narrow((float)sum, to[col]);
}

uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// Parts of the rows for the columns' sums: enough CTAs for every SM, at least 64 rows each.
uint32_t parts_of(uint64_t rows, uint64_t dim)
{
    const uint64_t most = ceil_div(rows, 64), want = ceil_div(148 * 8, ceil_div(dim, kColumns));
    return (uint32_t)(most < want ? (most < 1 ? 1 : most) : want);
}

template <int X, int Y> cudaError_t launch(const GradArgs& a, const NormGrads& out, cudaStream_t stream)
{
    cudaError_t err = cudaSuccess;
    if (out.dx != nullptr && a.rows != 0) err = launch_pdl(grad_long_kernel<X, Y>, (unsigned)a.rows, kLongThreads, stream, a);
    if (err != cudaSuccess || (out.dweight == nullptr && out.dbias == nullptr)) return err;
    const uint32_t parts = parts_of(a.rows, a.dim);
    err = launch_pdl_grid(columns_kernel<X, Y>, dim3((unsigned)ceil_div(a.dim, kColumns), parts), kColumns * kStripes, 0, stream, a,
                          ceil_div(a.rows, parts));
    if (err != cudaSuccess) return err;
    const unsigned blocks = (unsigned)ceil_div(2 * a.dim, 256);
    return out.dw_dtype == kF32
               ? launch_pdl(join_kernel<kF32>, blocks, 256, stream, a.partial, parts, a.dim, out.dweight, out.dbias, (int)out.add)
               : launch_pdl(join_kernel<kBf16>, blocks, 256, stream, a.partial, parts, a.dim, out.dweight, out.dbias, (int)out.add);
}

}  // namespace

size_t layer_norm_workspace_floats(uint64_t rows, uint64_t dim) { return (size_t)(parts_of(rows, dim) * 2 * dim); }

cudaError_t launch_layer_norm_grad(const void* dy, int dy_dtype, const NormRows& in, const float* stats, const NormGrads& out,
                                   float* workspace, cudaStream_t stream)
{
    const GradArgs a = {in.x, dy, in.weight, stats, out.dx, workspace, in.rows, in.dim, in.w_dtype};
    return in.x_dtype == kF32 ? (dy_dtype == kF32 ? launch<kF32, kF32>(a, out, stream) : launch<kF32, kBf16>(a, out, stream))
                              : (dy_dtype == kF32 ? launch<kBf16, kF32>(a, out, stream) : launch<kBf16, kBf16>(a, out, stream));
}

}  // namespace mqg
