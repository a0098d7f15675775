// The gradient of the layer norm, from the rows' means mu and reciprocal deviations r:
//   h = (x - mu) * r,  a = weight * dy
//   dx = r * (a - mean(a) - h * mean(a * h)),  dweight = sum over rows of dy * h,  dbias = sum over rows of dy
//
// Bound by memory: x and dy are read and dx is written.  A thread keeps the same columns of every row that its CTA takes, so the
// sums over the rows stay in its registers until the CTA's last row; the CTAs' sums are added up by a second launch.  Rows come by
// asynchronous copies, a few ahead, each thread its own elements: the copies that are on their way take no registers, and no
// thread waits for another's.
#include <atomic>

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

constexpr int kThreads = 512, kCtas = 148 * 2;
constexpr int kMostElements = 8;                        // of a row to a thread

template <int BYTES> __device__ __forceinline__ void copy_async(void* to, const void* from)
{
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// One thread's elements of a row: K vectors of V, `threads` vectors apart.
template <int X, int Y, int V, int K> struct Shares {
    static constexpr bool kAsync = V * kElemBytes<X> >= 4 && V * kElemBytes<Y> >= 4;
    static constexpr int kStages = kAsync ? (kElemBytes<X> + kElemBytes<Y> == 8 ? 3 : 4) : 1;
    struct Stage {
        Packed<X, V> x[K][kThreads];
        Packed<Y, V> dy[K][kThreads];
    };
};

// Sums of two values over the `threads` threads that have a row; `group` numbers these groups of a CTA.
struct RowSums {
    float2 of_warp[2][kThreads / 32];
    __device__ __forceinline__ float2 add(float2 v, uint32_t threads, uint32_t group, int turn)
    {
        v.x = lanes_sum(v.x, threads);
        v.y = lanes_sum(v.y, threads);
        if (threads <= 32) return v;
        const uint32_t warps = threads / 32, lane = threadIdx.x & 31;
        if (lane == 0) of_warp[turn][threadIdx.x >> 5] = v;
        asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(threads) : "memory");
        v = lane < warps ? of_warp[turn][group * warps + lane] : make_float2(0.0f, 0.0f);
        return make_float2(lanes_sum(v.x, 32), lanes_sum(v.y, 32));
    }
};

// threads: of a row, a power of two.
template <int X, int Y, int V, int K>
__global__ void __launch_bounds__(kThreads, 2) grad_rows_kernel(const GradArgs a, uint32_t threads, int sums)
{
    using S = Shares<X, Y, V, K>;
    extern __shared__ __align__(16) unsigned char memory[];
    auto* stage = reinterpret_cast<typename S::Stage*>(memory);
    __shared__ RowSums row_sums;
    const uint32_t place = threadIdx.x & (threads - 1), group = threadIdx.x / threads, groups = kThreads / threads;
    const uint32_t vectors = (uint32_t)(a.dim / V);
    const uint64_t stride = (uint64_t)gridDim.x * groups;
    const float n = (float)a.dim;
    grid_dependency_wait();
    const auto* x = static_cast<const typename Element<X>::type*>(a.x);
    const auto* dy = static_cast<const typename Element<Y>::type*>(a.dy);
    auto* dx = static_cast<typename Element<X>::type*>(a.dx);
    float w[K][V], dw[K][V], db[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const uint32_t at = place + k * threads;
        if (at < vectors) weights_at<V>(a.weight, a.w_dtype, at * V, 1.0f, w[k]);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (at >= vectors) w[k][e] = 0.0f;
            dw[k][e] = db[k][e] = 0.0f;
        }
    }
    const auto fetch = [&](uint64_t row, int slot) {
        if (row < a.rows)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const uint32_t at = place + k * threads;
                if (at >= vectors) continue;
                copy_async<V * kElemBytes<X>>(&stage[slot].x[k][threadIdx.x], x + row * a.dim + at * V);
                copy_async<V * kElemBytes<Y>>(&stage[slot].dy[k][threadIdx.x], dy + row * a.dim + at * V);
            }
        commit_copies();
    };
    const uint64_t first = (uint64_t)blockIdx.x * groups + group;
    if constexpr (S::kAsync)
#pragma unroll
        for (int s = 0; s < S::kStages - 1; ++s) fetch(first + s * stride, s);
    int slot = 0, turn = 0;
    // Every group of a CTA takes as many turns: the barriers of its warps are its own, but lanes of one warp stay together.
    for (uint64_t base = (uint64_t)blockIdx.x * groups; base < a.rows; base += stride) {
        const uint64_t row = base + group;
        const bool has = row < a.rows;
        Packed<X, V> px[K];
        Packed<Y, V> pdy[K];
        float2 stats = make_float2(0.0f, 0.0f);
        if (has) stats = make_float2(__ldg(a.stats + 2 * row), __ldg(a.stats + 2 * row + 1));
        if constexpr (S::kAsync) {
            fetch(row + (S::kStages - 1) * stride, slot == 0 ? S::kStages - 1 : slot - 1);
            wait_copies<S::kStages - 1>();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                px[k] = stage[slot].x[k][threadIdx.x];
                pdy[k] = stage[slot].dy[k][threadIdx.x];
            }
            slot = slot == S::kStages - 1 ? 0 : slot + 1;
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const uint32_t at = place + k * threads;
                if (!has || at >= vectors) continue;
                px[k].load(x + row * a.dim + at * V);
                pdy[k].load(dy + row * a.dim + at * V);
            }
        }
        float2 sum = make_float2(0.0f, 0.0f);
        float h[K][V], g[K][V];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const bool there = has && place + k * threads < vectors;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                h[k][e] = there ? (px[k].get(e) - stats.x) * stats.y : 0.0f;
                const float d = there ? pdy[k].get(e) : 0.0f;
                dw[k][e] = fmaf(d, h[k][e], dw[k][e]);
                db[k][e] += d;
                g[k][e] = d * w[k][e];
                sum.x += g[k][e];
                sum.y = fmaf(g[k][e], h[k][e], sum.y);
            }
        }
        if (dx == nullptr) continue;
        sum = row_sums.add(sum, threads, group, turn);
        turn ^= 1;
        const float m1 = __fdiv_rn(sum.x, n), m2 = __fdiv_rn(sum.y, n);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t at = place + k * threads;
            if (!has || at >= vectors) continue;
            Packed<X, V> out;
#pragma unroll
            for (int e = 0; e < V; ++e) out.set(e, stats.y * (g[k][e] - m1 - h[k][e] * m2));
            out.store(dx + row * a.dim + at * V);
        }
    }
    if (!sums) return;
    // The groups' sums, in their order, through shared memory.
    if constexpr (S::kAsync) wait_copies<0>();
    __syncthreads();
    float* all = reinterpret_cast<float*>(memory);      // [groups][dim] of one sum, then of the other
    const uint32_t dim = (uint32_t)a.dim;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t at = place + k * threads;
            if (at >= vectors) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) all[group * dim + at * V + e] = which == 0 ? dw[k][e] : db[k][e];
        }
        __syncthreads();
        for (uint32_t col = threadIdx.x; col < dim; col += kThreads) {
            float total = 0.0f;
            for (uint32_t i = 0; i < groups; ++i) total += all[i * dim + col];
            a.partial[((uint64_t)blockIdx.x * 2 + which) * dim + col] = total;
        }
        __syncthreads();
    }
}

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

// The parts' sums, in 64 bits: stripes of the parts side by side, then the stripes in order.
constexpr int kJoinColumns = 32, kJoinStripes = 32;
template <int W> __global__ void __launch_bounds__(kJoinColumns* kJoinStripes)
join_kernel(const float* __restrict__ partial, uint32_t parts, uint64_t dim, void* dweight, void* dbias, int add)
{
    __shared__ double sums[kJoinStripes][kJoinColumns];
    const uint32_t at = threadIdx.x % kJoinColumns, stripe = threadIdx.x / kJoinColumns;
    const uint64_t i = (uint64_t)blockIdx.x * kJoinColumns + at;
    grid_dependency_wait();
    double sum = 0.0;
    if (i < 2 * dim)
#pragma unroll 8
        for (uint32_t k = stripe; k < parts; k += kJoinStripes) sum += (double)__ldcg(partial + k * 2 * dim + i);
    sums[stripe][at] = sum;
    __syncthreads();
    if (stripe != 0 || i >= 2 * dim) return;
#pragma unroll
    for (int k = 1; k < kJoinStripes; ++k) sum += sums[k][at];
    auto* to = static_cast<typename Element<W>::type*>(i < dim ? dweight : dbias);
    if (to == nullptr) return;
    const uint64_t col = i < dim ? i : i - dim;
    if (add) sum += (double)widen(to[col]);
    narrow((float)sum, to[col]);
}

uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// Threads of a row in the kernel that keeps it in registers; 0: the row is too long.
uint32_t row_threads(uint64_t dim)
{
    uint32_t threads = 1;
    while (threads <= kThreads && (uint64_t)threads * kMostElements < dim) threads *= 2;
    return threads <= kThreads ? threads : 0;
}

// Parts of the rows that leave a sum each: the CTAs of that kernel, or, for long rows, enough for every SM of at least 64 rows.
uint32_t parts_of(uint64_t rows, uint64_t dim)
{
    uint64_t most, want = kCtas;
    if (const uint32_t threads = row_threads(dim)) {
        most = ceil_div(rows, kThreads / threads);
    } else {
        most = ceil_div(rows, 64);
        want = ceil_div(148 * 8, ceil_div(dim, kColumns));
    }
    return (uint32_t)(most < want ? (most < 1 ? 1 : most) : want);
}

template <int X, int Y, int V> cudaError_t launch_vectors(const GradArgs& a, uint32_t threads, uint32_t parts, int sums, cudaStream_t stream)
{
    using S = Shares<X, Y, V, kMostElements / V>;
    constexpr size_t kSums = kThreads * kMostElements * sizeof(float);
    constexpr size_t kRing = S::kAsync ? S::kStages * sizeof(typename S::Stage) : 0, kBytes = kRing > kSums ? kRing : kSums;
    const auto kernel = grad_rows_kernel<X, Y, V, kMostElements / V>;
    static std::atomic<bool> ready[64];                 // by device
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev].load(std::memory_order_relaxed)) {
        err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kBytes);
        if (err != cudaSuccess) return err;
        ready[dev].store(true, std::memory_order_relaxed);
    }
    return launch_pdl_smem(kernel, parts, kThreads, kBytes, stream, a, threads, sums);
}

template <int X, int Y> cudaError_t launch(const GradArgs& a, const NormGrads& out, cudaStream_t stream)
{
    const int sums = out.dweight != nullptr || out.dbias != nullptr;
    const uint32_t parts = parts_of(a.rows, a.dim), threads = row_threads(a.dim);
    cudaError_t err = cudaSuccess;
    if (threads != 0) {
        constexpr int V = kVector<X, Y>;
        const bool fit = vectors_fit(a.x, kElemBytes<X>, V, a.dim) && vectors_fit(a.dx, kElemBytes<X>, V, a.dim) &&
                         vectors_fit(a.dy, kElemBytes<Y>, V, a.dim) && vectors_fit(a.weight, element_bytes(a.w_dtype), V, a.dim);
        err = fit ? launch_vectors<X, Y, V>(a, threads, parts, sums, stream) : launch_vectors<X, Y, 1>(a, threads, parts, sums, stream);
    } else {
        if (a.dx != nullptr && a.rows != 0) err = launch_pdl(grad_long_kernel<X, Y>, (unsigned)a.rows, kLongThreads, stream, a);
        if (sums && err == cudaSuccess)
            err = launch_pdl_grid(columns_kernel<X, Y>, dim3((unsigned)ceil_div(a.dim, kColumns), parts), kColumns * kStripes, 0, stream, a,
                                  ceil_div(a.rows, parts));
    }
    if (err != cudaSuccess || !sums) return err;
    const unsigned blocks = (unsigned)ceil_div(2 * a.dim, kJoinColumns);
    const auto join = out.dw_dtype == kF32 ? join_kernel<kF32> : join_kernel<kBf16>;
    return launch_pdl(join, blocks, kJoinColumns * kJoinStripes, stream, a.partial, parts, a.dim, out.dweight, out.dbias, (int)out.add);
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
