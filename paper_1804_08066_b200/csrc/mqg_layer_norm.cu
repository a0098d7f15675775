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

// Rows on their way to shared memory, each thread's own elements.
template <int X, int V, int E> struct Ring {
    static constexpr bool kAsync = V > 1;
    static constexpr int kStageBytes = kRowThreads * E * kElemBytes<X>, kFit = (E <= 8 ? 100 : 200) * 1024 / kStageBytes;
    static constexpr int kStages = !kAsync ? 1 : kFit < 5 ? kFit : 5;
    Packed<X, V> x[kStages][E / V][kRowThreads];
};

template <int E> constexpr int kResident = E <= 8 ? 2 : 1;

// E elements to a thread, V to a vector.  FULL: rows of E times the threads of a group, without a condition on any vector.
template <int X, int Y, int V, int E, bool WIDE, bool FULL>
__global__ void __launch_bounds__(kRowThreads, kResident<E>) norm_rows_kernel(const NormArgs a, uint32_t threads)
{
    using R = Ring<X, V, E>;
    constexpr int K = E / V;
    extern __shared__ __align__(16) unsigned char memory[];
    auto& ring = *reinterpret_cast<R*>(memory);
    __shared__ RowSums sums;
    const uint32_t place = threadIdx.x % threads, group = threadIdx.x / threads, groups = blockDim.x / threads;
    const RowPlace<V, K, WIDE, FULL> at(a.dim, place, threads);
    const uint64_t stride = (uint64_t)gridDim.x * groups;
    const float per_element = __fdiv_rn(1.0f, (float)a.dim);
    grid_dependency_wait();
    const auto* x = static_cast<const typename Element<X>::type*>(a.x);
    auto* y = static_cast<typename Element<Y>::type*>(a.y);
    const auto fetch = [&](uint64_t row, int slot) {
        const auto* from = x + row * a.dim;
        if (row < a.rows)
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (at.has(k)) copy_async<V * kElemBytes<X>>(&ring.x[slot][k][threadIdx.x], from + at.element(k));
        commit_copies();
    };
    float w[E], b[E];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float wk[V], bk[V];
#pragma unroll
        for (int e = 0; e < V; ++e) wk[e] = bk[e] = 0.0f;
        if (at.has(k)) {
            weights_at<V>(a.weight, a.w_dtype, at.element(k), 1.0f, wk);
            weights_at<V>(a.bias, a.w_dtype, at.element(k), 0.0f, bk);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) { w[k * V + e] = wk[e]; b[k * V + e] = bk[e]; }
    }
    if constexpr (R::kAsync) {
        // places without elements hold zeros, which no copy overwrites
#pragma unroll
        for (int s = 0; s < R::kStages; ++s)
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (!at.has(k))
#pragma unroll
                    for (int e = 0; e < V; ++e) ring.x[s][k][threadIdx.x].set(e, 0.0f);
#pragma unroll
        for (int s = 0; s < R::kStages - 1; ++s) fetch((uint64_t)blockIdx.x * groups + group + s * stride, s);
    }
    // single elements: the next row, where registers hold one more
    constexpr bool kAhead = !R::kAsync && E <= 24;
    Packed<X, V> next[R::kAsync ? 1 : K];
    const auto load_next = [&](uint64_t row) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            next[k].set(0, 0.0f);
            if (row < a.rows && at.has(k)) next[k].load(x + row * a.dim + at.element(k));
        }
    };
    if constexpr (kAhead) load_next((uint64_t)blockIdx.x * groups + group);
    int slot = 0;
    for (uint64_t base = (uint64_t)blockIdx.x * groups; base < a.rows; base += stride) {
        const uint64_t row = base + group;
        const bool has = row < a.rows;
        float v[E];
        if constexpr (R::kAsync) {
            fetch(row + (R::kStages - 1) * stride, slot == 0 ? R::kStages - 1 : slot - 1);
            wait_copies<R::kStages - 1>();
#pragma unroll
            for (int k = 0; k < K; ++k) widen_to<X, V>(ring.x[slot][k][threadIdx.x], v + k * V);
            slot = slot == R::kStages - 1 ? 0 : slot + 1;
        } else {
            if constexpr (!kAhead) load_next(row);
#pragma unroll
            for (int k = 0; k < K; ++k) widen_to<X, V>(next[k], v + k * V);
            if constexpr (kAhead) load_next(row + stride);
        }
        float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int e = 0; e < E; e += 2) sum = __fadd2_rn(sum, make_float2(v[e], v[e + 1]));
        const float mean = sums.one(sum.x + sum.y, threads, group, 0) * per_element;
        float2 squares = make_float2(0.0f, 0.0f);
        const float2 minus = make_float2(-mean, -mean);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const float2 d = __fadd2_rn(make_float2(v[e], v[e + 1]), minus);
            v[e] = d.x;
            v[e + 1] = d.y;
            if constexpr (V > 1) {
                if (at.has(e / V)) squares = __ffma2_rn(d, d, squares);
            } else {
                squares.x = at.has(e) ? fmaf(d.x, d.x, squares.x) : squares.x;
                squares.y = at.has(e + 1) ? fmaf(d.y, d.y, squares.y) : squares.y;
            }
        }
        const float rstd = reciprocal_deviation(sums.one(squares.x + squares.y, threads, group, 1) * per_element, a.eps);
        if (!has) continue;
        if (place == 0 && a.stats != nullptr) { a.stats[2 * row] = mean; a.stats[2 * row + 1] = rstd; }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!at.has(k)) continue;
            Packed<Y, V> out;
            if constexpr (V > 1) {
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const int i = k * V + e;
                    const float2 h = __fmul2_rn(make_float2(v[i], v[i + 1]), make_float2(rstd, rstd));
                    const float2 r = __ffma2_rn(h, make_float2(w[i], w[i + 1]), make_float2(b[i], b[i + 1]));
                    out.set(e, r.x);
                    out.set(e + 1, r.y);
                }
            } else {
                out.set(0, fmaf(v[k] * rstd, w[k], b[k]));
            }
            out.store(y + row * a.dim + at.element(k));
        }
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

template <int X, int Y, int V, int E, bool WIDE, bool FULL> cudaError_t launch_groups(const NormArgs& a, const RowGroups& g, cudaStream_t stream)
{
    using R = Ring<X, V, E>;
    static std::atomic<bool> ready[64];
    const auto kernel = norm_rows_kernel<X, Y, V, E, WIDE, FULL>;
    constexpr size_t kBytes = R::kAsync ? sizeof(R) : 0;
    if (const cudaError_t err = allow_shared(kernel, kBytes, ready)) return err;
    return launch_pdl_smem(kernel, g.ctas, g.block, kBytes, stream, a, g.threads);
}

template <int X, int Y, int V, int E> cudaError_t launch_elements(const NormArgs& a, cudaStream_t stream)
{
    const RowGroups g = row_groups(a.rows, a.dim, E, kResident<E> * kRowThreads);
    const bool full = V > 1 && a.dim == (uint64_t)g.threads * E;
    if constexpr (V > 1 ? E < 32 : E <= 8)              // (rows that 32 elements to a thread are chosen for take whole warps)
        if (g.threads < 32) {
            if constexpr (V > 1)
                if (full) return launch_groups<X, Y, V, E, false, true>(a, g, stream);
            return launch_groups<X, Y, V, E, false, false>(a, g, stream);
        }
    if constexpr (V > 1)
        if (full) return launch_groups<X, Y, V, E, true, true>(a, g, stream);
    return launch_groups<X, Y, V, E, true, false>(a, g, stream);
}

// The more elements a thread has, the fewer shuffles and barriers there are to a row, and the more is under way: with 8 / 16 / 32 elements
// 65,536 rows of 4096 in bf16 take 268 / 242 / 164 us, 16,384 of 1024 19.7 / 16.8 / 13.6, 60,000 of 512 31.7 / 22.3 / 23.7, 131,072 of 64
// 9.6 / 7.8 / 10.7; in fp32 4096 of 4096 24.9 / 23.2 / 25.0.  A million rows of 16: 14 / 20 / 20, lanes then skip memory.  Rows that do not fill
// the threads of their group take 24 where that puts more of them on an SM, or as many with fewer threads idle: 24 million elements in
// rows of 264 in bf16 with 16 / 24 31.8 / 22.3, of 2304 with 32 / 24 22.6 / 19.6, of 1544 (fewer of them with 24) 22.7 / 26.8, in fp32 of 520 with
// 16 / 24 44.3 / 33.7, of 4104 45.2 / 35.8.
template <int X, int Y, int V> cudaError_t launch_vectors(const NormArgs& a, cudaStream_t stream)
{
    if (a.dim <= 32 || (a.dim <= 8 * kRowThreads && few_elements(a.rows, a.dim))) return launch_elements<X, Y, V, 8>(a, stream);
    const uint32_t e = a.dim <= (X == kF32 ? 16 * kRowThreads : 512) ? 16 : 32;
    if (a.dim > (X == kF32 ? 128 : 64) && a.dim <= 24 * kRowThreads && many_elements(a.rows, a.dim)) {
        const RowGroups g = row_groups(a.rows, a.dim, e, kRowThreads);
        const uint32_t by_24 = rows_at_once(a.dim, 24, kRowThreads), by_e = rows_at_once(a.dim, e, kRowThreads);
        if (a.dim != (uint64_t)g.threads * e && (e == 16 ? by_24 > by_e : by_24 >= by_e)) return launch_elements<X, Y, V, 24>(a, stream);
    }
    return e == 16 ? launch_elements<X, Y, V, 16>(a, stream) : launch_elements<X, Y, V, 32>(a, stream);
}

// Single elements are bound by instructions: with 8 / 24 elements 24 million in rows of 515 take 43 / 36 us in fp32, 42.6 / 27.1 in bf16, of 2050
// 39.8 / 35.0 and 35.9 / 28.1; of 770, of which an SM has as many at once either way, 40.5 / 41.5 and 37.1 / 39.6.  With less to do, 24
// have to put half as many rows again on an SM: 6 million in rows of 515 in bf16 13.2 / 10.7, of 1537 11.9 / 13.3, in fp32 13.1 / 12.8 and 12.6 / 14.4;
// 3 million of 515 8.2 / 8.3.
template <int X, int Y> cudaError_t launch_single(const NormArgs& a, cudaStream_t stream)
{
    if (a.dim > 24 * kRowThreads) return launch_elements<X, Y, 1, 32>(a, stream);
    bool by_24 = a.dim > 8 * kRowThreads;
    if (!by_24 && a.dim > 24 * 16 && many_elements(a.rows, a.dim)) {
        const uint32_t rows_24 = rows_at_once(a.dim, 24, kResident<24> * kRowThreads), rows_8 = rows_at_once(a.dim, 8, kResident<8> * kRowThreads);
        by_24 = a.rows * a.dim >= 12000000 ? rows_24 > rows_8 : X == kBf16 && 2 * rows_24 > 3 * rows_8;
    }
    return by_24 ? launch_elements<X, Y, 1, 24>(a, stream) : launch_elements<X, Y, 1, 8>(a, stream);
}

template <int X, int Y> cudaError_t launch(const NormArgs& a, cudaStream_t stream)
{
    if (a.dim > 32 * kRowThreads) return launch_pdl(norm_long_kernel<X, Y>, (unsigned)a.rows, kLongThreads, stream, a);
    constexpr int V = kVector<X, Y>;
    const int w = element_bytes(a.w_dtype);
    const bool fit = vectors_fit(a.x, kElemBytes<X>, V, a.dim) && vectors_fit(a.y, kElemBytes<Y>, V, a.dim) &&
                     vectors_fit(a.weight, w, V, a.dim) && vectors_fit(a.bias, w, V, a.dim);
    return fit ? launch_vectors<X, Y, V>(a, stream) : launch_single<X, Y>(a, stream);
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
