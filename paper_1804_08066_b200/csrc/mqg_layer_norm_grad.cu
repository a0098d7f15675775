// The gradient of the layer norm, from the rows' means mu and reciprocal deviations r:
//   h = (x - mu) * r,  a = weight * dy
//   dx = r * (a - mean(a) - h * mean(a * h)),  dweight = sum over rows of dy * h,  dbias = sum over rows of dy
//
// Bound by memory: x and dy are read and dx is written.  A thread keeps the same columns of every row that its CTA takes, so the
// sums over the rows stay in its registers until the CTA's last row; the CTAs' sums are added up by a second launch.  Rows come by
// asynchronous copies, a few ahead, each thread its own elements: the copies that are on their way take no registers, and no
// thread waits for another's.
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

// Rows on their way to shared memory: each thread's own elements, and the rows' stats, which the first thread of a group copies
// for those of its warp.
template <int X, int Y, int V, int E> struct Ring {
    static constexpr bool kAsync = V * kElemBytes<X> >= 4 && V * kElemBytes<Y> >= 4;
    static constexpr int kBytes = E * (kElemBytes<X> + kElemBytes<Y>);
    static constexpr int kStages = !kAsync ? 1 : kBytes <= 32 ? 5 : kBytes <= 48 ? 4 : kBytes <= 64 && E > 8 ? 5 : 3;
    Packed<X, V> x[kStages][E / V][kRowThreads];
    Packed<Y, V> dy[kStages][E / V][kRowThreads];
    float2 stats[kStages][kRowThreads];
};

template <int E> constexpr int kResident = E <= 8 ? 2 : 1;

// E elements to a thread, V to a vector.
template <int X, int Y, int V, int E>
__global__ void __launch_bounds__(kRowThreads, kResident<E>) grad_rows_kernel(const GradArgs a, uint32_t threads, int sums)
{
    using R = Ring<X, Y, V, E>;
    constexpr int K = E / V;
    extern __shared__ __align__(16) unsigned char memory[];
    auto& ring = *reinterpret_cast<R*>(memory);
    __shared__ RowSums row_sums;
    const uint32_t place = threadIdx.x % threads, group = threadIdx.x / threads, groups = blockDim.x / threads;
    const uint32_t vectors = (uint32_t)(a.dim / V);
    // the first thread of this one's group in its warp
    const uint32_t first = threads >= 32 ? threadIdx.x & ~31u : threadIdx.x - place;
    const uint64_t stride = (uint64_t)gridDim.x * groups;
    const float per_element = __fdiv_rn(1.0f, (float)a.dim);
    grid_dependency_wait();
    const auto* x = static_cast<const typename Element<X>::type*>(a.x);
    const auto* dy = static_cast<const typename Element<Y>::type*>(a.dy);
    auto* dx = static_cast<typename Element<X>::type*>(a.dx);
    const auto has_vector = [&](int k) { return place + k * threads < vectors; };
    const auto fetch = [&](uint64_t row, int slot) {
        if (row < a.rows) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (!has_vector(k)) continue;
                const uint64_t at = row * a.dim + (place + k * threads) * V;
                copy_async<V * kElemBytes<X>>(&ring.x[slot][k][threadIdx.x], x + at);
                copy_async<V * kElemBytes<Y>>(&ring.dy[slot][k][threadIdx.x], dy + at);
            }
            if (threadIdx.x == first) {
                copy_async<4>(&ring.stats[slot][first].x, a.stats + 2 * row);
                copy_async<4>(&ring.stats[slot][first].y, a.stats + 2 * row + 1);
            }
        }
        commit_copies();
    };
    float w[E];
    float2 dw[E / 2], db[E / 2];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float wk[V];
#pragma unroll
        for (int e = 0; e < V; ++e) wk[e] = 0.0f;
        if (has_vector(k)) weights_at<V>(a.weight, a.w_dtype, (place + k * threads) * V, 1.0f, wk);
#pragma unroll
        for (int e = 0; e < V; ++e) w[k * V + e] = wk[e];
    }
#pragma unroll
    for (int e = 0; e < E / 2; ++e) dw[e] = db[e] = make_float2(0.0f, 0.0f);
    if constexpr (R::kAsync) {
        // places without elements hold zeros, which no copy overwrites
#pragma unroll
        for (int s = 0; s < R::kStages; ++s)
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (!has_vector(k))
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        ring.x[s][k][threadIdx.x].set(e, 0.0f);
                        ring.dy[s][k][threadIdx.x].set(e, 0.0f);
                    }
#pragma unroll
        for (int s = 0; s < R::kStages - 1; ++s) fetch((uint64_t)blockIdx.x * groups + group + s * stride, s);
    }
    int slot = 0, turn = 0;
    // Every group of a CTA takes as many turns: the barriers of its warps are its own, but the lanes of one warp stay together.
    for (uint64_t base = (uint64_t)blockIdx.x * groups; base < a.rows; base += stride) {
        const uint64_t row = base + group;
        const bool has = row < a.rows;
        float vx[E], vd[E];
        float2 stats = make_float2(0.0f, 0.0f);
        if constexpr (R::kAsync) {
            __syncwarp();                               // the stats of the slot that is filled now have been read
            fetch(row + (R::kStages - 1) * stride, slot == 0 ? R::kStages - 1 : slot - 1);
            wait_copies<R::kStages - 1>();
            __syncwarp();
            if (has) stats = ring.stats[slot][first];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                widen_to<X, V>(ring.x[slot][k][threadIdx.x], vx + k * V);
                widen_to<Y, V>(ring.dy[slot][k][threadIdx.x], vd + k * V);
            }
            slot = slot == R::kStages - 1 ? 0 : slot + 1;
        } else {
            if (has) stats = make_float2(__ldg(a.stats + 2 * row), __ldg(a.stats + 2 * row + 1));
#pragma unroll
            for (int k = 0; k < K; ++k) {
                Packed<X, V> px;
                Packed<Y, V> pd;
#pragma unroll
                for (int e = 0; e < V; ++e) { px.set(e, 0.0f); pd.set(e, 0.0f); }
                if (has && has_vector(k)) {
                    px.load(x + row * a.dim + (place + k * threads) * V);
                    pd.load(dy + row * a.dim + (place + k * threads) * V);
                }
                widen_to<X, V>(px, vx + k * V);
                widen_to<Y, V>(pd, vd + k * V);
            }
        }
        float2 sum = make_float2(0.0f, 0.0f), along = make_float2(0.0f, 0.0f);
        const float2 minus = make_float2(-stats.x, -stats.x), rstd = make_float2(stats.y, stats.y);
        if (has) {
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const float2 d = make_float2(vd[e], vd[e + 1]);
                const float2 h = __fmul2_rn(__fadd2_rn(make_float2(vx[e], vx[e + 1]), minus), rstd);
                const float2 g = __fmul2_rn(d, make_float2(w[e], w[e + 1]));
                dw[e / 2] = __ffma2_rn(d, h, dw[e / 2]);
                db[e / 2] = __fadd2_rn(db[e / 2], d);
                sum = __fadd2_rn(sum, g);
                along = __ffma2_rn(g, h, along);
                vx[e] = h.x;
                vx[e + 1] = h.y;
                vd[e] = g.x;
                vd[e + 1] = g.y;
            }
        }
        if (dx == nullptr) continue;
        const float2 both = row_sums.two(make_float2(sum.x + sum.y, along.x + along.y), threads, group, turn);
        turn ^= 1;
        if (!has) continue;
        // r g - r m1 - h (r m2)
        const float c1 = -stats.y * (both.x * per_element), c2 = -stats.y * (both.y * per_element);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!has_vector(k)) continue;
            Packed<X, V> out;
            if constexpr (V > 1) {
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const int i = k * V + e;
                    const float2 h = make_float2(vx[i], vx[i + 1]), g = make_float2(vd[i], vd[i + 1]);
                    const float2 r = __ffma2_rn(g, rstd, __ffma2_rn(h, make_float2(c2, c2), make_float2(c1, c1)));
                    out.set(e, r.x);
                    out.set(e + 1, r.y);
                }
            } else {
                out.set(0, fmaf(vd[k], stats.y, fmaf(vx[k], c2, c1)));
            }
            out.store(dx + row * a.dim + (place + k * threads) * V);
        }
    }
    if (!sums) return;
    // The groups' sums, in their order, through shared memory.
    if constexpr (R::kAsync) wait_copies<0>();
    __syncthreads();
    float* all = reinterpret_cast<float*>(memory);      // [groups][dim] of one sum, then of the other
    const uint32_t dim = (uint32_t)a.dim;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float2 pair = which == 0 ? dw[e / 2] : db[e / 2];
            if (has_vector(e / V)) all[group * dim + (place + e / V * threads) * V + e % V] = e % 2 ? pair.y : pair.x;
        }
        __syncthreads();
        for (uint32_t col = threadIdx.x; col < dim; col += blockDim.x) {
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

// Elements of a row to a thread in the kernel that keeps it in registers; 0: the row is too long.
uint32_t row_elements(uint64_t dim) { return dim <= 8 * kRowThreads ? 8 : dim <= 16 * kRowThreads ? 16 : 0; }

RowGroups groups_of(uint64_t rows, uint64_t dim, uint32_t e) { return row_groups(rows, dim, e, (e <= 8 ? kResident<8> : kResident<16>)*kRowThreads); }

// Parts of the rows that leave a sum each: the CTAs of that kernel, or, for long rows, enough for every SM of at least 64 rows.
uint32_t parts_of(uint64_t rows, uint64_t dim)
{
    if (const uint32_t e = row_elements(dim)) return groups_of(rows, dim, e).ctas;
    const uint64_t most = ceil_div(rows, 64), want = ceil_div(148 * 8, ceil_div(dim, kColumns));
    return (uint32_t)(most < want ? (most < 1 ? 1 : most) : want);
}

template <int X, int Y, int V, int E> cudaError_t launch_elements(const GradArgs& a, int sums, cudaStream_t stream)
{
    using R = Ring<X, Y, V, E>;
    static std::atomic<bool> ready[64];
    const auto kernel = grad_rows_kernel<X, Y, V, E>;
    constexpr size_t kSums = kRowThreads * E * sizeof(float), kBytes = R::kAsync && sizeof(R) > kSums ? sizeof(R) : kSums;
    if (const cudaError_t err = allow_shared(kernel, kBytes, ready)) return err;
    const RowGroups g = groups_of(a.rows, a.dim, E);
    return launch_pdl_smem(kernel, g.ctas, g.block, kBytes, stream, a, g.threads, sums);
}

template <int X, int Y, int V> cudaError_t launch_vectors(const GradArgs& a, int sums, cudaStream_t stream)
{
    return row_elements(a.dim) == 8 ? launch_elements<X, Y, V, 8>(a, sums, stream) : launch_elements<X, Y, V, 16>(a, sums, stream);
}

template <int X, int Y> cudaError_t launch(const GradArgs& a, const NormGrads& out, cudaStream_t stream)
{
    const int sums = out.dweight != nullptr || out.dbias != nullptr;
    const uint32_t parts = parts_of(a.rows, a.dim);
    cudaError_t err = cudaSuccess;
    if (row_elements(a.dim) != 0) {
        constexpr int V = kVector<X, Y>;
        const bool fit = vectors_fit(a.x, kElemBytes<X>, V, a.dim) && vectors_fit(a.dx, kElemBytes<X>, V, a.dim) &&
                         vectors_fit(a.dy, kElemBytes<Y>, V, a.dim) && vectors_fit(a.weight, element_bytes(a.w_dtype), V, a.dim);
        err = fit ? launch_vectors<X, Y, V>(a, sums, stream) : launch_vectors<X, Y, 1>(a, sums, stream);
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
