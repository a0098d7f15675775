// The gradient of the layer norm, from the rows' means mu and reciprocal deviations r:
//   h = (x - mu) * r,  a = weight * dy
//   dx = r * (a - mean(a) - h * mean(a * h)),  dweight = sum over rows of dy * h,  dbias = sum over rows of dy
//
// Bound by memory: x and dy are read and dx is written.  A thread keeps the same columns of every row that its CTA takes, so the
// sums over the rows stay in its registers until the CTA's last row; the CTAs' sums are added up by a second launch.  Rows come by
// asynchronous copies, a few ahead, each thread its own elements: the copies that are on their way take no registers, and no
// thread waits for another's.
#include <algorithm>

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
    float* partial;          // [parts][2][dim]: sums for dweight and dbias; nullptr: the grid is one cluster, which adds them up itself
    void* dweight;
    void* dbias;
    int dw_dtype, add;
    uint64_t rows, dim;
    int w_dtype;
};

// Rows on their way to shared memory: each thread's own elements, and the rows' stats, which the first thread of a group copies
// for those of its warp.
template <int X, int Y, int V, int E> struct Ring {
    static constexpr bool kAsync = V > 1;
    static constexpr int kBytes = E * (kElemBytes<X> + kElemBytes<Y>);
    static constexpr int kStages = !kAsync ? 1 : kBytes <= 32 ? 5 : kBytes <= 48 ? 4 : kBytes <= 64 && E > 8 ? 5 : E > 16 ? (kBytes <= 128 ? 3 : kBytes <= 192 ? 2 : 1) : 3;
    Packed<X, V> x[kStages][E / V][kRowThreads];
    Packed<Y, V> dy[kStages][E / V][kRowThreads];
    float2 stats[kStages][kRowThreads];
};

// CTAs to an SM: what the registers leave room for, the next row's among them where it is loaded ahead.
template <int X, int Y, int V, int E> constexpr int kResident = E <= 8 && Ring<X, Y, V, E>::kAsync ? 2 : 1;

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// What the cluster's CTA `rank` has where this one has *p, in shared memory.
__device__ __forceinline__ float cluster_load(const float* p, uint32_t rank)
{
    uint32_t at;
    float v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at));
    return v;
}

constexpr uint32_t kClusterCtas = 8;                    // (portable)

__device__ __forceinline__ uint32_t cluster_ctas()
{
    uint32_t n;
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n));
    return n;
}
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// The sums of a row whose columns are shared out among a cluster's CTAs, in the CTAs' order.  Two turns' places: a CTA writes to a place
// again when all have been through the barrier of the turn between, and so have read it.
struct ClusterSums {
    float2 of_cta[2][kClusterCtas];

    __device__ __forceinline__ float2 operator()(float2 v, uint32_t ctas, uint32_t rank, int turn)
    {
        if (threadIdx.x < ctas) {
            uint32_t at;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(&of_cta[turn][rank])), "r"(threadIdx.x));
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(v.x), "f"(v.y) : "memory");
        }
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        float2 total = of_cta[turn][0];
        for (uint32_t k = 1; k < ctas; ++k) total = __fadd2_rn(total, of_cta[turn][k]);
        return total;
    }
};

// x rounded towards zero, its last bit set where that left something out: rounded to a bf16 then, it is x rounded once.
__device__ __forceinline__ float round_to_odd(double x)
{
    const float r = __double2float_rz(x);
    return (double)r == x ? r : __uint_as_float(__float_as_uint(r) | 1u);
}

// Column i of dweight, or i - dim of dbias.
template <int W> __device__ __forceinline__ void store_sum(void* dweight, void* dbias, uint64_t dim, uint64_t i, double sum, int add)
{
    auto* to = static_cast<typename Element<W>::type*>(i < dim ? dweight : dbias);
    if (to == nullptr) return;
    const uint64_t col = i < dim ? i : i - dim;
    if (add) sum += (double)widen(to[col]);
    narrow(W == kF32 ? (float)sum : round_to_odd(sum), to[col]);
}

// Rows of more elements leave the sums over the rows to a kernel of their own: registers hold no more.
template <int E> constexpr bool kSums = E <= 16;

// E elements to a thread, V to a vector.  FULL: rows of E times the threads of a group, without a condition on any vector.
// SPLIT: rows whose columns are shared out among the CTAs of a cluster, a group to a CTA.
template <int X, int Y, int V, int E, bool WIDE, bool FULL, bool SPLIT = false>
__global__ void __launch_bounds__(kRowThreads, (kResident<X, Y, V, E>)) grad_rows_kernel(const GradArgs a, uint32_t threads, int sums)
{
    using R = Ring<X, Y, V, E>;
    constexpr int K = E / V;
    extern __shared__ __align__(16) unsigned char memory[];
    auto& ring = *reinterpret_cast<R*>(memory);
    __shared__ RowSums row_sums;
    const uint32_t place = threadIdx.x % threads, group = threadIdx.x / threads, groups = blockDim.x / threads;
    __shared__ ClusterSums cluster_sums;
    const uint32_t ctas = SPLIT ? cluster_ctas() : 1, rank = SPLIT ? cluster_rank() : 0;
    const uint64_t share = SPLIT ? (a.dim + ctas * V - 1) / (ctas * V) * V : a.dim, first_column = rank * share;
    const RowPlace<V, K, WIDE, FULL> at(SPLIT ? min(share, a.dim - first_column) : a.dim, place, threads);
    // the first thread of this one's group in its warp
    const uint32_t first = threads >= 32 ? threadIdx.x & ~31u : threadIdx.x - place;
    const uint64_t stride = (uint64_t)(gridDim.x / ctas) * groups, first_row = (uint64_t)(blockIdx.x / ctas) * groups + group;
    const float per_element = __fdiv_rn(1.0f, (float)a.dim);
    if (SPLIT) cluster_arrive();                        // (all CTAs of the cluster are there before one writes to another)
    grid_dependency_wait();
    const auto* x = static_cast<const typename Element<X>::type*>(a.x) + first_column;
    const auto* dy = static_cast<const typename Element<Y>::type*>(a.dy) + first_column;
    auto* dx = static_cast<typename Element<X>::type*>(a.dx) + first_column;
    // Where this thread's elements of the row are that is fetched next, and of the one that is written next: kept where registers are
    // left for it (65,536 rows of 4096 in bf16 at the power limit: 7 % longer with two products for every row).
    constexpr bool kKept = R::kAsync && E > 8;
    const uint64_t row_step = stride * a.dim, from = first_row * a.dim + at.element(0);
    const auto* next_of_x = x + from;
    const auto* next_of_dy = dy + from;
    auto* next_of_dx = dx + from;
    const auto fetch = [&](uint64_t row, int slot) {
        const auto* row_x = kKept ? next_of_x : x + row * a.dim + at.element(0);
        const auto* row_dy = kKept ? next_of_dy : dy + row * a.dim + at.element(0);
        if (row < a.rows) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (!at.has(k)) continue;
                copy_async<V * kElemBytes<X>>(&ring.x[slot][k][threadIdx.x], row_x + at.beyond(k));
                copy_async<V * kElemBytes<Y>>(&ring.dy[slot][k][threadIdx.x], row_dy + at.beyond(k));
            }
            if (threadIdx.x == first) {
                copy_async<4>(&ring.stats[slot][first].x, a.stats + 2 * row);
                copy_async<4>(&ring.stats[slot][first].y, a.stats + 2 * row + 1);
            }
        }
        commit_copies();
        next_of_x += row_step;
        next_of_dy += row_step;
    };
    float w[E];
    float2 dw[E / 2], db[E / 2];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float wk[V];
#pragma unroll
        for (int e = 0; e < V; ++e) wk[e] = 0.0f;
        if (at.has(k)) weights_at<V>(a.weight, a.w_dtype, (uint32_t)first_column + at.element(k), 1.0f, wk);
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
                if (!at.has(k))
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        ring.x[s][k][threadIdx.x].set(e, 0.0f);
                        ring.dy[s][k][threadIdx.x].set(e, 0.0f);
                    }
#pragma unroll
        for (int s = 0; s < R::kStages - 1; ++s) fetch(first_row + s * stride, s);
    }
    // single elements: the next row, where registers hold one more
    constexpr bool kAhead = !R::kAsync && E <= 12;
    Packed<X, V> next_x[R::kAsync ? 1 : K];
    Packed<Y, V> next_dy[R::kAsync ? 1 : K];
    float2 next_stats = make_float2(0.0f, 0.0f);
    const auto load_next = [&](uint64_t row) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            next_x[k].set(0, 0.0f);
            next_dy[k].set(0, 0.0f);
            if (row < a.rows && at.has(k)) {
                next_x[k].load(x + row * a.dim + at.element(k));
                next_dy[k].load(dy + row * a.dim + at.element(k));
            }
        }
        if (row < a.rows) next_stats = make_float2(__ldg(a.stats + 2 * row), __ldg(a.stats + 2 * row + 1));
    };
    if constexpr (kAhead) load_next(first_row);
    int slot = 0, turn = 0;
    if (SPLIT) cluster_wait();
    // Every group of a CTA takes as many turns: the barriers of its warps are its own, but the lanes of one warp stay together.
    for (uint64_t base = first_row - group; base < a.rows; base += stride) {
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
            if constexpr (!kAhead) load_next(row);
            if (has) stats = next_stats;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                widen_to<X, V>(next_x[k], vx + k * V);
                widen_to<Y, V>(next_dy[k], vd + k * V);
            }
            if constexpr (kAhead) load_next(row + stride);
        }
        float2 sum = make_float2(0.0f, 0.0f), along = make_float2(0.0f, 0.0f);
        const float2 minus = make_float2(-stats.x, -stats.x), rstd = make_float2(stats.y, stats.y);
        if (has) {
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const float2 d = make_float2(vd[e], vd[e + 1]);
                const float2 h = __fmul2_rn(__fadd2_rn(make_float2(vx[e], vx[e + 1]), minus), rstd);
                const float2 g = __fmul2_rn(d, make_float2(w[e], w[e + 1]));
                if constexpr (kSums<E>) {
                    dw[e / 2] = __ffma2_rn(d, h, dw[e / 2]);
                    db[e / 2] = __fadd2_rn(db[e / 2], d);
                }
                sum = __fadd2_rn(sum, g);
                along = __ffma2_rn(g, h, along);
                vx[e] = h.x;
                vx[e + 1] = h.y;
                vd[e] = g.x;
                vd[e + 1] = g.y;
            }
            // (places without elements have x = dy = 0, and so h = -mu r: where that is infinite, its product with zero is left out)
            if (!FULL && !(fabsf(stats.x * stats.y) < INFINITY)) {
                along = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (at.has(e / V)) along.x = fmaf(vd[e], vx[e], along.x);
            }
        }
        if (a.dx == nullptr) continue;
        float2 both = row_sums.two(make_float2(sum.x + sum.y, along.x + along.y), threads, group, turn);
        if constexpr (SPLIT) both = cluster_sums(both, ctas, rank, turn);
        turn ^= 1;
        auto* row_dx = kKept ? next_of_dx : dx + row * a.dim + at.element(0);
        next_of_dx += row_step;
        if (!has) continue;
        // r g - r m1 - h (r m2)
        const float c1 = -stats.y * (both.x * per_element), c2 = -stats.y * (both.y * per_element);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!at.has(k)) continue;
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
            out.store(row_dx + at.beyond(k));
        }
    }
    if (!kSums<E> || !sums) return;
    // The groups' sums through shared memory, in 64 bits and a fixed order: where there are more threads than columns, each adds up the
    // groups of one of several stripes, and then one the stripes.
    if constexpr (R::kAsync) wait_copies<0>();
    __syncthreads();
    const uint32_t dim = (uint32_t)(SPLIT ? min(share, a.dim - first_column) : a.dim), columns = 2 * dim;        // of dweight and of dbias
    float* all = reinterpret_cast<float*>(memory);      // [2][groups][dim]
    float* totals = all + 2 * kRowThreads * E;          // [2][dim]; behind one for each thread, [stripes][2][dim]
    double* of_stripes = reinterpret_cast<double*>(totals + kRowThreads);
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (at.has(e / V)) {
            float* to = all + group * dim + at.element(e / V) + e % V;
            to[0] = e % 2 ? dw[e / 2].y : dw[e / 2].x;
            to[groups * dim] = e % 2 ? db[e / 2].y : db[e / 2].x;
        }
    __syncthreads();
    float* left = a.partial != nullptr ? a.partial + (uint64_t)(blockIdx.x / ctas) * 2 * a.dim + first_column : totals;
    if constexpr (SPLIT) {                              // (one group)
        for (uint32_t i = threadIdx.x; i < columns; i += blockDim.x) left[i < dim ? i : a.dim + i - dim] = all[i];
    } else if (columns >= blockDim.x) {
        for (uint32_t i = threadIdx.x; i < columns; i += blockDim.x) {
            const float* from = all + (i < dim ? i : groups * dim + i - dim);
            double total = (double)from[0];
            for (uint32_t g = 1; g < groups; ++g) total += (double)from[g * dim];
            left[i] = (float)total;
        }
    } else {
        const uint32_t stripes = blockDim.x / columns, stripe = threadIdx.x / columns, column = threadIdx.x - stripe * columns;
        double total = 0.0;
        if (stripe < stripes) {
            const float* from = all + (column < dim ? column : groups * dim + column - dim);
#pragma unroll 4
            for (uint32_t g = stripe; g < groups; g += stripes) total += (double)from[g * dim];
            of_stripes[threadIdx.x] = total;
        }
        __syncthreads();
        if (stripe == 0) {
            for (uint32_t k = 1; k < stripes; ++k) total += of_stripes[k * columns + column];
            left[column] = (float)total;
        }
    }
    if (a.partial != nullptr) return;
    // Every CTA of the cluster adds up the totals of its share of the columns, in the CTAs' order.
    cluster_arrive();
    cluster_wait();
    for (uint32_t i = blockIdx.x * blockDim.x + threadIdx.x; i < 2 * dim; i += gridDim.x * blockDim.x) {
        float of_cta[kClusterCtas];                     // all under way at once
#pragma unroll
        for (uint32_t rank = 0; rank < kClusterCtas; ++rank) of_cta[rank] = rank < gridDim.x ? cluster_load(totals + i, rank) : 0.0f;
        double total = 0.0;
#pragma unroll
        for (uint32_t rank = 0; rank < kClusterCtas; ++rank) total += (double)of_cta[rank];
        if (a.dw_dtype == kF32) store_sum<kF32>(a.dweight, a.dbias, dim, i, total, a.add);
        else store_sum<kBf16>(a.dweight, a.dbias, dim, i, total, a.add);
    }
    cluster_arrive();                                   // no CTA's totals go before all have read them
    cluster_wait();
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

// Sums over a part of the rows: a thread has C times V columns of every kStripes-th row.  Threads to an SM hide the loads better than rows
// ahead do: 2400 rows of 10,000, with dx, take 102.8 / 99.7 / 97.6 us in fp32 with 4 / 2 / 1 rows under way, 58.9 / 59.3 / 53.3 in bf16.
// Of single elements four columns share the row's stats: 2399 rows of 10,001 in fp32 156 us with one, 148 with four; 2926 of 8201 with 4 / 2 / 1
// rows under way 148.9 / 127.6 / 128.4, 132.3 / 106.7 / 108.7 in bf16, 1499 of 16,001 124.2 / 99.5 / 92.0, of two types 139.6 / 118.3 / 137.1.
constexpr int kStripes = 8, kColumnLanes = 32;
template <int X, int Y, int V> constexpr int kRowsAhead = V == 1 && X != Y ? 2 : 1;
template <int V> constexpr int kColumns = V == 1 ? 4 : 1;
template <int X, int Y, int V>
__global__ void __launch_bounds__(kColumnLanes* kStripes) columns_kernel(const GradArgs a, uint64_t per_part)
{
    constexpr int C = kColumns<V>, kAhead = kRowsAhead<X, Y, V>;
    __shared__ float2 sums[kStripes][C * V][kColumnLanes];
    const uint32_t lane = threadIdx.x % kColumnLanes, stripe = threadIdx.x / kColumnLanes;
    const uint64_t col = ((uint64_t)blockIdx.x * kColumnLanes * C + lane) * V;
    const uint64_t first = blockIdx.y * per_part, last = min(first + per_part, a.rows);
    grid_dependency_wait();
    const auto* x = static_cast<const typename Element<X>::type*>(a.x) + col;
    const auto* dy = static_cast<const typename Element<Y>::type*>(a.dy) + col;
    const auto has = [&](int c) { return col + c * kColumnLanes * V < a.dim; };
    float2 sum[C * V];                                  // of dweight and dbias
#pragma unroll
    for (int e = 0; e < C * V; ++e) sum[e] = make_float2(0.0f, 0.0f);
    if (col < a.dim)
#pragma unroll 1
        for (uint64_t row0 = first + stripe; row0 < last; row0 += kAhead * kStripes) {
            Packed<X, V> px[kAhead][C];
            Packed<Y, V> pd[kAhead][C];
            float2 stats[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const uint64_t row = min(row0 + i * kStripes, last - 1);
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const uint64_t from = row * a.dim + (has(c) ? c * kColumnLanes * V : 0);       // (what is added to no sum that counts)
                    px[i][c].load(x + from);
                    pd[i][c].load(dy + from);
                }
                stats[i] = make_float2(__ldg(a.stats + 2 * row), __ldg(a.stats + 2 * row + 1));
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (row0 + i * kStripes >= last) break;
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    float vx[V], vd[V];
                    widen_to<X, V>(px[i][c], vx);
                    widen_to<Y, V>(pd[i][c], vd);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        float2& to = sum[c * V + e];
                        to.x = fmaf(vd[e], (vx[e] - stats[i].x) * stats[i].y, to.x);
                        to.y += vd[e];
                    }
                }
            }
        }
#pragma unroll
    for (int e = 0; e < C * V; ++e) sums[stripe][e][lane] = sum[e];
    __syncthreads();
    static_assert(C * V <= kStripes, "a warp to each of a lane's columns");
    if (stripe >= C * V || !has(stripe / V)) return;
    double dw = 0.0, db = 0.0;
#pragma unroll
    for (int k = 0; k < kStripes; ++k) {
        dw += (double)sums[k][stripe][lane].x;
        db += (double)sums[k][stripe][lane].y;
    }
    const uint64_t i = col + stripe / V * kColumnLanes * V + stripe % V;
    a.partial[(blockIdx.y * 2ull + 0) * a.dim + i] = (float)dw;
    a.partial[(blockIdx.y * 2ull + 1) * a.dim + i] = (float)db;
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
    store_sum<W>(dweight, dbias, dim, i, sum, add);
}

uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// The longest row whose sums over the rows stay in registers: a row to a CTA.
constexpr uint64_t kSumsDim = 16 * kRowThreads;

// The CTAs of a cluster that does everything in one launch, for few elements; 0: a grid and a second launch.  (One row of 64: 4.6 us,
// 8.2 by two launches; 512 of 64 5.6 and 8.0, 256 of 256 5.7 and 5.6 to 7.8; 2048 of 64 7.3 and 5.6, one of 4096 7.5 and 7.0.)
uint32_t cluster_of(uint64_t rows, uint64_t dim, const RowGroups& g)
{
    if (dim > 1024 || rows * dim > 65536) return 0;
    uint32_t ctas = 1;
    while ((ctas < g.ctas || ctas * kRowThreads < 2 * dim) && ctas < kClusterCtas) ctas *= 2;
    return ctas;
}

// Parts of the rows that leave a sum each.  Longer rows: enough for every SM of at least 64 rows.
uint32_t long_parts(uint64_t rows, uint64_t dim)
{
    const uint64_t most = ceil_div(rows, 64), want = ceil_div(148 * 4, ceil_div(dim, kColumnLanes * 8));
    return (uint32_t)(most < want ? (most < 1 ? 1 : most) : want);
}

// Shared memory: the ring, then the sums.
template <int X, int Y, int V, int E>
constexpr size_t kGroupBytes = std::max<size_t>(Ring<X, Y, V, E>::kAsync ? sizeof(Ring<X, Y, V, E>) : 0,
                                                kSums<E> ? 3 * kRowThreads * E * sizeof(float) : 16);

template <typename Kernel>
cudaError_t launch_clusters(Kernel kernel, uint32_t ctas, uint32_t cluster, uint32_t block, size_t bytes, cudaStream_t stream, const GradArgs& a,
                            uint32_t threads, int sums)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a, threads, sums);
}

template <int X, int Y, int V, int E, bool WIDE, bool FULL>
cudaError_t launch_groups(const GradArgs& a, const RowGroups& g, uint32_t cluster, int sums, cudaStream_t stream)
{
    static std::atomic<bool> ready[64];
    const auto kernel = grad_rows_kernel<X, Y, V, E, WIDE, FULL>;
    constexpr size_t kBytes = kGroupBytes<X, Y, V, E>;
    if (const cudaError_t err = allow_shared(kernel, kBytes, ready)) return err;
    if (cluster == 0) return launch_pdl_smem(kernel, g.ctas, g.block, kBytes, stream, a, g.threads, sums);
    return launch_clusters(kernel, cluster, cluster, g.block, kBytes, stream, a, g.threads, sums);
}

template <int X, int Y, int V, int E> cudaError_t launch_elements(GradArgs a, int sums, uint32_t* parts, cudaStream_t stream)
{
    constexpr int kCtas = kResident<X, Y, V, E>;
    const RowGroups g = row_groups(a.rows, a.dim, E, kCtas * kRowThreads, kCtas);
    const uint32_t cluster = E <= 8 && sums ? cluster_of(a.rows, a.dim, g) : 0;
    *parts = g.ctas;
    if (cluster != 0) {
        a.partial = nullptr;
        *parts = 0;
    }
    const bool full = V > 1 && a.dim == (uint64_t)g.threads * E;
    if constexpr (V > 1 ? E < 32 : E <= 8)              // (rows that 32 elements to a thread are chosen for take whole warps)
        if (g.threads < 32) {
            if constexpr (V > 1 && !(E == 16 && X == kF32 && Y == kF32))        // (16 in fp32: where 8 leave threads of such groups idle)
                if (full) return launch_groups<X, Y, V, E, false, true>(a, g, cluster, sums, stream);
            return launch_groups<X, Y, V, E, false, false>(a, g, cluster, sums, stream);
        }
    if constexpr (V > 1)
        if (full) return launch_groups<X, Y, V, E, true, true>(a, g, cluster, sums, stream);
    return launch_groups<X, Y, V, E, true, false>(a, g, cluster, sums, stream);
}

// Rows longer than kSumsDim by two CTAs, on an SM each: the sums over the rows stay in registers and x and dy are read once, but the CTAs
// wait for one another in every row, 2 us for a pair.  Single elements (12 to a thread) where they fit: 2926 rows of 8201 in bf16 75 us,
// 109 by two kernels, 8 of 10,001 9.7 and 11.4.  Vectors where a row has bytes for that time, and rows enough to be worth it: 24 million
// elements in rows of 12,288 71 us and 94 in fp32, 60 and 64 of two types, of 9000 91 and 102, 66 and 66; in bf16 of 16,000 63 and 50;
// 300 of 16,000 in fp32 27.6 and 25.7, 74 16.2 and 13.2.
constexpr uint32_t kSplitCtas = 2;
template <int V> constexpr int kSplitE = V == 1 ? 12 : 16;
template <int X, int Y, int V> bool split(uint64_t rows, uint64_t dim)
{
    return dim > kSumsDim && dim <= kSplitCtas * kSplitE<V> * kRowThreads &&
           (V == 1 || (dim * (kElemBytes<X> + kElemBytes<Y>) >= 72000 && rows * dim >= 8000000));
}
uint32_t split_parts(uint64_t rows) { return (uint32_t)(rows < 148 / kSplitCtas ? (rows < 1 ? 1 : rows) : 148 / kSplitCtas); }

template <int X, int Y, int V> cudaError_t launch_split(const GradArgs& a, int sums, uint32_t* parts, cudaStream_t stream)
{
    constexpr int E = kSplitE<V>;
    static std::atomic<bool> ready[64];
    const auto kernel = grad_rows_kernel<X, Y, V, E, true, false, true>;
    constexpr size_t kBytes = kGroupBytes<X, Y, V, E>;
    if (const cudaError_t err = allow_shared(kernel, kBytes, ready)) return err;
    const uint32_t threads = (uint32_t)ceil_div(ceil_div(ceil_div(a.dim, kSplitCtas * V) * V, E), 32) * 32;
    *parts = split_parts(a.rows);
    return launch_clusters(kernel, *parts * kSplitCtas, kSplitCtas, threads, kBytes, stream, a, threads, sums);
}

// Elements to a thread.  More of them cost fewer shuffles and barriers to a row: 65,536 rows of 4096 in bf16 take a fifth longer with 8 than with
// 16 (then 260 to 285 us at the power limit, 252 after an idle moment); with 8 / 16 16,384 of 1024 27.7 / 24.0, but 64 of 4096 7.6 / 9.5; 4096 of
// 4096 in fp32 39.3 / 40.3; a million rows of 16 27 / 40.  In fp32 16 where 8 leave much of an SM's threads idle and 16 have as many rows on it:
// 24 million in rows of 264 61.5 / 51.4, of 2056 59.5 / 53.5, of 520 55.5 / 54.0, of 392 52.2 / 52.1, of 904 51.5 / 52.5.
// Single elements take 12 where that puts more rows on an SM: 24 million in rows of 515 with 8 / 12 in fp32 65.4 / 57.1, of 2050 75.4 / 57.7, of
// 3201 (one row either way) 62.4 / 63.1; 16 where these are a warp's, and 12 are more: of 385 with 8 / 12 / 16 60.9 / 63.9 / 54.9.
template <int X, int Y, int V> int elements_of(uint64_t rows, uint64_t dim)
{
    if (V == 1 && dim > 8 * kRowThreads) return dim <= 12 * kRowThreads ? 12 : 16;
    if (dim > 8 * kRowThreads) return 16;
    if (dim <= 32 || few_elements(rows, dim)) return 8;
    if (V == 1) {
        if (dim > 12 * 32 && dim <= 16 * 32) return 16;
        return dim > 12 * 16 && rows_at_once(dim, 12, kRowThreads) > rows_at_once(dim, 8, kRowThreads) ? 12 : 8;
    }
    if (X != kF32 || Y != kF32) return 16;
    const uint32_t by_8 = rows_at_once(dim, 8, 2 * kRowThreads, 2);
    return many_elements(rows, dim) && by_8 * dim * 10 < 2ull * kRowThreads * 8 * 6 && rows_at_once(dim, 16, kRowThreads) >= by_8 ? 16 : 8;
}

// dx, and the sums of `parts` parts of the rows (0: all of them are added up already).
template <int X, int Y, int V> cudaError_t launch_vectors(const GradArgs& a, int sums, uint32_t* parts, cudaStream_t stream)
{
    if (a.dim <= kSumsDim) {
        const int e = elements_of<X, Y, V>(a.rows, a.dim);
        if constexpr (V == 1)
            if (e == 12) return launch_elements<X, Y, V, 12>(a, sums, parts, stream);
        return e == 8 ? launch_elements<X, Y, V, 8>(a, sums, parts, stream) : launch_elements<X, Y, V, 16>(a, sums, parts, stream);
    }
    if constexpr (V == 1 || X == kF32 || Y == kF32)
        if (split<X, Y, V>(a.rows, a.dim)) return launch_split<X, Y, V>(a, sums, parts, stream);
    cudaError_t err = cudaSuccess;
    if (a.dx != nullptr && a.rows != 0) {
        if (a.dim <= 32 * kRowThreads) err = launch_elements<X, Y, V, 32>(a, 0, parts, stream);
        else err = launch_pdl(grad_long_kernel<X, Y>, (unsigned)a.rows, kLongThreads, stream, a);
    }
    if (!sums || err != cudaSuccess) return err;
    *parts = long_parts(a.rows, a.dim);
    return launch_pdl_grid(columns_kernel<X, Y, V>, dim3((unsigned)ceil_div(a.dim, kColumnLanes * kColumns<V> * V), *parts), kColumnLanes * kStripes, 0,
                           stream, a, ceil_div(a.rows, *parts));
}

template <int X, int Y> cudaError_t launch(const GradArgs& a, const NormGrads& out, cudaStream_t stream)
{
    const int sums = out.dweight != nullptr || out.dbias != nullptr;
    constexpr int V = kVector<X, Y>;
    const bool fit = vectors_fit(a.x, kElemBytes<X>, V, a.dim) && vectors_fit(a.dx, kElemBytes<X>, V, a.dim) &&
                     vectors_fit(a.dy, kElemBytes<Y>, V, a.dim) && vectors_fit(a.weight, element_bytes(a.w_dtype), V, a.dim);
    uint32_t parts = 0;
    const cudaError_t err = fit ? launch_vectors<X, Y, V>(a, sums, &parts, stream) : launch_vectors<X, Y, 1>(a, sums, &parts, stream);
    if (err != cudaSuccess || !sums || parts == 0) return err;
    const unsigned blocks = (unsigned)ceil_div(2 * a.dim, kJoinColumns);
    const auto join = out.dw_dtype == kF32 ? join_kernel<kF32> : join_kernel<kBf16>;
    return launch_pdl(join, blocks, kJoinColumns * kJoinStripes, stream, a.partial, parts, a.dim, out.dweight, out.dbias, (int)out.add);
}

}  // namespace

// (8 elements to a thread, two CTAs to an SM leave the most parts)
size_t layer_norm_workspace_floats(uint64_t rows, uint64_t dim)
{
    uint64_t parts = dim > kSumsDim ? long_parts(rows, dim) : row_groups(rows, dim, dim <= 8 * kRowThreads ? 8 : 16, 2 * kRowThreads).ctas;
    if (dim > kSumsDim && dim <= kSplitCtas * kSplitE<4> * kRowThreads) parts = std::max<uint64_t>(parts, split_parts(rows));
    return (size_t)(parts * 2 * dim);
}

cudaError_t launch_layer_norm_grad(const void* dy, int dy_dtype, const NormRows& in, const float* stats, const NormGrads& out,
                                   float* workspace, cudaStream_t stream)
{
    const GradArgs a = {in.x,  dy,           in.weight,    stats,   out.dx, workspace, out.dweight, out.dbias, out.dw_dtype,
                        out.add, in.rows, in.dim, in.w_dtype};
    return in.x_dtype == kF32 ? (dy_dtype == kF32 ? launch<kF32, kF32>(a, out, stream) : launch<kF32, kBf16>(a, out, stream))
                              : (dy_dtype == kF32 ? launch<kBf16, kF32>(a, out, stream) : launch<kBf16, kBf16>(a, out, stream));
}

}  // namespace mqg
