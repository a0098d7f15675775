// The global norm of many gradient tensors, and clipping by it.
//
//   N = sqrt(sum over all elements of x^2)        c = 1 where N <= max_norm, else max_norm / N
//   y = fl(c * x)
//
// The tensors are cut into tiles of 16 KB.  Up to 32 of them are one launch, a cluster whose CTAs hold one or four each.  Above that
// the measuring kernel's CTAs take the tiles in turn and leave one partial sum each, in a fixed order and without atomics, and
// every CTA of the kernel that scales adds them up itself (740 at most for each launch of the first kernel, from L2), so that
// no launch stands between the two, or, for long lists, a third kernel does.  The second reading comes from DRAM all the same
// where the tensors and what is written exceed about a quarter of L2: of 100 MB read twice, the second time backwards, 27 MB
// came from L2, whatever the eviction priorities.
// Squares are summed in fp32 inside a thread's share of a tile (at most 33 of them) and in 64 bits from there on.  A share
// whose sum of squares leaves the range where fp32 holds it is summed again in 64 bits: the norm is right for every finite
// gradient, also where single squares overflow or vanish in fp32.
#include <atomic>
#include <cmath>

#include "mqg_list.cuh"
#include "mqg_tma.cuh"
#include "mqg_training.h"
#include "mqg_vector.cuh"

namespace mqg {
namespace {

constexpr int kThreads = 256;
constexpr int kTileBytes = 16384;
// CTAs that are there at once, for 148 SMs: 5 to an SM of the measuring kernel (eight spill their vectors), 4 of the one that
// scales.
constexpr int kNormBlocks = 740, kScaleBlocks = 592;
// Above so many tiles a kernel of its own adds up the partial sums, and the one that scales has a CTA to a tile, which go
// through memory in the order of its addresses: 122 MB of bf16 into 245 of fp32 in 54 us where CTAs that take tiles in turn need
// 61.
constexpr uint64_t kApartTiles = 2 * kScaleBlocks;

// Tensors of one launch, passed by value: a kernel's parameters hold 32,764 bytes.
template <int CAP> struct TensorTable {
    int count;
    uint32_t tile_start[CAP + 1];
    uint64_t first[CAP + 1];                            // elements before the tensor in the whole list
    const void* ptr[CAP];
    uint8_t dtype[CAP];
};
constexpr int kLargeTable = 1024;

// Where a tile lies.
struct Tile {
    const void* ptr;         // its first element
    uint64_t at;             // elements before it in the whole list
    uint32_t count;          // its elements
    int dtype;
};

// The tensor that a tile is in.
template <int CAP> __device__ __forceinline__ int find_tensor(const TensorTable<CAP>& tab, uint32_t tile)
{
    return find_in_list<(CAP > 32)>(tab.tile_start, tab.count, tile);
}

template <int CAP> __device__ __forceinline__ Tile tile_of(const TensorTable<CAP>& tab, int tensor, uint32_t tile)
{
    Tile t;
    t.dtype = tab.dtype[tensor];
    const int shift = t.dtype == kF32 ? 2 : 1;
    const uint64_t n = tab.first[tensor + 1] - tab.first[tensor];
    const uint64_t e0 = (uint64_t)(tile - tab.tile_start[tensor]) * (kTileBytes >> shift);
    t.ptr = static_cast<const char*>(tab.ptr[tensor]) + (e0 << shift);
    t.at = tab.first[tensor] + e0;
    t.count = (uint32_t)min((uint64_t)(kTileBytes >> shift), n - e0);
    return t;
}

// A tile's elements before its first 16-byte boundary, its vectors and what is left behind them.
template <int DTYPE> struct Parts {
    static constexpr int V = 16 / kElemBytes<DTYPE>;
    uint32_t head, nvec, tail, count;
    __device__ __forceinline__ Parts(const void* p, uint32_t m) : count(m)
    {
        const uint32_t to_boundary = (uint32_t)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / kElemBytes<DTYPE>;
        head = to_boundary < m ? to_boundary : m;
        nvec = (m - head) / V;
        tail = m - head - nvec * V;
    }
    // The element outside the vectors that thread i takes care of, if there is one.
    __device__ __forceinline__ bool edge(uint32_t i, uint32_t& at) const
    {
        at = i < head ? i : count - tail + (i - head);
        return i < head + tail;
    }
};

template <int BLOCK = kThreads> __device__ __forceinline__ double block_sum(double v)
{
    __shared__ double warp_sum[BLOCK / 32];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = v;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int w = 0; w < BLOCK / 32; ++w) t += warp_sum[w];
    return t;
}

// What fp32 holds a sum of at most 33 squares in without loss: none overflows, and what vanishes of the smallest is below
// 2^-40 of the sum.
__device__ __forceinline__ bool squares_in_range(float s) { return s >= 0x1p-100f && s <= 0x1p120f; }

// Sum of the squares of K vectors and an edge element.
template <int DTYPE, int K>
__device__ __forceinline__ double squares(const Packed<DTYPE, 16 / kElemBytes<DTYPE>> (&x)[K], float edge)
{
    constexpr int V = 16 / kElemBytes<DTYPE>;
    float t = edge * edge;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float s = x[k].get(0) * x[k].get(0);
#pragma unroll
        for (int e = 1; e < V; ++e) s = __fmaf_rn(x[k].get(e), x[k].get(e), s);
        t += s;
    }
    if (squares_in_range(t)) return (double)t;
    double d = (double)edge * (double)edge;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) d = fma((double)x[k].get(e), (double)x[k].get(e), d);
    return d;
}

// The number of this thread among the kThreads that have a tile.
__device__ __forceinline__ uint32_t tile_thread() { return threadIdx.x % kThreads; }

// This thread's vectors of a tile, zeros where there are none, and its element outside them.
constexpr int kVectors = kTileBytes / 16 / kThreads;
struct Held { uint4 x[kVectors]; float edge; };
template <int DTYPE> struct Share {
    static constexpr int V = 16 / kElemBytes<DTYPE>;
    const typename Element<DTYPE>::type* p;
    Parts<DTYPE> parts;
    Packed<DTYPE, V> x[kVectors];
    float edge;
    uint32_t edge_at;
    bool has_edge;

    __device__ __forceinline__ Share(const Tile& t) : p(static_cast<const typename Element<DTYPE>::type*>(t.ptr)), parts(p, t.count)
    {
        const auto* from = p + first();
#pragma unroll
        for (int k = 0; k < kVectors; ++k) {
            if (has(k)) x[k].load(from + k * kThreads * V);
            else x[k].w[0] = make_uint4(0, 0, 0, 0);
        }
        has_edge = parts.edge(tile_thread(), edge_at);
        edge = has_edge ? widen(p[edge_at]) : 0.0f;
    }
    // as it was held by another of the same tile
    __device__ __forceinline__ Share(const Tile& t, const Held& h) : p(static_cast<const typename Element<DTYPE>::type*>(t.ptr)), parts(p, t.count)
    {
#pragma unroll
        for (int k = 0; k < kVectors; ++k) x[k].w[0] = h.x[k];
        has_edge = parts.edge(tile_thread(), edge_at);
        edge = h.edge;
    }
    __device__ __forceinline__ void hold(Held& h) const
    {
#pragma unroll
        for (int k = 0; k < kVectors; ++k) h.x[k] = x[k].w[0];
        h.edge = edge;
    }
    __device__ __forceinline__ bool has(int k) const { return tile_thread() + k * kThreads < parts.nvec; }
    // the first of its vectors' elements; the next are kThreads vectors further on
    __device__ __forceinline__ uint32_t first() const { return parts.head + tile_thread() * V; }
    __device__ __forceinline__ double sum() const { return squares<DTYPE, kVectors>(x, edge); }
};

// Bound by reading the tensors.  (CTAs of eight neighbouring tiles each, in the order of the addresses: 78.9 us on 500 MB against
// 79.6, and a turn of a few CTAs more on shorter lists.)
template <int CAP>
__global__ void __launch_bounds__(kThreads, kNormBlocks / 148)
norm_kernel(const __grid_constant__ TensorTable<CAP> tab, double* __restrict__ partial)
{
    const uint32_t ntiles = tab.tile_start[tab.count];
    double sum = 0.0;
    Tile t = tile_of(tab, find_tensor(tab, blockIdx.x), blockIdx.x);
    grid_dependency_wait();
    for (uint32_t tile = blockIdx.x; tile < ntiles;) {
        sum += t.dtype == kF32 ? Share<kF32>(t).sum() : Share<kBf16>(t).sum();
        tile += gridDim.x;
        if (tile < ntiles) t = tile_of(tab, find_tensor(tab, tile), tile);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

// The factor for a sum of squares S, and the norm, in 64 bits: 1 / sqrt(S) by one step of Newton's iteration from fp32's
// reciprocal root of S scaled to 1 .. 4 (an error of 2^-21 becomes 2^-41).  A division and a square root in 64 bits took every CTA
// that scales longer than adding up the partial sums.  A NaN among the elements makes norm and factor NaN, an infinity makes
// the factor 0.
__device__ __forceinline__ float factor_of(double s, float max_norm, float* norm)
{
    const int high = __double2hiint(s), even = ((high >> 20) - 1023) & ~1;          // exponent of the scale 2^even <= S
    if (!(s > 0.0) || (high >> 20) == 0x7FF) {          // zero, infinity, NaN
        *norm = (float)s;
        return s <= (double)max_norm ? 1.0f : s > 0.0 ? 0.0f : (float)s;
    }
    const double m = __hiloint2double(high - even * (1 << 20), __double2loint(s)), y0 = (double)rsqrtf((float)m);
    const double y = fma(y0, fma(-0.5 * m * y0, y0, 0.5), y0);
    const double up = __hiloint2double((even / 2 + 1023) << 20, 0), down = __hiloint2double((1023 - even / 2) << 20, 0);
    const double n = m * y * up;
    *norm = (float)n;
    return n <= (double)max_norm ? 1.0f : (float)((double)max_norm * (y * down));
}

__device__ __forceinline__ double sum_of_partials(const double* partial, int count)
{
    double s = 0.0;
#pragma unroll 4
    for (int i = threadIdx.x; i < count; i += kThreads) s += __ldcg(partial + i);
    return block_sum(s);
}

__global__ void __launch_bounds__(kThreads)
norm_result_kernel(const double* __restrict__ partial, int npartial, float max_norm, float* __restrict__ result)
{
    grid_dependency_wait();
    float norm;
    const float c = factor_of(sum_of_partials(partial, npartial), max_norm, &norm);
    if (threadIdx.x == 0) { result[0] = norm; result[1] = c; }
}

// y = c * x in place.
template <int DTYPE> __device__ __forceinline__ void scale_tile(const Tile& t, float c)
{
    auto* p = static_cast<typename Element<DTYPE>::type*>(const_cast<void*>(t.ptr));
    Share<DTYPE> s(t);
    if (s.has_edge) narrow(c * s.edge, p[s.edge_at]);
    p += s.first();
#pragma unroll
    for (int k = 0; k < kVectors; ++k) {
        if (!s.has(k)) continue;
#pragma unroll
        for (int e = 0; e < Share<DTYPE>::V; ++e) s.x[k].set(e, c * s.x[k].get(e));
        s.x[k].store(p + k * kThreads * Share<DTYPE>::V);
    }
}

// y = c * x into another buffer, by words of W elements from y's first 16-byte boundary on: 16 bytes of the wider type, so that
// every access of a warp covers whole sectors.  Where x does not lie on its words' boundaries there, element by element, lanes
// side by side.  (Words put together from the two that hold them took twice as long: ten times the instructions.)
template <int SRC, int DST>
__device__ __forceinline__ void copy_tile(const Tile& t, typename Element<DST>::type* y, float c)
{
    constexpr int W = 16 / (kElemBytes<SRC> > kElemBytes<DST> ? kElemBytes<SRC> : kElemBytes<DST>);
    constexpr int K = kTileBytes / kElemBytes<SRC> / W / kThreads;
    const auto* x = static_cast<const typename Element<SRC>::type*>(t.ptr);
    const uint32_t to_boundary = (uint32_t)((16 - (reinterpret_cast<uintptr_t>(y) & 15)) & 15) / kElemBytes<DST>;
    const uint32_t head = to_boundary < t.count ? to_boundary : t.count;
    if ((reinterpret_cast<uintptr_t>(x + head) & (W * kElemBytes<SRC> - 1)) != 0) {
        // (loads under a condition each took 7 registers an element: 40 million elements in 75 us instead of 68)
        constexpr int kAhead = 16;
#pragma unroll 1
        for (uint32_t i0 = threadIdx.x; i0 < t.count; i0 += kAhead * kThreads) {
            typename Element<SRC>::type v[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) v[k] = __ldcg(x + min(i0 + k * kThreads, t.count - 1));
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (i0 + k * kThreads < t.count) narrow(c * widen(v[k]), y[i0 + k * kThreads]);
        }
        return;
    }
    const uint32_t nvec = (t.count - head) / W, tail = t.count - head - nvec * W;
    const auto* from = x + head + threadIdx.x * W;
    auto* to = y + head + threadIdx.x * W;
    Packed<SRC, W> in[K];
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (threadIdx.x + k * kThreads < nvec) in[k].load(from + k * kThreads * W);
    if (threadIdx.x < head + tail) {
        const uint32_t i = threadIdx.x < head ? threadIdx.x : t.count - tail + (threadIdx.x - head);
        narrow(c * widen(x[i]), y[i]);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (threadIdx.x + k * kThreads >= nvec) continue;
        Packed<DST, W> out;
#pragma unroll
        for (int e = 0; e < W; ++e) out.set(e, c * in[k].get(e));
        out.store(to + k * kThreads * W);
    }
}

// Scales the tiles of one table, the last first: what the measuring kernel read last is what L2 still holds.
// partial == nullptr: the factor is at `factor`.  DST < 0: in place.
template <int CAP, int DST>
__global__ void __launch_bounds__(kThreads)
scale_kernel(const __grid_constant__ TensorTable<CAP> tab, const double* __restrict__ partial, int npartial, float max_norm,
             const float* __restrict__ factor, void* __restrict__ flat, float* __restrict__ result)
{
    uint32_t tile = tab.tile_start[tab.count] - 1 - blockIdx.x;
    Tile t = tile_of(tab, find_tensor(tab, tile), tile);
    grid_dependency_wait();
    float c;
    if (partial != nullptr) {
        float norm;
        c = factor_of(sum_of_partials(partial, npartial), max_norm, &norm);
        if (result != nullptr && blockIdx.x == 0 && threadIdx.x == 0) { result[0] = norm; result[1] = c; }
    } else {
        c = __ldcg(factor);
    }
    if (DST < 0 && c == 1.0f) return;                   // every product would be its own factor
    for (;;) {
        if constexpr (DST < 0) {
            if (t.dtype == kF32) scale_tile<kF32>(t, c);
            else scale_tile<kBf16>(t, c);
        } else {
            auto* y = static_cast<typename Element<DST>::type*>(flat) + t.at;
            if (t.dtype == kF32) copy_tile<kF32, DST>(t, y, c);
            else copy_tile<kBf16, DST>(t, y, c);
        }
        if (tile < gridDim.x) return;
        tile -= gridDim.x;
        t = tile_of(tab, find_tensor(tab, tile), tile);
    }
}

// ---- one launch ----
constexpr int kClusterTensors = 32;
constexpr unsigned kClusterCtas = 8, kClusterTiles = 4 * kClusterCtas;

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t rank;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    return rank;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ double peer_load(const double* p, uint32_t rank)
{
    uint32_t at;
    double v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(at) : "memory");
    return v;
}

// The sum of squares of a cluster's CTAs.
template <int BLOCK> __device__ __forceinline__ double cluster_sum(double v)
{
    __shared__ double cta_sum;
    v = block_sum<BLOCK>(v);
    if (threadIdx.x == 0) cta_sum = v;
    cluster_arrive();
    cluster_wait();
    double all = 0.0;
    for (uint32_t r = 0; r < gridDim.x; ++r) all += peer_load(&cta_sum, r);
    cluster_arrive();                                   // no CTA's sum goes before all have read it
    return all;
}

template <int SRC> __device__ __forceinline__ double measure_tile(const Tile& t, Held& h)
{
    const Share<SRC> s(t);
    s.hold(h);
    return s.sum();
}

// c times a tile as it is held.
template <int SRC, int DST> __device__ __forceinline__ void write_tile(const Tile& t, const Held& h, float c, void* flat)
{
    constexpr int V = Share<SRC>::V, D = DST < 0 ? SRC : DST;
    using Out = typename Element<D>::type;
    const Share<SRC> s(t, h);
    Out* y = DST < 0 ? static_cast<Out*>(const_cast<void*>(t.ptr)) : static_cast<Out*>(flat) + t.at;
    if (s.has_edge) narrow(c * s.edge, y[s.edge_at]);
    const bool aligned = (reinterpret_cast<uintptr_t>(y + s.parts.head) & (Packed<D, V>::kWordBytes - 1)) == 0;
    y += s.first();
#pragma unroll
    for (int k = 0; k < kVectors; ++k) {
        if (!s.has(k)) continue;
        Packed<D, V> out;
#pragma unroll
        for (int e = 0; e < V; ++e) out.set(e, c * s.x[k].get(e));
        if (aligned) {
            out.store(y + k * kThreads * V);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) y[k * kThreads * V + e] = out.e[e];
        }
    }
}

// Bound by latency: the launch, one turn to memory, the barrier.  Up to 8 tiles in CTAs of a tile each, up to 32 in CTAs of four: 9
// to 32 tiles measured in 3.4 to 3.7 us a call, written in 3.6 to 4.7, where two launches take 5.0 to 6.  (25 tiles in CTAs of 256
// threads that take them in turn: 5.8; clusters of 16 CTAs take 5.2 for whatever they hold.)  DST: -1 in place, -2 only the norm.
template <int DST, int BLOCK>
__global__ void __launch_bounds__(BLOCK)
clip_cluster_kernel(const __grid_constant__ TensorTable<kClusterTensors> tab, float max_norm, void* __restrict__ flat,
                    float* __restrict__ result)
{
    const uint32_t tile = cluster_rank() * (BLOCK / kThreads) + threadIdx.x / kThreads;
    const bool has_tile = tile < tab.tile_start[tab.count];     // others fill the cluster up, or there are no elements at all
    Tile t = {};
    if (has_tile) t = tile_of(tab, find_tensor(tab, tile), tile);
    grid_dependency_wait();
    Held h;
    double sum = 0.0;
    if (has_tile) sum = t.dtype == kF32 ? measure_tile<kF32>(t, h) : measure_tile<kBf16>(t, h);
    float norm;
    const float c = factor_of(cluster_sum<BLOCK>(sum), max_norm, &norm);
    if (cluster_rank() == 0 && threadIdx.x == 0) { result[0] = norm; result[1] = c; }
    if (DST != -2 && has_tile && !(DST == -1 && c == 1.0f)) {
        if (t.dtype == kF32) write_tile<kF32, DST>(t, h, c, flat);
        else write_tile<kBf16, DST>(t, h, c, flat);
    }
    cluster_wait();
}

template <int DST, int BLOCK>
cudaError_t launch_cluster(const TensorTable<kClusterTensors>& tab, float max_norm, void* flat, float* result, cudaStream_t stream)
{
    constexpr unsigned per = BLOCK / kThreads;
    unsigned ctas = 1;
    while (ctas * per < tab.tile_start[tab.count]) ctas *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(BLOCK);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ctas == 1 ? 1 : 2;
    return cudaLaunchKernelEx(&cfg, clip_cluster_kernel<DST, BLOCK>, tab, max_norm, flat, result);
}

template <int DST>
cudaError_t cluster_by_size(const TensorTable<kClusterTensors>& tab, float max_norm, void* flat, float* result, cudaStream_t stream)
{
    return tab.tile_start[tab.count] <= kClusterCtas ? launch_cluster<DST, kThreads>(tab, max_norm, flat, result, stream)
                                                     : launch_cluster<DST, 4 * kThreads>(tab, max_norm, flat, result, stream);
}

// params[i] <- fma(-lr, fl(c * acc[i]), params[i]), the last elements first: acc has mostly just been read, from the front on,
// by the call that measured it, and its end is what L2 still holds.  params pass through (evict-first), so that they do not
// displace it.
__global__ void __launch_bounds__(kThreads)
apply_clipped_kernel(float* __restrict__ params, const float* __restrict__ acc, float lr, const float* __restrict__ factor,
                     uint64_t n)
{
    const uint64_t n4 = n / 4, stride = (uint64_t)gridDim.x * kThreads;
    grid_dependency_wait();
    const float c = __ldcg(factor);
    for (uint64_t k = (uint64_t)blockIdx.x * kThreads + threadIdx.x; k < n4; k += stride) {
        const uint64_t i = n4 - 1 - k;
        float4 p = __ldcs(reinterpret_cast<const float4*>(params) + i);
        const float4 g = __ldcg(reinterpret_cast<const float4*>(acc) + i);
        p.x = __fmaf_rn(-lr, __fmul_rn(c, g.x), p.x);
        p.y = __fmaf_rn(-lr, __fmul_rn(c, g.y), p.y);
        p.z = __fmaf_rn(-lr, __fmul_rn(c, g.z), p.z);
        p.w = __fmaf_rn(-lr, __fmul_rn(c, g.w), p.w);
        __stcs(reinterpret_cast<float4*>(params) + i, p);
    }
    if (blockIdx.x == 0 && threadIdx.x < (n & 3)) {
        const uint64_t i = n4 * 4 + threadIdx.x;
        params[i] = __fmaf_rn(-lr, __fmul_rn(c, __ldcg(acc + i)), __ldcg(params + i));
    }
}

uint64_t tiles_of(const TensorList& list, int j)
{
    const uint64_t per_tile = list.dtype[j] == kF32 ? kTileBytes / 4 : kTileBytes / 2;
    return (list.size[j] + per_tile - 1) / per_tile;
}

template <int CAP> void fill_table(const TensorList& list, int first, int last, uint64_t before, TensorTable<CAP>& tab)
{
    uint64_t tiles = 0;
    int k = 0;
    for (int j = first; j < last; ++j, ++k) {
        tab.tile_start[k] = (uint32_t)tiles;
        tab.first[k] = before;
        tab.ptr[k] = list.ptr[j];
        tab.dtype[k] = (uint8_t)list.dtype[j];
        tiles += tiles_of(list, j);
        before += list.size[j];
    }
    tab.tile_start[k] = (uint32_t)tiles;
    tab.first[k] = before;
    tab.count = k;
}

template <int CAP, typename Fn> cudaError_t with_table(const TensorList& list, int first, int last, uint64_t& before, Fn& fn)
{
    TensorTable<CAP> tab;
    fill_table(list, first, last, before, tab);
    before = tab.first[tab.count];
    return fn(tab);
}

// Calls fn(table) for the list in tables of at most kLargeTable tensors, each as small as its tensors allow: a launch costs
// 0.25 us more for every 4 KB of parameters.
template <typename Fn> cudaError_t for_each_table(const TensorList& list, Fn&& fn)
{
    uint64_t before = 0;
    cudaError_t err = cudaSuccess;
    for (int first = 0; first < list.count && err == cudaSuccess; first += kLargeTable) {
        const int last = list.count - first > kLargeTable ? first + kLargeTable : list.count, n = last - first;
        err = n <= 32    ? with_table<32>(list, first, last, before, fn)
              : n <= 384 ? with_table<384>(list, first, last, before, fn)
                         : with_table<kLargeTable>(list, first, last, before, fn);
    }
    return err;
}

template <int CAP> unsigned blocks_of(const TensorTable<CAP>& tab, int most)
{
    const uint32_t tiles = tab.tile_start[tab.count];
    return tiles < (uint32_t)most ? tiles : (unsigned)most;
}

template <int DST, int CAP>
cudaError_t scale_table(const TensorTable<CAP>& tab, const double* partial, int npartial, float max_norm, const float* factor,
                        void* flat, float* result, cudaStream_t stream)
{
    // A CTA to a tile where the factor is there already and every tile is written; in place most calls write nothing.
    const unsigned blocks = blocks_of(tab, DST >= 0 && partial == nullptr ? 0x7FFFFFFF : kScaleBlocks);
    if (blocks == 0) return cudaSuccess;
    return launch_pdl(scale_kernel<CAP, DST>, blocks, kThreads, stream, tab, partial, npartial, max_norm, factor, flat, result);
}

}  // namespace

size_t norm_workspace_floats(int count)
{
    const size_t tables = count <= 0 ? 1 : ((size_t)count + kLargeTable - 1) / kLargeTable;
    return tables * kNormBlocks * 2;                    // a 64-bit sum for each CTA
}

cudaError_t launch_clip(const TensorList& list, float max_norm, ClipForm form, void* flat, int flat_dtype, float* result,
                        float* workspace, cudaStream_t stream)
{
    uint64_t tiles = 0;
    for (int j = 0; j < list.count; ++j) tiles += tiles_of(list, j);
    if (tiles == 0 || (list.count <= kClusterTensors && tiles <= kClusterTiles)) {
        TensorTable<kClusterTensors> tab;
        fill_table(list, 0, tiles == 0 ? 0 : list.count, 0, tab);   // any number of empty tensors are no tensors
        return form == kMeasureOnly ? cluster_by_size<-2>(tab, max_norm, nullptr, result, stream)
               : form == kInPlace   ? cluster_by_size<-1>(tab, max_norm, nullptr, result, stream)
               : flat_dtype == kF32 ? cluster_by_size<kF32>(tab, max_norm, flat, result, stream)
                                    : cluster_by_size<kBf16>(tab, max_norm, flat, result, stream);
    }
    double* partial = reinterpret_cast<double*>(workspace);
    int npartial = 0;
    cudaError_t err = for_each_table(list, [&](const auto& tab) {
        const unsigned blocks = blocks_of(tab, kNormBlocks);
        if (blocks == 0) return cudaSuccess;
        constexpr int CAP = sizeof(tab.dtype);          // a byte for each tensor
        const cudaError_t e = launch_pdl(norm_kernel<CAP>, blocks, kThreads, stream, tab, partial + npartial);
        npartial += (int)blocks;
        return e;
    });
    if (err != cudaSuccess) return err;
    if (form == kMeasureOnly || tiles > kApartTiles) {
        err = launch_pdl(norm_result_kernel, 1, kThreads, stream, partial, npartial, max_norm, result);
        if (err != cudaSuccess || form == kMeasureOnly) return err;
        partial = nullptr;
    }
    float* to = result;                                 // the first launch writes the result
    return for_each_table(list, [&](const auto& tab) {
        if (tab.tile_start[tab.count] == 0) return cudaSuccess;
        const cudaError_t e =
            form == kInPlace ? scale_table<-1>(tab, partial, npartial, max_norm, result + 1, nullptr, to, stream)
            : flat_dtype == kF32 ? scale_table<kF32>(tab, partial, npartial, max_norm, result + 1, flat, to, stream)
                                 : scale_table<kBf16>(tab, partial, npartial, max_norm, result + 1, flat, to, stream);
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
    if (blocks > 2 * kNormBlocks) blocks = 2 * kNormBlocks;
    return launch_pdl(apply_clipped_kernel, (unsigned)blocks, kThreads, stream, params, acc, lr, factor, n);
}

}  // namespace mqg
