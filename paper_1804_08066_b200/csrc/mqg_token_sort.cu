// Token ids sorted by id, stably, with the tokens' positions: least significant digit first, up to ten bits to a pass.
//
// Up to 65,536 tokens one thread-block cluster sorts in one launch.  A CTA holds K x 1024 pairs (key, token) of the order so
// far, K to a thread; a warp ranks its 32 K consecutive pairs by ballots, 32 at a time, the warps' digit counts are added up
// in shared memory and the CTAs' through distributed shared memory, and every pair is stored to its place in the CTA that
// holds it in the next pass (after the last one: to memory).  What bounds it is latency: two cluster barriers and about five
// dependent turns through shared memory for each pass.
// The launch's other CTAs set the buffer that the sums go to to zero meanwhile, which depends on nothing.
//
// More tokens take three launches a pass: count, scan, place.
#include <atomic>

#include "mqg_tma.cuh"
#include "mqg_token_sort.h"

namespace mqg {
namespace {

// An id as the key it is sorted by: those outside 0..rows-1 go behind all others.
template <typename ID> __device__ __forceinline__ uint32_t key_of(ID id, uint32_t rows)
{
    return id >= 0 && (uint64_t)id < rows ? (uint32_t)id : rows;
}

// The lanes of the warp that hold the same digit, among those that hold a key at all.
__device__ __forceinline__ uint32_t same_digit(uint32_t digit, int bits, uint32_t held)
{
    uint32_t same = held;
    for (int b = 0; b < bits; ++b) {
        const bool one = (digit >> b) & 1u;
        const uint32_t ones = __ballot_sync(0xFFFFFFFFu, one);
        same &= one ? ones : ~ones;
    }
    return same;
}

// ---- one launch ----
constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kMaxDigitBits = 10;

struct SortArgs {
    const void* ids;
    uint2* sorted;
    uint32_t* counter;       // set to zero for the kernels that follow
    void* zero;              // bytes to set to zero
    uint64_t zero_bytes;
    uint32_t tokens, rows;
    int bits, digit_bits;
    unsigned ctas;           // of the sort: the grid's first ones, one cluster
};

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t rank;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    return rank;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_address(const void* p, uint32_t rank)
{
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
    return at;
}
__device__ __forceinline__ uint32_t peer_load(const uint32_t* p, uint32_t rank)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(peer_address(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ void peer_store(uint2* p, uint32_t rank, uint2 v)
{
    asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(peer_address(p, rank)), "r"(v.x), "r"(v.y) : "memory");
}

__host__ __device__ constexpr size_t sort_smem(int per_thread, int bins)
{
    return (size_t)per_thread * kThreads * sizeof(uint2) + (size_t)bins * (kWarps * sizeof(uint16_t) + 2 * sizeof(uint32_t)) +
           kWarps * sizeof(uint32_t);
}

__device__ void set_zero(void* p, uint64_t bytes, unsigned cta, unsigned ctas)
{
    char* c = static_cast<char*>(p);
    const uint64_t to_boundary = (16 - (reinterpret_cast<uintptr_t>(c) & 15)) & 15;
    const uint64_t head = to_boundary < bytes ? to_boundary : bytes;
    const uint64_t nvec = (bytes - head) / 16, tail = bytes - head - nvec * 16;
    if (cta == 0 && threadIdx.x < head) c[threadIdx.x] = 0;
    if (cta == 0 && threadIdx.x < tail) c[bytes - tail + threadIdx.x] = 0;
    uint4* v = reinterpret_cast<uint4*>(c + head);
    const uint64_t stride = (uint64_t)ctas * kThreads;
    for (uint64_t i = (uint64_t)cta * kThreads + threadIdx.x; i < nvec; i += stride) v[i] = make_uint4(0, 0, 0, 0);
}

template <typename ID, int K>
__global__ void __launch_bounds__(kThreads) sort_cluster_kernel(const SortArgs a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr uint32_t kHeld = K * kThreads;            // pairs of a CTA
    const int bins = 1 << a.digit_bits;
    uint2* pairs = reinterpret_cast<uint2*>(smem);
    uint16_t* warp_count = reinterpret_cast<uint16_t*>(pairs + kHeld);               // [warp][digit]
    uint32_t* cta_count = reinterpret_cast<uint32_t*>(warp_count + kWarps * bins);   // [digit]
    uint32_t* place = cta_count + bins;                                              // [digit]
    uint32_t* warp_total = place + bins;                                             // [warp]
    const uint32_t d = threadIdx.x, lane = threadIdx.x & 31, w = threadIdx.x >> 5;

    grid_dependency_wait();
    if (blockIdx.x >= a.ctas) {
        set_zero(a.zero, a.zero_bytes, blockIdx.x - a.ctas, gridDim.x - a.ctas);
        return;
    }
    const uint32_t rank = cluster_rank();
    if (rank == 0 && threadIdx.x == 0) *a.counter = 0;
    const uint32_t local = w * (32 * K) + lane, first = rank * kHeld + local;
    uint16_t* mine = warp_count + w * bins;
    for (int shift = 0; shift < a.bits; shift += a.digit_bits) {
        const bool last = shift + a.digit_bits >= a.bits;
        uint2 pair[K];
#pragma unroll
        for (int r = 0; r < K; ++r) {
            const uint32_t i = first + r * 32;
            if (shift != 0) pair[r] = pairs[local + r * 32];
            else pair[r] = make_uint2(i < a.tokens ? key_of(__ldg(static_cast<const ID*>(a.ids) + i), a.rows) : 0u, i);
        }
        for (int i = lane; i < bins / 2; i += 32) reinterpret_cast<uint32_t*>(mine)[i] = 0;
        __syncwarp();
        uint32_t before[K];
#pragma unroll
        for (int r = 0; r < K; ++r) {
            const bool held = first + r * 32 < a.tokens;
            const uint32_t digit = (pair[r].x >> shift) & (bins - 1);
            const uint32_t same = same_digit(digit, a.digit_bits, __ballot_sync(0xFFFFFFFFu, held));
            const uint32_t so_far = mine[digit];
            __syncwarp();
            if (held && (same >> lane) == 1u) mine[digit] = (uint16_t)(so_far + __popc(same));
            __syncwarp();
            before[r] = so_far + __popc(same & ((1u << lane) - 1));
        }
        __syncthreads();
        uint32_t count = 0;
        if (d < (uint32_t)bins) {
#pragma unroll 8
            for (int v = 0; v < kWarps; ++v) {
                const uint32_t c = warp_count[v * bins + d];
                warp_count[v * bins + d] = (uint16_t)count;
                count += c;
            }
            cta_count[d] = count;
        }
        cluster_sync();                                 // the counts are there, and every CTA holds its pairs in registers
        uint32_t earlier = 0, total = 0;
        if (d < (uint32_t)bins) {
            for (uint32_t r = 0; r < a.ctas; ++r) {
                const uint32_t c = peer_load(cta_count + d, r);
                earlier += r < rank ? c : 0;
                total += c;
            }
        }
        uint32_t sum = total;                           // over the digits up to this one
#pragma unroll
        for (int step = 1; step < 32; step *= 2) {
            const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, sum, step);
            if (lane >= (uint32_t)step) sum += v;
        }
        if (lane == 31) warp_total[w] = sum;
        __syncthreads();
        uint32_t ahead = lane < w ? warp_total[lane] : 0;
#pragma unroll
        for (int step = 16; step > 0; step >>= 1) ahead += __shfl_xor_sync(0xFFFFFFFFu, ahead, step);
        if (d < (uint32_t)bins) place[d] = ahead + sum - total + earlier;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < K; ++r) {
            if (first + r * 32 >= a.tokens) continue;
            const uint32_t digit = (pair[r].x >> shift) & (bins - 1);
            const uint32_t at = place[digit] + mine[digit] + before[r];
            if (last) a.sorted[at] = pair[r];
            else peer_store(pairs + at % kHeld, at / kHeld, pair[r]);
        }
        cluster_sync();                                 // the pairs are there, and no CTA's counts go before they were read
    }
}

template <typename ID, int K> cudaError_t launch_cluster(const SortArgs& a, unsigned grid, cudaStream_t stream)
{
    static std::atomic<bool> ready[64];                 // per device (zero-initialised)
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev].load(std::memory_order_relaxed)) {
        err = cudaFuncSetAttribute(sort_cluster_kernel<ID, K>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                   (int)sort_smem(K, 1 << kMaxDigitBits));
        if (err != cudaSuccess) return err;
        ready[dev].store(true, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sort_smem(K, 1 << a.digit_bits);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = a.ctas == 0 ? 1 : a.ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, sort_cluster_kernel<ID, K>, a);
}

template <typename ID> cudaError_t launch_by_size(const SortArgs& a, uint32_t per_thread, unsigned grid, cudaStream_t stream)
{
    return per_thread <= 1 ? launch_cluster<ID, 1>(a, grid, stream)
           : per_thread <= 2 ? launch_cluster<ID, 2>(a, grid, stream)
           : per_thread <= 4 ? launch_cluster<ID, 4>(a, grid, stream)
                             : launch_cluster<ID, 8>(a, grid, stream);
}

// ---- three launches a pass ----
constexpr int kTile = 8 * kThreads;
constexpr int kBins = 256;

template <typename ID> struct PassInput {
    const ID* ids;           // of the first pass; null in the later ones
    const uint2* pairs;
    uint32_t count, rows;
    __device__ __forceinline__ uint2 get(uint32_t i) const
    {
        return ids != nullptr ? make_uint2(key_of(__ldg(ids + i), rows), i) : __ldcg(pairs + i);
    }
};

// Ranks a tile's pairs as above: before[r] of the warp's pairs with the same digit stand before this one.
template <typename ID>
__device__ __forceinline__ void rank_tile(const PassInput<ID>& in, int shift, uint16_t (*warp_count)[kBins], uint2 (&pair)[8],
                                          uint32_t (&before)[8])
{
    const uint32_t lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    for (int d = lane; d < kBins; d += 32) warp_count[w][d] = 0;
    const uint64_t first = (uint64_t)blockIdx.x * kTile + w * 256 + lane;
#pragma unroll
    for (int r = 0; r < 8; ++r) pair[r] = first + r * 32 < in.count ? in.get((uint32_t)first + r * 32) : make_uint2(0, 0);
    __syncwarp();
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const bool held = first + r * 32 < in.count;
        const uint32_t digit = (pair[r].x >> shift) & (kBins - 1);
        const uint32_t same = same_digit(digit, 8, __ballot_sync(0xFFFFFFFFu, held));
        const uint32_t so_far = warp_count[w][digit];
        __syncwarp();
        if (held && (same >> lane) == 1u) warp_count[w][digit] = (uint16_t)(so_far + __popc(same));
        __syncwarp();
        before[r] = so_far + __popc(same & ((1u << lane) - 1));
    }
}

template <typename ID>
__global__ void __launch_bounds__(kThreads)
count_kernel(const PassInput<ID> in, int shift, uint32_t* __restrict__ counts)
{
    __shared__ uint16_t warp_count[kWarps][kBins];
    uint2 pair[8];
    uint32_t before[8];
    grid_dependency_wait();
    rank_tile(in, shift, warp_count, pair, before);
    __syncthreads();
    if (threadIdx.x < kBins) {
        uint32_t sum = 0;
        for (int w = 0; w < kWarps; ++w) sum += warp_count[w][threadIdx.x];
        counts[(uint64_t)blockIdx.x * kBins + threadIdx.x] = sum;
    }
}

// counts[block][digit] becomes the first place of the block's keys of that digit.
__global__ void __launch_bounds__(kBins) scan_kernel(uint32_t* __restrict__ counts, uint32_t blocks, uint32_t* __restrict__ counter)
{
    __shared__ uint32_t total[kBins];
    const uint32_t d = threadIdx.x;
    grid_dependency_wait();
    if (d == 0) *counter = 0;
    uint32_t sum = 0;
#pragma unroll 8
    for (uint32_t b = 0; b < blocks; ++b) sum += __ldcg(counts + (uint64_t)b * kBins + d);
    total[d] = sum;
    __syncthreads();
    for (int step = 1; step < kBins; step *= 2) {
        const uint32_t v = d >= (uint32_t)step ? total[d - step] : 0;
        __syncthreads();
        total[d] += v;
        __syncthreads();
    }
    uint32_t at = total[d] - sum;
#pragma unroll 8
    for (uint32_t b = 0; b < blocks; ++b) {
        const uint32_t c = __ldcg(counts + (uint64_t)b * kBins + d);
        counts[(uint64_t)b * kBins + d] = at;
        at += c;
    }
}

template <typename ID>
__global__ void __launch_bounds__(kThreads)
place_kernel(const PassInput<ID> in, int shift, const uint32_t* __restrict__ counts, uint2* __restrict__ out)
{
    __shared__ uint16_t warp_count[kWarps][kBins];
    __shared__ uint32_t warp_first[kWarps][kBins];
    uint2 pair[8];
    uint32_t before[8];
    grid_dependency_wait();
    rank_tile(in, shift, warp_count, pair, before);
    __syncthreads();
    if (threadIdx.x < kBins) {
        uint32_t at = __ldcg(counts + (uint64_t)blockIdx.x * kBins + threadIdx.x);
        for (int w = 0; w < kWarps; ++w) {
            warp_first[w][threadIdx.x] = at;
            at += warp_count[w][threadIdx.x];
        }
    }
    __syncthreads();
    const uint32_t lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const uint64_t first = (uint64_t)blockIdx.x * kTile + w * 256 + lane;
#pragma unroll
    for (int r = 0; r < 8; ++r)
        if (first + r * 32 < in.count) out[warp_first[w][(pair[r].x >> shift) & (kBins - 1)] + before[r]] = pair[r];
}

// ---- host ----
constexpr uint32_t kMaxCluster = 8;
constexpr uint32_t kClusterTokens = kMaxCluster * 8 * kThreads;

int key_bits(uint32_t rows)                             // of the largest key, `rows`
{
    int bits = 1;
    while (bits < 32 && ((uint64_t)rows >> bits) != 0) ++bits;
    return bits;
}

template <typename ID>
cudaError_t sort_in_passes(const ID* ids, const SortArgs& s, uint2* spare, uint32_t* counts, cudaStream_t stream)
{
    const uint32_t blocks = (uint32_t)(((uint64_t)s.tokens + kTile - 1) / kTile);
    const int passes = (s.bits + 7) / 8;
    uint2 *out = passes % 2 ? s.sorted : spare, *other = passes % 2 ? spare : s.sorted;
    PassInput<ID> in = {ids, nullptr, s.tokens, s.rows};
    for (int shift = 0; shift < s.bits; shift += 8) {
        cudaError_t err = launch_pdl(count_kernel<ID>, blocks, kThreads, stream, in, shift, counts);
        if (err == cudaSuccess) err = launch_pdl(scan_kernel, 1, kBins, stream, counts, blocks, s.counter);
        if (err == cudaSuccess) err = launch_pdl(place_kernel<ID>, blocks, kThreads, stream, in, shift, counts, out);
        if (err != cudaSuccess) return err;
        in.ids = nullptr;
        in.pairs = out;
        uint2* t = out; out = other; other = t;
    }
    return cudaSuccess;
}

}  // namespace

uint64_t token_sort_words(uint64_t tokens)
{
    if (tokens <= kClusterTokens) return 0;
    return 2 * tokens + (tokens + kTile - 1) / kTile * kBins;
}

cudaError_t launch_token_sort(const TokenIds& ids, uint32_t rows, uint2* sorted, uint32_t* counter, uint32_t* scratch,
                              void* zero, uint64_t zero_bytes, cudaStream_t stream)
{
    SortArgs a = {ids.ptr, sorted, counter, zero, zero_bytes, (uint32_t)ids.count, rows, key_bits(rows), 1, 0};
    const bool one_launch = a.tokens <= kClusterTokens;
    uint32_t per_thread = 1;
    if (one_launch && a.tokens != 0) {
        // passes of equal digits; a CTA for each 2048 tokens, then more tokens to a CTA
        const int passes = (a.bits + kMaxDigitBits - 1) / kMaxDigitBits;
        a.digit_bits = (a.bits + passes - 1) / passes;
        a.ctas = 1;
        while (a.ctas < kMaxCluster && a.ctas * 2048u < a.tokens) a.ctas *= 2;
        per_thread = (a.tokens + a.ctas * kThreads - 1) / (a.ctas * kThreads);
    }
    if (one_launch || zero_bytes != 0) {
        int dev = 0, sms = 0;
        cudaError_t err = cudaGetDevice(&dev);
        if (err == cudaSuccess) err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        if (err != cudaSuccess) return err;
        // the CTAs that write zeros: 32 KB each at least, whole clusters of them, no more than fit beside the sort
        const unsigned size = a.ctas == 0 ? 1 : a.ctas;
        uint64_t extra = (zero_bytes + 32767) / 32768;
        const uint64_t room = (uint64_t)sms > size ? (uint64_t)sms - size : 1;
        if (extra > room) extra = room;
        extra = extra == 0 ? 0 : extra < size ? size : extra / size * size;
        const unsigned grid = a.ctas + (unsigned)extra;
        if (grid != 0) {
            err = ids.wide ? launch_by_size<int64_t>(a, per_thread, grid, stream) : launch_by_size<int32_t>(a, per_thread, grid, stream);
            if (err != cudaSuccess) return err;
        }
    }
    if (one_launch) return cudaSuccess;
    uint2* spare = reinterpret_cast<uint2*>(scratch);
    uint32_t* counts = scratch + 2 * (uint64_t)a.tokens;
    return ids.wide ? sort_in_passes(static_cast<const int64_t*>(ids.ptr), a, spare, counts, stream)
                    : sort_in_passes(static_cast<const int32_t*>(ids.ptr), a, spare, counts, stream);
}

}  // namespace mqg
