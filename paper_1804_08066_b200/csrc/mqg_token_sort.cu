// Token ids sorted by id, stably, with the tokens' positions: least significant digit first, up to ten bits to a pass.
//
// Up to 2048 tokens one CTA sorts, in shared memory, by digits of at most six bits: a pass costs little more than ranking.
// (2048 tokens of 16-bit ids: 8.5 us a launch; 4096: 13.0 in one CTA, 8.6 in a cluster.)
// Up to 131,072 a thread-block cluster of up to 16 CTAs does in one launch (fewer where the device, or the part of one, holds no
// cluster of 16: 8192 to a CTA), by digits of up to ten bits, since every pass has two cluster
// barriers.  In both a thread takes K pairs (key, token) of the order so far, a warp 32 K consecutive ones; it ranks them by
// ballots, the warps' digit counts are added up in shared memory (and the CTAs' through distributed shared memory), and every
// pair goes to its place: in shared memory, or, for the cluster, in memory, where the next pass reads it from L2.  (Stores to
// the shared memory of the CTA that holds the place took 10,000 cycles for 8192 pairs to a CTA, stores to memory 2,900.)  What
// bounds both is latency, and most SMs are idle meanwhile: further CTAs set a first part of the gradient to zero.
//
// More tokens take three launches a pass: count, scan, place.
#include <atomic>

#include "mqg_token_sort.cuh"

namespace mqg {
namespace {

// ---- one launch ----
constexpr int kThreads = kSortThreads, kWarps = kSortWarps;
constexpr unsigned kMaxCluster = 16;

struct SortArgs {
    const void* ids;
    uint2* sorted;
    uint2* spare;            // of the passes but the last
    uint32_t* counter;       // set to zero for the kernels that follow
    uint32_t tokens, rows;
    int bits, digit_bits;
    unsigned ctas;           // one cluster
    char* zero;              // what the CTAs behind them set to zero
    uint64_t zero_bytes;
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
__device__ __forceinline__ uint32_t peer_load(const uint32_t* p, uint32_t rank)
{
    uint32_t at, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at));
    return v;
}

__host__ __device__ constexpr size_t sort_smem(int bins)
{
    return (size_t)bins * (kWarps * sizeof(uint16_t) + 2 * sizeof(uint32_t)) + kWarps * sizeof(uint32_t);
}

// The sort leaves most SMs idle: the CTAs behind its own set memory to zero meanwhile, side by side, or, where it is little and
// there are no such, the sort's own before they begin.  Returns whether this CTA is one of those behind.
__device__ __forceinline__ bool zero_beside(const SortArgs& a)
{
    const bool apart = blockIdx.x >= a.ctas;
    if (!apart && gridDim.x != a.ctas) return false;
    const uint32_t index = apart ? blockIdx.x - a.ctas : blockIdx.x, count = apart ? gridDim.x - a.ctas : a.ctas;
    const uint64_t to_boundary = (16 - (reinterpret_cast<uintptr_t>(a.zero) & 15)) & 15;
    const uint64_t head = min(to_boundary, a.zero_bytes), nvec = (a.zero_bytes - head) / 16, behind = head + nvec * 16;
    uint4* to = reinterpret_cast<uint4*>(a.zero + head);
#pragma unroll 4
    for (uint64_t i = (uint64_t)index * kThreads + threadIdx.x; i < nvec; i += (uint64_t)count * kThreads) to[i] = make_uint4(0, 0, 0, 0);
    if (index == 0) {
        if (threadIdx.x < head) a.zero[threadIdx.x] = 0;
        if (threadIdx.x < a.zero_bytes - behind) a.zero[behind + threadIdx.x] = 0;
    }
    return apart;
}

// ---- one CTA ----
template <typename ID, int K>
__global__ void __launch_bounds__(kThreads, 1) sort_small_kernel(const SortArgs a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ SmallSort s;
    uint2* pairs = reinterpret_cast<uint2*>(smem);
    grid_dependency_wait();
    if (zero_beside(a)) return;
    if (threadIdx.x == 0) *a.counter = 0;
    uint2 pair[K];
    const uint32_t held = load_pairs<ID, K>(static_cast<const ID*>(a.ids), a.tokens, a.rows, (threadIdx.x >> 5) * (32 * K) + (threadIdx.x & 31), pair);
    sort_in_cta<K>(pair, held, a.tokens, a.bits, s, pairs);
    for (uint32_t i = threadIdx.x; i < a.tokens; i += kThreads) a.sorted[i] = pairs[i];
}

// ---- one cluster ----
template <typename ID, int K>
__global__ void __launch_bounds__(kThreads, 1) sort_cluster_kernel(const SortArgs a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    const int bins = 1 << a.digit_bits;
    uint16_t* warp_count = reinterpret_cast<uint16_t*>(smem);                        // [warp][digit]
    uint32_t* cta_count = reinterpret_cast<uint32_t*>(warp_count + kWarps * bins);   // [digit]
    uint32_t* place = cta_count + bins;                                              // [digit]
    uint32_t* warp_total = place + bins;                                             // [warp]
    const uint32_t d = threadIdx.x, lane = threadIdx.x & 31, w = threadIdx.x >> 5;

    grid_dependency_wait();
    if (zero_beside(a)) return;                         // another cluster, whole
    const uint32_t rank = cluster_rank();
    if (rank == 0 && threadIdx.x == 0) *a.counter = 0;
    const uint32_t first = rank * (K * kThreads) + w * (32 * K) + lane;
    uint16_t* mine = warp_count + w * bins;
    const int passes = (a.bits + a.digit_bits - 1) / a.digit_bits;
    uint2* to = passes & 1 ? a.sorted : a.spare;
    uint2* from = passes & 1 ? a.spare : a.sorted;
    uint2 pair[K];
    const uint32_t held = load_pairs<ID, K>(static_cast<const ID*>(a.ids), a.tokens, a.rows, first, pair);
    for (int shift = 0; shift < a.bits; shift += a.digit_bits) {
        if (shift != 0) {
#pragma unroll
            for (int r = 0; r < K; ++r)
                if ((held >> r) & 1u) pair[r] = __ldcg(from + first + r * 32);
        }
        for (int i = lane; i < bins / 2; i += 32) reinterpret_cast<uint32_t*>(mine)[i] = 0;
        __syncwarp();
        uint32_t rank_in_warp[K];
        rank_pairs<K>(pair, held, shift, a.digit_bits, mine, rank_in_warp);
        __syncthreads();
        uint32_t earlier = 0, total = 0;                // keys of this digit: of the CTAs before, of all
        if (d < (uint32_t)bins) {
#pragma unroll 16
            for (int v = 0; v < kWarps; ++v) {
                const uint32_t c = warp_count[v * bins + d];
                warp_count[v * bins + d] = (uint16_t)total;
                total += c;
            }
            cta_count[d] = total;
        }
        cluster_sync();                                 // the counts are there
        if (d < (uint32_t)bins) {
            total = 0;
#pragma unroll
            for (uint32_t half = 0; half < kMaxCluster; half += 8) {
                if (half >= a.ctas) break;
                uint32_t c[8];
#pragma unroll
                for (uint32_t r = 0; r < 8; ++r) c[r] = half + r < a.ctas ? peer_load(cta_count + d, half + r) : 0;
#pragma unroll
                for (uint32_t r = 0; r < 8; ++r) {
                    earlier += half + r < rank ? c[r] : 0;
                    total += c[r];
                }
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
            const uint32_t digit = (pair[r].x >> shift) & (bins - 1);
            if ((held >> r) & 1u) to[place[digit] + mine[digit] + rank_in_warp[r]] = pair[r];
        }
        cluster_sync();                                 // the pairs are there, and no CTA's counts go before they were read
        uint2* t = to; to = from; from = t;
    }
}

// ---- host: one launch ----
// Clusters of so many CTAs beside the sort's, at most `room`, that set memory to zero: none where it is up to 16 KB to a CTA.
unsigned zero_clusters(const SortArgs& a, unsigned room)
{
    const uint64_t share = 16384 * a.ctas, want = a.zero_bytes <= share ? 0 : (a.zero_bytes + share - 1) / share;
    return want < room ? (unsigned)want : room;
}

// The launch of one cluster of `ctas` CTAs; the attributes live as long as this.
struct ClusterConfig {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    ClusterConfig(unsigned ctas, size_t smem, cudaStream_t stream)
    {
        cfg.gridDim = dim3(ctas);
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = stream;
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = ctas;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
    }
};

// How many clusters of so many CTAs of a kernel the current device runs at once; 0: it cannot hold one.
template <typename ID, int K> cudaError_t clusters_at_once(int dev, unsigned ctas, int* clusters)
{
    static std::atomic<int> known[64][5];               // by device and log2(ctas): one more than the answer; 0: not asked yet
    std::atomic<int>& k = known[dev][31 - __builtin_clz(ctas)];
    int n = k.load(std::memory_order_relaxed);
    if (n == 0) {
        cudaError_t err = cudaFuncSetAttribute(sort_cluster_kernel<ID, K>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)sort_smem(1 << kMaxDigitBits));
        if (err == cudaSuccess)                         // clusters of 16 CTAs
            err = cudaFuncSetAttribute(sort_cluster_kernel<ID, K>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (err != cudaSuccess) return err;
        ClusterConfig c(ctas, sort_smem(1 << kMaxDigitBits), nullptr);
        c.cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&n, sort_cluster_kernel<ID, K>, &c.cfg) != cudaSuccess) {
            (void)cudaGetLastError();                   // a size that the device does not know
            n = 0;
        }
        k.store(++n, std::memory_order_relaxed);
    }
    *clusters = n - 1;
    return cudaSuccess;
}

cudaError_t current_device(int* dev)
{
    const cudaError_t err = cudaGetDevice(dev);
    if (err != cudaSuccess) return err;
    return *dev >= 0 && *dev < 64 ? cudaSuccess : cudaErrorInvalidDevice;
}

// The CTAs of the largest cluster that the current device holds, or 1: a part of a device may hold none of 16.
std::atomic<unsigned> g_most_ctas{kMaxCluster};
cudaError_t largest_cluster(unsigned* ctas)
{
    int dev, clusters = 0;
    cudaError_t err = current_device(&dev);
    *ctas = 2 * g_most_ctas.load(std::memory_order_relaxed);
    while (err == cudaSuccess && clusters == 0 && (*ctas /= 2) > 1) err = clusters_at_once<int64_t, 8>(dev, *ctas, &clusters);
    return err;
}

template <typename ID, int K> cudaError_t launch_cluster(const SortArgs& a, cudaStream_t stream)
{
    int dev, clusters;
    cudaError_t err = current_device(&dev);
    if (err == cudaSuccess) err = clusters_at_once<ID, K>(dev, a.ctas, &clusters);
    if (err != cudaSuccess) return err;
    ClusterConfig c(a.ctas, sort_smem(1 << a.digit_bits), stream);
    c.cfg.gridDim.x += zero_clusters(a, clusters > 1 ? clusters - 1 : 1) * a.ctas;
    return cudaLaunchKernelEx(&c.cfg, sort_cluster_kernel<ID, K>, a);
}

template <typename ID, int K> cudaError_t launch_small(const SortArgs& a, cudaStream_t stream)
{
    static std::atomic<bool> ready[64];                 // per device (zero-initialised)
    constexpr int kSmem = K * kThreads * (int)sizeof(uint2);
    int dev;
    cudaError_t err = current_device(&dev);
    if (err != cudaSuccess) return err;
    if (!ready[dev].load(std::memory_order_relaxed)) {
        err = cudaFuncSetAttribute(sort_small_kernel<ID, K>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (err != cudaSuccess) return err;
        ready[dev].store(true, std::memory_order_relaxed);
    }
    return launch_pdl_smem(sort_small_kernel<ID, K>, 1 + zero_clusters(a, 147), kThreads, kSmem, stream, a);
}

template <typename ID> cudaError_t launch_by_size(const SortArgs& a, uint32_t per_thread, cudaStream_t stream)
{
    if (a.ctas == 1)
        return per_thread <= 1 ? launch_small<ID, 1>(a, stream)
                               : launch_small<ID, 2>(a, stream);
    return per_thread <= 1 ? launch_cluster<ID, 1>(a, stream)
           : per_thread <= 2 ? launch_cluster<ID, 2>(a, stream)
           : per_thread <= 4 ? launch_cluster<ID, 4>(a, stream)
                             : launch_cluster<ID, 8>(a, stream);
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
constexpr uint32_t kTokensPerCta = 8 * kThreads, kSmallTokens = 2 * kThreads;

template <typename ID>
cudaError_t sort_in_passes(const ID* ids, const SortArgs& s, uint32_t* counts, cudaStream_t stream)
{
    const uint32_t blocks = (uint32_t)(((uint64_t)s.tokens + kTile - 1) / kTile);
    const int passes = (s.bits + 7) / 8;
    uint2 *out = passes % 2 ? s.sorted : s.spare, *other = passes % 2 ? s.spare : s.sorted;
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

int token_key_bits(uint32_t rows)
{
    int bits = 1;
    while (bits < 32 && ((uint64_t)rows >> bits) != 0) ++bits;
    return bits;
}

uint64_t token_sort_words(uint64_t tokens)
{
    // (counts of passes for what a cluster may sort, too: which clusters there are is the device's)
    return 2 * tokens + (tokens > kSmallTokens ? (tokens + kTile - 1) / kTile * kBins : 0);
}

void set_token_sort_cluster(unsigned most) { g_most_ctas.store(most, std::memory_order_relaxed); }

// What is set to zero beside the sort, by the SMs that it leaves idle, in about the time it takes: of 50,000 rows of 4 KB, 16,384
// tokens, 56 MB (49.8 us in all, with 32 MB 51.2, with 80 51.7); of 100,000 rows of 1 KB, 2048 tokens (one CTA sorts), 24.3 us,
// with 32 MB 26.9, with 96 25.9.
constexpr uint64_t kZeroBesideBytes = 56ull << 20;

cudaError_t launch_token_sort(const TokenIds& ids, uint32_t rows, uint2* sorted, uint32_t* counter, uint32_t* scratch, void* table,
                              uint64_t row_bytes, uint32_t* zeroed, cudaStream_t stream)
{
    SortArgs a = {ids.ptr, sorted, reinterpret_cast<uint2*>(scratch), counter, (uint32_t)ids.count, rows, token_key_bits(rows), 1, 1,
                  static_cast<char*>(table), 0};
    *zeroed = 0;
    unsigned most_ctas = 1;
    if (a.tokens > kSmallTokens) {
        const cudaError_t err = largest_cluster(&most_ctas);
        if (err != cudaSuccess) return err;
    }
    if (a.tokens > (most_ctas == 1 ? kSmallTokens : most_ctas * kTokensPerCta)) {
        uint32_t* counts = scratch + 2 * ids.count;
        return ids.wide ? sort_in_passes(static_cast<const int64_t*>(ids.ptr), a, counts, stream)
                        : sort_in_passes(static_cast<const int32_t*>(ids.ptr), a, counts, stream);
    }
    // the cluster: passes of equal digits; a CTA for each 1024 tokens, then more tokens to a thread (4096 tokens: 8.6 us a
    // launch with four CTAs, 10.5 with two)
    const int passes = (a.bits + kMaxDigitBits - 1) / kMaxDigitBits;
    a.digit_bits = (a.bits + passes - 1) / passes;
    while (a.tokens > kSmallTokens && a.ctas < most_ctas && a.ctas * kThreads < a.tokens) a.ctas *= 2;
    const uint32_t per_thread = (a.tokens + a.ctas * kThreads - 1) / (a.ctas * kThreads);
    if (table != nullptr) {
        const uint64_t fit = kZeroBesideBytes / row_bytes;
        *zeroed = fit < rows ? (uint32_t)fit : rows;
        a.zero_bytes = *zeroed * row_bytes;
    }
    return ids.wide ? launch_by_size<int64_t>(a, per_thread, stream) : launch_by_size<int32_t>(a, per_thread, stream);
}

}  // namespace mqg
