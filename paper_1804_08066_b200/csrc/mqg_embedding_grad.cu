// The gradient of a table of `rows` x `dim` from the gradient of the rows looked up in it:
//
//   grad[v] = fl((grad[v] +) scale * sum over t with ids[t] = v of dout[t])
//
// in fp32, tokens in ascending order.  Three steps:
//   1. the tokens are sorted by id (stable, least significant digit first; ids outside 0..rows-1 go behind all others), so
//      that the tokens of one row are neighbours and no atomic is needed: the order of every sum is fixed;
//   2. the sorted tokens are cut into chunks of kChunk; a thread takes V columns of a chunk and adds up its runs of equal
//      ids.  A run inside the chunk goes to its row; one that crosses the chunk's edge leaves a partial sum;
//   3. the partial sums of such a run are added up in the order of the chunks.
// Rows that no token uses are set to zero unless the gradient is added to what is there.
#include "mqg_tma.cuh"
#include "mqg_training.h"
#include "mqg_vector.cuh"

namespace mqg {
namespace {

// ---- the sort ----
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kKeysPerThread = 8, kSortTile = kSortThreads * kKeysPerThread;
constexpr int kDigitBits = 8, kBins = 1 << kDigitBits;

// An id as the key it is sorted by.
template <typename ID> __device__ __forceinline__ uint32_t key_of(ID id, uint32_t rows)
{
    return id >= 0 && (uint64_t)id < rows ? (uint32_t)id : rows;
}

// Where a pass reads its keys and tokens: the caller's ids (tokens = positions), or the pass before.
template <typename ID> struct SortInput {
    const ID* ids;
    const uint2* pairs;      // (key, token); used where ids is null
    uint32_t count, rows;
    __device__ __forceinline__ uint2 get(uint32_t i) const
    {
        return ids != nullptr ? make_uint2(key_of(__ldg(ids + i), rows), i) : __ldcg(pairs + i);
    }
};

// Ranks the tile's keys by digit, stably: rank[r] = how many keys of the warp before this one have its digit;
// warp_count[w][d] = how many of warp w's keys have digit d.  A warp takes 256 consecutive keys, 32 at a time.
template <typename ID>
__device__ __forceinline__ void rank_tile(const SortInput<ID>& in, int shift, uint16_t (*warp_count)[kBins],
                                          uint2 (&pair)[kKeysPerThread], uint32_t (&rank)[kKeysPerThread])
{
    const uint32_t lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    for (int d = lane; d < kBins; d += 32) warp_count[w][d] = 0;
    const uint32_t first = blockIdx.x * (uint32_t)kSortTile + w * (32 * kKeysPerThread) + lane;
#pragma unroll
    for (int r = 0; r < kKeysPerThread; ++r)
        pair[r] = first + r * 32 < in.count ? in.get(first + r * 32) : make_uint2(0, 0);
    __syncwarp();
#pragma unroll
    for (int r = 0; r < kKeysPerThread; ++r) {
        const bool held = first + r * 32 < in.count;
        const uint32_t d = held ? (pair[r].x >> shift) & (kBins - 1) : kBins;
        const uint32_t same = __match_any_sync(0xFFFFFFFFu, d);
        const uint32_t before = held ? warp_count[w][d] : 0;
        __syncwarp();
        if (held && (same >> lane) == 1u) warp_count[w][d] = (uint16_t)(before + __popc(same));
        __syncwarp();
        rank[r] = before + __popc(same & ((1u << lane) - 1));
    }
}

template <typename ID>
__global__ void __launch_bounds__(kSortThreads)
sort_count_kernel(const SortInput<ID> in, int shift, uint32_t* __restrict__ counts)
{
    __shared__ uint16_t warp_count[kSortWarps][kBins];
    uint2 pair[kKeysPerThread];
    uint32_t rank[kKeysPerThread];
    grid_dependency_wait();
    rank_tile(in, shift, warp_count, pair, rank);
    __syncthreads();
    if (threadIdx.x < kBins) {
        uint32_t sum = 0;
        for (int w = 0; w < kSortWarps; ++w) sum += warp_count[w][threadIdx.x];
        counts[(uint64_t)blockIdx.x * kBins + threadIdx.x] = sum;
    }
}

// counts[block][digit] becomes the first place of the block's keys of that digit.
__global__ void __launch_bounds__(kBins)
sort_scan_kernel(uint32_t* __restrict__ counts, uint32_t blocks)
{
    __shared__ uint32_t total[kBins];
    const uint32_t d = threadIdx.x;
    grid_dependency_wait();
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
__global__ void __launch_bounds__(kSortThreads)
sort_place_kernel(const SortInput<ID> in, int shift, const uint32_t* __restrict__ counts, uint2* __restrict__ out)
{
    __shared__ uint16_t warp_count[kSortWarps][kBins];
    __shared__ uint32_t warp_first[kSortWarps][kBins];
    uint2 pair[kKeysPerThread];
    uint32_t rank[kKeysPerThread];
    grid_dependency_wait();
    rank_tile(in, shift, warp_count, pair, rank);
    __syncthreads();
    if (threadIdx.x < kBins) {
        uint32_t at = __ldcg(counts + (uint64_t)blockIdx.x * kBins + threadIdx.x);
        for (int w = 0; w < kSortWarps; ++w) {
            warp_first[w][threadIdx.x] = at;
            at += warp_count[w][threadIdx.x];
        }
    }
    __syncthreads();
    const uint32_t lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const uint32_t first = blockIdx.x * (uint32_t)kSortTile + w * (32 * kKeysPerThread) + lane;
#pragma unroll
    for (int r = 0; r < kKeysPerThread; ++r)
        if (first + r * 32 < in.count) out[warp_first[w][(pair[r].x >> shift) & (kBins - 1)] + rank[r]] = pair[r];
}

// ---- the sums ----
constexpr int kChunk = 32;                              // sorted tokens of one thread
constexpr int kSumThreads = 128;
constexpr int kAhead = 8;                               // rows whose loads are in flight together

struct GradArgs {
    const uint2* sorted;     // (row, token), rows ascending; a row of `rows` = none
    const void* dout;
    void* grad;
    float* partial;          // [chunk][2][dim]: the sum of the run that enters the chunk, and of the one that begins there
                             // and leaves it
    uint64_t dim;
    uint32_t tokens, rows, chunks;
    float scale;
};

template <int DST, int V, bool ADD>
__device__ __forceinline__ void write_row(const GradArgs& a, uint32_t row, uint64_t col, const float (&sum)[V])
{
    auto* p = static_cast<typename Element<DST>::type*>(a.grad) + (uint64_t)row * a.dim + col;
    Packed<DST, V> y;
    if (ADD) y.load(p);
#pragma unroll
    for (int e = 0; e < V; ++e) y.set(e, ADD ? __fadd_rn(y.get(e), __fmul_rn(a.scale, sum[e])) : __fmul_rn(a.scale, sum[e]));
    y.store(p);
}

template <int V> __device__ __forceinline__ float* partial_at(const GradArgs& a, uint32_t chunk, int leaves, uint64_t col)
{
    return a.partial + ((uint64_t)chunk * 2 + leaves) * a.dim + col;
}

// Threads: x = columns, V of them each; y = chunks.
template <int SRC, int DST, int V, bool ADD>
__global__ void __launch_bounds__(kSumThreads) grad_sum_kernel(const GradArgs a)
{
    const uint64_t col = ((uint64_t)blockIdx.y * blockDim.x + threadIdx.x) * V;
    const uint32_t chunk = blockIdx.x * blockDim.y + threadIdx.y;
    grid_dependency_wait();
    if (col >= a.dim || chunk >= a.chunks) return;
    const uint32_t first = chunk * kChunk, last = min(first + kChunk, a.tokens);
    uint32_t row = __ldcg(&a.sorted[first]).x;
    if (row == a.rows) return;
    bool enters = first > 0 && __ldcg(&a.sorted[first - 1]).x == row;
    float sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = 0.0f;
    const auto* dout = static_cast<const typename Element<SRC>::type*>(a.dout) + col;
    for (uint32_t p = first; p < last && row != a.rows; p += kAhead) {
        uint2 k[kAhead];
        Packed<SRC, V> x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) k[u] = p + u < last ? __ldcg(&a.sorted[p + u]) : make_uint2(row, ~0u);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (p + u < last && k[u].x != a.rows) x[u].load(dout + (uint64_t)k[u].y * a.dim);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (p + u >= last || row == a.rows) break;
            if (k[u].x != row) {
                if (enters) {
#pragma unroll
                    for (int e = 0; e < V; ++e) partial_at<V>(a, chunk, 0, col)[e] = sum[e];
                } else {
                    write_row<DST, V, ADD>(a, row, col, sum);
                }
                row = k[u].x;
                enters = false;
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] = 0.0f;
                if (row == a.rows) break;
            }
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] = __fadd_rn(sum[e], x[u].get(e));
        }
    }
    if (row == a.rows) return;
    const bool leaves = last < a.tokens && __ldcg(&a.sorted[last]).x == row;
    if (enters || leaves) {
#pragma unroll
        for (int e = 0; e < V; ++e) partial_at<V>(a, chunk, enters ? 0 : 1, col)[e] = sum[e];
    } else {
        write_row<DST, V, ADD>(a, row, col, sum);
    }
}

// The rows whose runs cross chunks: by the chunk where the run begins.
template <int DST, int V, bool ADD>
__global__ void __launch_bounds__(kSumThreads) grad_join_kernel(const GradArgs a)
{
    const uint64_t col = ((uint64_t)blockIdx.y * blockDim.x + threadIdx.x) * V;
    uint32_t chunk = blockIdx.x * blockDim.y + threadIdx.y;
    grid_dependency_wait();
    if (col >= a.dim || chunk + 1 >= a.chunks) return;
    const uint32_t first = chunk * kChunk, end = first + kChunk;
    const uint32_t row = __ldcg(&a.sorted[end - 1]).x;
    if (row == a.rows || __ldcg(&a.sorted[end]).x != row) return;                     // nothing leaves the chunk
    if (first > 0 && __ldcg(&a.sorted[first - 1]).x == row) return;                   // it began before
    float sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = __ldcg(partial_at<V>(a, chunk, 1, col) + e);
    do {
        ++chunk;
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] = __fadd_rn(sum[e], __ldcg(partial_at<V>(a, chunk, 0, col) + e));
    } while (chunk + 1 < a.chunks && __ldcg(&a.sorted[(chunk + 1) * kChunk]).x == row);
    write_row<DST, V, ADD>(a, row, col, sum);
}

// Zeros in the rows that no token uses: 32 rows for each block, whose first warp looks each up among the sorted tokens.
template <int DST, int V>
__global__ void __launch_bounds__(kSumThreads) grad_zero_kernel(const GradArgs a)
{
    __shared__ uint32_t used;
    const uint32_t row0 = blockIdx.x * 32u, rows = min(32u, a.rows - row0);
    grid_dependency_wait();
    if (threadIdx.x < 32) {
        const uint32_t row = row0 + threadIdx.x;
        uint32_t lo = 0, hi = a.tokens;                 // the first sorted token whose row is not below
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (__ldcg(&a.sorted[mid]).x < row) lo = mid + 1; else hi = mid;
        }
        const uint32_t u = __ballot_sync(0xFFFFFFFFu, lo < a.tokens && __ldcg(&a.sorted[lo]).x == row);
        if (threadIdx.x == 0) used = u;
    }
    __syncthreads();
    Packed<DST, V> zero;
#pragma unroll
    for (int e = 0; e < V; ++e) zero.set(e, 0.0f);
    auto* p = static_cast<typename Element<DST>::type*>(a.grad) + (uint64_t)row0 * a.dim;
    for (uint32_t r = 0; r < rows; ++r)
        if (!((used >> r) & 1u))
            for (uint64_t c = (uint64_t)threadIdx.x * V; c < a.dim; c += kSumThreads * V) zero.store(p + r * a.dim + c);
}

// ---- host ----
constexpr uint64_t round4(uint64_t words) { return (words + 3) & ~3ull; }

template <typename... KArgs, typename... Args>
cudaError_t launch_pdl_block(void (*kernel)(KArgs...), dim3 grid, dim3 block, cudaStream_t stream, Args&&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

struct Layout {
    uint32_t chunks, sort_blocks;
    uint64_t pairs, counts, partial, total;             // sizes in words
    Layout(uint64_t tokens, uint64_t dim)
    {
        chunks = (uint32_t)((tokens + kChunk - 1) / kChunk);
        sort_blocks = (uint32_t)((tokens + kSortTile - 1) / kSortTile);
        pairs = round4(2 * tokens);
        counts = round4((uint64_t)sort_blocks * kBins);
        partial = 2 * (uint64_t)chunks * dim;
        total = 2 * pairs + counts + partial;
    }
};

template <typename ID>
cudaError_t sort_tokens(const ID* ids, uint32_t tokens, uint32_t rows, uint2* a, uint2* b, uint32_t* counts, const Layout& lay,
                        cudaStream_t stream, const uint2** sorted)
{
    int bits = 1;
    while (bits < 32 && ((uint64_t)rows >> bits) != 0) ++bits;                        // of the largest key, `rows`
    SortInput<ID> in = {ids, nullptr, tokens, rows};
    for (int shift = 0; shift < bits; shift += kDigitBits) {
        cudaError_t err = launch_pdl(sort_count_kernel<ID>, lay.sort_blocks, kSortThreads, stream, in, shift, counts);
        if (err == cudaSuccess) err = launch_pdl(sort_scan_kernel, 1, kBins, stream, counts, lay.sort_blocks);
        if (err == cudaSuccess) err = launch_pdl(sort_place_kernel<ID>, lay.sort_blocks, kSortThreads, stream, in, shift, counts, a);
        if (err != cudaSuccess) return err;
        in.ids = nullptr;
        in.pairs = a;
        *sorted = a;
        uint2* t = a; a = b; b = t;
    }
    return cudaSuccess;
}

template <int SRC, int DST, int V, bool ADD> cudaError_t launch_sums(const GradArgs& a, cudaStream_t stream)
{
    if (!ADD) {
        const cudaError_t err = launch_pdl(grad_zero_kernel<DST, V>, (a.rows + 31) / 32, kSumThreads, stream, a);
        if (err != cudaSuccess) return err;
    }
    if (a.chunks == 0) return cudaSuccess;
    const uint64_t cols = a.dim / V;
    unsigned bx = 1;
    while (bx < (unsigned)kSumThreads && bx < cols) bx *= 2;
    const unsigned by = kSumThreads / bx;
    const dim3 grid((a.chunks + by - 1) / by, (unsigned)((cols + bx - 1) / bx));
    cudaError_t err = launch_pdl_block(grad_sum_kernel<SRC, DST, V, ADD>, grid, dim3(bx, by), stream, a);
    if (err == cudaSuccess && a.chunks > 1) err = launch_pdl_block(grad_join_kernel<DST, V, ADD>, grid, dim3(bx, by), stream, a);
    return err;
}

template <int SRC, int DST, int V> cudaError_t by_add(const GradArgs& a, bool add, cudaStream_t stream)
{
    return add ? launch_sums<SRC, DST, V, true>(a, stream) : launch_sums<SRC, DST, V, false>(a, stream);
}

template <int SRC, int DST> cudaError_t by_vector(const GradArgs& a, bool add, cudaStream_t stream)
{
    constexpr int most = SRC == kF32 && DST == kF32 ? 4 : 8;
    switch (row_vector(most, a.dim, a.dout, kElemBytes<SRC>, a.grad, kElemBytes<DST>)) {
        case 8: if constexpr (most == 8) return by_add<SRC, DST, 8>(a, add, stream);
        case 4: return by_add<SRC, DST, 4>(a, add, stream);
        case 2: return by_add<SRC, DST, 2>(a, add, stream);
    }
    return by_add<SRC, DST, 1>(a, add, stream);
}

}  // namespace

size_t embedding_workspace_floats(uint64_t tokens, uint64_t rows, uint64_t dim)
{
    return tokens == 0 || rows == 0 || dim == 0 ? 0 : (size_t)Layout(tokens, dim).total;
}

cudaError_t launch_embedding_grad(const void* dout, int dout_dtype, const TokenIds& ids, uint64_t rows, uint64_t dim,
                                  float scale, void* grad, int grad_dtype, bool add, float* workspace, cudaStream_t stream)
{
    const Layout lay(ids.count, dim);
    const uint32_t tokens = (uint32_t)ids.count;
    uint2* first = reinterpret_cast<uint2*>(workspace);
    uint2* second = reinterpret_cast<uint2*>(workspace + lay.pairs);
    uint32_t* counts = reinterpret_cast<uint32_t*>(workspace + 2 * lay.pairs);
    GradArgs a = {nullptr, dout, grad, workspace + 2 * lay.pairs + lay.counts, dim, tokens, (uint32_t)rows, lay.chunks, scale};
    cudaError_t err = cudaSuccess;
    if (tokens != 0)
        err = ids.wide ? sort_tokens(static_cast<const int64_t*>(ids.ptr), tokens, a.rows, first, second, counts, lay, stream, &a.sorted)
                       : sort_tokens(static_cast<const int32_t*>(ids.ptr), tokens, a.rows, first, second, counts, lay, stream, &a.sorted);
    if (err != cudaSuccess) return err;
    if (dout_dtype == kF32)
        return grad_dtype == kF32 ? by_vector<kF32, kF32>(a, add, stream) : by_vector<kF32, kBf16>(a, add, stream);
    return grad_dtype == kF32 ? by_vector<kBf16, kF32>(a, add, stream) : by_vector<kBf16, kBf16>(a, add, stream);
}

}  // namespace mqg
