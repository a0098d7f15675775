// The gradient of a table of `rows` x `dim` from the gradient of the rows looked up in it:
//
//   grad[v] = fl((grad[v] +) scale * sum over t with ids[t] = v of dout[t])
//
// in fp32, tokens in ascending order.  Three launches:
//   1. the tokens are sorted by id (mqg_token_sort.cu), so that the tokens of a row are neighbours (a run) and no atomic is
//      needed: the order of every sum is fixed.  Unless the gradient is added to what is there, the same launch sets it to
//      zero;
//   2. the sorted tokens are cut into chunks of C; a thread takes V columns of a chunk and adds up its runs.  A run that
//      crosses chunks belongs to the chunk it begins in, which follows it, as long as it covers no chunk as a whole (less
//      than 2 C tokens); of a longer one every chunk leaves its part's sum in the workspace;
//   3. the parts of the long runs are added up in the order of the chunks.
#include "mqg_tma.cuh"
#include "mqg_token_sort.h"
#include "mqg_vector.cuh"

namespace mqg {
namespace {

constexpr int kThreads = 128;

struct GradArgs {
    const uint2* sorted;     // (row, token), rows ascending; the row `rows` = none
    const void* dout;
    void* grad;
    float* parts;            // [chunk][2][dim]: the sum of the long run that enters the chunk, and of the one that begins in it
    uint32_t* long_runs;     // how many there are, then the chunks that they begin in
    uint64_t dim;
    uint32_t tokens, rows, chunks;
    int chunk_bits;
    float scale;
};

__device__ __forceinline__ uint32_t row_at(const GradArgs& a, uint32_t i) { return __ldg(&a.sorted[i].x); }

template <int V> __device__ __forceinline__ float* part_at(const GradArgs& a, uint32_t chunk, bool begins, uint64_t col)
{
    return a.parts + ((uint64_t)chunk * 2 + (begins ? 1 : 0)) * a.dim + col;
}

// grad's row from the sum and, with ADD, what was there.
template <int DST, int V, bool ADD>
__device__ __forceinline__ void finish_row(typename Element<DST>::type* p, Packed<DST, V>& y, float scale, const float (&sum)[V])
{
#pragma unroll
    for (int e = 0; e < V; ++e) y.set(e, ADD ? __fadd_rn(y.get(e), __fmul_rn(scale, sum[e])) : __fmul_rn(scale, sum[e]));
    y.store(p);
}

template <int V> __device__ __forceinline__ void store_part(float* p, const float (&sum)[V])
{
    Packed<kF32, V> y;
#pragma unroll
    for (int e = 0; e < V; ++e) y.set(e, sum[e]);
    y.store(p);
}

// Threads: x = columns, V of them each; y = chunks.
template <int SRC, int DST, int V, bool ADD>
__global__ void __launch_bounds__(kThreads) grad_sum_kernel(const GradArgs a)
{
    constexpr int kAhead = ADD ? 4 : 8;                 // tokens whose loads are in flight together
    const uint64_t col = ((uint64_t)blockIdx.y * blockDim.x + threadIdx.x) * V;
    const uint32_t chunk = blockIdx.x * blockDim.y + threadIdx.y;
    grid_dependency_wait();
    if (col >= a.dim || chunk >= a.chunks) return;
    const uint32_t size = 1u << a.chunk_bits, first = chunk << a.chunk_bits, end = min(first + size, a.tokens);
    const uint32_t row0 = row_at(a, first), row1 = row_at(a, end - 1);
    if (row0 == a.rows) return;
    const bool enters = first != 0 && row_at(a, first - 1) == row0;
    const bool leaves = row1 != a.rows && end < a.tokens && row_at(a, end) == row1;
    // long: covers this chunk, the one before or the one behind as a whole
    const bool long_in = enters && (row0 == row1 || row_at(a, first - size) == row0);
    const bool long_out = leaves && (row0 == row1 || row_at(a, min(end + size, a.tokens) - 1) == row1);
    const uint32_t limit = leaves && !long_out ? min(end + size, a.tokens) - 1 : end;
    if (long_out && !(long_in && row0 == row1) && col == 0) a.long_runs[1 + atomicAdd(a.long_runs, 1u)] = chunk;

    const auto* dout = static_cast<const typename Element<SRC>::type*>(a.dout) + col;
    auto* grad = static_cast<typename Element<DST>::type*>(a.grad) + col;
    float sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = 0.0f;
    for (uint32_t p = first; p < limit; p += kAhead) {
        uint2 k[kAhead + 1];
#pragma unroll
        for (int u = 0; u <= kAhead; ++u) k[u] = p + u < a.tokens ? __ldg(a.sorted + p + u) : make_uint2(a.rows, 0);
        if (p >= end && k[0].x != row1) break;
        Packed<SRC, V> x[kAhead];
        Packed<DST, V> y[kAhead];
        bool used[kAhead], ends[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            // what stands before a short run's end belongs to the chunk before; what stands behind this chunk's to its run
            used[u] = p + u < limit && k[u].x != a.rows && (p + u < end || k[u].x == row1) && !(enters && !long_in && k[u].x == row0);
            ends[u] = used[u] && k[u + 1].x != k[u].x;
            if (used[u]) x[u].load(dout + (uint64_t)k[u].y * a.dim);
            if (ADD && ends[u] && !(long_in && k[u].x == row0)) y[u].load(grad + (uint64_t)k[u].x * a.dim);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (!used[u]) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] = __fadd_rn(sum[e], x[u].get(e));
            if (!ends[u]) continue;
            if (long_in && k[u].x == row0) store_part<V>(part_at<V>(a, chunk, false, col), sum);
            else finish_row<DST, V, ADD>(grad + (uint64_t)k[u].x * a.dim, y[u], a.scale, sum);
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] = 0.0f;
        }
    }
    if (long_out) store_part<V>(part_at<V>(a, chunk, !(long_in && row0 == row1), col), sum);
}

// The long runs: a CTA takes the columns of kThreads / kSplits vectors of one run after another, kSplits groups of threads
// equal shares of its parts.
constexpr int kSplits = 8, kColumns = kThreads / kSplits;

template <int DST, int V, bool ADD>
__global__ void __launch_bounds__(kThreads) grad_join_kernel(const GradArgs a, uint32_t column_tiles)
{
    __shared__ float share[kSplits][V][kColumns];
    grid_dependency_wait();
    const uint64_t items = (uint64_t)__ldcg(a.long_runs) * column_tiles;
    const uint32_t x = threadIdx.x % kColumns, s = threadIdx.x / kColumns, lane = threadIdx.x & 31;
    for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t begin = __ldcg(a.long_runs + 1 + item / column_tiles);
        const uint64_t col = ((uint64_t)(item % column_tiles) * kColumns + x) * V;
        const uint32_t row = row_at(a, ((begin + 1) << a.chunk_bits) - 1);
        uint32_t n = 1;                                 // chunks that the run has a part in
        for (bool more = true; more;) {
            const uint64_t next = ((uint64_t)(begin + n + lane)) << a.chunk_bits;
            const uint32_t on = __ballot_sync(0xFFFFFFFFu, next < a.tokens && row_at(a, (uint32_t)next) == row);
            n += on == 0xFFFFFFFFu ? 32 : __ffs(~on) - 1;
            more = on == 0xFFFFFFFFu;
        }
        const uint32_t per = (n + kSplits - 1) / kSplits, from = min(s * per, n), to = min(from + per, n);
        float sum[V];
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] = 0.0f;
        if (col < a.dim) {
#pragma unroll 8
            for (uint32_t i = from; i < to; ++i) {
                Packed<kF32, V> y;
                y.load(part_at<V>(a, begin + i, i == 0, col));
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] = __fadd_rn(sum[e], y.get(e));
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) share[s][e][x] = sum[e];
        __syncthreads();
        if (s == 0 && col < a.dim) {
#pragma unroll
            for (int t = 1; t < kSplits; ++t)
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] = __fadd_rn(sum[e], share[t][e][x]);
            auto* p = static_cast<typename Element<DST>::type*>(a.grad) + (uint64_t)row * a.dim + col;
            Packed<DST, V> y;
            if (ADD) y.load(p);
            finish_row<DST, V, ADD>(p, y, a.scale, sum);
        }
        __syncthreads();
    }
}

// ---- host ----
constexpr uint64_t round4(uint64_t words) { return (words + 3) & ~3ull; }

// Tokens of a chunk: as many as leave the sums' launch a few CTAs for each SM.
int chunk_bits_of(uint64_t tokens, uint64_t dim)
{
    int bits = 5;
    while (bits > 3 && ((tokens * dim) >> bits) < 1024 * 1024) --bits;
    return bits;
}

struct Layout {
    int chunk_bits;
    uint32_t chunks;
    uint64_t sorted, runs, scratch, parts, total;       // sizes in words
    Layout(uint64_t tokens, uint64_t dim)
    {
        chunk_bits = chunk_bits_of(tokens, dim);
        chunks = (uint32_t)((tokens + (1u << chunk_bits) - 1) >> chunk_bits);
        sorted = round4(2 * tokens);
        runs = round4(1 + (uint64_t)chunks);
        scratch = round4(token_sort_words(tokens));
        parts = 2 * (uint64_t)chunks * round4(dim);
        total = sorted + runs + scratch + parts;
    }
};

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

template <int SRC, int DST, int V, bool ADD> cudaError_t launch_sums(const GradArgs& a, cudaStream_t stream)
{
    const uint64_t cols = a.dim / V;
    unsigned bx = 1;
    while (bx < (unsigned)kThreads && bx < cols) bx *= 2;
    const unsigned by = kThreads / bx;
    const dim3 grid((a.chunks + by - 1) / by, (unsigned)((cols + bx - 1) / bx));
    cudaError_t err = launch_pdl_block(grad_sum_kernel<SRC, DST, V, ADD>, grid, dim3(bx, by), stream, a);
    if (err != cudaSuccess || a.chunks < 2) return err;
    const uint32_t tiles = (uint32_t)((cols + kColumns - 1) / kColumns);
    const uint64_t most = (uint64_t)(a.chunks - 1) * tiles;
    return launch_pdl(grad_join_kernel<DST, V, ADD>, (unsigned)(most < 592 ? most : 592), kThreads, stream, a, tiles);
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
    uint2* sorted = reinterpret_cast<uint2*>(workspace);
    uint32_t* runs = reinterpret_cast<uint32_t*>(workspace + lay.sorted);
    uint32_t* scratch = runs + lay.runs;
    const GradArgs a = {sorted, dout, grad, workspace + lay.sorted + lay.runs + lay.scratch, runs, dim, (uint32_t)ids.count,
                        (uint32_t)rows, lay.chunks, lay.chunk_bits, scale};
    const uint64_t zero_bytes = add ? 0 : rows * dim * (grad_dtype == kF32 ? 4 : 2);
    const cudaError_t err = launch_token_sort(ids, a.rows, sorted, runs, scratch, grad, zero_bytes, stream);
    if (err != cudaSuccess || a.chunks == 0) return err;
    if (dout_dtype == kF32)
        return grad_dtype == kF32 ? by_vector<kF32, kF32>(a, add, stream) : by_vector<kF32, kBf16>(a, add, stream);
    return grad_dtype == kF32 ? by_vector<kBf16, kF32>(a, add, stream) : by_vector<kBf16, kBf16>(a, add, stream);
}

}  // namespace mqg
