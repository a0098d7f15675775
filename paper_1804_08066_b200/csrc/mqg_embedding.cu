// Rows of a table for a batch of token ids:  out[t] = fl(scale * table[ids[t]]), a row of zeros for an id outside 0..rows-1.
//
// Bound by memory: the rows that are used are read, the output is written.  A thread takes words of V elements, 16 bytes of the
// wider type, so that every access of a warp covers whole sectors, and eight of them so that their dependent loads (id, then
// row) overlap.
#include "mqg_tma.cuh"
#include "mqg_training.h"
#include "mqg_vector.cuh"

namespace mqg {
namespace {

constexpr int kThreads = 256;
constexpr int kVectors = 8;                             // of each thread

struct LookupArgs {
    const void* table;
    const void* ids;
    void* out;
    uint64_t rows, dim, tokens;
    float scale;
};

template <int SRC, int DST, int V, typename ID>
__global__ void __launch_bounds__(kThreads) embedding_kernel(const LookupArgs a)
{
    const uint32_t row_vectors = (uint32_t)(a.dim / V);
    const uint64_t n = a.tokens * row_vectors, first = (uint64_t)blockIdx.x * (kThreads * kVectors);
    const uint64_t token0 = first / row_vectors;
    const uint32_t col0 = (uint32_t)(first - token0 * row_vectors);
    grid_dependency_wait();
    uint64_t at[kVectors], from[kVectors];
#pragma unroll
    for (int k = 0; k < kVectors; ++k) {
        const uint32_t local = col0 + threadIdx.x + k * kThreads, over = local / row_vectors;
        const uint32_t col = local - over * row_vectors;
        const uint64_t token = token0 + over;
        at[k] = first + threadIdx.x + k * kThreads;
        from[k] = ~0ull;
        if (at[k] < n) {
            const int64_t id = (int64_t)__ldg(static_cast<const ID*>(a.ids) + token);
            if (id >= 0 && (uint64_t)id < a.rows) from[k] = (uint64_t)id * row_vectors + col;
        }
    }
    Packed<SRC, V> x[kVectors];
#pragma unroll
    for (int k = 0; k < kVectors; ++k)
        if (from[k] != ~0ull) x[k].load(static_cast<const typename Element<SRC>::type*>(a.table) + from[k] * V);
#pragma unroll
    for (int k = 0; k < kVectors; ++k) {
        if (at[k] >= n) continue;
        Packed<DST, V> y;
#pragma unroll
        for (int e = 0; e < V; ++e) y.set(e, from[k] != ~0ull ? a.scale * x[k].get(e) : 0.0f);
        y.store(static_cast<typename Element<DST>::type*>(a.out) + at[k] * V);
    }
}

// The same where rows start anywhere: the output, a row of rows without gaps, is written by words of W elements on their
// boundaries, and a word's elements are put together from the two words of the table that hold them.  A word that crosses into
// the next row (there is none longer than a row), or whose two words are not both inside the table, is read element by
// element.
template <int SRC, int DST, int W, typename ID>
__global__ void __launch_bounds__(kThreads) embedding_across_kernel(const LookupArgs a)
{
    using S = typename Element<SRC>::type;
    using D = typename Element<DST>::type;
    constexpr int kWords = 4;                           // of each thread
    constexpr uint32_t kWordBytes = W * kElemBytes<SRC>;
    const uint32_t dim = (uint32_t)a.dim;
    const uint64_t n = a.tokens * dim, first = (uint64_t)blockIdx.x * (kThreads * kWords * W), token0 = first / dim;
    const uint32_t col0 = (uint32_t)(first - token0 * dim);
    const S* table = static_cast<const S*>(a.table);
    const char *low = reinterpret_cast<const char*>(table), *high = reinterpret_cast<const char*>(table + a.rows * dim);
    D* out = static_cast<D*>(a.out) + first;
    const auto row_of = [&](uint64_t token) -> const S* {
        const int64_t id = token < a.tokens ? (int64_t)__ldg(static_cast<const ID*>(a.ids) + token) : -1;
        return id >= 0 && (uint64_t)id < a.rows ? table + (uint64_t)id * dim : nullptr;
    };
    grid_dependency_wait();
    const S *x[kWords], *next[kWords];                  // where the word's first row has its elements; the next row
    uint32_t here[kWords];                              // how many of them are the first row's
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
        const uint32_t local = (threadIdx.x + k * kThreads) * W, over = (col0 + local) / dim, col = col0 + local - over * dim;
        here[k] = dim - col < (uint32_t)W ? dim - col : (uint32_t)W;
        const S* row = row_of(token0 + over);
        x[k] = row != nullptr ? row + col : nullptr;
        next[k] = here[k] < (uint32_t)W ? row_of(token0 + over + 1) : nullptr;
    }
    Packed<SRC, W> v[kWords];
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
        const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(x[k]) & (kWordBytes - 1));
        const char* word = reinterpret_cast<const char*>(x[k]) - off;
        if (here[k] == (uint32_t)W && x[k] != nullptr && word >= low && word + 2 * kWordBytes <= high) {
            v[k] = load_across<SRC, W>(x[k], off);
        } else {
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const bool first_row = (uint32_t)e < here[k];
                const S* from = first_row ? x[k] : next[k];
                narrow(0.0f, v[k].e[e]);
                if (from != nullptr) v[k].e[e] = first_row ? x[k][e] : next[k][e - here[k]];
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
        const uint32_t local = (threadIdx.x + k * kThreads) * W;
        Packed<DST, W> y;
#pragma unroll
        for (int e = 0; e < W; ++e)                     // +0 in empty places, whatever the scale
            y.set(e, ((uint32_t)e < here[k] ? x[k] : next[k]) != nullptr ? a.scale * v[k].get(e) : 0.0f);
        if (first + local + W <= n) {
            y.store(out + local);
        } else {
#pragma unroll
            for (int e = 0; e < W; ++e)
                if (first + local + e < n) out[local + e] = y.e[e];
        }
    }
}

template <int SRC, int DST, int V, typename ID>
cudaError_t launch(const LookupArgs& a, cudaStream_t stream)
{
    const uint64_t n = a.tokens * (a.dim / V), per_block = kThreads * kVectors;
    return launch_pdl(embedding_kernel<SRC, DST, V, ID>, (unsigned)((n + per_block - 1) / per_block), kThreads, stream, a);
}

template <int SRC, int DST, int V> cudaError_t by_ids(const LookupArgs& a, int wide, cudaStream_t stream)
{
    return wide ? launch<SRC, DST, V, int64_t>(a, stream) : launch<SRC, DST, V, int32_t>(a, stream);
}

template <int SRC, int DST, int W> cudaError_t launch_across(const LookupArgs& a, int wide, cudaStream_t stream)
{
    const uint64_t per_block = kThreads * 4 * W, blocks = (a.tokens * a.dim + per_block - 1) / per_block;
    return wide ? launch_pdl(embedding_across_kernel<SRC, DST, W, int64_t>, (unsigned)blocks, kThreads, stream, a)
                : launch_pdl(embedding_across_kernel<SRC, DST, W, int32_t>, (unsigned)blocks, kThreads, stream, a);
}

// Words of 16 bytes of the wider type where they divide the rows and both sides start on their boundaries.  Where they do not,
// words put together from two, as long as the output starts on a word and a row has several; or shorter words.
template <int SRC, int DST> cudaError_t by_vector(const LookupArgs& a, int wide, cudaStream_t stream)
{
    constexpr int most = SRC == kF32 || DST == kF32 ? 4 : 8;
    const int v = row_vector(most, a.dim, a.table, kElemBytes<SRC>, a.out, kElemBytes<DST>);
    if (v < most && a.dim >= 4 * most && (reinterpret_cast<uintptr_t>(a.out) & (most * kElemBytes<DST> - 1)) == 0)
        return launch_across<SRC, DST, most>(a, wide, stream);
    switch (v) {
        case 8: if constexpr (most == 8) return by_ids<SRC, DST, 8>(a, wide, stream);
        case 4: return by_ids<SRC, DST, 4>(a, wide, stream);
        case 2: return by_ids<SRC, DST, 2>(a, wide, stream);
    }
    return by_ids<SRC, DST, 1>(a, wide, stream);
}

}  // namespace

cudaError_t launch_embedding(const void* table, int table_dtype, uint64_t rows, uint64_t dim, const TokenIds& ids, float scale,
                             void* out, int out_dtype, cudaStream_t stream)
{
    const LookupArgs a = {table, ids.ptr, out, rows, dim, ids.count, scale};
    if (table_dtype == kF32)
        return out_dtype == kF32 ? by_vector<kF32, kF32>(a, ids.wide, stream) : by_vector<kF32, kBf16>(a, ids.wide, stream);
    return out_dtype == kF32 ? by_vector<kBf16, kF32>(a, ids.wide, stream) : by_vector<kBf16, kBf16>(a, ids.wide, stream);
}

}  // namespace mqg
