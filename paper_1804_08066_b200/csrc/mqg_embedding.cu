// Rows of a table for a batch of token ids:  out[t] = fl(scale * table[ids[t]]), a row of zeros for an id outside 0..rows-1.
//
// Bound by memory: the rows that are used are read, the output is written.  A thread takes vectors of V elements (up to
// 16 bytes of the narrower type), several of them so that their dependent loads (id, then row) overlap.
#include "mqg_tma.cuh"
#include "mqg_training.h"
#include "mqg_vector.cuh"

namespace mqg {
namespace {

constexpr int kThreads = 256;
constexpr int kVectors = 4;                             // of each thread

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

// The longest vector that divides the rows and that both sides' addresses allow.
template <int SRC, int DST> cudaError_t by_vector(const LookupArgs& a, int wide, cudaStream_t stream)
{
    constexpr int most = SRC == kF32 && DST == kF32 ? 4 : 8;
    switch (row_vector(most, a.dim, a.table, kElemBytes<SRC>, a.out, kElemBytes<DST>)) {
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
