// Rows of a table for a batch of token ids:  out[t] = fl(scale * table[ids[t]]), a row of zeros for an id outside 0..rows-1.
//
// Bound by memory: the rows that are used are read, the output is written.  A thread takes words of V elements, 16 bytes of the
// wider type, so that every access of a warp covers whole sectors, and four of them so that their dependent loads (id, then
// row) overlap.  (16,384 rows of 1024 from fp32 to bf16: 12.6 us, with eight 13.7, two 14.8; 13.0 with a division for every
// word.)
#include "mqg_tma.cuh"
#include "mqg_training.h"
#include "mqg_vector.cuh"

namespace mqg {
namespace {

constexpr int kThreads = 256;
constexpr int kVectors = 4;                             // of each thread

__device__ __forceinline__ uint64_t quotient(uint64_t a, uint32_t b) { return (a >> 32) == 0 ? (uint32_t)a / b : a / b; }

struct LookupArgs {
    const void* table;
    const void* ids;
    void* out;
    uint64_t rows, dim, tokens;
    float scale;
    uint32_t reciprocal;     // of the words of a row: ceil(2^32 / words); 0: 1 word, or more than kMostWords
};

// Rows a CTA's word `local` (counted from the first row it begins in) is beyond the first: a division by the words of a row, of a
// number below words + kThreads * kVectors, without the 25 instructions that a division is.  The high word of the product with
// the reciprocal is exact up to kMostWords: the product's error, below words * local, stays below 2^32.
constexpr uint32_t kMostWords = 32768;
__device__ __forceinline__ uint32_t rows_beyond(uint32_t local, uint32_t words, uint32_t reciprocal)
{
    if (reciprocal != 0) return __umulhi(local, reciprocal);
    return words == 1 ? local : local >= words ? 1 : 0;
}

template <int SRC, int DST, int V, typename ID>
__global__ void __launch_bounds__(kThreads) embedding_kernel(const LookupArgs a)
{
    const uint32_t row_vectors = (uint32_t)(a.dim / V);
    const uint64_t n = a.tokens * row_vectors, first = (uint64_t)blockIdx.x * (kThreads * kVectors);
    const uint64_t token0 = quotient(first, row_vectors);
    const uint32_t col0 = (uint32_t)(first - token0 * row_vectors);
    grid_dependency_wait();
    const uint32_t held = (uint32_t)min(n - first, (uint64_t)(kThreads * kVectors));
    const ID* ids = static_cast<const ID*>(a.ids) + token0;
    const auto* table = static_cast<const typename Element<SRC>::type*>(a.table);
    const typename Element<SRC>::type* from[kVectors];  // the word of the table, null where the place is empty
#pragma unroll
    for (int k = 0; k < kVectors; ++k) {
        const uint32_t i = threadIdx.x + k * kThreads, local = col0 + i, over = rows_beyond(local, row_vectors, a.reciprocal);
        const int64_t id = i < held ? (int64_t)__ldg(ids + over) : -1;
        const bool there = (uint64_t)id < a.rows;       // (a negative id is above every count of rows)
        from[k] = there ? table + ((uint64_t)id * row_vectors + (local - over * row_vectors)) * V : nullptr;
    }
    Packed<SRC, V> x[kVectors];
#pragma unroll
    for (int k = 0; k < kVectors; ++k)
        if (from[k] != nullptr) x[k].load(from[k]);
    auto* out = static_cast<typename Element<DST>::type*>(a.out) + first * V;
#pragma unroll
    for (int k = 0; k < kVectors; ++k) {
        const uint32_t i = threadIdx.x + k * kThreads;
        if (i >= held) continue;
        Packed<DST, V> y;
#pragma unroll
        for (int e = 0; e < V; ++e) y.set(e, a.scale * x[k].get(e));
        if (from[k] == nullptr) {
#pragma unroll
            for (int j = 0; j < Packed<DST, V>::kWords; ++j) y.w[j] = {};
        }
        y.store(out + i * V);
    }
}

// The same where rows start anywhere, by vectors of one element or two: threads stand side by side over a row, and a thread
// takes every so many-th vector of four rows.  Without divisions, and with few instructions to an element, which is what bounds
// it: 65,536 rows of 515 from fp32 to bf16 in 53 us, where 16-byte words put together from the two that hold them took 71.
struct RowArgs {
    LookupArgs a;
    int thread_bits;         // 2^this threads side by side
    uint32_t tiles;          // CTAs side by side
};

template <int SRC, int DST, int V, typename ID>
__global__ void __launch_bounds__(kThreads) embedding_rows_kernel(const RowArgs args)
{
    using S = typename Element<SRC>::type;
    using D = typename Element<DST>::type;
    constexpr int kRows = 4, kGroups = 4;
    const LookupArgs& a = args.a;
    const uint32_t dim = (uint32_t)a.dim, across = 1u << args.thread_bits, down = kThreads >> args.thread_bits;
    const uint32_t group = blockIdx.x / args.tiles, tile = blockIdx.x - group * args.tiles, apart = across * V;
    const uint32_t col = tile * (apart * kGroups) + (threadIdx.x & (across - 1)) * V;
    const uint64_t token0 = (uint64_t)group * (down * kRows) + (threadIdx.x >> args.thread_bits);
    grid_dependency_wait();
    const S* x[kRows];                                  // the row, null where the place is empty
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const uint64_t token = token0 + r * down;
        const int64_t id = token < a.tokens ? (int64_t)__ldg(static_cast<const ID*>(a.ids) + token) : -1;
        x[r] = id >= 0 && (uint64_t)id < a.rows ? static_cast<const S*>(a.table) + (uint64_t)id * dim + col : nullptr;
    }
    Packed<SRC, V> v[kRows][kGroups];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
            if (x[r] != nullptr && col + g * apart < dim) v[r][g].load(x[r] + g * apart);
    D* y = static_cast<D*>(a.out) + token0 * dim + col;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        if (token0 + r * down >= a.tokens) break;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            if (col + g * apart >= dim) break;
            Packed<DST, V> out;
#pragma unroll
            for (int e = 0; e < V; ++e) out.set(e, x[r] != nullptr ? a.scale * v[r][g].get(e) : 0.0f);
            out.store(y + g * apart);
        }
        y += (uint64_t)down * dim;
    }
}

template <int SRC, int DST, int V, typename ID>
cudaError_t launch(LookupArgs a, cudaStream_t stream)
{
    const uint64_t words = a.dim / V, n = a.tokens * words, per_block = kThreads * kVectors;
    a.reciprocal = words > 1 && words <= kMostWords ? (uint32_t)(((1ull << 32) + words - 1) / words) : 0;
    return launch_pdl(embedding_kernel<SRC, DST, V, ID>, (unsigned)((n + per_block - 1) / per_block), kThreads, stream, a);
}

template <int SRC, int DST, int V> cudaError_t by_ids(const LookupArgs& a, int wide, cudaStream_t stream)
{
    return wide ? launch<SRC, DST, V, int64_t>(a, stream) : launch<SRC, DST, V, int32_t>(a, stream);
}

template <int SRC, int DST, int V> cudaError_t launch_rows(const LookupArgs& a, int wide, cudaStream_t stream)
{
    RowArgs x = {a, 0, 1};
    while ((1 << x.thread_bits) < 128 && ((uint64_t)V * 4) << x.thread_bits < a.dim) ++x.thread_bits;
    const uint64_t tile = ((uint64_t)V * 4) << x.thread_bits, rows = (uint64_t)(kThreads >> x.thread_bits) * 4;
    x.tiles = (uint32_t)((a.dim + tile - 1) / tile);
    const unsigned blocks = (unsigned)((a.tokens + rows - 1) / rows * x.tiles);
    return wide ? launch_pdl(embedding_rows_kernel<SRC, DST, V, int64_t>, blocks, kThreads, stream, x)
                : launch_pdl(embedding_rows_kernel<SRC, DST, V, int32_t>, blocks, kThreads, stream, x);
}

// Words of 16 bytes of the wider type where they divide the rows and both sides start on their boundaries, or as long ones as do.
template <int SRC, int DST> cudaError_t by_vector(const LookupArgs& a, int wide, cudaStream_t stream)
{
    constexpr int most = SRC == kF32 || DST == kF32 ? 4 : 8;
    switch (row_vector(most, a.dim, a.table, kElemBytes<SRC>, a.out, kElemBytes<DST>)) {
        case 8: if constexpr (most == 8) return by_ids<SRC, DST, 8>(a, wide, stream);
        case 4: return by_ids<SRC, DST, 4>(a, wide, stream);
        case 2: return launch_rows<SRC, DST, 2>(a, wide, stream);
    }
    return launch_rows<SRC, DST, 1>(a, wide, stream);
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
