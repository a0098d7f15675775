// The gradient of a table of `rows` x `dim` from the gradient of the rows looked up in it:
//
//   grad[v] = fl((grad[v] +) scale * sum over t with ids[t] = v of dout[t])
//
// in fp32, tokens in ascending order:
//   1. the tokens are sorted by id (mqg_token_sort.cu), so that the tokens of a row are neighbours (a run) and no atomic is
//      needed: the order of every sum is fixed;
//   2. the sorted tokens are cut into chunks of C; a thread takes eight columns of a chunk and adds up its runs.  A run that
//      crosses chunks belongs to the chunk it begins in, which follows it, as long as it covers no chunk as a whole (less
//      than 2 C tokens); of a longer one every chunk leaves its part's sum in the workspace.  Unless the gradient is added to
//      what is there, further CTAs of the sort's launch set a first part of it to zero, and of this one the rest of the rows
//      that have no tokens.  (Zeros by a launch of their own that the sort let begin early, beside itself, took as long or up to
//      3 % less, but they began to write before any wait of theirs said that what came before was done);
//   3. the parts of the long runs are added up in the order of the chunks.
#include <atomic>

#include "mqg_token_sort.cuh"
#include "mqg_vector.cuh"

namespace mqg {
namespace {

constexpr int kThreads = 128;
constexpr int kColumns = 8;                             // of a thread, in groups of W neighbours
constexpr int kMaxChunkBits = 5, kLeastThreadBits = 3;
constexpr int kMaxDown = kThreads >> kLeastThreadBits;  // chunks of a CTA

struct GradArgs {
    const uint2* sorted;     // (row, token), rows ascending; the row `rows` = none
    const void* dout;
    void* grad;
    float4* parts;           // [chunk][2][words]: the sums of the long run that enters the chunk, and of the one that begins in it
    uint32_t* run_count;
    uint4* long_runs;        // (chunk that it begins in, chunks that it has parts in, row, 0)
    uint32_t dim, tokens, rows, chunks;
    int chunk_bits;
    uint32_t tiles;          // CTAs side by side over the columns
    int thread_bits;         // 2^this threads of a CTA over the columns, the others over chunks
    float scale;
    uint32_t sum_ctas;       // the CTAs behind them set rows without tokens to zero,
    uint32_t zero_from;      // from this one on:
    uint32_t zero_rows;      // so many each, or,
    uint32_t zero_parts;     // where a row is more than a CTA's share, one of so many parts of a row
    uint32_t reciprocal;     // of a row's bytes: ceil(2^32 / bytes), where a CTA has several rows
};

// The sums of a thread's eight columns are two words of a part: word j of thread t of tile i is word (2 i + j) * threads + t.
__device__ __forceinline__ uint32_t part_words(const GradArgs& a) { return a.tiles * 2 << a.thread_bits; }
__device__ __forceinline__ float4* part_at(const GradArgs& a, uint32_t chunk, bool begins)
{
    return a.parts + ((uint64_t)chunk * 2 + (begins ? 1 : 0)) * part_words(a);
}

// The sorted tokens that a CTA's chunks look at, in shared memory: its chunks', and a chunk more on both sides.
struct Window {
    uint2 token[(kMaxDown + 2) << kMaxChunkBits];
    uint32_t begin;                                     // token[0] is sorted token `begin`, modulo 2^32

    __device__ __forceinline__ void load(const GradArgs& a, uint32_t first_chunk, uint32_t chunks)
    {
        const uint32_t from = (first_chunk - 1) << a.chunk_bits, n = (chunks + 2) << a.chunk_bits;
        for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
            const uint32_t p = from + i;                // wraps in the chunk before the first
            // (not by way of L1: this launch may have begun before the sort was done)
            token[i] = p < a.tokens ? __ldcg(a.sorted + p) : make_uint2(a.rows, 0);
        }
        if (threadIdx.x == 0) begin = from;
        __syncthreads();
    }
    __device__ __forceinline__ uint2 at(uint32_t p) const { return token[p - begin]; }
    __device__ __forceinline__ uint32_t row(uint32_t p) const { return token[p - begin].x; }
};

// What a thread has to do in its chunk: sorted tokens begin..end - 1.
struct ChunkWork {
    uint32_t begin, end;
    uint32_t entering;       // the row of a long run that enters the chunk, or `rows`
    uint32_t leaving;        // the row of a long run that leaves it, or `rows`
    bool begins;             // the one that leaves it begins here

    template <typename Args, typename Tokens>
    __device__ __forceinline__ ChunkWork(const Args& a, const Tokens& s, uint32_t chunk)
    {
        const uint32_t size = 1u << a.chunk_bits, first = chunk << a.chunk_bits;
        begin = first;
        end = min(first + size, a.tokens);
        const uint32_t row0 = s.row(first), row1 = s.row(end - 1);
        const bool enters = first != 0 && s.row(first - 1) == row0;
        const bool crosses = row1 != a.rows && end < a.tokens && s.row(end) == row1;
        // long: covers this chunk, the one before or the one behind as a whole
        const bool long_in = enters && row0 != a.rows && (row0 == row1 || s.row(first - size) == row0);
        const bool long_out = crosses && (row0 == row1 || s.row(min(end + size, a.tokens) - 1) == row1);
        begins = long_out && !(long_in && row0 == row1);
        entering = long_in ? row0 : a.rows;
        leaving = long_out ? row1 : a.rows;
        if (enters && !long_in) {                       // a short run's end, which belongs to the chunk before
            for (uint32_t step = size / 2; step != 0; step /= 2)
                if (begin + step < end && s.row(begin + step - 1) == row0) begin += step;
            while (begin < end && s.row(begin) == row0) ++begin;
        }
        if (crosses && !long_out) {                     // a short run's end in the chunk behind
            while (s.row(end) == row1) ++end;
        } else if (row1 == a.rows) {                    // ids outside the table
            while (end > begin && s.row(end - 1) == a.rows) --end;
        }
    }
};

// A copy of 4, 8 or 16 bytes to shared memory that only the copying thread reads.
template <int BYTES> __device__ __forceinline__ void copy_async(void* smem, const void* p)
{
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(smem)), "l"(p) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_u32(smem)), "l"(p), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A thread's columns of DEPTH rows under way: in slots of shared memory that the thread alone writes and reads, or, for groups
// of less than the 4 bytes that asynchronous copies take (bf16 rows of an odd length), in registers.
template <int DTYPE, int W, int DEPTH> struct Flight {
    static constexpr int kGroups = kColumns / W;
    static constexpr bool kAsync = W * kElemBytes<DTYPE> >= 4;
    using Group = Packed<DTYPE, W>;
    static_assert(Group::kWords == 1, "a group is one access");
    struct Shared { typename Group::word slot[kAsync ? DEPTH : 1][kGroups][kAsync ? kThreads : 1]; };
    Group held[kAsync ? 1 : DEPTH][kGroups];

    // The groups whose bit is set, `apart` elements from one to the next.
    __device__ __forceinline__ void fetch(Shared& s, int i, const typename Element<DTYPE>::type* p, uint32_t apart, uint32_t groups)
    {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            if (!((groups >> g) & 1u)) continue;
            if constexpr (kAsync) copy_async<Group::kBytes>(&s.slot[i][g][threadIdx.x], p + g * apart);
            else held[i][g].load(p + g * apart);
        }
    }
    __device__ __forceinline__ Group get(const Shared& s, int i, int g) const
    {
        if constexpr (kAsync) {
            Group x;
            x.w[0] = s.slot[i][g][threadIdx.x];
            return x;
        } else {
            return held[i][g];
        }
    }
};

// One group of a row of grad: the sum times the scale and, with ADD, what was there.
template <int DST, int W, bool ADD>
__device__ __forceinline__ void finish(typename Element<DST>::type* p, Packed<DST, W> y, float scale, const float* sum)
{
#pragma unroll
    for (int e = 0; e < W; ++e) y.set(e, ADD ? __fadd_rn(y.get(e), __fmul_rn(scale, sum[e])) : __fmul_rn(scale, sum[e]));
    y.store(p);
}

// How many chunks the long run that begins in `chunk` has parts in: 32 looks at a time, 32 chunks apart and then one.
__device__ __forceinline__ uint32_t chunks_of_run(const GradArgs& a, uint32_t chunk, uint32_t row)
{
    uint32_t n = 1;
#pragma unroll
    for (int bits = 5; bits >= 0; bits -= 5) {
        uint32_t on;
        do {
            on = 0;
#pragma unroll
            for (uint32_t k = 1; k <= 32; ++k) {        // the run covers a first part of the chunks: as many as are on
                const uint64_t p = ((uint64_t)chunk + n + (k << bits) - 1) << a.chunk_bits;
                on += p < a.tokens && __ldcg(&a.sorted[p].x) == row ? 1 : 0;
            }
            n += on << bits;
        } while (on == 32);
    }
    return n;
}

// ---- rows without tokens ----
// A CTA has up to 32 KB of the gradient.  It finds the sorted tokens of its rows, marks the rows that have some and sets the
// others to zero.  It writes no row that has tokens, so that it need not be ordered with the sums, and it begins, like them,
// when the sort is done.  Bound by the writes to DRAM (200,000 rows of 1000 in fp32, 16,384 tokens: 134 us in all, 800 MB
// written and 66 read) as long as the turns to memory before them are few: as a rule two, a look at 128 tokens far apart and one
// at the 512 behind the last of them that is of a row before.  (With 16 KB the CTAs are too short for that: 159 us; with 64
// there are too few of them at the end: 50,000 rows of 4 KB, 16,384 tokens, 51.6 us instead of 49.4.)
constexpr uint32_t kZeroBytes = 32768;
constexpr uint32_t kMaxZeroRows = 1024, kMaxScan = 4096;
constexpr int kRowsPerThread = kMaxZeroRows / kThreads;

struct UsedRows {
    uint32_t bits[kMaxZeroRows / 32];
    uint32_t any;
    __device__ __forceinline__ bool has(uint32_t row) const { return (bits[row / 32] >> (row & 31)) & 1u; }
};

// Marks which of the `rows` rows from row0 on have tokens; returns whether any has.
__device__ __forceinline__ bool find_used(const GradArgs& a, uint32_t row0, uint32_t rows, UsedRows& used)
{
    constexpr uint32_t kLooks = 4;
    const uint32_t lane = threadIdx.x & 31, end = a.tokens;
    if (threadIdx.x < kMaxZeroRows / 32) used.bits[threadIdx.x] = 0;
    if (threadIdx.x == 0) used.any = 0;
    uint32_t begin = 0;                                 // the tokens before are of rows before
    for (uint32_t n = end; n > kLooks * kThreads;) {
        const uint32_t step = (n + kThreads - 1) / kThreads, p = begin + (threadIdx.x + 1) * step - 1;
        begin += step * __syncthreads_count(p < end && __ldcg(&a.sorted[p].x) < row0);
        n = min(step - 1, end - begin);
    }
    for (uint32_t from = begin; from - begin < kMaxScan; from += kLooks * kThreads) {
        uint32_t row[kLooks];
#pragma unroll
        for (uint32_t u = 0; u < kLooks; ++u) {
            const uint32_t p = from + u * kThreads + threadIdx.x;
            row[u] = p < end ? __ldcg(&a.sorted[p].x) : ~0u;
        }
        if (from == begin) __syncthreads();             // (nothing is marked before all is clear)
#pragma unroll
        for (uint32_t u = 0; u < kLooks; ++u) {
            const uint32_t before = __shfl_up_sync(0xFFFFFFFFu, row[u], 1), r = row[u] - row0;
            if (row[u] < row0 || r >= rows || (lane != 0 && row[u] == before)) continue;
            atomicOr(&used.bits[r / 32], 1u << (r & 31));
            used.any = 1;
        }
        const bool beyond = row[kLooks - 1] >= row0 && row[kLooks - 1] - row0 >= rows;
        if (__syncthreads_or(beyond)) return used.any != 0;
    }
    // more tokens than are worth looking at (all but the first 512 are of these rows): a search for every row
    uint32_t at[kRowsPerThread];                        // the last token whose row is not above, or the first
#pragma unroll
    for (int u = 0; u < kRowsPerThread; ++u) at[u] = begin;
    for (uint32_t left = end - begin; left > 1;) {
        const uint32_t half = left / 2;
#pragma unroll
        for (int u = 0; u < kRowsPerThread; ++u) {
            if (u * kThreads >= rows) break;
            if (__ldcg(&a.sorted[at[u] + half].x) <= row0 + u * kThreads + threadIdx.x) at[u] += half;
        }
        left -= half;
    }
#pragma unroll
    for (int u = 0; u < kRowsPerThread; ++u) {
        if (u * kThreads >= rows) break;
        const bool there = u * kThreads + threadIdx.x < rows && __ldcg(&a.sorted[at[u]].x) == row0 + u * kThreads + threadIdx.x;
        const uint32_t bits = __ballot_sync(0xFFFFFFFFu, there);
        if (lane == 0) used.bits[u * (kThreads / 32) + threadIdx.x / 32] = bits;
    }
    __syncthreads();
    return true;
}

// Zeros into `bytes` bytes of elements T, by `count` threads of which this is number `i`.
template <typename T> __device__ __forceinline__ void write_zeros(char* p, uint32_t bytes, uint32_t i, uint32_t count)
{
    const uint32_t to_boundary = (uint32_t)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15);
    const uint32_t head = min(to_boundary, bytes), behind = bytes - (bytes - head) % 16;
#pragma unroll 4
    for (uint32_t at = head + i * 16; at < behind; at += count * 16) *reinterpret_cast<uint4*>(p + at) = make_uint4(0, 0, 0, 0);
    const uint32_t at = i * (uint32_t)sizeof(T);
    if (at < head) *reinterpret_cast<T*>(p + at) = T();
    if (at < bytes - behind) *reinterpret_cast<T*>(p + behind + at) = T();
}

// The same for rows of row_bytes of which those that are used stay: of long rows a warp takes one at a time, of others threads go
// through the vectors side by side.
constexpr uint32_t kLongRow = 512;
template <typename T>
__device__ __forceinline__ void write_zeros_between(char* p, uint32_t rows, uint32_t row_bytes, uint32_t reciprocal, const UsedRows& used)
{
    if (row_bytes >= kLongRow) {
        for (uint32_t r = threadIdx.x / 32; r < rows; r += kThreads / 32)
            if (!used.has(r)) write_zeros<T>(p + r * row_bytes, row_bytes, threadIdx.x & 31, 32);
        return;
    }
    const uint32_t bytes = rows * row_bytes, to_boundary = (uint32_t)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15);
    const uint32_t head = min(to_boundary, bytes), behind = bytes - (bytes - head) % 16;
    const auto row_of = [&](uint32_t at) { return __umulhi(at, reciprocal); };
    const auto element = [&](uint32_t at) {
        if (!used.has(row_of(at))) *reinterpret_cast<T*>(p + at) = T();
    };
    for (uint32_t at = head + threadIdx.x * 16; at < behind; at += kThreads * 16) {
        const uint32_t row = row_of(at), last = row_of(at + 16 - (uint32_t)sizeof(T));
        bool any = used.has(row), all = any;
        for (uint32_t r = row + 1; r <= last; ++r) {    // rows that start anywhere: some end in the vector
            any |= used.has(r);
            all &= used.has(r);
        }
        if (!any) {
            *reinterpret_cast<uint4*>(p + at) = make_uint4(0, 0, 0, 0);
        } else if (!all) {
#pragma unroll 1
            for (uint32_t e = 0; e < 16; e += sizeof(T)) element(at + e);
        }
    }
    const uint32_t at = threadIdx.x * (uint32_t)sizeof(T);
    if (at < head) element(at);
    if (at < bytes - behind) element(behind + at);
}

template <typename T> __device__ __forceinline__ void zero_unused_rows(const GradArgs& a, uint32_t cta, UsedRows& used)
{
    const uint32_t group = cta / a.zero_parts, part = cta - group * a.zero_parts;
    const uint32_t row0 = a.zero_from + group * a.zero_rows, rows = min(a.zero_rows, a.rows - row0);
    const bool any = find_used(a, row0, rows, used);
    if (any && a.zero_rows == 1) return;
    const uint64_t row_bytes = (uint64_t)a.dim * sizeof(T), from = (uint64_t)part * kZeroBytes;
    char* p = static_cast<char*>(a.grad) + row0 * row_bytes + from;
    if (any) write_zeros_between<T>(p, rows, (uint32_t)row_bytes, a.reciprocal, used);
    else write_zeros<T>(p, (uint32_t)min(rows * row_bytes - from, (uint64_t)kZeroBytes), threadIdx.x, kThreads);
}

// CTAs that read the same rows are neighbours in the grid.  Lanes take neighbouring groups, so that every access of a warp
// covers whole sectors (two 16-byte stores per thread, 32 bytes apart from lane to lane, made the fp32 sums write half
// sectors).  kDepth rows are under way for each thread: four with 23 KB of shared memory to a CTA did as well as six, and
// left room for more CTAs whose beginnings and ends overlap; eight were 10 % slower.
template <int SRC, int DST, int W, bool ADD>
__global__ void __launch_bounds__(kThreads) grad_sum_kernel(const GradArgs a)
{
    constexpr int kDepth = 4, kGroups = kColumns / W;
    using X = Flight<SRC, W, kDepth>;
    using Y = Flight<DST, W, ADD ? kDepth : 1>;
    __shared__ typename X::Shared xs;
    __shared__ typename Y::Shared ys;
    __shared__ Window tokens;
    if constexpr (!ADD) {
        if (blockIdx.x >= a.sum_ctas) {
            __shared__ UsedRows used;
            grid_dependency_wait();
            zero_unused_rows<typename Element<DST>::type>(a, blockIdx.x - a.sum_ctas, used);
            return;
        }
    }
    const uint32_t across = 1u << a.thread_bits, down = blockIdx.x / a.tiles, tile = blockIdx.x - down * a.tiles;
    const uint32_t t = threadIdx.x & (across - 1), first_chunk = down * (kThreads >> a.thread_bits);
    const uint32_t chunk = first_chunk + (threadIdx.x >> a.thread_bits);
    const uint32_t col = (tile * across * kGroups + t) * W, apart = across * W;
    grid_dependency_wait();
    tokens.load(a, first_chunk, kThreads >> a.thread_bits);
    if (col >= a.dim || chunk >= a.chunks) return;
    uint32_t groups = 0;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) groups |= col + g * apart < a.dim ? 1u << g : 0u;

    const ChunkWork w(a, tokens, chunk);
    if (w.begins && col == 0) a.long_runs[atomicAdd(a.run_count, 1u)] = make_uint4(chunk, chunks_of_run(a, chunk, w.leaving), w.leaving, 0);
    const auto* dout = static_cast<const typename Element<SRC>::type*>(a.dout) + col;
    auto* grad = static_cast<typename Element<DST>::type*>(a.grad) + col;
    X x;
    Y y;
    uint2 next = tokens.at(w.begin);
    uint32_t row[kDepth], ends = 0;                     // of the tokens under way; bits: those that end a run
    const auto fetch = [&](uint32_t p, int i) {         // called for one token after the other
        if (p < w.end) {
            const uint2 k = next;
            next = tokens.at(p + 1);
            row[i] = k.x;
            x.fetch(xs, i, dout + (uint64_t)k.y * a.dim, apart, groups);
            if (next.x != k.x) {
                ends |= 1u << i;
                if (ADD && k.x != w.entering) y.fetch(ys, i, grad + (uint64_t)k.x * a.dim, apart, groups);
            }
        }
        copies_commit();
    };
    float sum[kColumns];
#pragma unroll
    for (int e = 0; e < kColumns; ++e) sum[e] = 0.0f;
    const auto store_part = [&](bool begins) {
        float4* p = part_at(a, chunk, begins) + (tile * 2 << a.thread_bits) + t;
        p[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
        p[across] = make_float4(sum[4], sum[5], sum[6], sum[7]);
    };
#pragma unroll
    for (int i = 0; i < kDepth; ++i) fetch(w.begin + i, i);
    for (uint32_t p = w.begin; p < w.end; p += kDepth) {
#pragma unroll
        for (int i = 0; i < kDepth; ++i) {
            if (p + i >= w.end) break;
            copies_wait<kDepth - 1>();
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const auto v = x.get(xs, i, g);
#pragma unroll
                for (int e = 0; e < W; ++e) sum[g * W + e] = __fadd_rn(sum[g * W + e], v.get(e));
            }
            if ((ends >> i) & 1u) {
                ends &= ~(1u << i);
                if (row[i] == w.entering) {
                    store_part(false);
                } else {
#pragma unroll
                    for (int g = 0; g < kGroups; ++g) {
                        if (!((groups >> g) & 1u)) continue;
                        Packed<DST, W> old;
                        if (ADD) old = y.get(ys, ADD ? i : 0, g);
                        finish<DST, W, ADD>(grad + (uint64_t)row[i] * a.dim + g * apart, old, a.scale, sum + g * W);
                    }
                }
#pragma unroll
                for (int e = 0; e < kColumns; ++e) sum[e] = 0.0f;
            }
            fetch(p + kDepth + i, i);
        }
    }
    if (w.leaving != a.rows) store_part(w.begins);
}

// The long runs: a CTA takes kJoinWords words of one run after another, kSplits groups of threads equal shares of its parts.
// What bounds it is the chain of dependent loads: the run, its length, its parts, in that order.
constexpr int kJoinThreads = 256, kSplits = 8, kJoinWords = kJoinThreads / kSplits;

template <int DST, int W, bool ADD>
__global__ void __launch_bounds__(kJoinThreads) grad_join_kernel(const GradArgs a)
{
    __shared__ float4 share[kSplits][kJoinWords];
    grid_dependency_wait();
    const uint32_t words = part_words(a), tiles = (words + kJoinWords - 1) / kJoinWords;
    const uint64_t items = (uint64_t)__ldcg(a.run_count) * tiles;
    const uint32_t s = threadIdx.x / kJoinWords;
    for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t run = (uint32_t)(item / tiles), word = (uint32_t)(item - (uint64_t)run * tiles) * kJoinWords + threadIdx.x % kJoinWords;
        const uint4 r = __ldcg(a.long_runs + run);
        const uint32_t n = word < words ? r.y : 0;
        const uint32_t per = (n + kSplits - 1) / kSplits, from = min(s * per, n), to = min(from + per, n);
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
        for (uint32_t i = from; i < to; ++i) {
            const float4 v = __ldcg(part_at(a, r.x + i, i == 0) + word);
            sum.x = __fadd_rn(sum.x, v.x);
            sum.y = __fadd_rn(sum.y, v.y);
            sum.z = __fadd_rn(sum.z, v.z);
            sum.w = __fadd_rn(sum.w, v.w);
        }
        share[s][threadIdx.x % kJoinWords] = sum;
        __syncthreads();
        if (s == 0 && word < words) {
#pragma unroll
            for (int k = 1; k < kSplits; ++k) {
                const float4 v = share[k][threadIdx.x];
                sum.x = __fadd_rn(sum.x, v.x);
                sum.y = __fadd_rn(sum.y, v.y);
                sum.z = __fadd_rn(sum.z, v.z);
                sum.w = __fadd_rn(sum.w, v.w);
            }
            // the word's columns: a group of four, half a group of eight, or several smaller groups
            constexpr int G = W < 4 ? W : 4;
            const uint32_t across = 1u << a.thread_bits, tile = word / (2 * across), half = (word / across) & 1, t = word & (across - 1);
            const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
            for (int g = 0; g < 4 / G; ++g) {
                const uint32_t group = W == 8 ? 0 : half * (4 / G) + g;
                const uint32_t col = ((tile * (kColumns / W) + group) * across + t) * W + (W == 8 ? half * 4 : 0);
                if (col >= a.dim) continue;
                auto* p = static_cast<typename Element<DST>::type*>(a.grad) + (uint64_t)r.z * a.dim + col;
                Packed<DST, G> old;
                if (ADD) old.load(p);
                finish<DST, G, ADD>(p, old, a.scale, v + g * G);
            }
        }
        __syncthreads();
    }
}

// ---- one launch, for few tokens ----
// A CTA has up to 32 columns of every G-th row of the table (every G-th, so that the frequent ids, which often are neighbours, do
// not meet in one CTA).  It sets them to zero, finds its rows' tokens among all and sorts them in shared memory, adds them up in
// chunks, a thread to each column of a chunk, and joins the long runs' parts, which stay in shared memory.  Bound by latency: of
// the launch, the search, the sort (one pass where the CTA has at most 64 rows) and two turns to memory.  (64 columns: 2048
// tokens, a seventh of them the same, 1000 rows of 64 take 9.4 us against 8, as many evenly spread 6.2 against 6.4.)
constexpr int kSmallColumnBits = 5, kLeastColumnBits = 3, kSmallPerThread = 8;
constexpr uint32_t kSmallTokens = kSmallPerThread * kSortThreads;
static_assert(kSmallTokens <= 1u << PairWord::kTokenBits, "a token is part of a word");
constexpr uint32_t kFewChunks = 64;                     // 4 tokens to a chunk, up to 32 where that makes more chunks than this

__host__ __device__ constexpr uint32_t small_chunks(uint32_t tokens)
{
    return tokens >> kMaxChunkBits > kFewChunks ? (tokens + (1u << kMaxChunkBits) - 1) >> kMaxChunkBits : kFewChunks;
}

struct SmallArgs {
    const void* ids;
    const void* dout;
    void* grad;
    uint32_t dim, tokens, rows;
    uint32_t groups;         // G
    uint32_t reciprocal;     // ceil(2^32 / G): a row's number in its group is the high word of the product; 0: G = 1
    int key_bits;            // of that number
    int column_bits;         // 2^this columns of a CTA
    int wide;
    float scale;
};
constexpr uint64_t kSmallRows = 1 << 24;                // what the reciprocal is exact for, up to G = 148

// The CTA's tokens, sorted by row.
struct SmallWindow {
    const PairWord* pairs;
    uint32_t tokens, rows;
    int chunk_bits;
    __device__ __forceinline__ uint32_t row(uint32_t p) const { return p < tokens ? pairs[p].key() : rows; }
};

// The tokens of the CTA's rows into `pairs`, in order; returns how many.
template <typename ID>
__device__ __forceinline__ uint32_t find_tokens(const SmallArgs& a, uint32_t group, PairWord* pairs, uint32_t* warp_total)
{
    const uint32_t lane = threadIdx.x & 31, w = threadIdx.x >> 5, per = (a.tokens + kSortThreads - 1) / kSortThreads;
    const uint32_t first = w * 32 * per + lane;
    const ID* ids = static_cast<const ID*>(a.ids);
    uint32_t row[kSmallPerThread];
#pragma unroll
    for (int r = 0; r < kSmallPerThread; ++r) {
        const uint32_t i = first + r * 32;
        row[r] = (uint32_t)r < per && i < a.tokens ? key_of(__ldg(ids + i), a.rows) : a.rows;
    }
    uint32_t count = 0, held = 0;
#pragma unroll
    for (int r = 0; r < kSmallPerThread; ++r) {
        if ((uint32_t)r >= per) break;
        const uint32_t k = a.reciprocal != 0 ? __umulhi(row[r], a.reciprocal) : row[r];
        const bool mine = row[r] < a.rows && row[r] - k * a.groups == group;
        held |= mine ? 1u << r : 0u;
        row[r] = k;
        count += __popc(__ballot_sync(0xFFFFFFFFu, mine));
    }
    if (lane == 0) warp_total[w] = count;
    __syncthreads();
    const uint32_t total = warp_total[lane], up_to = sum_up_to_lane(total);
    uint32_t at = __shfl_sync(0xFFFFFFFFu, up_to - total, w);
#pragma unroll
    for (int r = 0; r < kSmallPerThread; ++r) {
        if ((uint32_t)r >= per) break;
        const bool mine = (held >> r) & 1u;
        const uint32_t all = __ballot_sync(0xFFFFFFFFu, mine);
        if (mine) pairs[at + __popc(all & ((1u << lane) - 1))].v = row[r] << PairWord::kTokenBits | (first + r * 32);
        at += __popc(all);
    }
    __syncthreads();
    return __shfl_sync(0xFFFFFFFFu, up_to, 31);
}

template <int K> __device__ __forceinline__ void sort_small(PairWord* pairs, uint32_t n, int bits, SmallSort& s)
{
    PairWord pair[K];
    sort_in_cta<K>(pair, take_pairs<K>(pair, pairs, n), n, bits, s, pairs);
}

// Zeros into the first `columns` columns at `grad` of every groups-th row.
template <typename T>
__device__ __forceinline__ void zero_rows(T* grad, uint32_t rows, uint64_t pitch, uint32_t columns, int column_bits)
{
    constexpr uint32_t V = 16 / sizeof(T);
    if (((reinterpret_cast<uintptr_t>(grad) | pitch * sizeof(T) | columns * sizeof(T)) & 15) == 0) {
        const int bits = column_bits - (sizeof(T) == 4 ? 2 : 3);
        const uint32_t at = (threadIdx.x & ((1u << bits) - 1)) * V;
        if (at >= columns) return;
        for (uint32_t row = threadIdx.x >> bits; row < rows; row += kSortThreads >> bits)
            *reinterpret_cast<uint4*>(grad + row * pitch + at) = make_uint4(0, 0, 0, 0);
    } else {
        const uint32_t at = threadIdx.x & ((1u << column_bits) - 1);
        if (at >= columns) return;
        for (uint32_t row = threadIdx.x >> column_bits; row < rows; row += kSortThreads >> column_bits)
            narrow(0.0f, grad[row * pitch + at]);
    }
}

template <int SRC, int DST, bool ADD>
__global__ void __launch_bounds__(kSortThreads, 1) grad_small_kernel(const SmallArgs a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ SmallSort sort;
    __shared__ uint32_t warp_total[kSortWarps], long_runs[small_chunks(kSmallTokens)], run_count;
    float* parts = reinterpret_cast<float*>(smem);      // [chunk][2][column]
    PairWord* pairs = reinterpret_cast<PairWord*>(parts + (small_chunks(a.tokens) * 2 << a.column_bits));
    const uint32_t across = 1u << a.column_bits, chunks = kSortThreads >> a.column_bits;
    const uint32_t c = threadIdx.x & (across - 1), first_chunk = threadIdx.x >> a.column_bits;
    const uint32_t tile = blockIdx.x / a.groups, group = blockIdx.x - tile * a.groups, col0 = tile * across;
    const uint32_t rows = (a.rows - 1 - group) / a.groups + 1;
    const uint64_t pitch = (uint64_t)a.groups * a.dim;
    const auto* dout = static_cast<const typename Element<SRC>::type*>(a.dout) + col0 + c;
    auto* grad = static_cast<typename Element<DST>::type*>(a.grad) + (uint64_t)group * a.dim + col0;
    const auto finish_one = [&](uint32_t row, float sum, float old) {
        narrow(ADD ? __fadd_rn(old, __fmul_rn(a.scale, sum)) : __fmul_rn(a.scale, sum), grad[row * pitch + c]);
    };
    if (threadIdx.x == 0) run_count = 0;
    grid_dependency_wait();
    if (!ADD) zero_rows(grad, rows, pitch, min(across, a.dim - col0), a.column_bits);
    const uint32_t n = a.wide ? find_tokens<int64_t>(a, group, pairs, warp_total) : find_tokens<int32_t>(a, group, pairs, warp_total);
    if (n > 1 && rows > 1) {
        if (n <= kSortThreads) sort_small<1>(pairs, n, a.key_bits, sort);
        else if (n <= 2 * kSortThreads) sort_small<2>(pairs, n, a.key_bits, sort);
        else if (n <= 4 * kSortThreads) sort_small<4>(pairs, n, a.key_bits, sort);
        else sort_small<kSmallPerThread>(pairs, n, a.key_bits, sort);
    }

    SmallWindow tokens = {pairs, n, rows, 2};
    while (tokens.chunk_bits < kMaxChunkBits && n > min(chunks, kFewChunks) << tokens.chunk_bits) ++tokens.chunk_bits;
    for (uint32_t chunk = first_chunk; col0 + c < a.dim && (chunk << tokens.chunk_bits) < n; chunk += chunks) {
        constexpr int kAhead = 16;                      // as a rule, all of a chunk
        const ChunkWork w(tokens, tokens, chunk);
        if (w.begins && c == 0) long_runs[atomicAdd(&run_count, 1u)] = chunk;
        float sum = 0.0f;
        for (uint32_t p = w.begin; p < w.end; p += kAhead) {
            typename Element<SRC>::type x[kAhead];      // (widened here, every load would be waited for before the next)
            typename Element<DST>::type old[ADD ? kAhead : 1];
            uint32_t ends = 0;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (p + u >= w.end) break;
                const PairWord k = pairs[p + u];
                x[u] = dout[(uint64_t)k.token() * a.dim];
                if (tokens.row(p + u + 1) != k.key()) {
                    ends |= 1u << u;
                    if (ADD && k.key() != w.entering) old[ADD ? u : 0] = grad[k.key() * pitch + c];
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (p + u >= w.end) break;
                sum = __fadd_rn(sum, widen(x[u]));
                if (!((ends >> u) & 1u)) continue;
                const uint32_t row = pairs[p + u].key();
                if (row == w.entering) parts[(chunk * 2) * across + c] = sum;
                else finish_one(row, sum, ADD ? widen(old[ADD ? u : 0]) : 0.0f);
                sum = 0.0f;
            }
        }
        if (w.leaving != rows) parts[(chunk * 2 + (w.begins ? 1 : 0)) * across + c] = sum;
    }
    __syncthreads();
    if (col0 + c >= a.dim) return;
    for (uint32_t i = first_chunk; i < run_count; i += chunks) {
        const uint32_t begin = long_runs[i], row = tokens.row(((begin + 1) << tokens.chunk_bits) - 1);
        const float old = ADD ? widen(grad[row * pitch + c]) : 0.0f;
        float sum = parts[(begin * 2 + 1) * across + c];
        for (uint32_t k = begin + 1;; k += 8) {         // the chunks that the run goes on in, eight looks at a time
            float part[8];
            bool on[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                on[u] = tokens.row((k + u) << tokens.chunk_bits) == row;
                part[u] = on[u] ? parts[(k + u) * 2 * across + c] : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (on[u]) sum = __fadd_rn(sum, part[u]);
            if (!on[7]) break;
        }
        finish_one(row, sum, old);
    }
}

// ---- host ----
// Sizes in the workspace are whole lines of 128 bytes: with parts that begin in the middle of a sector, 73,903 tokens of 512
// took 61 us instead of 57.
constexpr uint64_t whole_lines(uint64_t words) { return (words + 31) & ~31ull; }

struct Layout {
    int chunk_bits, thread_bits;
    uint32_t chunks, tiles;
    uint64_t sorted, runs, scratch, parts, total;       // sizes in words
    Layout(uint64_t tokens, uint64_t dim)
    {
        // 32 tokens to a chunk, down to 8 where that leaves less than a CTA for each of 1024 x 1024 elements
        chunk_bits = kMaxChunkBits;
        while (chunk_bits > 3 && ((tokens * dim) >> chunk_bits) < 1024 * 1024) --chunk_bits;
        chunks = (uint32_t)((tokens + (1u << chunk_bits) - 1) >> chunk_bits);
        thread_bits = kLeastThreadBits;
        while ((1 << thread_bits) < kThreads && (uint64_t)kColumns << thread_bits < dim) ++thread_bits;
        const uint64_t tile = (uint64_t)kColumns << thread_bits;
        tiles = (uint32_t)((dim + tile - 1) / tile);
        sorted = whole_lines(2 * tokens);
        runs = whole_lines(4 + 4 * (uint64_t)chunks);
        scratch = whole_lines(token_sort_words(tokens));
        parts = 2 * (uint64_t)chunks * tiles * tile;
        total = sorted + runs + scratch + parts;
    }
};

template <int SRC, int DST, int W, bool ADD> cudaError_t launch_sums(GradArgs a, cudaStream_t stream)
{
    const uint32_t down = kThreads >> a.thread_bits;
    a.sum_ctas = (a.chunks + down - 1) / down * a.tiles;
    uint32_t zero_ctas = 0;
    if (!ADD) {
        const uint64_t row_bytes = (uint64_t)a.dim * kElemBytes<DST>;
        const uint64_t fit = kZeroBytes / row_bytes;
        a.zero_rows = fit < 1 ? 1 : fit > kMaxZeroRows ? kMaxZeroRows : (uint32_t)fit;
        a.zero_parts = (uint32_t)((row_bytes + kZeroBytes - 1) / kZeroBytes);
        a.reciprocal = fit < 1 ? 0 : (uint32_t)(((1ull << 32) + row_bytes - 1) / row_bytes);
        zero_ctas = (uint32_t)(((uint64_t)a.rows - a.zero_from + a.zero_rows - 1) / a.zero_rows * a.zero_parts);
    }
    const cudaError_t err = launch_pdl(grad_sum_kernel<SRC, DST, W, ADD>, a.sum_ctas + zero_ctas, kThreads, stream, a);
    if (err != cudaSuccess || a.chunks < 2) return err;                              // a long run is in two chunks at least
    const uint64_t most = (uint64_t)(a.chunks - 1) * (((a.tiles * 2 << a.thread_bits) + kJoinWords - 1) / kJoinWords);
    return launch_pdl(grad_join_kernel<DST, W, ADD>, (unsigned)(most < 1184 ? most : 1184), kJoinThreads, stream, a);
}

template <int SRC, int DST, int W> cudaError_t by_add(const GradArgs& a, bool add, cudaStream_t stream)
{
    return add ? launch_sums<SRC, DST, W, true>(a, stream) : launch_sums<SRC, DST, W, false>(a, stream);
}

// Groups of up to 16 bytes of the wider type, as long as they divide the rows and start on their boundaries.
template <int SRC, int DST> cudaError_t by_group(const GradArgs& a, bool add, cudaStream_t stream)
{
    constexpr int most = SRC == kF32 || DST == kF32 ? 4 : 8;
    switch (row_vector(most, a.dim, a.dout, kElemBytes<SRC>, a.grad, kElemBytes<DST>)) {
        case 8: if constexpr (most == 8) return by_add<SRC, DST, 8>(a, add, stream);
        case 4: return by_add<SRC, DST, 4>(a, add, stream);
        case 2: return by_add<SRC, DST, 2>(a, add, stream);
    }
    return by_add<SRC, DST, 1>(a, add, stream);
}

}  // namespace

namespace {

// One launch instead of three: 2048 tokens, 1000 rows of 64 take 6 to 7 us against 12 to 16, 64 tokens 5 against 8, 8192 tokens,
// 1000 rows of 256 11 to 18 against 18 to 19, 4096 tokens, 8000 rows of 515 15 against 18 to 20.  Not where there is more to add up
// (4096 tokens of 1024 18 us against 17 to 18, 1024 of 4096 15 to 18 against 12 to 16, 8192 of 1024 27 to 30 against 20 to 21),
// where there are more columns than SMs for them (every CTA searches), or where the zeros are what takes the time: the CTAs
// write a piece of a row at a time, single elements where rows start anywhere (one token, 30,000 rows of 515 in bf16: 12 us
// against 8; 30,000 of 1024 11 either way; 100,000 of 64 in fp32 5.6 against 8).
constexpr uint64_t kSmallElements = 3 << 20;

bool small_shape(SmallArgs& a)
{
    a.column_bits = kLeastColumnBits;
    while (a.column_bits < kSmallColumnBits && 1u << a.column_bits < a.dim) ++a.column_bits;
    const uint32_t tiles = (a.dim + (1u << a.column_bits) - 1) >> a.column_bits;
    if (tiles > 148) return false;
    a.groups = 148 / tiles;                             // a CTA to each SM
    if (a.groups > a.rows) a.groups = a.rows;
    a.reciprocal = a.groups > 1 ? (uint32_t)(((1ull << 32) + a.groups - 1) / a.groups) : 0;
    a.key_bits = token_key_bits((a.rows - 1) / a.groups);
    return a.key_bits <= PairWord::kKeyBits;
}

bool small_applies(const TokenIds& ids, uint64_t rows, uint64_t dim, bool add, const void* grad, uint64_t element, SmallArgs& a)
{
    if (ids.count == 0 || ids.count > kSmallTokens || ids.count * dim > kSmallElements || rows > kSmallRows) return false;
    const bool words = (reinterpret_cast<uintptr_t>(grad) | dim * element) % 16 == 0;
    if (!add && rows * dim > (words ? (32u << 20) / element : 4u << 20)) return false;
    a.ids = ids.ptr;
    a.dim = (uint32_t)dim;
    a.tokens = (uint32_t)ids.count;
    a.rows = (uint32_t)rows;
    a.wide = ids.wide;
    return small_shape(a);
}

template <int SRC, int DST, bool ADD> cudaError_t launch_small(const SmallArgs& a, cudaStream_t stream)
{
    static std::atomic<bool> ready[64];                 // per device (zero-initialised)
    const auto bytes = [](uint32_t tokens, int column_bits) { return (small_chunks(tokens) * 2 << column_bits) * 4 + tokens * 4; };
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev].load(std::memory_order_relaxed)) {
        err = cudaFuncSetAttribute(grad_small_kernel<SRC, DST, ADD>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                   (int)bytes(kSmallTokens, kSmallColumnBits));
        if (err != cudaSuccess) return err;
        ready[dev].store(true, std::memory_order_relaxed);
    }
    const uint32_t tiles = (a.dim + (1u << a.column_bits) - 1) >> a.column_bits;
    return launch_pdl_smem(grad_small_kernel<SRC, DST, ADD>, tiles * a.groups, kSortThreads, bytes(a.tokens, a.column_bits), stream, a);
}

template <int SRC, int DST> cudaError_t small_by_add(const SmallArgs& a, bool add, cudaStream_t stream)
{
    return add ? launch_small<SRC, DST, true>(a, stream) : launch_small<SRC, DST, false>(a, stream);
}

}  // namespace

size_t embedding_workspace_floats(uint64_t tokens, uint64_t rows, uint64_t dim)
{
    return tokens == 0 || rows == 0 || dim == 0 ? 0 : (size_t)Layout(tokens, dim).total;
}

cudaError_t launch_embedding_grad(const void* dout, int dout_dtype, const TokenIds& ids, uint64_t rows, uint64_t dim,
                                  float scale, void* grad, int grad_dtype, bool add, float* workspace, cudaStream_t stream)
{
    SmallArgs s = {};
    if (small_applies(ids, rows, dim, add, grad, grad_dtype == kF32 ? 4 : 2, s)) {
        s.dout = dout;
        s.grad = grad;
        s.scale = scale;
        if (dout_dtype == kF32)
            return grad_dtype == kF32 ? small_by_add<kF32, kF32>(s, add, stream) : small_by_add<kF32, kBf16>(s, add, stream);
        return grad_dtype == kF32 ? small_by_add<kBf16, kF32>(s, add, stream) : small_by_add<kBf16, kBf16>(s, add, stream);
    }
    const Layout lay(ids.count, dim);
    uint2* sorted = reinterpret_cast<uint2*>(workspace);
    uint32_t* runs = reinterpret_cast<uint32_t*>(workspace + lay.sorted);
    uint32_t* scratch = runs + lay.runs;
    GradArgs a = {sorted, dout, grad, reinterpret_cast<float4*>(scratch + lay.scratch), runs,
                        reinterpret_cast<uint4*>(runs + 4), (uint32_t)dim, (uint32_t)ids.count, (uint32_t)rows, lay.chunks,
                        lay.chunk_bits, lay.tiles, lay.thread_bits, scale, 0, 0, 0, 0, 0};
    if (ids.count != 0) {
        const cudaError_t err = launch_token_sort(ids, a.rows, sorted, runs, scratch, add ? nullptr : grad,
                                                  dim * (grad_dtype == kF32 ? 4 : 2), &a.zero_from, stream);
        if (err != cudaSuccess) return err;
    }
    if (dout_dtype == kF32)
        return grad_dtype == kF32 ? by_group<kF32, kF32>(a, add, stream) : by_group<kF32, kBf16>(a, add, stream);
    return grad_dtype == kF32 ? by_group<kBf16, kF32>(a, add, stream) : by_group<kBf16, kBf16>(a, add, stream);
}

}  // namespace mqg
