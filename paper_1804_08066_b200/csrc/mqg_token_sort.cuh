// Sorting pairs (key, token) by key within a CTA: the ranking of a warp's pairs, and the sort in shared memory.
#pragma once

#include "mqg_tma.cuh"
#include "mqg_token_sort.h"

namespace mqg {

constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;

// An id as the key it is sorted by: those outside 0..rows-1 go behind all others.
template <typename ID> __device__ __forceinline__ uint32_t key_of(ID id, uint32_t rows)
{
    return id >= 0 && (uint64_t)id < rows ? (uint32_t)id : rows;
}

constexpr int kMaxDigitBits = 10;

// A key of up to 19 bits and one of 8192 tokens in a word.
struct PairWord {
    static constexpr int kTokenBits = 13, kKeyBits = 32 - kTokenBits;
    uint32_t v;
    __device__ __forceinline__ uint32_t key() const { return v >> kTokenBits; }
    __device__ __forceinline__ uint32_t token() const { return v & ((1u << kTokenBits) - 1); }
};
__device__ __forceinline__ uint32_t key_in(const uint2& pair) { return pair.x; }
__device__ __forceinline__ uint32_t key_in(const PairWord& pair) { return pair.key(); }

// The lanes of the warp that hold the same digit, among those that hold a key at all.  (Straight through the digit's bits: with a
// branch at every bit a round of ballots took half as long again.)
__device__ __forceinline__ uint32_t same_digit(uint32_t digit, int bits, uint32_t held)
{
    uint32_t same = held;
    const auto bit = [&](int b) {
        const bool one = (digit & (1u << b)) != 0;
        const uint32_t ones = __ballot_sync(0xFFFFFFFFu, one);
        same &= one ? ones : ~ones;
    };
    switch (bits) {
        case 10: bit(9);
        case 9: bit(8);
        case 8: bit(7);
        case 7: bit(6);
        case 6: bit(5);
        case 5: bit(4);
        case 4: bit(3);
        case 3: bit(2);
        case 2: bit(1);
        default: bit(0);
    }
    return same;
}

// This thread's pairs of the ids, `first` and every 32nd behind it; returns a bit for each that exists.
template <typename ID, int K>
__device__ __forceinline__ uint32_t load_pairs(const ID* ids, uint32_t tokens, uint32_t rows, uint32_t first, uint2 (&pair)[K])
{
    uint32_t held = 0;
#pragma unroll
    for (int r = 0; r < K; ++r) {
        const uint32_t i = first + r * 32;
        pair[r] = make_uint2(0, i);
        if (i < tokens) {
            held |= 1u << r;
            pair[r].x = key_of(__ldg(ids + i), rows);
        }
    }
    return held;
}

// Ranks a warp's pairs, 32 at a time: rank[r] = how many of the warp's pairs with the same digit stand before this one;
// count[digit] = how many the warp has.  `held`: a bit for each r.
template <int K, typename Pair>
__device__ __forceinline__ void rank_pairs(const Pair (&pair)[K], uint32_t held, int shift, int bits, uint16_t* count, uint32_t (&rank)[K])
{
    const uint32_t lane = threadIdx.x & 31, mask = (1u << bits) - 1;
    uint32_t there[K];
#pragma unroll
    for (int r = 0; r < K; ++r) {
        there[r] = __ballot_sync(0xFFFFFFFFu, (held >> r) & 1u);
        rank[r] = there[r] == 0 ? 0 : same_digit((key_in(pair[r]) >> shift) & mask, bits, there[r]);
    }
#pragma unroll
    for (int r = 0; r < K; ++r) {
        if (there[r] == 0) continue;
        const uint32_t digit = (key_in(pair[r]) >> shift) & mask, same = rank[r], so_far = count[digit];
        __syncwarp();
        if (((held >> r) & 1u) && (same >> lane) == 1u) count[digit] = (uint16_t)(so_far + __popc(same));
        __syncwarp();
        rank[r] = so_far + __popc(same & ((1u << lane) - 1));
    }
}

__device__ __forceinline__ uint32_t sum_up_to_lane(uint32_t v)
{
#pragma unroll
    for (int step = 1; step < 32; step *= 2) {
        const uint32_t before = __shfl_up_sync(0xFFFFFFFFu, v, step);
        if ((threadIdx.x & 31) >= (uint32_t)step) v += before;
    }
    return v;
}

constexpr int kSmallBits = 6;                           // of a digit at most (1024 tokens of 16-bit ids: 6.8 us; digits of 8 bits, in two passes, 13.1)
struct SmallSort {
    uint16_t count[kSortWarps][(1 << kSmallBits) + 2];  // (a column is read by a warp: no two of its words in one bank)
    uint32_t total[1 << kSmallBits];
};

// This thread's pairs of n in shared memory.
template <int K, typename Pair>
__device__ __forceinline__ uint32_t take_pairs(Pair (&pair)[K], const Pair* pairs, uint32_t n)
{
    const uint32_t local = (threadIdx.x >> 5) * (32 * K) + (threadIdx.x & 31);
    uint32_t held = 0;
#pragma unroll
    for (int r = 0; r < K; ++r) {
        if (local + r * 32 >= n) continue;
        pair[r] = pairs[local + r * 32];
        held |= 1u << r;
    }
    return held;
}

// n pairs, of which `held` are this thread's; the sorted ones are in `pairs`, in shared memory, at the end.
template <int K, typename Pair>
__device__ __forceinline__ void sort_in_cta(Pair (&pair)[K], uint32_t held, uint32_t n, int bits, SmallSort& s, Pair* pairs)
{
    const uint32_t lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int passes = (bits + kSmallBits - 1) / kSmallBits, digit_bits = (bits + passes - 1) / passes, bins = 1 << digit_bits;
    for (int shift = 0; shift < bits; shift += digit_bits) {
        if (shift != 0) held = take_pairs<K>(pair, pairs, n);
        for (int i = lane; i < (bins + 1) / 2; i += 32) reinterpret_cast<uint32_t*>(s.count[w])[i] = 0;
        __syncwarp();
        uint32_t rank[K];
        rank_pairs<K>(pair, held, shift, digit_bits, s.count[w], rank);
        __syncthreads();
#pragma unroll 4
        for (int d = w; d < bins; d += kSortWarps) {    // a warp takes a digit, a lane the count of a warp
            const uint32_t c = s.count[lane][d], sum = sum_up_to_lane(c);
            s.count[lane][d] = (uint16_t)(sum - c);
            if (lane == 31) s.total[d] = sum;
        }
        __syncthreads();
        // every warp adds the digits' first places to its own counts, neighbouring digits to a lane
        const int per = (bins + 31) / 32;
        uint32_t total = 0;
        for (int i = 0; i < per; ++i)
            if ((int)lane * per + i < bins) total += s.total[lane * per + i];
        uint32_t at = sum_up_to_lane(total) - total;
        for (int i = 0; i < per; ++i) {
            if ((int)lane * per + i >= bins) break;
            s.count[w][lane * per + i] += (uint16_t)at;
            at += s.total[lane * per + i];
        }
        __syncwarp();
#pragma unroll
        for (int r = 0; r < K; ++r) {
            const uint32_t digit = (key_in(pair[r]) >> shift) & (bins - 1);
            if ((held >> r) & 1u) pairs[s.count[w][digit] + rank[r]] = pair[r];
        }
        __syncthreads();
    }
}

}  // namespace mqg
