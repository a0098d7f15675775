// Token ids sorted by id: mqg_token_sort.cu.
#pragma once

#include "mqg_training.h"

namespace mqg {

// Bits of the largest key, `rows`.
int token_key_bits(uint32_t rows);

// 32-bit words of scratch memory (8-byte aligned) that the sort needs beside its output.
uint64_t token_sort_words(uint64_t tokens);

// sorted[i] = (key, token): keys ascending, a key's tokens ascending; an id outside 0..rows-1 has the key `rows`.  Sets
// *counter to zero as well and, unless `table` is null, the first *zeroed rows of row_bytes there, as many as take no longer
// than the sort.  At least one token.
cudaError_t launch_token_sort(const TokenIds& ids, uint32_t rows, uint2* sorted, uint32_t* counter, uint32_t* scratch, void* table,
                              uint64_t row_bytes, uint32_t* zeroed, cudaStream_t stream);

// For tests, process-wide: clusters of at most `most` CTAs, a power of two (1: none) up to 16, which is the default.
void set_token_sort_cluster(unsigned most);

}  // namespace mqg
