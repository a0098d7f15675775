// Token ids sorted by id: mqg_token_sort.cu.
#pragma once

#include "mqg_training.h"

namespace mqg {

// Bits of the largest key, `rows`.
int token_key_bits(uint32_t rows);

// 32-bit words of scratch memory (8-byte aligned) that the sort needs beside its output.
uint64_t token_sort_words(uint64_t tokens, uint64_t rows);

// sorted[i] = (key, token): keys ascending, a key's tokens ascending; an id outside 0..rows-1 has the key `rows`.  Sets
// *counter to zero as well and, unless `zero` is null, of the `rows` rows of row_bytes there those that no token has (others may
// be set to zero, too).
cudaError_t launch_token_sort(const TokenIds& ids, uint32_t rows, uint2* sorted, uint32_t* counter, uint32_t* scratch,
                              void* zero, uint64_t row_bytes, cudaStream_t stream);

}  // namespace mqg
