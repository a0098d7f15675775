// Token ids sorted by id: mqg_token_sort.cu.
#pragma once

#include "mqg_training.h"

namespace mqg {

// 32-bit words of scratch memory (8-byte aligned) that the sort needs beside its output.
uint64_t token_sort_words(uint64_t tokens);

// sorted[i] = (key, token): keys ascending, a key's tokens ascending; an id outside 0..rows-1 has the key `rows`.  Sets
// *counter and `zero_bytes` bytes at `zero` to zero as well.
cudaError_t launch_token_sort(const TokenIds& ids, uint32_t rows, uint2* sorted, uint32_t* counter, uint32_t* scratch,
                              void* zero, uint64_t zero_bytes, cudaStream_t stream);

}  // namespace mqg
