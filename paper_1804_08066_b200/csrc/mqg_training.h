// Host-side launchers of the operators around the codec: the global norm of many gradient tensors, clipping, and the
// table of a model over tokens (arguments already validated by mqg_api_training.cu).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace mqg {

// A list of gradient tensors as the C ABI gets it.
struct TensorList {
    const void* const* ptr;
    const uint64_t* size;
    const int* dtype;
    int count;
};

// Where the clipped tensors go.
enum ClipForm { kMeasureOnly, kInPlace, kFlatten };

size_t norm_workspace_floats(int count);
// The norm of all tensors and the factor that clips it into result[0..1]; then, by `form`, the tensors scaled in place, or
// written one after another into `flat`.
cudaError_t launch_clip(const TensorList& list, float max_norm, ClipForm form, void* flat, int flat_dtype, float* result,
                        float* workspace, cudaStream_t stream);
cudaError_t launch_scale_tensors(const TensorList& list, const float* factor, cudaStream_t stream);
cudaError_t launch_apply_clipped(float* params, const float* acc, float lr, const float* factor, uint64_t n,
                                 cudaStream_t stream);

// The table of a model over tokens: `rows` rows of `dim` elements.
struct TokenIds {
    const void* ptr;
    uint64_t count;
    int wide;                // 64-bit ids
};
cudaError_t launch_embedding(const void* table, int table_dtype, uint64_t rows, uint64_t dim, const TokenIds& ids, float scale,
                             void* out, int out_dtype, cudaStream_t stream);
size_t embedding_workspace_floats(uint64_t tokens, uint64_t rows, uint64_t dim);
cudaError_t launch_embedding_grad(const void* dout, int dout_dtype, const TokenIds& ids, uint64_t rows, uint64_t dim,
                                  float scale, void* grad, int grad_dtype, bool add, float* workspace, cudaStream_t stream);

}  // namespace mqg
