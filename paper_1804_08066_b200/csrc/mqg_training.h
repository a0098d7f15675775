// Host-side launchers of the operators around the codec: the global norm of many gradient tensors, clipping, AdamW, and the
// table and the layer norm of a model over tokens (arguments already validated by mqg_api_training.cu and mqg_api_model.cu).
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


// Parameters, gradients and states of AdamW, tensor by tensor; scales == nullptr: states in 32 bits.  Host arrays.
struct AdamwList {
    void* const* p;
    const int* p_dtype;
    const void* const* g;
    const int* g_dtype;
    void* const* m;
    void* const* v;
    float* const* scales;
    const uint64_t* size;
    const float* decay;      // nullptr: none
    int count;
};
struct AdamwStep {
    double lr, beta1, beta2, eps;
    uint32_t t;
    uint64_t seed;
    float grad_scale;
    const float* factor;     // on the device; may be nullptr, as the next
    const float* schedule;   // lr, 1 - beta1^t, 1 - beta2^t, t
};
cudaError_t launch_adamw(const AdamwList& list, const AdamwStep& step, cudaStream_t stream);

// Layer norm over rows of `dim` elements.  weight and bias: nullptr = ones, zeros.
struct NormRows {
    const void* x;
    int x_dtype;
    uint64_t rows, dim;
    const void* weight;
    const void* bias;
    int w_dtype;
};
cudaError_t launch_layer_norm(const NormRows& in, float eps, void* y, int y_dtype, float* stats, cudaStream_t stream);
// dx, dweight and dbias may be nullptr.
struct NormGrads {
    void* dx;
    void* dweight;
    void* dbias;
    int dw_dtype;
    bool add;
};
size_t layer_norm_workspace_floats(uint64_t rows, uint64_t dim);
cudaError_t launch_layer_norm_grad(const void* dy, int dy_dtype, const NormRows& in, const float* stats, const NormGrads& out,
                                   float* workspace, cudaStream_t stream);

}  // namespace mqg
