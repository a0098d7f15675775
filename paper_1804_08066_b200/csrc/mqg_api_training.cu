// C ABI of the operators around the codec: argument checks and dispatch to the launchers of mqg_training.h.
#include <cmath>

#include "../../include/mqgrad.h"
#include "mqg_internal.h"
#include "mqg_token_sort.h"
#include "mqg_training.h"

namespace {

using mqg::report_error;

constexpr uint64_t kMaxRows = 0x7FFFFFFF, kMaxDim = 1u << 22;

bool aligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
bool known(mqg_dtype t) { return t == MQG_F32 || t == MQG_BF16; }
uintptr_t bytes_of(mqg_dtype t) { return t == MQG_F32 ? 4 : 2; }
uintptr_t bytes_of(mqg_index t) { return t == MQG_I64 ? 8 : 4; }

mqg_status cuda_status(const char* what, cudaError_t err)
{
    return err == cudaSuccess ? MQG_OK : report_error(MQG_ERR_CUDA, "%s: %s", what, cudaGetErrorString(err));
}

// Memory that a call reads or writes; `bytes` = 0: none.
struct Region {
    const char* name;
    const void* p;
    uint64_t bytes;
    bool meets(const Region& r) const
    {
        const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(r.p);
        return bytes != 0 && r.bytes != 0 && (a < b ? b - a < bytes : a - b < r.bytes);
    }
};

// Whether what is written shares memory with anything else: MQG_OK if not.
template <int N> mqg_status check_apart(const char* what, const Region& written, const Region (&others)[N])
{
    for (const Region& r : others)
        if (written.meets(r)) return report_error(MQG_ERR_INVALID, "%s: %s and %s share memory", what, written.name, r.name);
    return MQG_OK;
}

template <int N>
mqg_status check_list_apart(const char* what, const void* const* grads, const uint64_t* sizes, const mqg_dtype* dtypes, int count,
                            const Region (&others)[N])
{
    for (int j = 0; j < count; ++j) {
        const Region tensor = {"", grads[j], sizes[j] * bytes_of(dtypes[j])};
        for (const Region& r : others)
            if (tensor.meets(r)) return report_error(MQG_ERR_INVALID, "%s: tensor %d and %s share memory", what, j, r.name);
    }
    return MQG_OK;
}

// A list of tensors.  A launch counts its 16 KB tiles in 32 bits, so a list holds less than 2^44 bytes.
mqg_status check_list(const char* what, const void* const* grads, const uint64_t* sizes, const mqg_dtype* dtypes, int count)
{
    if (count < 0) return report_error(MQG_ERR_INVALID, "%s: count = %d is negative", what, count);
    if (count == 0) return MQG_OK;
    if (!grads || !sizes || !dtypes) return report_error(MQG_ERR_INVALID, "%s: grads, sizes or dtypes is null", what);
    uint64_t bytes = 0;
    for (int j = 0; j < count; ++j) {
        if (!known(dtypes[j])) return report_error(MQG_ERR_INVALID, "%s: unknown dtype %d of tensor %d", what, (int)dtypes[j], j);
        if (sizes[j] == 0) continue;
        if (!grads[j]) return report_error(MQG_ERR_INVALID, "%s: tensor %d is null", what, j);
        if (!aligned(grads[j], bytes_of(dtypes[j])))
            return report_error(MQG_ERR_ALIGN, "%s: tensor %d is not aligned to its elements", what, j);
        if (sizes[j] >= (1ull << 42) || (bytes += sizes[j] * 4) >= (1ull << 44))
            return report_error(MQG_ERR_INVALID, "%s: the tensors hold more than 2^44 bytes", what);
    }
    return MQG_OK;
}

mqg_status check_norm(const char* what, int count, float max_norm, const float* result, const float* workspace,
                      size_t workspace_floats)
{
    if (!(max_norm >= 0.0f)) return report_error(MQG_ERR_INVALID, "%s: max_norm = %g is negative or NaN", what, (double)max_norm);
    if (!result) return report_error(MQG_ERR_INVALID, "%s: result is null", what);
    if (!aligned(result, 4)) return report_error(MQG_ERR_ALIGN, "%s: result not 4-byte aligned", what);
    const size_t need = mqg_norm_workspace_floats(count);
    if (workspace_floats < need)
        return report_error(MQG_ERR_INVALID, "%s: workspace holds %llu floats, %llu needed (mqg_norm_workspace_floats)", what,
                            (unsigned long long)workspace_floats, (unsigned long long)need);
    if (!workspace) return report_error(MQG_ERR_INVALID, "%s: workspace is null", what);
    if (!aligned(workspace, 8)) return report_error(MQG_ERR_ALIGN, "%s: workspace not 8-byte aligned", what);
    return MQG_OK;
}

// What a call that measures writes lies apart: `flat`, if there is one, the result and the workspace.
mqg_status check_norm_apart(const char* what, const void* const* grads, const uint64_t* sizes, const mqg_dtype* dtypes, int count,
                            const float* result, const float* workspace, const Region& flat = {"flat", nullptr, 0})
{
    const Region out = {"result", result, 8}, scratch = {"workspace", workspace, mqg_norm_workspace_floats(count) * 4};
    if (mqg_status st = check_apart(what, out, {scratch})) return st;
    if (mqg_status st = check_apart(what, flat, {out, scratch})) return st;
    return check_list_apart(what, grads, sizes, dtypes, count, {out, scratch, flat});
}

mqg::TensorList list_of(const void* const* grads, const uint64_t* sizes, const mqg_dtype* dtypes, int count)
{
    static_assert(sizeof(mqg_dtype) == sizeof(int), "the list's types are passed on as int");
    return {grads, sizes, reinterpret_cast<const int*>(dtypes), count};
}

mqg_status check_table(const char* what, uint64_t rows, uint64_t dim, uint64_t tokens, const void* ids, mqg_index ids_type)
{
    if (rows > kMaxRows || tokens > kMaxRows)
        return report_error(MQG_ERR_INVALID, "%s: %llu rows, %llu tokens: at most 2^31 - 1 of each", what,
                            (unsigned long long)rows, (unsigned long long)tokens);
    if (dim > kMaxDim) return report_error(MQG_ERR_INVALID, "%s: dim = %llu is above 2^22", what, (unsigned long long)dim);
    if (ids_type != MQG_I32 && ids_type != MQG_I64) return report_error(MQG_ERR_INVALID, "%s: unknown index type %d", what, (int)ids_type);
    if (tokens != 0 && dim != 0) {
        if (!ids) return report_error(MQG_ERR_INVALID, "%s: ids is null", what);
        if (!aligned(ids, bytes_of(ids_type))) return report_error(MQG_ERR_ALIGN, "%s: ids not aligned", what);
    }
    return MQG_OK;
}

mqg_status check_buffer(const char* what, const char* name, const void* p, mqg_dtype t, bool empty)
{
    if (!known(t)) return report_error(MQG_ERR_INVALID, "%s: unknown dtype %d of %s", what, (int)t, name);
    if (empty) return MQG_OK;
    if (!p) return report_error(MQG_ERR_INVALID, "%s: %s is null", what, name);
    if (!aligned(p, bytes_of(t))) return report_error(MQG_ERR_ALIGN, "%s: %s is not aligned to its elements", what, name);
    return MQG_OK;
}

}  // namespace

extern "C" {

size_t mqg_norm_workspace_floats(int count) { return mqg::norm_workspace_floats(count); }

mqg_status mqg_grad_norm(const void* const* grads, const uint64_t* sizes, const mqg_dtype* dtypes, int count, float max_norm,
                         float* result, float* workspace, size_t workspace_floats, void* cuda_stream)
{
    const char* what = "mqg_grad_norm";
    if (mqg_status st = check_list(what, grads, sizes, dtypes, count)) return st;
    if (mqg_status st = check_norm(what, count, max_norm, result, workspace, workspace_floats)) return st;
    if (mqg_status st = check_norm_apart(what, grads, sizes, dtypes, count, result, workspace)) return st;
    return cuda_status(what, mqg::launch_clip(list_of(grads, sizes, dtypes, count), max_norm, mqg::kMeasureOnly, nullptr, 0,
                                              result, workspace, static_cast<cudaStream_t>(cuda_stream)));
}

mqg_status mqg_clip_grad_norm(void* const* grads, const uint64_t* sizes, const mqg_dtype* dtypes, int count, float max_norm,
                              float* result, float* workspace, size_t workspace_floats, void* cuda_stream)
{
    const char* what = "mqg_clip_grad_norm";
    if (mqg_status st = check_list(what, grads, sizes, dtypes, count)) return st;
    if (mqg_status st = check_norm(what, count, max_norm, result, workspace, workspace_floats)) return st;
    if (mqg_status st = check_norm_apart(what, grads, sizes, dtypes, count, result, workspace)) return st;
    return cuda_status(what, mqg::launch_clip(list_of(grads, sizes, dtypes, count), max_norm, mqg::kInPlace, nullptr, 0,
                                              result, workspace, static_cast<cudaStream_t>(cuda_stream)));
}

mqg_status mqg_clip_flatten(const void* const* grads, const uint64_t* sizes, const mqg_dtype* dtypes, int count,
                            float max_norm, void* flat, mqg_dtype flat_dtype, float* result, float* workspace,
                            size_t workspace_floats, void* cuda_stream)
{
    const char* what = "mqg_clip_flatten";
    if (mqg_status st = check_list(what, grads, sizes, dtypes, count)) return st;
    if (mqg_status st = check_norm(what, count, max_norm, result, workspace, workspace_floats)) return st;
    uint64_t total = 0;
    for (int j = 0; j < count; ++j) total += sizes[j];
    if (mqg_status st = check_buffer(what, "flat", flat, flat_dtype, total == 0)) return st;
    const Region to = {"flat", flat, total * bytes_of(flat_dtype)};
    if (mqg_status st = check_norm_apart(what, grads, sizes, dtypes, count, result, workspace, to)) return st;
    return cuda_status(what, mqg::launch_clip(list_of(grads, sizes, dtypes, count), max_norm, mqg::kFlatten, flat,
                                              (int)flat_dtype, result, workspace, static_cast<cudaStream_t>(cuda_stream)));
}

mqg_status mqg_scale_grads(void* const* grads, const uint64_t* sizes, const mqg_dtype* dtypes, int count, const float* factor,
                           void* cuda_stream)
{
    const char* what = "mqg_scale_grads";
    if (mqg_status st = check_list(what, grads, sizes, dtypes, count)) return st;
    if (mqg_status st = check_buffer(what, "factor", factor, MQG_F32, false)) return st;
    if (mqg_status st = check_list_apart(what, grads, sizes, dtypes, count, {{"factor", factor, 4}})) return st;
    return cuda_status(what, mqg::launch_scale_tensors(list_of(grads, sizes, dtypes, count), factor,
                                                       static_cast<cudaStream_t>(cuda_stream)));
}

mqg_status mqg_apply_clipped(float* params, const float* acc, float lr, const float* factor, uint64_t n, void* cuda_stream)
{
    const char* what = "mqg_apply_clipped";
    if (n == 0) return MQG_OK;
    if (!params || !acc) return report_error(MQG_ERR_INVALID, "%s: params or acc is null", what);
    if (!aligned(params, 16) || !aligned(acc, 16)) return report_error(MQG_ERR_ALIGN, "%s: params or acc not 16-byte aligned", what);
    if (mqg_status st = check_buffer(what, "factor", factor, MQG_F32, false)) return st;
    const Region from = {"acc", acc, params == acc ? 0 : n * 4};         // (every element is read before it is written)
    if (mqg_status st = check_apart(what, {"params", params, n * 4}, {from, {"factor", factor, 4}})) return st;
    return cuda_status(what, mqg::launch_apply_clipped(params, acc, lr, factor, n, static_cast<cudaStream_t>(cuda_stream)));
}

mqg_status mqg_embedding(const void* table, mqg_dtype table_dtype, uint64_t rows, uint64_t dim, const void* ids,
                         mqg_index ids_type, uint64_t tokens, float scale, void* out, mqg_dtype out_dtype, void* cuda_stream)
{
    const char* what = "mqg_embedding";
    const bool empty = tokens == 0 || dim == 0;
    if (mqg_status st = check_table(what, rows, dim, tokens, ids, ids_type)) return st;
    if (mqg_status st = check_buffer(what, "table", table, table_dtype, empty || rows == 0)) return st;
    if (mqg_status st = check_buffer(what, "out", out, out_dtype, empty)) return st;
    if (empty) return MQG_OK;
    const Region written = {"out", out, tokens * dim * bytes_of(out_dtype)};
    if (mqg_status st = check_apart(what, written, {{"table", table, rows * dim * bytes_of(table_dtype)},
                                                    {"ids", ids, tokens * bytes_of(ids_type)}})) return st;
    return cuda_status(what, mqg::launch_embedding(table, (int)table_dtype, rows, dim, {ids, tokens, ids_type == MQG_I64}, scale,
                                                   out, (int)out_dtype, static_cast<cudaStream_t>(cuda_stream)));
}

size_t mqg_embedding_workspace_floats(uint64_t tokens, uint64_t rows, uint64_t dim)
{
    if (tokens > kMaxRows || rows > kMaxRows || dim > kMaxDim) return 0;
    return mqg::embedding_workspace_floats(tokens, rows, dim);
}

mqg_status mqg_embedding_grad(const void* dout, mqg_dtype dout_dtype, const void* ids, mqg_index ids_type, uint64_t tokens,
                              uint64_t rows, uint64_t dim, float scale, void* grad, mqg_dtype grad_dtype, int add_into_grad,
                              float* workspace, size_t workspace_floats, void* cuda_stream)
{
    const char* what = "mqg_embedding_grad";
    if (mqg_status st = check_table(what, rows, dim, tokens, ids, ids_type)) return st;
    const bool nothing = rows == 0 || dim == 0 || (tokens == 0 && add_into_grad);
    if (mqg_status st = check_buffer(what, "dout", dout, dout_dtype, nothing || tokens == 0)) return st;
    if (mqg_status st = check_buffer(what, "grad", grad, grad_dtype, nothing)) return st;
    if (nothing) return MQG_OK;
    const size_t need = mqg::embedding_workspace_floats(tokens, rows, dim);
    if (workspace_floats < need)
        return report_error(MQG_ERR_INVALID, "%s: workspace holds %llu floats, %llu needed (mqg_embedding_workspace_floats)",
                            what, (unsigned long long)workspace_floats, (unsigned long long)need);
    if (need != 0 && !workspace) return report_error(MQG_ERR_INVALID, "%s: workspace is null", what);
    if (!aligned(workspace, 16)) return report_error(MQG_ERR_ALIGN, "%s: workspace not 16-byte aligned", what);
    const Region from = {"dout", dout, tokens * dim * bytes_of(dout_dtype)}, by = {"ids", ids, tokens * bytes_of(ids_type)};
    const Region written = {"grad", grad, rows * dim * bytes_of(grad_dtype)}, scratch = {"workspace", workspace, need * 4};
    if (mqg_status st = check_apart(what, written, {from, by, scratch})) return st;
    if (mqg_status st = check_apart(what, scratch, {from, by})) return st;
    return cuda_status(what, mqg::launch_embedding_grad(dout, (int)dout_dtype, {ids, tokens, ids_type == MQG_I64}, rows, dim,
                                                        scale, grad, (int)grad_dtype, add_into_grad != 0, workspace,
                                                        static_cast<cudaStream_t>(cuda_stream)));
}

mqg_status mqg_test_sort_cluster(uint32_t most_ctas)
{
    if (most_ctas == 0) most_ctas = 16;
    if (most_ctas > 16 || (most_ctas & (most_ctas - 1)) != 0)
        return report_error(MQG_ERR_INVALID, "mqg_test_sort_cluster: %u is no power of two up to 16", most_ctas);
    mqg::set_token_sort_cluster(most_ctas);
    return MQG_OK;
}

}  // extern "C"
