// C ABI of AdamW over many tensors and of the layer norm: argument checks and dispatch to the launchers of mqg_training.h.
#include <algorithm>
#include <cmath>
#include <exception>
#include <vector>

#include "mqg_checks.h"
#include "mqg_training.h"

namespace {

using namespace mqg;

constexpr uint64_t kMaxRows = 0x7FFFFFFF, kMaxDim = 1u << 22;
constexpr uint64_t kStateBlock = 256;

uint64_t state_blocks(uint64_t n) { return n / kStateBlock + (n % kStateBlock != 0); }

// One of the lists of a call: where its buffers are and how long.
struct BufferList {
    const char* name;
    const void* const* ptr;
    const mqg_dtype* dtype;                             // of the elements; nullptr: `unit` bytes each
    uint64_t unit;                                      // 0: two floats to a block of elements
    bool written;

    uint64_t bytes(const uint64_t* sizes, int j) const
    {
        return dtype ? sizes[j] * bytes_of(dtype[j]) : unit ? sizes[j] * unit : state_blocks(sizes[j]) * 8;
    }
};

// What a look at every buffer of a call finds, without a branch for each: a reason to look closely, or none.  Lists of slices of
// one vector each, in its order, are seen to share no memory.
template <int N>
bool plainly_good(const BufferList (&lists)[N], const uint64_t* sizes, const float* decays, int count, const Region (&scalars)[2])
{
    struct Span { uintptr_t from, to; };
    Span span[N];
    for (Span& s : span) s = {~(uintptr_t)0, 0};
    uint64_t total = 0;
    bool bad = false;
    for (int j = 0; j < count; ++j) {
        const uint64_t n = sizes[j];
        bad |= n >= (1ull << 42) || (unsigned)lists[0].dtype[j] > 1u || (unsigned)lists[1].dtype[j] > 1u;
        bad |= decays != nullptr && !(decays[j] >= 0.0f && decays[j] <= 3.4e38f);
        total += n;
        if (n == 0) continue;
        bad |= total >= (1ull << 42);
        for (int k = 0; k < N; ++k) {
            const BufferList& l = lists[k];
            const uintptr_t p = reinterpret_cast<uintptr_t>(l.ptr[j]);
            const unsigned shift = k < 2 ? 2u - (unsigned)(lists[k].dtype[j] & 1) : k < 4 && l.unit == 1 ? 0u : 2u;
            const uint64_t bytes = k < 4 ? n << shift : state_blocks(n) * 8;
            bad |= p == 0 || (p & ((1u << shift) - 1)) != 0 || (l.written && p < span[k].to);
            span[k].from = std::min(span[k].from, p);
            span[k].to = std::max(span[k].to, p + bytes);
        }
    }
    for (int k = 0; k < N; ++k) {
        for (int i = 0; i < k; ++i)
            bad |= (lists[k].written || lists[i].written) && span[k].from < span[i].to && span[i].from < span[k].to;
        for (const Region& r : scalars) {
            const uintptr_t p = reinterpret_cast<uintptr_t>(r.p);
            bad |= lists[k].written && r.bytes != 0 && span[k].from < p + r.bytes && p < span[k].to;
        }
    }
    return !bad;
}

// Whether everything that is written shares no memory with anything else: the buffers in the order of their addresses.
mqg_status check_lists_apart(const char* what, const BufferList* lists, int nlists, const uint64_t* sizes, int count,
                             const Region (&scalars)[2])
{
    struct Piece { uintptr_t from, to; int list, tensor; };
    std::vector<Piece> pieces;
    pieces.reserve((size_t)nlists * count + 2);
    for (int k = 0; k < nlists; ++k)
        for (int j = 0; j < count; ++j) {
            const uintptr_t p = reinterpret_cast<uintptr_t>(lists[k].ptr[j]);
            if (const uint64_t n = lists[k].bytes(sizes, j)) pieces.push_back({p, p + n, k, j});
        }
    for (int i = 0; i < 2; ++i)
        if (scalars[i].bytes != 0) {
            const uintptr_t p = reinterpret_cast<uintptr_t>(scalars[i].p);
            pieces.push_back({p, p + scalars[i].bytes, nlists + i, -1});
        }
    std::sort(pieces.begin(), pieces.end(), [](const Piece& a, const Piece& b) { return a.from < b.from; });
    const auto written = [&](const Piece& p) { return p.list < nlists && lists[p.list].written; };
    const auto name = [&](const Piece& p) { return p.list < nlists ? lists[p.list].name : scalars[p.list - nlists].name; };
    const Piece *last = nullptr, *last_written = nullptr;           // of those so far, the ones that reach furthest
    for (const Piece& p : pieces) {
        const Piece* other = written(p) ? last : last_written;
        if (other && other->to > p.from)
            return report_error(MQG_ERR_INVALID, "%s: %s (tensor %d) and %s (tensor %d) share memory", what, name(*other), other->tensor,
                                name(p), p.tensor);
        if (!last || p.to > last->to) last = &p;
        if (written(p) && (!last_written || p.to > last_written->to)) last_written = &p;
    }
    return MQG_OK;
}

template <int N>
mqg_status check_adamw(const char* what, const BufferList (&lists)[N], const uint64_t* sizes, const float* decays, int count,
                       const AdamwStep& s)
{
    if (count < 0) return report_error(MQG_ERR_INVALID, "%s: count = %d is negative", what, count);
    if (!(s.lr >= 0.0 && s.lr <= 3.4e38)) return report_error(MQG_ERR_INVALID, "%s: lr = %g is not a finite number from 0 on", what, s.lr);
    for (const double beta : {s.beta1, s.beta2})
        if (!(beta >= 0.0 && (float)beta < 1.0f))
            return report_error(MQG_ERR_INVALID, "%s: beta = %.9g is outside [0, 1) in fp32", what, beta);
    if (!(s.eps >= 0x1p-50 && s.eps <= 3.4e38))
        return report_error(MQG_ERR_INVALID, "%s: eps = %g is not a finite number from 2^-50 on", what, s.eps);
    if (!std::isfinite(s.grad_scale)) return report_error(MQG_ERR_INVALID, "%s: grad_scale is not finite", what);
    if (s.t == 0 && !s.schedule) return report_error(MQG_ERR_INVALID, "%s: step counts from 1", what);
    if (!aligned(s.factor, 4) || !aligned(s.schedule, 4)) return report_error(MQG_ERR_ALIGN, "%s: factor or schedule not 4-byte aligned", what);
    if (count == 0) return MQG_OK;
    if (!sizes) return report_error(MQG_ERR_INVALID, "%s: sizes is null", what);
    for (int k = 0; k < N; ++k)
        if (!lists[k].ptr) return report_error(MQG_ERR_INVALID, "%s: %s is null", what, lists[k].name);
    const Region scalars[2] = {{"factor", s.factor, s.factor ? 4u : 0u}, {"schedule", s.schedule, s.schedule ? 16u : 0u}};
    if (plainly_good(lists, sizes, decays, count, scalars)) return MQG_OK;
    uint64_t total = 0;
    for (int j = 0; j < count; ++j) {
        for (int k = 0; k < 2; ++k)
            if (!known(lists[k].dtype[j]))
                return report_error(MQG_ERR_INVALID, "%s: unknown dtype %d of %s, tensor %d", what, (int)lists[k].dtype[j], lists[k].name, j);
        if (decays && !(decays[j] >= 0.0f && decays[j] <= 3.4e38f))
            return report_error(MQG_ERR_INVALID, "%s: decay %g of tensor %d is not a finite number from 0 on", what, (double)decays[j], j);
        if (sizes[j] == 0) continue;
        if (sizes[j] >= (1ull << 42) || (total += sizes[j]) >= (1ull << 42))
            return report_error(MQG_ERR_INVALID, "%s: the tensors hold 2^42 elements or more", what);
        for (int k = 0; k < N; ++k) {
            const BufferList& l = lists[k];
            if (!l.ptr[j]) return report_error(MQG_ERR_INVALID, "%s: %s, tensor %d is null", what, l.name, j);
            if (!aligned(l.ptr[j], l.dtype ? bytes_of(l.dtype[j]) : l.unit ? l.unit : 4))
                return report_error(MQG_ERR_ALIGN, "%s: %s, tensor %d is not aligned to its elements", what, l.name, j);
        }
    }
    return check_lists_apart(what, lists, N, sizes, count, scalars);
}

template <int N>
mqg_status run_adamw(const char* what, const BufferList (&lists)[N], const AdamwList& list, const AdamwStep& step, void* stream)
{
    static_assert(sizeof(mqg_dtype) == sizeof(int), "the lists' types are passed on as int");
    try {
        if (mqg_status st = check_adamw(what, lists, list.size, list.decay, list.count, step)) return st;
    } catch (const std::exception& e) {                 // no memory to sort the list in
        return report_error(MQG_ERR_INVALID, "%s: %s", what, e.what());
    }
    return cuda_status(what, launch_adamw(list, step, static_cast<cudaStream_t>(stream)));
}

const int* as_int(const mqg_dtype* t) { return reinterpret_cast<const int*>(t); }

mqg_status check_rows(const char* what, uint64_t rows, uint64_t dim)
{
    if (rows > kMaxRows) return report_error(MQG_ERR_INVALID, "%s: %llu rows: at most 2^31 - 1", what, (unsigned long long)rows);
    if (dim > kMaxDim) return report_error(MQG_ERR_INVALID, "%s: dim = %llu is above 2^22", what, (unsigned long long)dim);
    return MQG_OK;
}

// A buffer that may be left out.
mqg_status check_optional(const char* what, const char* name, const void* p, mqg_dtype t)
{
    return check_buffer(what, name, p, t, p == nullptr);
}

}  // namespace

extern "C" {

size_t mqg_adamw8_scale_floats(uint64_t n) { return (size_t)(2 * state_blocks(n)); }

mqg_status mqg_adamw(void* const* params, const mqg_dtype* param_dtypes, const void* const* grads, const mqg_dtype* grad_dtypes,
                     float* const* m, float* const* v, const uint64_t* sizes, const float* decays, int count, double lr, double beta1,
                     double beta2, double eps, uint32_t step, float grad_scale, const float* factor, const float* schedule,
                     void* cuda_stream)
{
    const char* what = "mqg_adamw";
    if (count > 0 && (!param_dtypes || !grad_dtypes)) return report_error(MQG_ERR_INVALID, "%s: param_dtypes or grad_dtypes is null", what);
    void* const* states[2] = {reinterpret_cast<void* const*>(m), reinterpret_cast<void* const*>(v)};
    const BufferList lists[4] = {{"params", params, param_dtypes, 0, true},
                                 {"grads", grads, grad_dtypes, 0, false},
                                 {"m", states[0], nullptr, 4, true},
                                 {"v", states[1], nullptr, 4, true}};
    const AdamwList list = {params, as_int(param_dtypes), grads, as_int(grad_dtypes), states[0], states[1], nullptr, sizes, decays, count};
    return run_adamw(what, lists, list, {lr, beta1, beta2, eps, step, 0, grad_scale, factor, schedule}, cuda_stream);
}

mqg_status mqg_adamw8(void* const* params, const mqg_dtype* param_dtypes, const void* const* grads, const mqg_dtype* grad_dtypes,
                      uint8_t* const* m, uint8_t* const* v, float* const* scales, const uint64_t* sizes, const float* decays, int count,
                      double lr, double beta1, double beta2, double eps, uint32_t step, uint64_t seed, float grad_scale,
                      const float* factor, const float* schedule, void* cuda_stream)
{
    const char* what = "mqg_adamw8";
    if (count > 0 && (!param_dtypes || !grad_dtypes)) return report_error(MQG_ERR_INVALID, "%s: param_dtypes or grad_dtypes is null", what);
    if (count > 0 && !scales) return report_error(MQG_ERR_INVALID, "%s: scales is null", what);
    void* const* states[2] = {reinterpret_cast<void* const*>(m), reinterpret_cast<void* const*>(v)};
    const BufferList lists[5] = {{"params", params, param_dtypes, 0, true},
                                 {"grads", grads, grad_dtypes, 0, false},
                                 {"m", states[0], nullptr, 1, true},
                                 {"v", states[1], nullptr, 1, true},
                                 {"scales", reinterpret_cast<void* const*>(scales), nullptr, 0, true}};
    const AdamwList list = {params, as_int(param_dtypes), grads, as_int(grad_dtypes), states[0], states[1], scales, sizes, decays, count};
    return run_adamw(what, lists, list, {lr, beta1, beta2, eps, step, seed, grad_scale, factor, schedule}, cuda_stream);
}

mqg_status mqg_layer_norm(const void* x, mqg_dtype x_dtype, uint64_t rows, uint64_t dim, const void* weight, const void* bias,
                          mqg_dtype weight_dtype, float eps, void* y, mqg_dtype y_dtype, float* stats, void* cuda_stream)
{
    const char* what = "mqg_layer_norm";
    const bool empty = rows == 0 || dim == 0;
    if (mqg_status st = check_rows(what, rows, dim)) return st;
    if (!(eps > 0.0f && std::isfinite(eps))) return report_error(MQG_ERR_INVALID, "%s: eps = %g is not a finite number above 0", what, (double)eps);
    if (mqg_status st = check_buffer(what, "x", x, x_dtype, empty)) return st;
    if (mqg_status st = check_buffer(what, "y", y, y_dtype, empty)) return st;
    if (mqg_status st = check_optional(what, "weight", weight, weight_dtype)) return st;
    if (mqg_status st = check_optional(what, "bias", bias, weight_dtype)) return st;
    if (mqg_status st = check_optional(what, "stats", stats, MQG_F32)) return st;
    if (empty) return MQG_OK;
    const Region from = {"x", x, rows * dim * bytes_of(x_dtype)}, to = {"y", y, rows * dim * bytes_of(y_dtype)};
    const Region w = {"weight", weight, weight ? dim * bytes_of(weight_dtype) : 0}, b = {"bias", bias, bias ? dim * bytes_of(weight_dtype) : 0};
    const Region kept = {"stats", stats, stats ? rows * 8 : 0};
    if (mqg_status st = check_apart(what, to, {from, w, b, kept})) return st;
    if (mqg_status st = check_apart(what, kept, {from, w, b})) return st;
    const NormRows in = {x, (int)x_dtype, rows, dim, weight, bias, (int)weight_dtype};
    return cuda_status(what, launch_layer_norm(in, eps, y, (int)y_dtype, stats, static_cast<cudaStream_t>(cuda_stream)));
}

size_t mqg_layer_norm_workspace_floats(uint64_t rows, uint64_t dim)
{
    if (rows > kMaxRows || dim > kMaxDim) return 0;
    return layer_norm_workspace_floats(rows, dim);
}

mqg_status mqg_layer_norm_grad(const void* dy, mqg_dtype dy_dtype, const void* x, mqg_dtype x_dtype, uint64_t rows, uint64_t dim,
                               const void* weight, mqg_dtype weight_dtype, const float* stats, void* dx, void* dweight, void* dbias,
                               mqg_dtype dweight_dtype, int add_into_grads, float* workspace, size_t workspace_floats,
                               void* cuda_stream)
{
    const char* what = "mqg_layer_norm_grad";
    if (mqg_status st = check_rows(what, rows, dim)) return st;
    const bool empty = rows == 0 || dim == 0, sums = dweight != nullptr || dbias != nullptr;
    if (mqg_status st = check_buffer(what, "dy", dy, dy_dtype, empty)) return st;
    if (mqg_status st = check_buffer(what, "x", x, x_dtype, empty)) return st;
    if (mqg_status st = check_optional(what, "weight", weight, weight_dtype)) return st;
    if (mqg_status st = check_buffer(what, "stats", stats, MQG_F32, empty)) return st;
    if (mqg_status st = check_optional(what, "dx", dx, x_dtype)) return st;
    if (mqg_status st = check_optional(what, "dweight", dweight, dweight_dtype)) return st;
    if (mqg_status st = check_optional(what, "dbias", dbias, dweight_dtype)) return st;
    if (dim == 0 || (rows == 0 && (add_into_grads || !sums)) || (!dx && !sums)) return MQG_OK;
    const size_t need = sums ? layer_norm_workspace_floats(rows, dim) : 0;
    if (workspace_floats < need)
        return report_error(MQG_ERR_INVALID, "%s: workspace holds %llu floats, %llu needed (mqg_layer_norm_workspace_floats)", what,
                            (unsigned long long)workspace_floats, (unsigned long long)need);
    if (need != 0 && !workspace) return report_error(MQG_ERR_INVALID, "%s: workspace is null", what);
    if (!aligned(workspace, 16)) return report_error(MQG_ERR_ALIGN, "%s: workspace not 16-byte aligned", what);
    const uint64_t n = rows * dim, dw_bytes = dim * bytes_of(dweight_dtype);
    const Region g = {"dy", dy, n * bytes_of(dy_dtype)}, in = {"x", x, n * bytes_of(x_dtype)}, st = {"stats", stats, rows * 8};
    const Region w = {"weight", weight, weight ? dim * bytes_of(weight_dtype) : 0}, scratch = {"workspace", workspace, need * 4};
    const Region to = {"dx", dx, dx ? n * bytes_of(x_dtype) : 0}, dw = {"dweight", dweight, dweight ? dw_bytes : 0};
    const Region db = {"dbias", dbias, dbias ? dw_bytes : 0};
    if (mqg_status s = check_apart(what, to, {g, in, st, w, dw, db, scratch})) return s;
    if (mqg_status s = check_apart(what, dw, {g, in, st, w, db, scratch})) return s;
    if (mqg_status s = check_apart(what, db, {g, in, st, w, scratch})) return s;
    if (mqg_status s = check_apart(what, scratch, {g, in, st, w})) return s;
    const NormRows rows_in = {x, (int)x_dtype, rows, dim, weight, nullptr, (int)weight_dtype};
    const NormGrads out = {dx, dweight, dbias, (int)dweight_dtype, add_into_grads != 0};
    return cuda_status(what, launch_layer_norm_grad(dy, (int)dy_dtype, rows_in, stats, out, workspace, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
