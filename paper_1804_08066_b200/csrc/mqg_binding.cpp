// The Python entry points that enqueue work, as native functions over the C ABI of include/mqgrad.h: they
// take torch tensors, read the device pointers and torch's current stream, and make the call.
//
// Why native: a call's work on the device takes 2 to 4 us for gradients up to a million elements, and a
// launch about as long on the host.  Marshalling through ctypes (a Python frame, a type check and a
// data_ptr() call per tensor, a pointer table per list, a stream object, argument conversion) took 7 us for
// the call with the fewest arguments and 22 us for one that takes three lists of eight tensors, so the
// device waited for the host.
#include <Python.h>

#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstring>
#include <memory>
#include <vector>

#include "../../include/mqgrad.h"

namespace {

constexpr int kMaxArgs = 16;

// One entry point's parameters, in order; the last `ndefaults` may be left out (a null slot).
struct Signature {
    const char* function;
    int nargs, ndefaults;
    const char* names[kMaxArgs];
    PyObject* interned[kMaxArgs];
};

// Positional and keyword arguments of a call into slots (borrowed references).
bool bind_arguments(Signature& sig, PyObject* const* args, Py_ssize_t npos, PyObject* kwnames, PyObject** slot)
{
    if (npos > sig.nargs) {
        PyErr_Format(PyExc_TypeError, "%s() takes at most %d arguments (%zd given)", sig.function, sig.nargs, npos);
        return false;
    }
    for (int i = 0; i < sig.nargs; ++i) slot[i] = i < npos ? args[i] : nullptr;
    const Py_ssize_t nkw = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
    for (Py_ssize_t k = 0; k < nkw; ++k) {
        PyObject* key = PyTuple_GET_ITEM(kwnames, k);
        int at = -1;
        for (int i = 0; i < sig.nargs && at < 0; ++i)
            if (key == sig.interned[i]) at = i;
        for (int i = 0; i < sig.nargs && at < 0; ++i)
            if (PyUnicode_CompareWithASCIIString(key, sig.names[i]) == 0) at = i;
        if (at < 0) {
            PyErr_Format(PyExc_TypeError, "%s() got an unexpected keyword argument '%U'", sig.function, key);
            return false;
        }
        if (slot[at]) {
            PyErr_Format(PyExc_TypeError, "%s() got multiple values for argument '%s'", sig.function, sig.names[at]);
            return false;
        }
        slot[at] = args[npos + k];
    }
    for (int i = 0; i < sig.nargs - sig.ndefaults; ++i)
        if (!slot[i]) {
            PyErr_Format(PyExc_TypeError, "%s() missing required argument: '%s'", sig.function, sig.names[i]);
            return false;
        }
    return true;
}

// Thrown with a Python error set.
struct PythonError {};

uint64_t to_u64(PyObject* o, uint64_t absent = 0)
{
    if (!o) return absent;
    const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);      // wraps like a C conversion
    if (v == (unsigned long long)-1 && PyErr_Occurred()) throw PythonError();
    return v;
}
uint32_t to_u32(PyObject* o) { return (uint32_t)to_u64(o); }
int to_int(PyObject* o) { return (int)(uint32_t)to_u64(o); }
float to_float(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PythonError();
    return (float)v;
}
double to_double(PyObject* o, double absent = 0.0)
{
    if (!o) return absent;
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PythonError();
    return v;
}
bool to_bool(PyObject* o)
{
    if (!o) return false;
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PythonError();
    return v != 0;
}

// THPVariable_Check asks isinstance(), which an object can answer without being a tensor.
bool is_tensor(PyObject* o) { return PyObject_TypeCheck(o, reinterpret_cast<PyTypeObject*>(THPVariableClass)); }

// Device pointer of a contiguous CUDA tensor.  `index` >= 0: the tensor is that item of a list.
void* device_ptr(PyObject* o, const char* what, Py_ssize_t index = -1)
{
    char name[64];
    auto called = [&]() -> const char* {
        if (index < 0) return what;
        snprintf(name, sizeof(name), "%s[%zd]", what, index);
        return name;
    };
    if (!is_tensor(o) || !THPVariable_Unpack(o).is_cuda()) {
        PyErr_Format(PyExc_TypeError, "%s must be a CUDA tensor (libmqgrad has no CPU path)", called());
        throw PythonError();
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s must be contiguous", called());
        throw PythonError();
    }
    return t.data_ptr();
}

mqg_dtype grad_dtype(PyObject* o)
{
    if (is_tensor(o)) {
        const at::ScalarType s = THPVariable_Unpack(o).scalar_type();
        if (s == at::kFloat) return MQG_F32;
        if (s == at::kBFloat16) return MQG_BF16;
        PyErr_Format(PyExc_TypeError, "grad must be float32 or bfloat16, got %s", c10::toString(s));
    } else {
        PyErr_SetString(PyExc_TypeError, "grad must be a tensor");
    }
    throw PythonError();
}

// Tensors of a list that live as long as this: while the call runs without the interpreter lock, another thread could take them out of
// the list.
struct HeldItems {
    PyObject** at;                                      // room for them
    size_t count = 0;
    void hold(PyObject* o) { at[count++] = Py_NewRef(o); }
    explicit HeldItems(PyObject** room = nullptr) : at(room) {}
    HeldItems(const HeldItems&) = delete;
    ~HeldItems()
    {
        while (count != 0) Py_DECREF(at[--count]);
    }
};

// A list (or tuple, or any iterable) of W tensors as a table of device pointers.  Everything that is wanted of the
// items is read at once: later arguments may run Python code that changes the list.  They live as long as this.
struct PointerTable {
    void* ptr[MQG_MAX_WORKERS];
    PyObject* item[MQG_MAX_WORKERS];
    HeldItems kept{item};
    PyObject* items = nullptr;
    Py_ssize_t count = 0;
    ~PointerTable() { Py_XDECREF(items); }

    // `exact`: the list has to hold exactly W tensors; otherwise at least W.
    void read(PyObject* o, const char* what, int W, bool exact)
    {
        items = PySequence_Fast(o, "a list of tensors is expected");
        if (!items) throw PythonError();
        count = PySequence_Fast_GET_SIZE(items);
        // a worker count outside the library's range is the C ABI's to reject: it reads no table then
        if (exact ? count != W : count < W && W <= MQG_MAX_WORKERS) {
            PyErr_Format(PyExc_ValueError, "%s must hold %s%d tensors, got %zd", what, exact ? "" : "at least ", W, count);
            throw PythonError();
        }
        const Py_ssize_t n = count < MQG_MAX_WORKERS ? count : MQG_MAX_WORKERS;
        for (Py_ssize_t i = 0; i < n; ++i) {
            ptr[i] = device_ptr(PySequence_Fast_GET_ITEM(items, i), what, i);
            kept.hold(PySequence_Fast_GET_ITEM(items, i));
        }
    }
    template <typename T> T* const* as() const { return reinterpret_cast<T* const*>(ptr); }
};

struct GradientTable : PointerTable {
    mqg_dtype dtype;

    // `all_alike`: every gradient must have the first one's type.
    void read(PyObject* o, int W, bool exact, bool all_alike)
    {
        PointerTable::read(o, "grads", W, exact);
        if (count == 0) {
            if (all_alike) PyErr_SetString(PyExc_TypeError, "all gradients must have the same dtype: there are none");
            else PyErr_SetString(PyExc_IndexError, "grads is empty");
            throw PythonError();
        }
        dtype = grad_dtype(PySequence_Fast_GET_ITEM(items, 0));
        for (Py_ssize_t i = 1; all_alike && i < count; ++i)
            if (grad_dtype(PySequence_Fast_GET_ITEM(items, i)) != dtype) {
                PyErr_SetString(PyExc_TypeError, "all gradients must have the same dtype");
                throw PythonError();
            }
    }
};

struct Reference {
    PyObject* object;
    ~Reference() { Py_XDECREF(object); }
};

// A segment table: 64-bit integers from an array that exposes them, or from any sequence of numbers.  Copied: the
// library checks the table and then uses it, without the interpreter lock.
struct OffsetTable {
    uint64_t inline_store[65];
    std::vector<uint64_t> store;
    const uint64_t* data = nullptr;
    Py_ssize_t count = 0;

    void read(PyObject* o)
    {
        if (!PyList_Check(o) && !PyTuple_Check(o) && PyObject_CheckBuffer(o) && read_buffer(o)) return;
        const Reference items = {PySequence_Tuple(o)};  // a list could change while its items are converted
        if (!items.object) throw PythonError();
        uint64_t* to = room(PyTuple_GET_SIZE(items.object));
        for (Py_ssize_t i = 0; i < count; ++i) {
            PyObject* v = PyTuple_GET_ITEM(items.object, i);
            const Reference whole = {PyLong_CheckExact(v) ? Py_NewRef(v) : PyNumber_Long(v)};
            if (!whole.object) throw PythonError();
            to[i] = to_u64(whole.object);
        }
    }

private:
    uint64_t* room(Py_ssize_t n)
    {
        uint64_t* to = inline_store;
        if (n > 65) { store.resize((size_t)n); to = store.data(); }
        data = to;
        count = n;
        return to;
    }
    bool read_buffer(PyObject* o)
    {
        struct View : Py_buffer { ~View() { PyBuffer_Release(this); } } view;       // (releasing an empty one does nothing)
        if (PyObject_GetBuffer(o, &view, PyBUF_FORMAT | PyBUF_C_CONTIGUOUS) != 0) {
            PyErr_Clear();
            return false;
        }
        const bool offsets = view.ndim == 1 && view.itemsize == 8 && view.format && view.format[0] != '\0' &&
                             view.format[1] == '\0' && std::strchr("lLqQ", view.format[0]);
        if (offsets) std::memcpy(room(view.len / 8), view.buf, (size_t)view.len);
        return offsets;
    }
};

// seg_off and code_off of a call; returns the number of segments.
int read_segments(PyObject* seg_off, PyObject* code_off, OffsetTable& seg, OffsetTable& code)
{
    seg.read(seg_off);
    code.read(code_off);
    if (code.count < seg.count) {
        PyErr_Format(PyExc_ValueError, "code_off holds %zd offsets, seg_off %zd", code.count, seg.count);
        throw PythonError();
    }
    return (int)seg.count - 1;
}

void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

PyObject* g_error_class = nullptr;      // MqgError of the package

// None, or the package's MqgError with the library's message.
PyObject* finish(mqg_status st)
{
    if (st == MQG_OK) Py_RETURN_NONE;
    PyObject* e = PyObject_CallFunction(g_error_class, "is", (int)st, mqg_last_error());
    if (e) { PyErr_SetObject(g_error_class, e); Py_DECREF(e); }
    return nullptr;
}

// The call itself runs without the interpreter lock: a full launch queue blocks it.  The lock is back whichever way
// the call ends.
struct WithoutLock {
    PyThreadState* state = PyEval_SaveThread();
    ~WithoutLock() { PyEval_RestoreThread(state); }
};
template <typename Fn> PyObject* enqueue(Fn&& fn)
{
    mqg_status st;
    {
        const WithoutLock unlocked;
        st = fn();
    }
    return finish(st);
}

// Defines the native function `name`: binds the arguments to `v[]` and runs the body that follows.
#define MQG_ENTRY(name, ndefaults, nargs, ...)                                                                      \
    Signature sig_##name = {#name, nargs, ndefaults, {__VA_ARGS__}, {}};                                            \
    PyObject* body_##name(PyObject** v);                                                                            \
    PyObject* py_##name(PyObject*, PyObject* const* args, Py_ssize_t npos, PyObject* kwnames)                       \
    {                                                                                                               \
        PyObject* v[kMaxArgs];                                                                                      \
        if (!bind_arguments(sig_##name, args, npos, kwnames, v)) return nullptr;                                    \
        try {                                                                                                       \
            return body_##name(v);                                                                                  \
        } catch (const PythonError&) {                                                                              \
        } catch (const std::exception& e) {                                                                         \
            PyErr_SetString(PyExc_RuntimeError, e.what());                                                          \
        }                                                                                                           \
        return nullptr;                                                                                             \
    }                                                                                                               \
    PyObject* body_##name(PyObject** v)

MQG_ENTRY(mqg_quantize, 3, 10, "grad", "n", "bits", "bucket", "seed", "codes", "scales", "worker", "step", "elem_offset")
{
    const uint64_t n = to_u64(v[1]), bucket = to_u64(v[3]), seed = to_u64(v[4]), off = to_u64(v[9]);
    const int bits = to_int(v[2]);
    const uint32_t worker = to_u32(v[7]), step = to_u32(v[8]);
    const mqg_dtype dt = grad_dtype(v[0]);
    const void* grad = n ? device_ptr(v[0], "grad") : nullptr;
    uint32_t* codes = n ? static_cast<uint32_t*>(device_ptr(v[5], "codes")) : nullptr;
    float* scales = n ? static_cast<float*>(device_ptr(v[6], "scales")) : nullptr;
    void* s = stream();
    return enqueue([=] { return mqg_quantize(grad, n, bits, bucket, seed, codes, scales, dt, worker, step, off, s); });
}

MQG_ENTRY(mqg_quantize_l2, 3, 10, "grad", "n", "bits", "bucket", "seed", "codes", "scales", "worker", "step", "elem_offset")
{
    const uint64_t n = to_u64(v[1]), bucket = to_u64(v[3]), seed = to_u64(v[4]), off = to_u64(v[9]);
    const int bits = to_int(v[2]);
    const uint32_t worker = to_u32(v[7]), step = to_u32(v[8]);
    const void* grad = device_ptr(v[0], "grad");
    const mqg_dtype dt = grad_dtype(v[0]);
    uint32_t* codes = static_cast<uint32_t*>(device_ptr(v[5], "codes"));
    float* scales = static_cast<float*>(device_ptr(v[6], "scales"));
    void* s = stream();
    return enqueue([=] { return mqg_quantize_l2(grad, n, bits, bucket, seed, codes, scales, dt, worker, step, off, s); });
}

template <typename Fn> PyObject* quantize_workers(PyObject** v, Fn fn)
{
    const int W = to_int(v[1]), bits = to_int(v[3]);
    const uint64_t n = to_u64(v[2]), bucket = to_u64(v[4]), seed = to_u64(v[5]), off = to_u64(v[10]);
    const uint32_t first = to_u32(v[8]), step = to_u32(v[9]);
    GradientTable g;
    PointerTable c, sc;
    g.read(v[0], W, true, true);
    c.read(v[6], "codes", W, true);
    sc.read(v[7], "scales", W, true);
    void* s = stream();
    return enqueue([&] { return fn(g.as<const void>(), W, n, bits, bucket, seed, c.as<uint32_t>(), sc.as<float>(), g.dtype,
                                   first, step, off, s); });
}

MQG_ENTRY(mqg_quantize_workers, 3, 11, "grads", "W", "n", "bits", "bucket", "seed", "codes", "scales", "first_worker",
          "step", "elem_offset")
{
    return quantize_workers(v, ::mqg_quantize_workers);
}

MQG_ENTRY(mqg_quantize_workers_l2, 3, 11, "grads", "W", "n", "bits", "bucket", "seed", "codes", "scales", "first_worker",
          "step", "elem_offset")
{
    return quantize_workers(v, ::mqg_quantize_workers_l2);
}

MQG_ENTRY(mqg_quantize_workers_minmax, 0, 7, "grads", "W", "n", "bits", "bucket", "codes", "ranges")
{
    const int W = to_int(v[1]), bits = to_int(v[3]);
    const uint64_t n = to_u64(v[2]), bucket = to_u64(v[4]);
    GradientTable g;
    PointerTable c, r;
    g.read(v[0], W, true, true);
    c.read(v[5], "codes", W, true);
    r.read(v[6], "ranges", W, true);
    void* s = stream();
    return enqueue([&] { return ::mqg_quantize_workers_minmax(g.as<const void>(), W, n, bits, bucket, c.as<uint32_t>(),
                                                              r.as<float>(), g.dtype, s); });
}

MQG_ENTRY(mqg_quantize_minmax, 0, 6, "grad", "n", "bits", "bucket", "codes", "ranges")
{
    const uint64_t n = to_u64(v[1]), bucket = to_u64(v[3]);
    const int bits = to_int(v[2]);
    const mqg_dtype dt = grad_dtype(v[0]);
    const void* grad = n ? device_ptr(v[0], "grad") : nullptr;
    uint32_t* codes = n ? static_cast<uint32_t*>(device_ptr(v[4], "codes")) : nullptr;
    float* ranges = n ? static_cast<float*>(device_ptr(v[5], "ranges")) : nullptr;
    void* s = stream();
    return enqueue([=] { return mqg_quantize_minmax(grad, n, bits, bucket, codes, ranges, dt, s); });
}

MQG_ENTRY(mqg_quantize_1bit_ef, 0, 6, "grad", "residual", "n", "bucket", "codes", "ranges")
{
    const uint64_t n = to_u64(v[2]), bucket = to_u64(v[3]);
    const void* grad = device_ptr(v[0], "grad");
    float* residual = static_cast<float*>(device_ptr(v[1], "residual"));
    uint32_t* codes = static_cast<uint32_t*>(device_ptr(v[4], "codes"));
    float* ranges = static_cast<float*>(device_ptr(v[5], "ranges"));
    const mqg_dtype dt = grad_dtype(v[0]);
    void* s = stream();
    return enqueue([=] { return mqg_quantize_1bit_ef(grad, residual, n, bucket, codes, ranges, dt, s); });
}

template <typename Fn> PyObject* dequant_accumulate(PyObject** v, const char* second, Fn fn)
{
    const int W = to_int(v[2]), bits = to_int(v[3]);
    const uint64_t n = to_u64(v[4]), bucket = to_u64(v[6]);
    const int add = to_bool(v[7]) ? 1 : 0;
    PointerTable c, sc;
    c.read(v[0], "codes", W, false);
    sc.read(v[1], second, W, false);
    float* acc = n ? static_cast<float*>(device_ptr(v[5], "acc")) : nullptr;
    void* s = stream();
    return enqueue([&] { return fn(c.as<const uint32_t>(), sc.as<const float>(), W, bits, n, acc, bucket, add, s); });
}

MQG_ENTRY(mqg_dequant_accumulate, 1, 8, "codes", "scales", "W", "bits", "n", "acc", "bucket", "add_into_acc")
{
    return dequant_accumulate(v, "scales", ::mqg_dequant_accumulate);
}

MQG_ENTRY(mqg_dequant_accumulate_minmax, 1, 8, "codes", "ranges", "W", "bits", "n", "acc", "bucket", "add_into_acc")
{
    return dequant_accumulate(v, "ranges", ::mqg_dequant_accumulate_minmax);
}

float* optional_ptr(PyObject* o, const char* what)
{
    return o && o != Py_None ? static_cast<float*>(device_ptr(o, what)) : nullptr;
}

template <typename Fn> PyObject* server_step(PyObject** v, const char* second, Fn fn)
{
    const int W = to_int(v[2]), bits = to_int(v[3]);
    const uint64_t n = to_u64(v[4]), bucket = to_u64(v[5]);
    const float lr = to_float(v[7]);
    PointerTable c, sc;
    c.read(v[0], "codes", W, false);
    sc.read(v[1], second, W, false);
    float* params = n ? static_cast<float*>(device_ptr(v[6], "params")) : nullptr;
    float* acc = optional_ptr(v[8], "acc_out");
    void* s = stream();
    return enqueue([&] { return fn(c.as<const uint32_t>(), sc.as<const float>(), W, bits, n, bucket, params, lr, acc, s); });
}

MQG_ENTRY(mqg_server_step, 1, 9, "codes", "scales", "W", "bits", "n", "bucket", "params", "lr", "acc_out")
{
    return server_step(v, "scales", ::mqg_server_step);
}

MQG_ENTRY(mqg_server_step_minmax, 1, 9, "codes", "ranges", "W", "bits", "n", "bucket", "params", "lr", "acc_out")
{
    return server_step(v, "ranges", ::mqg_server_step_minmax);
}

MQG_ENTRY(mqg_apply, 0, 4, "params", "acc", "lr", "n")
{
    const uint64_t n = to_u64(v[3]);
    const float lr = to_float(v[2]);
    float* params = n ? static_cast<float*>(device_ptr(v[0], "params")) : nullptr;
    const float* acc = n ? static_cast<const float*>(device_ptr(v[1], "acc")) : nullptr;
    void* s = stream();
    return enqueue([=] { return mqg_apply(params, acc, lr, n, s); });
}

MQG_ENTRY(mqg_server_requantize, 2, 12, "codes", "scales", "W", "bits", "n", "bucket", "mean_scale", "seed", "codes_out",
          "scales_out", "worker", "step")
{
    const int W = to_int(v[2]), bits = to_int(v[3]);
    const uint64_t n = to_u64(v[4]), bucket = to_u64(v[5]), seed = to_u64(v[7]);
    const float mean_scale = to_float(v[6]);
    const uint32_t worker = to_u32(v[10]), step = to_u32(v[11]);
    PointerTable c, sc;
    c.read(v[0], "codes", W, false);
    sc.read(v[1], "scales", W, false);
    uint32_t* codes_out = n ? static_cast<uint32_t*>(device_ptr(v[8], "codes_out")) : nullptr;
    float* scales_out = n ? static_cast<float*>(device_ptr(v[9], "scales_out")) : nullptr;
    void* s = stream();
    return enqueue([&] { return ::mqg_server_requantize(c.as<const uint32_t>(), sc.as<const float>(), W, bits, n, bucket,
                                                        mean_scale, seed, codes_out, scales_out, worker, step, s); });
}

MQG_ENTRY(mqg_quantize_segments, 3, 10, "grad", "seg_off", "code_off", "bits", "seed", "codes", "scales", "worker", "step",
          "elem_offset")
{
    OffsetTable seg, code;
    const int nseg = read_segments(v[1], v[2], seg, code), bits = to_int(v[3]);
    const uint64_t seed = to_u64(v[4]), off = to_u64(v[9]);
    const uint32_t worker = to_u32(v[7]), step = to_u32(v[8]);
    const void* grad = device_ptr(v[0], "grad");
    const mqg_dtype dt = grad_dtype(v[0]);
    uint32_t* codes = static_cast<uint32_t*>(device_ptr(v[5], "codes"));
    float* scales = static_cast<float*>(device_ptr(v[6], "scales"));
    void* s = stream();
    return enqueue([&] { return ::mqg_quantize_segments(grad, nseg, seg.data, code.data, bits, seed, codes, scales, dt,
                                                        worker, step, off, s); });
}

MQG_ENTRY(mqg_quantize_segments_l2, 3, 11, "grad", "seg_off", "code_off", "bits", "seed", "codes", "scales", "workspace",
          "worker", "step", "elem_offset")
{
    OffsetTable seg, code;
    const int nseg = read_segments(v[1], v[2], seg, code), bits = to_int(v[3]);
    const uint64_t seed = to_u64(v[4]), off = to_u64(v[10]);
    const uint32_t worker = to_u32(v[8]), step = to_u32(v[9]);
    const void* grad = device_ptr(v[0], "grad");
    const mqg_dtype dt = grad_dtype(v[0]);
    uint32_t* codes = static_cast<uint32_t*>(device_ptr(v[5], "codes"));
    float* scales = static_cast<float*>(device_ptr(v[6], "scales"));
    float* workspace = static_cast<float*>(device_ptr(v[7], "workspace"));
    const size_t floats = (size_t)THPVariable_Unpack(v[7]).numel();
    void* s = stream();
    return enqueue([&] { return ::mqg_quantize_segments_l2(grad, nseg, seg.data, code.data, bits, seed, codes, scales, dt,
                                                           worker, step, off, workspace, floats, s); });
}

MQG_ENTRY(mqg_quantize_segments_l2_static, 3, 10, "grad", "seg_off", "code_off", "bits", "seed", "codes", "scales",
          "worker", "step", "elem_offset")
{
    OffsetTable seg, code;
    const int nseg = read_segments(v[1], v[2], seg, code), bits = to_int(v[3]);
    const uint64_t seed = to_u64(v[4]), off = to_u64(v[9]);
    const uint32_t worker = to_u32(v[7]), step = to_u32(v[8]);
    const void* grad = device_ptr(v[0], "grad");
    const mqg_dtype dt = grad_dtype(v[0]);
    uint32_t* codes = static_cast<uint32_t*>(device_ptr(v[5], "codes"));
    float* scales = static_cast<float*>(device_ptr(v[6], "scales"));
    void* s = stream();
    return enqueue([&] { return ::mqg_quantize_segments_l2_static(grad, nseg, seg.data, code.data, bits, seed, codes,
                                                                  scales, dt, worker, step, off, s); });
}

MQG_ENTRY(mqg_quantize_segments_workers, 3, 11, "grads", "W", "seg_off", "code_off", "bits", "seed", "codes", "scales",
          "first_worker", "step", "elem_offset")
{
    OffsetTable seg, code;
    const int W = to_int(v[1]), nseg = read_segments(v[2], v[3], seg, code), bits = to_int(v[4]);
    const uint64_t seed = to_u64(v[5]), off = to_u64(v[10]);
    const uint32_t first = to_u32(v[8]), step = to_u32(v[9]);
    GradientTable g;
    PointerTable c, sc;
    g.read(v[0], W, false, false);
    c.read(v[6], "codes", W, false);
    sc.read(v[7], "scales", W, false);
    void* s = stream();
    return enqueue([&] { return ::mqg_quantize_segments_workers(g.as<const void>(), W, nseg, seg.data, code.data, bits,
                                                                seed, c.as<uint32_t>(), sc.as<float>(), g.dtype, first, step,
                                                                off, s); });
}

MQG_ENTRY(mqg_server_step_segments, 1, 9, "codes", "scales", "W", "bits", "seg_off", "code_off", "params", "lr", "acc_out")
{
    OffsetTable seg, code;
    const int W = to_int(v[2]), bits = to_int(v[3]), nseg = read_segments(v[4], v[5], seg, code);
    const float lr = to_float(v[7]);
    PointerTable c, sc;
    c.read(v[0], "codes", W, false);
    sc.read(v[1], "scales", W, false);
    float* params = static_cast<float*>(device_ptr(v[6], "params"));
    float* acc = optional_ptr(v[8], "acc_out");
    void* s = stream();
    return enqueue([&] { return ::mqg_server_step_segments(c.as<const uint32_t>(), sc.as<const float>(), W, bits, nseg,
                                                           seg.data, code.data, params, lr, acc, s); });
}

// ---- around the codec: the global norm, clipping, and the table of a model over tokens ----
// These calls check types and sizes of every tensor, and run on the tensors' device, on its current stream.

struct Operands {
    int device = -1;

    // A contiguous CUDA tensor of at least `least` elements; all of a call's are on one device.
    const at::Tensor& tensor(PyObject* o, const char* what, uint64_t least, Py_ssize_t index = -1)
    {
        if (!is_tensor(o)) device_ptr(o, what, index);  // (says so)
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || !t.is_contiguous()) device_ptr(o, what, index);
        if ((uint64_t)t.numel() < least) {
            PyErr_Format(PyExc_ValueError, "%s holds %lld elements, %llu are needed", what, (long long)t.numel(),
                         (unsigned long long)least);
            throw PythonError();
        }
        const int on = t.get_device();
        if (device >= 0 && on != device) {
            PyErr_Format(PyExc_ValueError, "%s is on cuda:%d, the tensors before it on cuda:%d", what, on, device);
            throw PythonError();
        }
        device = on;
        return t;
    }
    float* floats(PyObject* o, const char* what, uint64_t least, uint64_t* count = nullptr)
    {
        const at::Tensor& t = tensor(o, what, least);
        if (t.scalar_type() != at::kFloat) {
            PyErr_Format(PyExc_TypeError, "%s must be float32, got %s", what, c10::toString(t.scalar_type()));
            throw PythonError();
        }
        if (count) *count = (uint64_t)t.numel();
        return static_cast<float*>(t.data_ptr());
    }
    void* values(PyObject* o, const char* what, uint64_t least, mqg_dtype* dtype, Py_ssize_t index = -1, uint64_t* count = nullptr)
    {
        const at::Tensor& t = tensor(o, what, least, index);
        const at::ScalarType s = t.scalar_type();
        if (s != at::kFloat && s != at::kBFloat16) {
            PyErr_Format(PyExc_TypeError, "%s must be float32 or bfloat16, got %s", what, c10::toString(s));
            throw PythonError();
        }
        *dtype = s == at::kFloat ? MQG_F32 : MQG_BF16;
        if (count) *count = (uint64_t)t.numel();
        return t.data_ptr();
    }
    const void* ids(PyObject* o, uint64_t least, mqg_index* type)
    {
        const at::Tensor& t = tensor(o, "ids", least);
        const at::ScalarType s = t.scalar_type();
        if (s != at::kInt && s != at::kLong) {
            PyErr_Format(PyExc_TypeError, "ids must be int32 or int64, got %s", c10::toString(s));
            throw PythonError();
        }
        *type = s == at::kLong ? MQG_I64 : MQG_I32;
        return t.data_ptr();
    }
};

template <typename Fn> PyObject* enqueue_on(const Operands& on, Fn&& fn)
{
    if (c10::cuda::current_device() == on.device) {
        void* s = stream();
        return enqueue([&] { return fn(s); });
    }
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)on.device);
    void* s = stream();
    return enqueue([&] { return fn(s); });
}

// The product of two sizes, with what does not fit 64 bits as the largest value (which no tensor holds).
uint64_t area(uint64_t a, uint64_t b)
{
    uint64_t r;
    return __builtin_mul_overflow(a, b, &r) ? ~0ull : r;
}

// A list (or tuple, or any iterable) of gradient tensors of any sizes.  Everything that is wanted of the items is read at once,
// and no Python code runs meanwhile.  The items live as long as this: tensors that an iterable made for the call alone, or that
// another thread takes out of the list, are not freed before the launch.
struct TensorTable {
    static constexpr size_t kInline = 64;
    void* inline_ptr[kInline];
    uint64_t inline_size[kInline];
    mqg_dtype inline_dtype[kInline];
    PyObject* inline_item[kInline];
    std::unique_ptr<char[]> store;                      // (not filled with zeros first)
    HeldItems kept{inline_item};
    void** ptr = inline_ptr;
    uint64_t* size = inline_size;
    mqg_dtype* dtype = inline_dtype;
    size_t n = 0;
    uint64_t total = 0;
    Reference items = {nullptr};

    void read(PyObject* o, Operands& on)
    {
        items.object = PySequence_Fast(o, "a list of tensors is expected");
        if (!items.object) throw PythonError();
        n = (size_t)PySequence_Fast_GET_SIZE(items.object);
        if (n > kInline) {
            store.reset(new char[n * (2 * sizeof(void*) + sizeof(uint64_t) + sizeof(mqg_dtype))]);
            ptr = reinterpret_cast<void**>(store.get());
            kept.at = reinterpret_cast<PyObject**>(ptr + n);
            size = reinterpret_cast<uint64_t*>(kept.at + n);
            dtype = reinterpret_cast<mqg_dtype*>(size + n);
        }
        PyObject** item = PySequence_Fast_ITEMS(items.object);
        for (size_t i = 0; i < n; ++i) {
            ptr[i] = on.values(item[i], "grads", 0, &dtype[i], (Py_ssize_t)i, &size[i]);
            total += size[i];
            kept.hold(item[i]);
        }
    }
    const char* end(size_t i) const { return static_cast<const char*>(ptr[i]) + size[i] * (dtype[i] == MQG_F32 ? 4 : 2); }
    // Tensors that are written: no two of them share memory.
    void check_apart() const
    {
        bool ascending = true;
        for (size_t i = 1; i < n && ascending; ++i) ascending = end(i - 1) <= ptr[i];
        if (ascending) return;
        std::vector<size_t> order;
        for (size_t i = 0; i < n; ++i)
            if (size[i] != 0) order.push_back(i);
        std::sort(order.begin(), order.end(), [&](size_t a, size_t b) { return ptr[a] < ptr[b]; });
        for (size_t k = 1; k < order.size(); ++k)
            if (end(order[k - 1]) > ptr[order[k]]) {
                PyErr_Format(PyExc_ValueError, "grads[%zu] and grads[%zu] share memory", std::min(order[k - 1], order[k]),
                             std::max(order[k - 1], order[k]));
                throw PythonError();
            }
    }
    int count() const { return (int)n; }
};

struct NormArgs {
    TensorTable g;
    float max_norm, *result, *workspace;
    uint64_t floats;
    // What may run Python code (a number's conversion, an iterable) comes before the pointers of the other tensors.
    void read(PyObject* grads, PyObject* limit, PyObject* res, PyObject* work, Operands& on)
    {
        max_norm = to_float(limit);
        g.read(grads, on);
        result = on.floats(res, "result", 2);
        workspace = on.floats(work, "workspace", 0, &floats);
    }
};

MQG_ENTRY(mqg_grad_norm, 0, 4, "grads", "max_norm", "result", "workspace")
{
    Operands on;
    NormArgs a;
    a.read(v[0], v[1], v[2], v[3], on);
    return enqueue_on(on, [&](void* s) { return ::mqg_grad_norm(a.g.ptr, a.g.size, a.g.dtype, a.g.count(), a.max_norm,
                                                                a.result, a.workspace, a.floats, s); });
}

MQG_ENTRY(mqg_clip_grad_norm, 0, 4, "grads", "max_norm", "result", "workspace")
{
    Operands on;
    NormArgs a;
    a.read(v[0], v[1], v[2], v[3], on);
    a.g.check_apart();
    return enqueue_on(on, [&](void* s) { return ::mqg_clip_grad_norm(a.g.ptr, a.g.size, a.g.dtype, a.g.count(), a.max_norm,
                                                                     a.result, a.workspace, a.floats, s); });
}

MQG_ENTRY(mqg_clip_flatten, 0, 5, "grads", "max_norm", "flat", "result", "workspace")
{
    Operands on;
    NormArgs a;
    mqg_dtype type;
    a.read(v[0], v[1], v[3], v[4], on);
    const TensorTable& g = a.g;
    char* flat = static_cast<char*>(on.values(v[2], "flat", g.total, &type));
    const char* end = flat + g.total * (type == MQG_F32 ? 4 : 2);
    for (size_t i = 0; i < g.n; ++i)
        if (g.ptr[i] < end && g.end(i) > flat && g.size[i] != 0) {
            PyErr_Format(PyExc_ValueError, "grads[%zu] and flat share memory", i);
            return nullptr;
        }
    return enqueue_on(on, [&](void* s) { return ::mqg_clip_flatten(g.ptr, g.size, g.dtype, g.count(), a.max_norm, flat, type,
                                                                   a.result, a.workspace, a.floats, s); });
}

MQG_ENTRY(mqg_scale_grads, 0, 2, "grads", "factor")
{
    Operands on;
    TensorTable g;
    g.read(v[0], on);
    const float* factor = on.floats(v[1], "factor", 1);
    g.check_apart();
    return enqueue_on(on, [&](void* s) { return ::mqg_scale_grads(g.ptr, g.size, g.dtype, g.count(), factor, s); });
}

MQG_ENTRY(mqg_apply_clipped, 0, 5, "params", "acc", "lr", "factor", "n")
{
    Operands on;
    const uint64_t n = to_u64(v[4]);
    const float lr = to_float(v[2]);
    float* params = on.floats(v[0], "params", n);
    const float* acc = on.floats(v[1], "acc", n);
    const float* factor = on.floats(v[3], "factor", 1);
    return enqueue_on(on, [&](void* s) { return ::mqg_apply_clipped(params, acc, lr, factor, n, s); });
}

MQG_ENTRY(mqg_embedding, 0, 7, "table", "rows", "dim", "ids", "tokens", "scale", "out")
{
    Operands on;
    const uint64_t rows = to_u64(v[1]), dim = to_u64(v[2]), tokens = to_u64(v[4]);
    const float scale = to_float(v[5]);
    mqg_dtype table_type, out_type;
    mqg_index ids_type;
    const void* table = on.values(v[0], "table", area(rows, dim), &table_type);
    const void* ids = on.ids(v[3], tokens, &ids_type);
    void* out = on.values(v[6], "out", area(tokens, dim), &out_type);
    return enqueue_on(on, [&](void* s) { return ::mqg_embedding(table, table_type, rows, dim, ids, ids_type, tokens, scale, out,
                                                                out_type, s); });
}

MQG_ENTRY(mqg_embedding_grad, 1, 9, "dout", "ids", "tokens", "rows", "dim", "scale", "grad", "workspace", "add_into_grad")
{
    Operands on;
    const uint64_t tokens = to_u64(v[2]), rows = to_u64(v[3]), dim = to_u64(v[4]);
    const float scale = to_float(v[5]);
    const int add = to_bool(v[8]) ? 1 : 0;
    mqg_dtype dout_type, grad_type;
    mqg_index ids_type;
    uint64_t floats;
    const void* dout = on.values(v[0], "dout", area(tokens, dim), &dout_type);
    const void* ids = on.ids(v[1], tokens, &ids_type);
    void* grad = on.values(v[6], "grad", area(rows, dim), &grad_type);
    float* workspace = on.floats(v[7], "workspace", 0, &floats);
    return enqueue_on(on, [&](void* s) { return ::mqg_embedding_grad(dout, dout_type, ids, ids_type, tokens, rows, dim, scale,
                                                                     grad, grad_type, add, workspace, floats, s); });
}

// ---- beside the codec: AdamW over many tensors, and the layer norm of a model over tokens ----

bool absent(PyObject* o) { return !o || o == Py_None; }

// The lists of an AdamW step.  Numbers and iterables, whose conversion may run Python code, are converted before any tensor is
// looked at; the tensors live as long as this.
struct AdamwLists {
    static constexpr int kMost = 5;
    static constexpr size_t kInline = 64;
    Reference items[kMost] = {};
    int nlists = 0;
    size_t n = 0;
    std::unique_ptr<char[]> store;                      // (not filled with zeros first)
    static constexpr size_t kPer = 2 * kMost * sizeof(void*) + sizeof(uint64_t) + 2 * sizeof(mqg_dtype) + sizeof(float);
    alignas(8) char inline_store[kInline * kPer];
    HeldItems kept;
    void** ptr[kMost];
    uint64_t* size;
    mqg_dtype* dtype[2];
    float* decay;
    bool has_decay = false;
    Operands on;
    const c10::StorageImpl* last_storage = nullptr;
    char* last_start = nullptr;

    AdamwLists(PyObject* const* lists, int count, PyObject* decays, PyObject* factor, PyObject* schedule) : nlists(count)
    {
        for (int k = 0; k < count; ++k) {
            items[k].object = PySequence_Fast(lists[k], "lists of tensors are expected");
            if (!items[k].object) throw PythonError();
        }
        n = (size_t)PySequence_Fast_GET_SIZE(items[0].object);
        const bool several = !absent(decays) && (PySequence_Check(decays) || PyIter_Check(decays)), one = !absent(decays) && !several;
        const Reference numbers = {several ? PySequence_Tuple(decays) : nullptr};
        if (several && !numbers.object) throw PythonError();
        const double all = one ? to_double(decays) : 0.0;
        has_decay = !absent(decays);
        if (n > kInline) store.reset(new char[n * kPer]);
        char* at = n > kInline ? store.get() : inline_store;
        for (int k = 0; k < kMost; ++k, at += n * sizeof(void*)) ptr[k] = reinterpret_cast<void**>(at);
        kept.at = reinterpret_cast<PyObject**>(at);
        size = reinterpret_cast<uint64_t*>(at + kMost * n * sizeof(void*));
        dtype[0] = reinterpret_cast<mqg_dtype*>(size + n);
        dtype[1] = dtype[0] + n;
        decay = reinterpret_cast<float*>(dtype[1] + n);
        if (numbers.object && (size_t)PyTuple_GET_SIZE(numbers.object) != n) {
            PyErr_Format(PyExc_ValueError, "decays holds %zd numbers, params %zu tensors", PyTuple_GET_SIZE(numbers.object), n);
            throw PythonError();
        }
        for (size_t j = 0; j < n; ++j) decay[j] = (float)(numbers.object ? to_double(PyTuple_GET_ITEM(numbers.object, j)) : all);
        // from here on no Python code runs
        for (int k = 0; k < count; ++k)
            if ((size_t)PySequence_Fast_GET_SIZE(items[k].object) != n) {
                PyErr_Format(PyExc_ValueError, "%s holds %zd tensors, params %zu", name(k), PySequence_Fast_GET_SIZE(items[k].object), n);
                throw PythonError();
            }
        read_list<0>();
        read_list<1>();
        read_list<2>();
        read_list<3>();
        if (count == kMost) read_list<4>();
        this->factor = absent(factor) ? nullptr : on.floats(factor, "factor", 1);
        this->schedule = absent(schedule) ? nullptr : on.floats(schedule, "schedule", 4);
    }
    AdamwLists(const AdamwLists&) = delete;

    const float *factor, *schedule;

    static const char* name(int k)
    {
        static constexpr const char* kNames[kMost] = {"params", "grads", "m", "v", "scales"};
        return kNames[k];
    }

    // A tensor's address.  Of tensors one after the other that are slices of one vector, only the first one's is asked for, which takes
    // as long as everything else that is wanted of a tensor.
    void* address(const at::Tensor& t, uint64_t held, int64_t bytes)
    {
        const at::TensorImpl* impl = t.unsafeGetTensorImpl();
        const c10::StorageImpl* from = impl->unsafe_storage().unsafeGetStorageImpl();
        if (held != 0 && from == last_storage) return last_start + impl->storage_offset() * bytes;
        void* p = t.data_ptr();
        if (held != 0) {
            last_storage = from;
            last_start = static_cast<char*>(p) - impl->storage_offset() * bytes;
        }
        return p;
    }
    // (a template: what differs from list to list is not asked for every tensor, which makes up for half of what holding it costs)
    template <int k> void read_list()
    {
        PyObject** item = PySequence_Fast_ITEMS(items[k].object);
        for (size_t j = 0; j < n; ++j) {
            read<k>(j, item[j]);
            kept.hold(item[j]);
        }
    }
    template <int k> void read(size_t j, PyObject* o)
    {
        const at::Tensor& t = on.tensor(o, name(k), 0, (Py_ssize_t)j);
        const at::ScalarType s = t.scalar_type();
        const uint64_t held = (uint64_t)t.numel();
        if constexpr (k < 2) {
            if (s != at::kFloat && s != at::kBFloat16) wrong_type(k, j, "float32 or bfloat16", s);
            dtype[k][j] = s == at::kFloat ? MQG_F32 : MQG_BF16;
            if (k == 0) size[j] = held;
        } else if (k == 4 || nlists == 4) {
            if (s != at::kFloat) wrong_type(k, j, "float32", s);
        } else if (s != at::kByte && s != (k == 2 ? at::kFloat8_e4m3fn : at::kFloat8_e5m2)) {
            wrong_type(k, j, k == 2 ? "float8_e4m3fn or uint8" : "float8_e5m2 or uint8", s);
        }
        ptr[k][j] = address(t, held, s == at::kFloat ? 4 : s == at::kBFloat16 ? 2 : 1);
        if (k < 4) return check_size(k, j, held);
        if (held != ::mqg_adamw8_scale_floats(size[j])) {
            PyErr_Format(PyExc_ValueError, "scales[%zu] holds %llu floats, params[%zu] needs %zu (mqg_adamw8_scale_floats)", j,
                         (unsigned long long)held, j, ::mqg_adamw8_scale_floats(size[j]));
            throw PythonError();
        }
    }
    [[noreturn]] static void wrong_type(int k, size_t j, const char* wanted, at::ScalarType s)
    {
        PyErr_Format(PyExc_TypeError, "%s[%zu] must be %s, got %s", name(k), j, wanted, c10::toString(s));
        throw PythonError();
    }
    void check_size(int k, size_t j, uint64_t held) const
    {
        if (held == size[j]) return;
        PyErr_Format(PyExc_ValueError, "%s[%zu] holds %llu elements, params[%zu] %llu", name(k), j, (unsigned long long)held, j,
                     (unsigned long long)size[j]);
        throw PythonError();
    }
    template <typename T> T* const* as(int k) const { return reinterpret_cast<T* const*>(ptr[k]); }
    const float* decays() const { return has_decay ? decay : nullptr; }
};

uint32_t to_step(PyObject* o)
{
    const uint64_t t = to_u64(o);
    if (t > 0xFFFFFFFFull) {
        PyErr_SetString(PyExc_ValueError, "step must be below 2^32");
        throw PythonError();
    }
    return (uint32_t)t;
}

MQG_ENTRY(mqg_adamw, 3, 13, "params", "grads", "m", "v", "decays", "lr", "beta1", "beta2", "eps", "step", "grad_scale", "factor",
          "schedule")
{
    const double lr = to_double(v[5]), beta1 = to_double(v[6]), beta2 = to_double(v[7]), eps = to_double(v[8]);
    const uint32_t step = to_step(v[9]);
    const float grad_scale = (float)to_double(v[10], 1.0);
    const AdamwLists a(v, 4, v[4], v[11], v[12]);
    return enqueue_on(a.on, [&](void* s) { return ::mqg_adamw(a.as<void>(0), a.dtype[0], a.as<const void>(1), a.dtype[1], a.as<float>(2),
                                                              a.as<float>(3), a.size, a.decays(), (int)a.n, lr, beta1, beta2, eps, step,
                                                              grad_scale, a.factor, a.schedule, s); });
}

MQG_ENTRY(mqg_adamw8, 3, 15, "params", "grads", "m", "v", "scales", "decays", "lr", "beta1", "beta2", "eps", "step", "seed",
          "grad_scale", "factor", "schedule")
{
    const double lr = to_double(v[6]), beta1 = to_double(v[7]), beta2 = to_double(v[8]), eps = to_double(v[9]);
    const uint32_t step = to_step(v[10]);
    const uint64_t seed = to_u64(v[11]);
    const float grad_scale = (float)to_double(v[12], 1.0);
    const AdamwLists a(v, 5, v[5], v[13], v[14]);
    return enqueue_on(a.on, [&](void* s) { return ::mqg_adamw8(a.as<void>(0), a.dtype[0], a.as<const void>(1), a.dtype[1],
                                                               a.as<uint8_t>(2), a.as<uint8_t>(3), a.as<float>(4), a.size, a.decays(),
                                                               (int)a.n, lr, beta1, beta2, eps, step, seed, grad_scale, a.factor,
                                                               a.schedule, s); });
}

// `weight` and `bias` (or `dweight` and `dbias`): either may be None; both have one type.
struct Pair {
    void* ptr[2] = {nullptr, nullptr};
    mqg_dtype dtype = MQG_F32;
    Pair(PyObject* a, const char* a_name, PyObject* b, const char* b_name, uint64_t dim, Operands& on)
    {
        mqg_dtype types[2];
        if (!absent(a)) ptr[0] = on.values(a, a_name, dim, &types[0]);
        if (!absent(b)) ptr[1] = on.values(b, b_name, dim, &types[1]);
        if (ptr[0] || ptr[1]) dtype = types[ptr[0] ? 0 : 1];
        if (!absent(a) && !absent(b) && types[0] != types[1]) {
            PyErr_Format(PyExc_TypeError, "%s and %s must be of one type", a_name, b_name);
            throw PythonError();
        }
    }
};

MQG_ENTRY(mqg_layer_norm, 1, 8, "x", "rows", "dim", "weight", "bias", "eps", "y", "stats")
{
    Operands on;
    const uint64_t rows = to_u64(v[1]), dim = to_u64(v[2]);
    const float eps = to_float(v[5]);
    mqg_dtype x_type, y_type;
    const void* x = on.values(v[0], "x", area(rows, dim), &x_type);
    const Pair w(v[3], "weight", v[4], "bias", dim, on);
    void* y = on.values(v[6], "y", area(rows, dim), &y_type);
    float* stats = absent(v[7]) ? nullptr : on.floats(v[7], "stats", area(rows, 2));
    return enqueue_on(on, [&](void* s) { return ::mqg_layer_norm(x, x_type, rows, dim, w.ptr[0], w.ptr[1], w.dtype, eps, y, y_type,
                                                                 stats, s); });
}

MQG_ENTRY(mqg_layer_norm_grad, 1, 11, "dy", "x", "rows", "dim", "weight", "stats", "dx", "dweight", "dbias", "workspace",
          "add_into_grads")
{
    Operands on;
    const uint64_t rows = to_u64(v[2]), dim = to_u64(v[3]);
    const int add = to_bool(v[10]) ? 1 : 0;
    mqg_dtype dy_type, x_type, dx_type, w_type = MQG_F32;
    uint64_t floats = 0;
    const void* dy = on.values(v[0], "dy", area(rows, dim), &dy_type);
    const void* x = on.values(v[1], "x", area(rows, dim), &x_type);
    const void* weight = absent(v[4]) ? nullptr : on.values(v[4], "weight", dim, &w_type);
    const float* stats = on.floats(v[5], "stats", area(rows, 2));
    void* dx = absent(v[6]) ? nullptr : on.values(v[6], "dx", area(rows, dim), &dx_type);
    if (dx && dx_type != x_type) {
        PyErr_SetString(PyExc_TypeError, "dx and x must be of one type");
        return nullptr;
    }
    const Pair d(v[7], "dweight", v[8], "dbias", dim, on);
    float* workspace = absent(v[9]) ? nullptr : on.floats(v[9], "workspace", 0, &floats);
    return enqueue_on(on, [&](void* s) { return ::mqg_layer_norm_grad(dy, dy_type, x, x_type, rows, dim, weight, w_type, stats, dx,
                                                                      d.ptr[0], d.ptr[1], d.dtype, add, workspace, floats, s); });
}

PyObject* set_error_class(PyObject*, PyObject* cls)
{
    Py_XSETREF(g_error_class, Py_NewRef(cls));
    Py_RETURN_NONE;
}

#define MQG_METHOD(name, signature, doc)                                                                            \
    {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL | METH_KEYWORDS, #name signature "\n--\n\n" doc}

PyMethodDef kMethods[] = {
    MQG_METHOD(mqg_quantize, "(grad, n, bits, bucket, seed, codes, scales, worker=0, step=0, elem_offset=0)",
               "Quantize(g, K): writes `codes` (uint32/int32 words) and `scales` (float32)."),
    MQG_METHOD(mqg_quantize_workers,
               "(grads, W, n, bits, bucket, seed, codes, scales, first_worker=0, step=0, elem_offset=0)",
               "Quantize(g_p, K) for W workers' gradients (lists of W tensors) in one launch."),
    MQG_METHOD(mqg_quantize_workers_l2,
               "(grads, W, n, bits, bucket, seed, codes, scales, first_worker=0, step=0, elem_offset=0)",
               "The L2-norm scale variant for W workers' gradients (lists of W tensors) in one launch."),
    MQG_METHOD(mqg_dequant_accumulate, "(codes, scales, W, bits, n, acc, bucket, add_into_acc=False)",
               "De-quantize and sum W workers' buffers into `acc`."),
    MQG_METHOD(mqg_apply, "(params, acc, lr, n)", "params <- params - lr * acc."),
    MQG_METHOD(mqg_server_step, "(codes, scales, W, bits, n, bucket, params, lr, acc_out=None)",
               "De-quantize, sum and apply W workers' buffers in one pass."),
    MQG_METHOD(mqg_quantize_workers_minmax, "(grads, W, n, bits, bucket, codes, ranges)",
               "The (min, max) variant for W workers' gradients (lists of W tensors) in one launch."),
    MQG_METHOD(mqg_quantize_minmax, "(grad, n, bits, bucket, codes, ranges)",
               "(min, max) nearest-rounding variant: writes `codes` and `ranges` (lo, hi per bucket)."),
    MQG_METHOD(mqg_dequant_accumulate_minmax, "(codes, ranges, W, bits, n, acc, bucket, add_into_acc=False)",
               "mqg_dequant_accumulate for the (min, max) variant."),
    MQG_METHOD(mqg_server_step_minmax, "(codes, ranges, W, bits, n, bucket, params, lr, acc_out=None)",
               "mqg_server_step for the (min, max) variant."),
    MQG_METHOD(mqg_server_requantize,
               "(codes, scales, W, bits, n, bucket, mean_scale, seed, codes_out, scales_out, worker=0, step=0)",
               "Downlink: de-quantize + sum + scale to the mean + quantize again, in one pass."),
    MQG_METHOD(mqg_quantize_segments,
               "(grad, seg_off, code_off, bits, seed, codes, scales, worker=0, step=0, elem_offset=0)",
               "Quantize with one scale per segment of the flat gradient."),
    MQG_METHOD(mqg_quantize_segments_workers,
               "(grads, W, seg_off, code_off, bits, seed, codes, scales, first_worker=0, step=0, elem_offset=0)",
               "mqg_quantize_segments for W workers' gradients that share one segment table."),
    MQG_METHOD(mqg_server_step_segments, "(codes, scales, W, bits, seg_off, code_off, params, lr, acc_out=None)",
               "mqg_server_step for buffers written by mqg_quantize_segments."),
    MQG_METHOD(mqg_quantize_1bit_ef, "(grad, residual, n, bucket, codes, ranges)",
               "One bit with error feedback; `residual` (float32, n elements) is read and updated in place."),
    MQG_METHOD(mqg_quantize_l2, "(grad, n, bits, bucket, seed, codes, scales, worker=0, step=0, elem_offset=0)",
               "mqg_quantize with the bucket's L2 norm as its scale."),
    MQG_METHOD(mqg_quantize_segments_l2,
               "(grad, seg_off, code_off, bits, seed, codes, scales, workspace, worker=0, step=0, elem_offset=0)",
               "`workspace`: float32 CUDA tensor of at least mqg_l2_workspace_floats(seg_off) elements."),
    MQG_METHOD(mqg_quantize_segments_l2_static,
               "(grad, seg_off, code_off, bits, seed, codes, scales, worker=0, step=0, elem_offset=0)",
               "mqg_quantize_segments_l2 for callers that cannot supply a workspace: the partial sums use an array\n"
               "inside the library (at most MQG_L2_STATIC_WORKSPACE_FLOATS of them); calls that may overlap on the\n"
               "device must be ordered by the caller."),
    MQG_METHOD(mqg_grad_norm, "(grads, max_norm, result, workspace)",
               "The norm of a list of gradient tensors and the factor that clips it to max_norm: `result` (float32, 2).\n"
               "`workspace`: float32 CUDA tensor of at least mqg_norm_workspace_floats(len(grads)) elements."),
    MQG_METHOD(mqg_clip_grad_norm, "(grads, max_norm, result, workspace)",
               "mqg_grad_norm, and the tensors scaled by the factor in place."),
    MQG_METHOD(mqg_clip_flatten, "(grads, max_norm, flat, result, workspace)",
               "mqg_grad_norm, and the tensors, times the factor, one after another in `flat` (float32 or bfloat16)."),
    MQG_METHOD(mqg_scale_grads, "(grads, factor)",
               "Scales a list of tensors in place by a float32 that is on the device."),
    MQG_METHOD(mqg_apply_clipped, "(params, acc, lr, factor, n)", "params <- params - lr * (factor * acc)."),
    MQG_METHOD(mqg_embedding, "(table, rows, dim, ids, tokens, scale, out)",
               "out[t] = scale * table[ids[t]]; zeros where an id is outside 0..rows-1."),
    MQG_METHOD(mqg_embedding_grad,
               "(dout, ids, tokens, rows, dim, scale, grad, workspace, add_into_grad=False)",
               "The gradient of mqg_embedding's table, written to `grad` or added to it; `workspace`: float32 CUDA tensor\n"
               "of at least mqg_embedding_workspace_floats(tokens, rows, dim) elements."),
    MQG_METHOD(mqg_adamw,
               "(params, grads, m, v, decays, lr, beta1, beta2, eps, step, grad_scale=1.0, factor=None, schedule=None)",
               "One step of AdamW over lists of tensors, in place; m and v are float32.  `decays`: None, a number, or one for\n"
               "each tensor; `factor` and `schedule`: float32 on the device (1 and 4 elements)."),
    MQG_METHOD(mqg_adamw8,
               "(params, grads, m, v, scales, decays, lr, beta1, beta2, eps, step, seed, grad_scale=1.0, factor=None, "
               "schedule=None)",
               "mqg_adamw with m (float8_e4m3fn or uint8) and v (float8_e5m2 or uint8) in 8 bits; `scales`: float32 tensors\n"
               "of mqg_adamw8_scale_floats(numel) elements."),
    MQG_METHOD(mqg_layer_norm, "(x, rows, dim, weight, bias, eps, y, stats=None)",
               "Layer norm of rows; `stats` (float32, rows x 2) takes their means and reciprocal deviations."),
    MQG_METHOD(mqg_layer_norm_grad, "(dy, x, rows, dim, weight, stats, dx, dweight, dbias, workspace, add_into_grads=False)",
               "The gradients of mqg_layer_norm (each of dx, dweight, dbias may be None); `workspace`: float32 CUDA tensor of at\n"
               "least mqg_layer_norm_workspace_floats(rows, dim) elements."),
    {"_set_error_class", set_error_class, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

Signature* const kSignatures[] = {
    &sig_mqg_quantize, &sig_mqg_quantize_workers, &sig_mqg_quantize_workers_l2, &sig_mqg_dequant_accumulate,
    &sig_mqg_apply, &sig_mqg_server_step, &sig_mqg_quantize_workers_minmax, &sig_mqg_quantize_minmax,
    &sig_mqg_dequant_accumulate_minmax, &sig_mqg_server_step_minmax, &sig_mqg_server_requantize,
    &sig_mqg_quantize_segments, &sig_mqg_quantize_segments_workers, &sig_mqg_server_step_segments,
    &sig_mqg_quantize_1bit_ef, &sig_mqg_quantize_l2, &sig_mqg_quantize_segments_l2,
    &sig_mqg_quantize_segments_l2_static, &sig_mqg_grad_norm, &sig_mqg_clip_grad_norm, &sig_mqg_clip_flatten,
    &sig_mqg_scale_grads, &sig_mqg_apply_clipped, &sig_mqg_embedding, &sig_mqg_embedding_grad,
    &sig_mqg_adamw, &sig_mqg_adamw8, &sig_mqg_layer_norm, &sig_mqg_layer_norm_grad,
};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_binding", "Native entry points of libmqgrad.", -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void)
{
    for (Signature* s : kSignatures)
        for (int i = 0; i < s->nargs; ++i) {
            s->interned[i] = PyUnicode_InternFromString(s->names[i]);
            if (!s->interned[i]) return nullptr;
        }
    return PyModule_Create(&kModule);
}
