// The marshalling of binding.Handle's scoring calls, natively: a decoding step's call takes a few microseconds on the
// GPU, and reading a tensor's attributes, allocating the result and converting arguments from Python took more than
// that.  Checks of tensors (TypeError), allocation of results, the current stream, one call through the C ABI, its status
// (binding.ExcpError).  The addresses of the C functions come from the library that binding.py has loaded.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <stdexcept>
#include <string>

#include "../../include/excp.h"

namespace {

struct Api {
    decltype(&excp_mx4_bytes) mx4_bytes;
    decltype(&excp_mx4_tensor_scale) mx4_tensor_scale;
    decltype(&excp_mx4_quantize) mx4_quantize;
    decltype(&excp_mx4_dequantize) mx4_dequantize;
    decltype(&excp_mx4_matmul) mx4_matmul;
    decltype(&excp_mx4_linear_scratch) mx4_linear_scratch;
    decltype(&excp_mx4_linear) mx4_linear;
    decltype(&excp_token_logprobs) token_logprobs;
    decltype(&excp_token_logprobs_grad) token_logprobs_grad;
} api;
PyObject* excp_error;                              // binding.ExcpError

struct Refused : std::runtime_error {              // becomes a TypeError
    using std::runtime_error::runtime_error;
};
struct Status {                                    // becomes an ExcpError
    int code;
    const char* call;
};
struct PythonError {};                             // already set

void check(excp_status s, const char* call) {
    if (s != EXCP_OK) throw Status{(int)s, call};
}

long long integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PythonError{};
    return v;
}
excp_handle handle(PyObject* o) { return reinterpret_cast<excp_handle>(integer(o)); }

const at::Tensor& tensor(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) throw Refused(std::string(what) + ": expected a tensor");
    return THPVariable_Unpack(o);
}
PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }

int dtype_code(at::ScalarType t) {
    return t == at::kFloat ? EXCP_F32 : t == at::kHalf ? EXCP_F16 : t == at::kBFloat16 ? EXCP_BF16 : -1;
}
at::ScalarType wanted(PyObject* o) {
    if (!THPDtype_Check(o)) throw Refused("dtype: expected a torch.dtype");
    const at::ScalarType t = reinterpret_cast<THPDtype*>(o)->scalar_type;
    if (dtype_code(t) < 0) throw Refused("dtype: expected float32, float16 or bfloat16");
    return t;
}

bool on(const at::Tensor& t, int device) { return t.is_cuda() && t.get_device() == device; }
// A new tensor straight from torch's allocator for the device.
at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType t, int device) {
    return at::detail::empty_cuda(sizes, t, at::Device(at::kCUDA, (c10::DeviceIndex)device), std::nullopt);
}
// A contiguous tensor within the bytes of another one.
at::Tensor within(const at::Tensor& base, at::ScalarType t, at::IntArrayRef sizes, int64_t at_byte) {
    auto impl = c10::make_intrusive<c10::TensorImpl>(c10::Storage(base.storage()), base.key_set(), c10::scalarTypeToTypeMeta(t));
    impl->set_sizes_contiguous(sizes);
    impl->set_storage_offset(at_byte / (int64_t)c10::elementSize(t));
    return at::Tensor(std::move(impl));
}
void* stream(int device) { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }

struct Rows {                                      // a 2-D tensor whose last dimension is dense
    void* p;
    int dtype;
    size_t rows, cols, stride;
};
Rows rows(const at::Tensor& t, int device, const char* what) {
    const int dt = dtype_code(t.scalar_type());
    if (t.dim() != 2 || dt < 0 || !on(t, device))
        throw Refused(std::string(what) + ": expected a 2-D float32, float16 or bfloat16 tensor on cuda:" + std::to_string(device));
    const int64_t r = t.size(0), c = t.size(1);
    if (c > 1 && t.stride(1) != 1) throw Refused(std::string(what) + ": the last dimension must be dense");
    return Rows{t.data_ptr(), dt, (size_t)r, (size_t)c, (size_t)(r > 1 ? t.stride(0) : c)};
}
void* vector(PyObject* o, int device, at::ScalarType type, int64_t n, const char* what) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, what);
    if (t.scalar_type() != type || t.numel() != n || !on(t, device) || !t.is_contiguous())
        throw Refused(std::string(what) + ": expected " + std::to_string(n) + " contiguous values of the right type on cuda:" + std::to_string(device));
    return t.data_ptr();
}
void* packed(const at::Tensor& t, int device, size_t need, const char* what) {
    if (t.scalar_type() != at::kByte || !on(t, device) || !t.is_contiguous() || (size_t)t.numel() < need)
        throw Refused(std::string(what) + ": expected at least " + std::to_string(need) + " contiguous uint8 values on cuda:" + std::to_string(device));
    return t.data_ptr();
}
// `out`, or a new [r, c] tensor where it is None.
at::Tensor result(PyObject* out, int device, at::ScalarType type, int64_t r, int64_t c) {
    if (out == Py_None) return fresh({r, c}, type, device);
    const at::Tensor& t = tensor(out, "out");
    if (t.dim() != 2 || t.size(0) != r || t.size(1) != c)
        throw Refused("out: expected the shape [" + std::to_string(r) + ", " + std::to_string(c) + "]");
    return t;
}

// (handle, device, x, out or None)
PyObject* tensor_scale(PyObject* const* a) {
    const int device = (int)integer(a[1]);
    const Rows x = rows(tensor(a[2], "x"), device, "x");
    const at::Tensor out = a[3] == Py_None ? fresh({}, at::kFloat, device) : tensor(a[3], "out");
    if (out.scalar_type() != at::kFloat || out.numel() != 1 || !on(out, device)) throw Refused("out: expected one float32 value on the handle's device");
    check(api.mx4_tensor_scale(handle(a[0]), x.p, x.dtype, x.rows, x.cols, x.stride, static_cast<float*>(out.data_ptr()), stream(device)), "excp_mx4_tensor_scale");
    return wrap(out);
}

// (handle, device, x, format, scale or None, out or None)
PyObject* quantize(PyObject* const* a) {
    const int device = (int)integer(a[1]), format = (int)integer(a[3]);
    const Rows x = rows(tensor(a[2], "x"), device, "x");
    const size_t need = api.mx4_bytes(x.rows, x.cols, format);
    const at::Tensor out = a[5] == Py_None ? fresh({(int64_t)need}, at::kByte, device) : tensor(a[5], "out");
    check(api.mx4_quantize(handle(a[0]), x.p, x.dtype, x.rows, x.cols, x.stride, format,
                           static_cast<float*>(vector(a[4], device, at::kFloat, 1, "tensor_scale")), packed(out, device, need, "out"), stream(device)), "excp_mx4_quantize");
    return wrap(out);
}

// (handle, device, data, rows, cols, format, scale or None, dtype, out or None)
PyObject* dequantize(PyObject* const* a) {
    const int device = (int)integer(a[1]), format = (int)integer(a[5]);
    const long long r = integer(a[3]), c = integer(a[4]);
    void* p = packed(tensor(a[2], "m"), device, api.mx4_bytes(r, c, format), "m");
    const at::Tensor out = result(a[8], device, wanted(a[7]), r, c);
    const Rows y = rows(out, device, "out");
    check(api.mx4_dequantize(handle(a[0]), p, r, c, format, static_cast<float*>(vector(a[6], device, at::kFloat, 1, "scale")), y.p, y.dtype, y.stride, stream(device)), "excp_mx4_dequantize");
    return wrap(out);
}

// (handle, device, a, a rows, a scale, b, b rows, b scale, cols, format, bias or None, dtype, out or None)
PyObject* matmul(PyObject* const* a) {
    const int device = (int)integer(a[1]), format = (int)integer(a[9]);
    const long long ar = integer(a[3]), br = integer(a[6]), c = integer(a[8]);
    void* pa = packed(tensor(a[2], "a"), device, api.mx4_bytes(ar, c, format), "a");
    void* pb = packed(tensor(a[5], "b"), device, api.mx4_bytes(br, c, format), "b");
    const at::Tensor out = result(a[12], device, wanted(a[11]), ar, br);
    const Rows y = rows(out, device, "out");
    check(api.mx4_matmul(handle(a[0]), pa, ar, static_cast<float*>(vector(a[4], device, at::kFloat, 1, "a.scale")), pb, br,
                         static_cast<float*>(vector(a[7], device, at::kFloat, 1, "b.scale")), c, format,
                         static_cast<float*>(vector(a[10], device, at::kFloat, br, "bias")), y.p, y.dtype, y.stride, stream(device)), "excp_mx4_matmul");
    return wrap(out);
}

// (handle, device, x, x scale, w, w rows, w scale, cols, format, bias or None, dtype or None, out or None, room or None)
PyObject* linear(PyObject* const* a) {
    const excp_handle h = handle(a[0]);
    const int device = (int)integer(a[1]), format = (int)integer(a[8]);
    const at::Tensor& xt = tensor(a[2], "x");
    const Rows x = rows(xt, device, "x");
    const long long wr = integer(a[5]), c = integer(a[7]);
    if ((long long)x.cols != c) throw Refused("x: expected " + std::to_string(c) + " columns");
    void* w = packed(tensor(a[4], "w"), device, api.mx4_bytes(wr, c, format), "w");
    const at::Tensor out = result(a[11], device, a[10] == Py_None ? xt.scalar_type() : wanted(a[10]), (int64_t)x.rows, wr);
    const Rows y = rows(out, device, "out");
    const size_t need = api.mx4_linear_scratch(h, x.rows, wr, c, format);
    at::Tensor room;                               // torch's allocator hands it out again only behind this call's work
    void* px = nullptr;
    if (a[12] != Py_None) px = packed(tensor(a[12], "x_packed"), device, need, "x_packed");
    else if (need) px = (room = fresh({(int64_t)need}, at::kByte, device)).data_ptr();
    check(api.mx4_linear(h, x.p, x.dtype, x.rows, x.stride, static_cast<float*>(vector(a[3], device, at::kFloat, 1, "tensor_scale")), w, wr,
                         static_cast<float*>(vector(a[6], device, at::kFloat, 1, "w.scale")), c, format,
                         static_cast<float*>(vector(a[9], device, at::kFloat, wr, "bias")), y.p, y.dtype, y.stride, px, stream(device)), "excp_mx4_linear");
    return wrap(out);
}

// What torch's allocator hands out at least, so that results which fit it hold no more together than one of them alone.  Every
// further allocation costs a call about 0.5 us (three alternatives: one allocation 4.6 us of host time, three 5.6, five 6.6).
constexpr int64_t ONE_BLOCK = 512;

// (handle, device, logits, tokens, top, scale) -> (logprob, entropy, top_logprob or None, top_index or None, row_stats)
PyObject* logprobs(PyObject* const* a) {
    const int device = (int)integer(a[1]);
    const Rows x = rows(tensor(a[2], "logits"), device, "logits");
    const long long top = integer(a[4]);
    const double scale = PyFloat_AsDouble(a[5]);
    if (scale == -1.0 && PyErr_Occurred()) throw PythonError{};
    const int64_t r = (int64_t)x.rows;
    const long long* tokens = static_cast<long long*>(vector(a[3], device, at::kLong, r, "tokens"));
    const int64_t k = top > 0 && top <= (1 << 20) ? top : 0;
    const int number = top < 0 || top > INT_MAX ? -1 : (int)top;           // what does not fit is refused, not cut
    // Bytes: row statistics 16 a row, alternatives 8 and 4 each, log probability and entropy 4 and 4 a row.  What is kept or saved
    // on its own has memory of its own: the statistics, the alternatives, and the two values a row.
    at::Tensor all, some;
    if (r * (24 + 12 * k) <= ONE_BLOCK) all = some = fresh({r * (24 + 12 * k)}, at::kByte, device);
    const int64_t some_at = all.defined() ? 16 * r : 0, two_at = all.defined() ? 16 * r + 12 * r * k : 0;
    const at::Tensor stats = all.defined() ? within(all, at::kFloat, {r, 4}, 0) : fresh({r, 4}, at::kFloat, device);
    at::Tensor tl, ti;
    if (k) {
        if (!all.defined()) some = fresh({12 * r * k}, at::kByte, device);
        ti = within(some, at::kLong, {r, k}, some_at);
        tl = within(some, at::kFloat, {r, k}, some_at + 8 * r * k);
    }
    const at::Tensor two = all.defined() ? all : fresh({8 * r}, at::kByte, device);
    const at::Tensor lp = within(two, at::kFloat, {r}, two_at), h = within(two, at::kFloat, {r}, two_at + 4 * r);
    check(api.token_logprobs(handle(a[0]), x.p, x.dtype, x.rows, x.cols, x.stride, tokens, (float)scale, number, static_cast<float*>(lp.data_ptr()),
                             static_cast<float*>(h.data_ptr()), static_cast<float*>(stats.data_ptr()), tl.defined() ? static_cast<float*>(tl.data_ptr()) : nullptr,
                             ti.defined() ? static_cast<long long*>(ti.data_ptr()) : nullptr, stream(device)), "excp_token_logprobs");
    PyObject* out = PyTuple_New(5);
    if (!out) throw PythonError{};
    PyTuple_SET_ITEM(out, 0, wrap(lp));
    PyTuple_SET_ITEM(out, 1, wrap(h));
    PyTuple_SET_ITEM(out, 2, tl.defined() ? wrap(tl) : Py_NewRef(Py_None));
    PyTuple_SET_ITEM(out, 3, ti.defined() ? wrap(ti) : Py_NewRef(Py_None));
    PyTuple_SET_ITEM(out, 4, wrap(stats));
    return out;
}

// (handle, device, logits, tokens, row_stats, scale, g_logprob or None, g_entropy or None, out or None)
PyObject* logprobs_grad(PyObject* const* a) {
    const int device = (int)integer(a[1]);
    const at::Tensor& xt = tensor(a[2], "logits");
    const Rows x = rows(xt, device, "logits");
    const double scale = PyFloat_AsDouble(a[5]);
    if (scale == -1.0 && PyErr_Occurred()) throw PythonError{};
    const int64_t r = (int64_t)x.rows;
    const at::Tensor out = result(a[8], device, xt.scalar_type(), r, (int64_t)x.cols);
    const Rows y = rows(out, device, "out");
    if (y.dtype != x.dtype) throw Refused("out: expected the logits' type");
    check(api.token_logprobs_grad(handle(a[0]), x.p, x.dtype, x.rows, x.cols, x.stride, static_cast<long long*>(vector(a[3], device, at::kLong, r, "tokens")), (float)scale,
                                  static_cast<float*>(vector(a[4], device, at::kFloat, r * 4, "row_stats")), static_cast<float*>(vector(a[6], device, at::kFloat, r, "g_logprob")),
                                  static_cast<float*>(vector(a[7], device, at::kFloat, r, "g_entropy")), y.p, y.stride, stream(device)), "excp_token_logprobs_grad");
    return wrap(out);
}

// Python's side: argument count, and no C++ exception leaves.
template <PyObject* (*F)(PyObject* const*), Py_ssize_t N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments", N);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const PythonError&) {
    } catch (const Refused& e) {
        PyErr_SetString(PyExc_TypeError, e.what());
    } catch (const Status& s) {
        PyObject* e = PyObject_CallFunction(excp_error, "is", s.code, s.call);
        if (e) {
            PyErr_SetObject(excp_error, e);
            Py_DECREF(e);
        }
    } catch (const std::exception& e) {            // torch's own, out of memory among them
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

// (addresses in the order of Api, ExcpError)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    constexpr Py_ssize_t count = sizeof(Api) / sizeof(void*);
    if (n != count + 1) {
        PyErr_SetString(PyExc_TypeError, "bind: wrong number of addresses");
        return nullptr;
    }
    void* at[count];
    for (Py_ssize_t i = 0; i < count; ++i) {
        at[i] = PyLong_AsVoidPtr(args[i]);
        if (!at[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "bind: null address");
            return nullptr;
        }
    }
    static_assert(sizeof(Api) == sizeof(at), "function pointers");
    memcpy(&api, at, sizeof(api));
    Py_XDECREF(excp_error);
    excp_error = Py_NewRef(args[count]);
    Py_RETURN_NONE;
}

#define EXCP_ENTRY(name, f, n) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<f, n>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&bind)), METH_FASTCALL, nullptr},
    EXCP_ENTRY("mx4_tensor_scale", tensor_scale, 4),
    EXCP_ENTRY("mx4_quantize", quantize, 6),
    EXCP_ENTRY("mx4_dequantize", dequantize, 9),
    EXCP_ENTRY("mx4_matmul", matmul, 13),
    EXCP_ENTRY("mx4_linear", linear, 13),
    EXCP_ENTRY("token_logprobs", logprobs, 6),
    EXCP_ENTRY("token_logprobs_grad", logprobs_grad, 9),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_score", "Native marshalling of the scoring calls.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__score() { return PyModule_Create(&module); }
