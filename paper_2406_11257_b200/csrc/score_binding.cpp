// The marshalling of binding.Handle's scoring calls and layers, natively: a decoding step's call takes a few microseconds on the
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
    decltype(&excp_act8_bytes) act8_bytes;
    decltype(&excp_act8_quantize) act8_quantize;
    decltype(&excp_act8_restore) act8_restore;
    decltype(&excp_act_grad_scratch) act_grad_scratch;
    decltype(&excp_act_grad) act_grad;
    decltype(&excp_layer_norm) layer_norm;
    decltype(&excp_layer_norm_grad_scratch) layer_norm_grad_scratch;
    decltype(&excp_layer_norm_grad) layer_norm_grad;
    decltype(&excp_linear_scratch) linear_scratch;
    decltype(&excp_linear) linear;
    decltype(&excp_linear_grad_input) linear_grad_input;
    decltype(&excp_linear_grad_weight) linear_grad_weight;
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

// A result, behind the call that wrote it.  Where it is a tensor of the caller's (`given` is not None), autograd is told that it has changed.
PyObject* wrap_written(const at::Tensor& t, PyObject* given) {
    if (given != Py_None && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    return wrap(t);
}

// (handle, device, x, out or None)
PyObject* tensor_scale(PyObject* const* a) {
    const int device = (int)integer(a[1]);
    const Rows x = rows(tensor(a[2], "x"), device, "x");
    const at::Tensor out = a[3] == Py_None ? fresh({}, at::kFloat, device) : tensor(a[3], "out");
    if (out.scalar_type() != at::kFloat || out.numel() != 1 || !on(out, device)) throw Refused("out: expected one float32 value on the handle's device");
    check(api.mx4_tensor_scale(handle(a[0]), x.p, x.dtype, x.rows, x.cols, x.stride, static_cast<float*>(out.data_ptr()), stream(device)), "excp_mx4_tensor_scale");
    return wrap_written(out, a[3]);
}

// (handle, device, x, format, scale or None, out or None)
PyObject* quantize(PyObject* const* a) {
    const int device = (int)integer(a[1]), format = (int)integer(a[3]);
    const Rows x = rows(tensor(a[2], "x"), device, "x");
    const size_t need = api.mx4_bytes(x.rows, x.cols, format);
    const at::Tensor out = a[5] == Py_None ? fresh({(int64_t)need}, at::kByte, device) : tensor(a[5], "out");
    check(api.mx4_quantize(handle(a[0]), x.p, x.dtype, x.rows, x.cols, x.stride, format,
                           static_cast<float*>(vector(a[4], device, at::kFloat, 1, "tensor_scale")), packed(out, device, need, "out"), stream(device)), "excp_mx4_quantize");
    return wrap_written(out, a[5]);
}

// (handle, device, data, rows, cols, format, scale or None, dtype, out or None)
PyObject* dequantize(PyObject* const* a) {
    const int device = (int)integer(a[1]), format = (int)integer(a[5]);
    const long long r = integer(a[3]), c = integer(a[4]);
    void* p = packed(tensor(a[2], "m"), device, api.mx4_bytes(r, c, format), "m");
    const at::Tensor out = result(a[8], device, wanted(a[7]), r, c);
    const Rows y = rows(out, device, "out");
    check(api.mx4_dequantize(handle(a[0]), p, r, c, format, static_cast<float*>(vector(a[6], device, at::kFloat, 1, "scale")), y.p, y.dtype, y.stride, stream(device)), "excp_mx4_dequantize");
    return wrap_written(out, a[8]);
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
    return wrap_written(out, a[12]);
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
    return wrap_written(out, a[11]);
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
    return wrap_written(out, a[8]);
}

// ---- the layers before the logits --------------------------------------------------------------------------------------------------
excp_matrix matrix(const at::Tensor& t, int device, const char* what) {
    const Rows r = rows(t, device, what);
    return excp_matrix{r.p, r.dtype, r.rows, r.cols, r.stride};
}
excp_matrix shaped(const at::Tensor& t, int device, const char* what, size_t r, size_t c) {
    const excp_matrix m = matrix(t, device, what);
    if (m.rows != r || m.cols != c) throw Refused(std::string(what) + ": expected the shape [" + std::to_string(r) + ", " + std::to_string(c) + "]");
    return m;
}
// None, or a matrix of that shape.
const excp_matrix* optional(PyObject* o, int device, const char* what, size_t r, size_t c, excp_matrix& room) {
    if (o == Py_None) return nullptr;
    room = shaped(tensor(o, what), device, what, r, c);
    return &room;
}
// What a matrix of 8 bits says: without the bytes behind its last scale, which no call reads.
size_t act8_said(size_t r, size_t c) { return api.act8_bytes(r, c) ? r * ((c + 31) / 32) * 34 : 0; }
// A plain matrix, or the data of a packed one of 8 bits (where `is_packed`).
excp_matrix kept(PyObject* o, bool is_packed, int device, const char* what, size_t r, size_t c) {
    const at::Tensor& t = tensor(o, what);
    if (!is_packed) return shaped(t, device, what, r, c);
    return excp_matrix{packed(t, device, act8_said(r, c), what), EXCP_ACT8, r, c, c};
}
// One value per column, of type float32 or any 16-bit one.
void* columns(PyObject* o, int device, int64_t n, int& dtype, const char* what) {
    dtype = EXCP_F32;
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, what);
    dtype = dtype_code(t.scalar_type());
    if (dtype < 0 || t.dim() != 1 || t.numel() != n || !on(t, device) || !t.is_contiguous())
        throw Refused(std::string(what) + ": expected " + std::to_string(n) + " contiguous float32, float16 or bfloat16 values on cuda:" + std::to_string(device));
    return t.data_ptr();
}
// Scratch from torch's allocator, which hands it out again only behind this call's work.
struct Scratch {
    at::Tensor t;
    void* p = nullptr;
    Scratch(size_t need, int device) {
        if (need) p = (t = fresh({(int64_t)need}, at::kByte, device)).data_ptr();
    }
};
bool flag(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PythonError{};
    return v != 0;
}
PyObject* or_none(const at::Tensor& t) { return t.defined() ? wrap(t) : Py_NewRef(Py_None); }
template <typename... O>
PyObject* tuple(O... items) {
    PyObject* out = PyTuple_New(sizeof...(items));
    if (!out) throw PythonError{};
    Py_ssize_t i = 0;
    (PyTuple_SET_ITEM(out, i++, items), ...);
    return out;
}

// (handle, device, x, out or None)
PyObject* act8_quantize(PyObject* const* a) {
    const int device = (int)integer(a[1]);
    const excp_matrix x = matrix(tensor(a[2], "x"), device, "x");
    const size_t need = api.act8_bytes(x.rows, x.cols);
    const at::Tensor out = a[3] == Py_None ? fresh({(int64_t)need}, at::kByte, device) : tensor(a[3], "out");
    check(api.act8_quantize(handle(a[0]), &x, packed(out, device, need, "out"), stream(device)), "excp_act8_quantize");
    return wrap_written(out, a[3]);
}

// (handle, device, data, rows, cols, dtype, out or None)
PyObject* act8_restore(PyObject* const* a) {
    const int device = (int)integer(a[1]);
    const long long r = integer(a[3]), c = integer(a[4]);
    void* p = packed(tensor(a[2], "m"), device, act8_said(r, c), "m");
    const at::Tensor out = result(a[6], device, wanted(a[5]), r, c);
    const excp_matrix y = matrix(out, device, "out");
    check(api.act8_restore(handle(a[0]), p, &y, stream(device)), "excp_act8_restore");
    return wrap_written(out, a[6]);
}

// (handle, device, dy, pre or None, pre is packed, act, dpre wanted, again wanted, dbias wanted, out or None) -> (dpre, a, dbias), each or None
PyObject* act_grad(PyObject* const* a) {
    const excp_handle h = handle(a[0]);
    const int device = (int)integer(a[1]), act = (int)integer(a[5]);
    const at::Tensor& t = tensor(a[2], "dy");
    const excp_matrix dy = matrix(t, device, "dy");
    excp_matrix pre, dpre, again;
    const bool has_pre = a[3] != Py_None;
    if (has_pre) pre = kept(a[3], flag(a[4]), device, "pre", dy.rows, dy.cols);
    const int64_t r = (int64_t)dy.rows, c = (int64_t)dy.cols;
    at::Tensor out, value, db;
    if (flag(a[6])) dpre = shaped(out = result(a[9], device, t.scalar_type(), r, c), device, "out", r, c);
    if (flag(a[7])) again = shaped(value = fresh({r, c}, t.scalar_type(), device), device, "again", r, c);
    if (flag(a[8])) db = fresh({c}, at::kFloat, device);
    const Scratch room(db.defined() ? api.act_grad_scratch(h, dy.rows, dy.cols) : 0, device);
    check(api.act_grad(h, act, &dy, has_pre ? &pre : nullptr, out.defined() ? &dpre : nullptr, value.defined() ? &again : nullptr,
                       db.defined() ? static_cast<float*>(db.data_ptr()) : nullptr, room.p, stream(device)), "excp_act_grad");
    return tuple(out.defined() ? wrap_written(out, a[9]) : Py_NewRef(Py_None), or_none(value), or_none(db));
}

// (handle, device, x, weight or None, bias or None, eps, rms, kept wanted, out or None) -> (y, row_stats, kept or None)
PyObject* layer_norm(PyObject* const* a) {
    const int device = (int)integer(a[1]);
    const at::Tensor& t = tensor(a[2], "x");
    const excp_matrix x = matrix(t, device, "x");
    int wt, bt;
    void* w = columns(a[3], device, (int64_t)x.cols, wt, "weight");
    void* b = columns(a[4], device, (int64_t)x.cols, bt, "bias");
    if (w && b && wt != bt) throw Refused("weight, bias: expected the same type");
    const double eps = PyFloat_AsDouble(a[5]);
    if (eps == -1.0 && PyErr_Occurred()) throw PythonError{};
    const int64_t r = (int64_t)x.rows;
    const at::Tensor out = result(a[8], device, t.scalar_type(), r, (int64_t)x.cols);
    const excp_matrix y = matrix(out, device, "out");
    const at::Tensor stats = fresh({r, 2}, at::kFloat, device);
    at::Tensor k;
    if (flag(a[7])) k = fresh({(int64_t)api.act8_bytes(x.rows, x.cols)}, at::kByte, device);
    check(api.layer_norm(handle(a[0]), &x, w, b, w ? wt : bt, (float)eps, flag(a[6]), &y, static_cast<float*>(stats.data_ptr()), k.defined() ? k.data_ptr() : nullptr,
                         stream(device)), "excp_layer_norm");
    return tuple(wrap_written(out, a[8]), wrap(stats), or_none(k));
}

// (handle, device, dy, x, x is packed, weight or None, rms, row_stats, add or None, out or None, vectors wanted) -> (dx, dweight, dbias), the last two or None
PyObject* layer_norm_grad(PyObject* const* a) {
    const excp_handle h = handle(a[0]);
    const int device = (int)integer(a[1]);
    const at::Tensor& t = tensor(a[2], "dy");
    const excp_matrix dy = matrix(t, device, "dy"), x = kept(a[3], flag(a[4]), device, "x", dy.rows, dy.cols);
    const int64_t r = (int64_t)dy.rows, c = (int64_t)dy.cols;
    int wt;
    void* w = columns(a[5], device, c, wt, "weight");
    const bool rms = flag(a[6]), vectors = flag(a[10]);
    excp_matrix add_room;
    const excp_matrix* add = optional(a[8], device, "add", dy.rows, dy.cols, add_room);
    const at::Tensor out = result(a[9], device, t.scalar_type(), r, c);
    const excp_matrix dx = matrix(out, device, "out");
    at::Tensor dw, db;
    if (vectors) dw = fresh({c}, at::kFloat, device);
    if (vectors && !rms) db = fresh({c}, at::kFloat, device);
    const Scratch room(api.layer_norm_grad_scratch(h, dy.rows, dy.cols), device);
    check(api.layer_norm_grad(h, &dy, &x, w, wt, rms, static_cast<float*>(vector(a[7], device, at::kFloat, 2 * r, "row_stats")), add, &dx,
                              dw.defined() ? static_cast<float*>(dw.data_ptr()) : nullptr, db.defined() ? static_cast<float*>(db.data_ptr()) : nullptr, room.p,
                              stream(device)), "excp_layer_norm_grad");
    return tuple(wrap_written(out, a[9]), or_none(dw), or_none(db));
}

// (handle, device, x, w, bias or None, act, residual or None, dtype or None, out or None, keep: None, a dtype or True for 8 bits) -> (y, kept or None)
PyObject* plain_linear(PyObject* const* a) {
    const int device = (int)integer(a[1]), act = (int)integer(a[5]);
    const at::Tensor& t = tensor(a[2], "x");
    const excp_matrix x = matrix(t, device, "x"), w = matrix(tensor(a[3], "w"), device, "w");
    int bt;
    void* b = columns(a[4], device, (int64_t)w.rows, bt, "bias");
    const int64_t r = (int64_t)x.rows, n = (int64_t)w.rows;
    excp_matrix residual_room, keep;
    const excp_matrix* residual = optional(a[6], device, "residual", x.rows, w.rows, residual_room);
    const at::Tensor out = result(a[8], device, a[7] == Py_None ? t.scalar_type() : wanted(a[7]), r, n);
    const excp_matrix y = matrix(out, device, "out");
    at::Tensor k;
    if (a[9] == Py_True) {
        k = fresh({(int64_t)api.act8_bytes(x.rows, w.rows)}, at::kByte, device);
        keep = excp_matrix{k.data_ptr(), EXCP_ACT8, x.rows, w.rows, w.rows};
    } else if (a[9] != Py_None) {
        keep = matrix(k = fresh({r, n}, wanted(a[9]), device), device, "kept");
    }
    const Scratch room(api.linear_scratch(&x, &w), device);
    check(api.linear(handle(a[0]), &x, &w, b, bt, act, residual, &y, k.defined() ? &keep : nullptr, room.p, stream(device)), "excp_linear");
    return tuple(wrap_written(out, a[8]), or_none(k));
}

// (handle, device, dy, w, add or None, dtype or None, out or None)
PyObject* linear_grad_input(PyObject* const* a) {
    const int device = (int)integer(a[1]);
    const at::Tensor& t = tensor(a[2], "dy");
    const excp_matrix dy = matrix(t, device, "dy"), w = matrix(tensor(a[3], "w"), device, "w");
    excp_matrix add_room;
    const excp_matrix* add = optional(a[4], device, "add", dy.rows, w.cols, add_room);
    const at::Tensor out = result(a[6], device, a[5] == Py_None ? t.scalar_type() : wanted(a[5]), (int64_t)dy.rows, (int64_t)w.cols);
    const excp_matrix dx = matrix(out, device, "out");
    const Scratch room(api.linear_scratch(&dy, &w), device);
    check(api.linear_grad_input(handle(a[0]), &dy, &w, add, &dx, room.p, stream(device)), "excp_linear_grad_input");
    return wrap_written(out, a[6]);
}

// (handle, device, dy, x, add or None, dtype, out or None)
PyObject* linear_grad_weight(PyObject* const* a) {
    const int device = (int)integer(a[1]);
    const excp_matrix dy = matrix(tensor(a[2], "dy"), device, "dy"), x = matrix(tensor(a[3], "x"), device, "x");
    excp_matrix add_room;
    const excp_matrix* add = optional(a[4], device, "add", dy.cols, x.cols, add_room);
    const at::Tensor out = result(a[6], device, wanted(a[5]), (int64_t)dy.cols, (int64_t)x.cols);
    const excp_matrix dw = matrix(out, device, "out");
    const Scratch room(api.linear_scratch(&dy, &x), device);
    check(api.linear_grad_weight(handle(a[0]), &dy, &x, add, &dw, room.p, stream(device)), "excp_linear_grad_weight");
    return wrap_written(out, a[6]);
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
    EXCP_ENTRY("act8_quantize", act8_quantize, 4),
    EXCP_ENTRY("act8_restore", act8_restore, 7),
    EXCP_ENTRY("act_grad", act_grad, 10),
    EXCP_ENTRY("layer_norm", layer_norm, 9),
    EXCP_ENTRY("layer_norm_grad", layer_norm_grad, 11),
    EXCP_ENTRY("linear", plain_linear, 10),
    EXCP_ENTRY("linear_grad_input", linear_grad_input, 7),
    EXCP_ENTRY("linear_grad_weight", linear_grad_weight, 7),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_score", "Native marshalling of the scoring calls.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__score() { return PyModule_Create(&module); }
