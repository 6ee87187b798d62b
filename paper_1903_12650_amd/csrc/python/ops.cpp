// The calls of one operation that a Python program makes once per layer, marshalled natively: argument checks, descriptor, output
// and workspace tensors, the call of the C ABI.  At small batches such a call is a few microseconds of GPU time, and what it
// costs in the interpreter (a tensor allocation 1.3 us, an address with its checks 0.3, a converted argument 0.1, five to fifteen
// of each) is longer: a float bottleneck block at batch 2, 21 calls, forward, backward and LARS, took 250 us for 188 us of GPU
// time with the same steps in Python, and takes 218 with them here.
// Signatures and defaults are those of the functions of the same names in binding.py, which are the callers.  Errors are raised as
// there (AssertionError, TypeError, ValueError, Rn50Error), and torch's own as torch raises them from Python (an allocation that
// does not fit: torch.OutOfMemoryError), without a C++ backtrace in the text.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <algorithm>
#include <exception>
#include <string>
#include <vector>

#include <ATen/ATen.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../../include/rn50_hip.h"

namespace {

PyObject *g_error = nullptr, *g_stream = nullptr, *g_device = nullptr;  // Rn50Error; torch's current stream of a device and current device

struct PyError {  // (a Python exception is set)
};

// The call itself, without the interpreter's lock (a launch may have to wait for room in its queue).
template <typename F>
void call(F f) {
  PyThreadState* state = PyEval_SaveThread();
  const int rc = f();
  PyEval_RestoreThread(state);
  if (rc == 0) return;
  PyObject* e = PyObject_CallFunction(g_error, "is", rc, rn50_last_error());
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  throw PyError();
}
[[noreturn]] void raise(PyObject* type, const char* text) {
  PyErr_SetString(type, text);
  throw PyError();
}

const at::Tensor* tensor(PyObject* o) {  // null: None
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) raise(PyExc_TypeError, "expected a tensor");
  return &THPVariable_Unpack(o);
}
const at::Tensor& required(PyObject* o) {
  const at::Tensor* t = tensor(o);
  if (!t) raise(PyExc_TypeError, "expected a tensor");
  return *t;
}
template <typename T = void>
T* addr(const at::Tensor* t) {
  if (!t) return nullptr;
  if (!t->is_cuda() || !t->is_contiguous()) raise(PyExc_AssertionError, "device, contiguous tensors only");
  return static_cast<T*>(t->data_ptr());
}
template <typename T = void>
T* addr(const at::Tensor& t) { return addr<T>(&t); }

int dtype_of(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return RN50_F32;
  if (t.scalar_type() == at::kBFloat16) return RN50_BF16;
  raise(PyExc_TypeError, (std::string("unsupported dtype ") + c10::toString(t.scalar_type())).c_str());
}
int to_int(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw PyError();
  if (v != static_cast<int>(v)) raise(PyExc_OverflowError, "Python int too large to convert to C int");
  return static_cast<int>(v);
}
double to_double(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PyError();
  return v;
}
struct Shape4 {
  int64_t d[4];
};
Shape4 shape4(const at::Tensor& t) {
  if (t.dim() != 4) raise(PyExc_ValueError, "a tensor of four dimensions is expected");
  return {{t.size(0), t.size(1), t.size(2), t.size(3)}};
}
Shape4 shape4(PyObject* shape) {  // (any iterable of four numbers)
  Shape4 s;
  PyObject* seq = PySequence_Fast(shape, "a shape of four dimensions is expected");  // (a tuple or list is taken as it is)
  if (!seq) throw PyError();
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
  for (Py_ssize_t i = 0; i < 4 && n == 4 && !PyErr_Occurred(); ++i) s.d[i] = PyLong_AsLongLong(PySequence_Fast_GET_ITEM(seq, i));
  Py_DECREF(seq);
  if (PyErr_Occurred()) throw PyError();
  if (n != 4) raise(PyExc_ValueError, "a shape of four dimensions is expected");
  return s;
}
rn50_conv_desc conv_desc(const Shape4& x, const Shape4& w, PyObject* stride, PyObject* pad, int dtype) {
  if (x.d[3] != w.d[3]) raise(PyExc_AssertionError, "channels of the input and of the weights");
  auto i = [](int64_t v) { return static_cast<int>(v); };
  return rn50_conv_desc{i(x.d[0]), i(x.d[1]), i(x.d[2]), i(x.d[3]), i(w.d[0]), i(w.d[1]), i(w.d[2]), to_int(stride), to_int(pad), dtype};
}
at::Tensor empty(at::IntArrayRef size, at::ScalarType type, const at::Tensor& like) {
  return at::empty(size, at::TensorOptions().dtype(type).device(like.device()));
}
// A workspace of at least `need` bytes; none is made where none is needed.
struct Workspace {
  at::Tensor made;
  void* p = nullptr;
  size_t bytes = 0;
  Workspace(PyObject* given, size_t need, const at::Tensor& like) {
    const at::Tensor* t = tensor(given);
    if (!t && need) {
      made = empty({static_cast<int64_t>(need)}, at::kByte, like);
      t = &made;
    }
    p = addr(t);
    bytes = t ? static_cast<size_t>(t->numel()) : 0;
  }
};
// The tensor that is given, or a new one.
at::Tensor output(PyObject* given, at::IntArrayRef size, at::ScalarType type, const at::Tensor& like) {
  const at::Tensor* t = tensor(given);
  return t ? *t : empty(size, type, like);
}
PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }

template <typename F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F f) {
  if (n != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, n);
    return nullptr;
  }
  try {
    return f();
  } catch (const PyError&) {
    return nullptr;
  } catch (const std::exception&) {
    torch::translate_exception_to_python(std::current_exception());
    return nullptr;
  }
}
void* current_stream() {  // (asked for after the arguments were checked: without a GPU it raises)
  PyObject* dev = PyObject_CallNoArgs(g_device);
  if (!dev) throw PyError();
  PyObject* num = PyObject_CallOneArg(g_stream, dev);
  Py_DECREF(dev);
  if (!num) throw PyError();
  void* s = PyLong_AsVoidPtr(num);
  Py_DECREF(num);
  if (!s && PyErr_Occurred()) throw PyError();
  return s;
}

// conv_fwd(x, w, stride, pad, y, workspace)
PyObject* conv_fwd_py(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    const at::Tensor &x = required(a[0]), &w = required(a[1]);
    const rn50_conv_desc d = conv_desc(shape4(x), shape4(w), a[2], a[3], dtype_of(x));
    if (d.stride == 0) raise(PyExc_ZeroDivisionError, "stride");
    auto extent = [&](int64_t span) { return (span >= 0 ? span / d.stride : -1 - (-1 - span) / d.stride) + 1; };
    const at::Tensor y = output(a[4], {d.N, extent(d.H + 2 * d.pad - d.R), extent(d.W + 2 * d.pad - d.S), d.Cout}, x.scalar_type(), x);
    const Workspace ws(a[5], a[5] == Py_None ? conv_fwd_workspace_bytes(&d) : 0, x);
    void* const p[] = {addr(x), addr(w), addr(y), current_stream()};
    call([&] { return conv_fwd(&d, p[0], p[1], p[2], ws.p, ws.bytes, p[3]); });
    return wrap(y);
  });
}
// conv_dgrad(dy, w, x_shape, stride, pad, dx, workspace)
PyObject* conv_dgrad_py(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject* {
    const at::Tensor &dy = required(a[0]), &w = required(a[1]);
    const Shape4 xs = shape4(a[2]);
    const rn50_conv_desc d = conv_desc(xs, shape4(w), a[3], a[4], dtype_of(dy));
    const at::Tensor dx = output(a[5], {xs.d, 4}, dy.scalar_type(), dy);
    const Workspace ws(a[6], a[6] == Py_None ? conv_dgrad_workspace_bytes(&d) : 0, dy);
    void* const p[] = {addr(dy), addr(w), addr(dx), current_stream()};
    call([&] { return conv_dgrad(&d, p[0], p[1], p[2], ws.p, ws.bytes, p[3]); });
    return wrap(dx);
  });
}
// conv_wgrad(x, dy, w_shape, stride, pad, dw, workspace)
PyObject* conv_wgrad_py(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject* {
    const at::Tensor &x = required(a[0]), &dy = required(a[1]);
    const Shape4 ws_ = shape4(a[2]);
    const rn50_conv_desc d = conv_desc(shape4(x), ws_, a[3], a[4], dtype_of(x));
    const at::Tensor dw = output(a[5], {ws_.d, 4}, at::kFloat, x);
    const Workspace ws(a[6], a[6] == Py_None ? conv_wgrad_workspace_bytes(&d) : 0, x);
    void* const p[] = {addr(x), addr(dy), addr(dw), current_stream()};
    call([&] { return conv_wgrad(&d, p[0], p[1], static_cast<float*>(p[2]), ws.p, ws.bytes, p[3]); });
    return wrap(dw);
  });
}
rn50_bn_desc bn_desc(const at::Tensor& x, PyObject* eps, PyObject* mode) {
  const int64_t C = x.size(-1);
  if (x.dim() != 4 && C == 0) raise(PyExc_ZeroDivisionError, "channels");
  rn50_bn_desc d{1, 1, static_cast<int>(C ? x.numel() / C : 0), static_cast<int>(C), static_cast<float>(to_double(eps)), dtype_of(x), to_int(mode)};
  if (x.dim() == 4) {
    d.N = static_cast<int>(x.size(0)); d.H = static_cast<int>(x.size(1)); d.W = static_cast<int>(x.size(2));
  }
  return d;
}
// bn_relu_fwd(x, gamma, beta, residual, eps, mode, running_mean, running_var, momentum, workspace, relu_mask)
PyObject* bn_relu_fwd_py(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&]() -> PyObject* {
    const at::Tensor& x = required(a[0]);
    const rn50_bn_desc d = bn_desc(x, a[4], a[5]);
    const at::Tensor y = at::empty_like(x), mean = empty({d.C}, at::kFloat, x), rstd = empty({d.C}, at::kFloat, x);
    const Workspace ws(a[9], a[9] == Py_None ? bn_relu_fwd_workspace_bytes(&d) : 0, x);
    const float momentum = static_cast<float>(to_double(a[8]));
    float* const f[] = {addr<float>(tensor(a[1])), addr<float>(tensor(a[2])), addr<float>(mean), addr<float>(rstd),
                        addr<float>(tensor(a[6])), addr<float>(tensor(a[7]))};
    uint8_t* const mask = addr<uint8_t>(tensor(a[10]));
    void* const p[] = {addr(x), addr(tensor(a[3])), addr(y), current_stream()};
    call([&] { return bn_relu_fwd(&d, p[0], f[0], f[1], p[1], p[2], mask, f[2], f[3], f[4], f[5], momentum, ws.p, ws.bytes, p[3]); });
    return Py_BuildValue("NNN", wrap(y), wrap(mean), wrap(rstd));
  });
}
// bn_relu_bwd(dz, x, z, gamma, mean, rstd, mode, beta, dz2, eps, workspace, relu_mask)
PyObject* bn_relu_bwd_py(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject* {
    const at::Tensor& x = required(a[1]);
    const rn50_bn_desc d = bn_desc(x, a[9], a[6]);
    const at::Tensor dx = at::empty_like(x);
    at::Tensor dres;
    if (d.mode == 2) dres = at::empty_like(x);
    const at::Tensor dgamma = empty({d.C}, at::kFloat, x), dbeta = empty({d.C}, at::kFloat, x);
    const Workspace ws(a[10], a[10] == Py_None ? bn_relu_bwd_workspace_bytes(&d) : 0, x);
    float* const f[] = {addr<float>(tensor(a[3])), addr<float>(tensor(a[7])), addr<float>(tensor(a[4])), addr<float>(tensor(a[5])),
                        addr<float>(dgamma), addr<float>(dbeta)};
    uint8_t* const mask = addr<uint8_t>(tensor(a[11]));
    void* const p[] = {addr(tensor(a[0])), addr(tensor(a[8])), addr(x), addr(tensor(a[2])), addr(dx),
                       dres.defined() ? addr(dres) : nullptr, current_stream()};
    call([&] {
      return bn_relu_bwd(&d, p[0], p[1], p[2], p[3], mask, f[0], f[1], f[2], f[3], p[4], p[5], f[4], f[5], ws.p, ws.bytes, p[6]);
    });
    PyObject* res = Py_None;
    if (d.mode == 2) res = wrap(dres); else Py_INCREF(Py_None);
    return Py_BuildValue("NNNN", wrap(dx), res, wrap(dgamma), wrap(dbeta));
  });
}
// ------------------------------------------- 8-bit products and distillation
// A matrix whose rows are contiguous, on the current device; `ld`: elements from one row to the next.
struct Rows {
  void* p;
  int64_t n, c, ld;
};
void on_current_device(const at::Tensor& t) {
  PyObject* dev = PyObject_CallNoArgs(g_device);
  if (!dev) throw PyError();
  const long i = PyLong_AsLong(dev);
  Py_DECREF(dev);
  if (i == -1 && PyErr_Occurred()) throw PyError();
  if (t.device().index() != i) raise(PyExc_ValueError, "tensors of the current device are expected");
}
Rows rows_of(const at::Tensor& t) {
  if (t.dim() != 2) raise(PyExc_ValueError, "a matrix is expected");
  const int64_t n = t.size(0), c = t.size(1);
  if (n > INT32_MAX || c > INT32_MAX) raise(PyExc_ValueError, "a matrix of at most 2^31 - 1 rows and columns is expected");
  if (!t.is_cuda() || (c > 1 && t.stride(1) != 1)) raise(PyExc_AssertionError, "device tensors with contiguous rows only");
  return {t.data_ptr(), n, c, n > 1 ? t.stride(0) : std::max<int64_t>(t.stride(0), c)};
}
// A contiguous tensor of one type and size (None: null, where that is allowed).
template <typename T>
T* vec(PyObject* o, at::ScalarType type, at::IntArrayRef size, const char* what, const at::Tensor& like, bool optional = false) {
  if (optional && o == Py_None) return nullptr;
  const at::Tensor& t = required(o);
  if (t.scalar_type() != type) raise(PyExc_TypeError, (std::string(what) + ": " + c10::toString(type) + " is expected, got " + c10::toString(t.scalar_type())).c_str());
  if (t.sizes() != size) raise(PyExc_ValueError, (std::string(what) + ": the size does not fit").c_str());
  T* p = addr<T>(t);
  if (t.device() != like.device()) raise(PyExc_ValueError, (std::string(what) + ": on another device").c_str());
  return p;
}
at::ScalarType float_type(PyObject* o) {
  if (!THPDtype_Check(o)) raise(PyExc_TypeError, "a torch.dtype is expected");
  const at::ScalarType t = reinterpret_cast<THPDtype*>(o)->scalar_type;
  if (t != at::kFloat && t != at::kBFloat16) raise(PyExc_TypeError, (std::string("unsupported dtype ") + c10::toString(t)).c_str());
  return t;
}
// quant_rows_i8(x)
PyObject* quant_rows_i8_py(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 1, [&]() -> PyObject* {
    const at::Tensor& x = required(a[0]);
    const int dt = dtype_of(x);
    const Rows r = rows_of(x);
    on_current_device(x);
    const at::Tensor q = empty({r.n, static_cast<int64_t>(quant_i8_row_bytes(static_cast<int>(r.c)))}, at::kChar, x), scale = empty({r.n}, at::kFloat, x);
    int8_t* const pq = addr<int8_t>(q);
    float* const ps = addr<float>(scale);
    void* const s = current_stream();
    call([&] { return quant_rows_i8(static_cast<int>(r.n), static_cast<int>(r.c), dt, r.p, r.ld, pq, ps, s); });
    return Py_BuildValue("NN", wrap(q), wrap(scale));
  });
}
// The output of a product: a matrix of `rows` x `cols`, given or made.
at::Tensor product_out(PyObject* given, PyObject* dtype, int64_t rows, int64_t cols, const at::Tensor& like) {
  const at::Tensor* t = tensor(given);
  if (!t) return empty({rows, cols}, float_type(dtype), like);
  if (t->dim() != 2 || t->size(0) != rows || t->size(1) != cols) raise(PyExc_ValueError, "y: the size does not fit");
  if (t->device() != like.device()) raise(PyExc_ValueError, "y: on another device");
  return *t;
}
// matmul_i8(K, q, q_scale, w, w_scale, bias, dtype, y)
PyObject* matmul_i8_py(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const int K = to_int(a[0]);
    const at::Tensor &q = required(a[1]), &w = required(a[3]);
    if (q.dim() != 2 || w.dim() != 2) raise(PyExc_ValueError, "a matrix is expected");
    const int64_t row = static_cast<int64_t>(quant_i8_row_bytes(K)), M = q.size(0), N = w.size(0);
    if (M > INT32_MAX || N > INT32_MAX) raise(PyExc_ValueError, "a matrix of at most 2^31 - 1 rows is expected");
    const int8_t *pq = vec<int8_t>(a[1], at::kChar, {M, row}, "q", q), *pw = vec<int8_t>(a[3], at::kChar, {N, row}, "w", q);
    const float *qs = vec<float>(a[2], at::kFloat, {M}, "q_scale", q), *ws = vec<float>(a[4], at::kFloat, {N}, "w_scale", q);
    const float* bias = vec<float>(a[5], at::kFloat, {N}, "bias", q, true);
    on_current_device(q);
    const at::Tensor y = product_out(a[7], a[6], M, N, q);
    const Rows r = rows_of(y);
    const int dt = dtype_of(y);
    void* const s = current_stream();
    call([&] { return matmul_i8(static_cast<int>(M), static_cast<int>(N), K, pq, qs, pw, ws, bias, dt, r.p, r.ld, s); });
    return wrap(y);
  });
}
// fc_i8_fwd(x, w, w_scale, bias, dtype, y, workspace)
PyObject* fc_i8_fwd_py(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject* {
    const at::Tensor &x = required(a[0]), &w = required(a[1]);
    const int xt = dtype_of(x);
    const Rows rx = rows_of(x);
    if (w.dim() != 2) raise(PyExc_ValueError, "a matrix is expected");
    const int M = static_cast<int>(rx.n), K = static_cast<int>(rx.c);
    const int64_t N = w.size(0);
    if (N > INT32_MAX) raise(PyExc_ValueError, "a matrix of at most 2^31 - 1 rows is expected");
    const int8_t* pw = vec<int8_t>(a[1], at::kChar, {N, static_cast<int64_t>(quant_i8_row_bytes(K))}, "w", x);
    const float *ws = vec<float>(a[2], at::kFloat, {N}, "w_scale", x), *bias = vec<float>(a[3], at::kFloat, {N}, "bias", x, true);
    on_current_device(x);
    const at::Tensor y = product_out(a[5], a[4], M, N, x);
    const Rows ry = rows_of(y);
    const int yt = dtype_of(y);
    const Workspace work(a[6], a[6] == Py_None ? fc_i8_workspace_bytes(M, K) : 0, x);
    void* const s = current_stream();
    call([&] { return fc_i8_fwd(M, static_cast<int>(N), K, xt, rx.p, rx.ld, pw, ws, bias, yt, ry.p, ry.ld, work.p, work.bytes, s); });
    return wrap(y);
  });
}
// topk_rows(logits, k, temperature, tail, workspace)
PyObject* topk_rows_py(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&]() -> PyObject* {
    const at::Tensor& z = required(a[0]);
    const int dt = dtype_of(z), k = to_int(a[1]);
    const Rows r = rows_of(z);
    const int N = static_cast<int>(r.n), C = static_cast<int>(r.c);
    const float temperature = static_cast<float>(to_double(a[2]));
    const int want = PyObject_IsTrue(a[3]);
    if (want < 0) throw PyError();
    if (k < 0) raise(PyExc_ValueError, "k is negative");
    on_current_device(z);
    const at::Tensor values = empty({r.n, k}, at::kFloat, z), indices = empty({r.n, k}, at::kInt, z);
    at::Tensor tail;
    if (want) tail = empty({r.n}, at::kFloat, z);
    const Workspace ws(a[4], a[4] == Py_None ? topk_rows_workspace_bytes(N, C, k) : 0, z);
    float *const pv = addr<float>(values), *const pt = want ? addr<float>(tail) : nullptr;
    int32_t* const pi = addr<int32_t>(indices);
    void* const s = current_stream();
    call([&] { return topk_rows(N, C, k, dt, r.p, r.ld, temperature, pv, pi, pt, ws.p, ws.bytes, s); });
    PyObject* t = Py_None;
    if (want) t = wrap(tail); else Py_INCREF(Py_None);
    return Py_BuildValue("NNN", wrap(values), wrap(indices), t);
  });
}
// distill_fwd_bwd(logits, t_values, t_indices, t_tail, labels, temperature, alpha, label_smoothing, row_weight, grad_scale, grad, dlogits, workspace)
PyObject* distill_fwd_bwd_py(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 13, [&]() -> PyObject* {
    const at::Tensor& z = required(a[0]);
    rn50_distill_desc d{};
    d.dtype = dtype_of(z);
    const Rows r = rows_of(z);
    d.N = static_cast<int>(r.n);
    d.C = static_cast<int>(r.c);
    d.ld = r.ld;
    const at::Tensor* entries = tensor(a[1]);
    if (entries && (entries->dim() != 2 || entries->size(1) > INT32_MAX)) raise(PyExc_ValueError, "t_values: a matrix is expected");
    d.k = entries ? static_cast<int>(entries->size(1)) : 0;
    const float* tv = vec<float>(a[1], at::kFloat, {r.n, d.k}, "t_values", z, true);
    const int32_t* ti = vec<int32_t>(a[2], at::kInt, {r.n, d.k}, "t_indices", z, entries == nullptr);
    const float* tt = vec<float>(a[3], at::kFloat, {r.n}, "t_tail", z, true);
    const int32_t* labels = vec<int32_t>(a[4], at::kInt, {r.n}, "labels", z, true);
    d.temperature = static_cast<float>(to_double(a[5]));
    d.alpha = static_cast<float>(to_double(a[6]));
    d.label_smoothing = static_cast<float>(to_double(a[7]));
    const float* weight = vec<float>(a[8], at::kFloat, {r.n}, "row_weight", z, true);
    d.grad_scale = static_cast<float>(to_double(a[9]));
    const int grad = PyObject_IsTrue(a[10]);
    if (grad < 0) throw PyError();
    on_current_device(z);
    at::Tensor dz;
    Rows g{nullptr, 0, 0, d.C};
    if (grad) {
      const at::Tensor* given = tensor(a[11]);
      dz = given ? *given : empty({r.n, r.c}, z.scalar_type(), z);
      if (dz.scalar_type() != z.scalar_type()) raise(PyExc_TypeError, "dlogits: the logits' type is expected");
      if (dz.sizes() != z.sizes()) raise(PyExc_ValueError, "dlogits: the size does not fit");
      if (dz.device() != z.device()) raise(PyExc_ValueError, "dlogits: on another device");
      g = rows_of(dz);
    }
    d.grad_ld = g.ld;
    const at::Tensor loss = empty({1}, at::kFloat, z), row = empty({r.n}, at::kFloat, z);
    const Workspace ws(a[12], a[12] == Py_None ? distill_workspace_bytes(&d) : 0, z);
    float *const pl = addr<float>(loss), *const pr = addr<float>(row);
    void* const s = current_stream();
    call([&] { return distill_fwd_bwd(&d, r.p, tv, ti, tt, labels, weight, pl, pr, g.p, ws.p, ws.bytes, s); });
    PyObject* out = Py_None;
    if (grad) out = wrap(dz); else Py_INCREF(Py_None);
    return Py_BuildValue("NNN", wrap(loss), wrap(row), out);
  });
}
// setup(Rn50Error, current raw stream of a device, current device)
PyObject* setup_py(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 3, [&]() -> PyObject* {
    PyObject** const kept[] = {&g_error, &g_stream, &g_device};
    for (int i = 0; i < 3; ++i) {
      Py_INCREF(a[i]);
      Py_XSETREF(*kept[i], a[i]);
    }
    Py_RETURN_NONE;
  });
}

#define FAST(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {FAST("conv_fwd", conv_fwd_py), FAST("conv_dgrad", conv_dgrad_py), FAST("conv_wgrad", conv_wgrad_py),
                          FAST("bn_relu_fwd", bn_relu_fwd_py), FAST("bn_relu_bwd", bn_relu_bwd_py),
                          FAST("quant_rows_i8", quant_rows_i8_py), FAST("matmul_i8", matmul_i8_py), FAST("fc_i8_fwd", fc_i8_fwd_py),
                          FAST("topk_rows", topk_rows_py), FAST("distill_fwd_bwd", distill_fwd_bwd_py),
                          FAST("setup", setup_py), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_ops", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops() { return PyModule_Create(&kModule); }
