// The dense operators' calls on tensors: argument checks, output allocation and
// the C entries (include/bmlp.h), without a Python-level step in between.  A
// call on small tensors is bound by the host: norm_quant takes 15 us of it as
// Python with ctypes and four torch.empty, and the launches themselves 3.
//
// Loaded by paper_2412_00119_amd/dense.py, which documents the functions.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/ops/empty_cuda_dispatch.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <optional>

#include "bmlp.h"

namespace {

// Python callables kept by bind(): device index -> raw stream handle; (status,
// name) -> raises the package's error.
PyObject *g_stream = nullptr, *g_fail = nullptr;

// a Python error is set already
struct PyError {};

void refuse(const char *format, const char *what) {
  PyErr_Format(PyExc_ValueError, format, what);
  throw PyError{};
}

// The calls record nothing for autograd: results would leave a tensor's
// gradient, or its forward-mode tangent, out without a word.
void no_gradient(const at::Tensor &x, const char *what) {
  if ((c10::GradMode::is_enabled() && x.requires_grad()) || x._fw_grad(0).defined())
    refuse("%s requires a gradient, which this call does not record: pass it detached (or call under torch.no_grad()) and "
           "chain the gradient that norm_quant_backward or distill returns", what);
}
const at::Tensor &tensor(PyObject *o, const char *what) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s must be a tensor", what);
    throw PyError{};
  }
  const at::Tensor &x = THPVariable_Unpack(o);
  no_gradient(x, what);
  return x;
}
const at::Tensor *tensor_or_none(PyObject *o, const char *what) { return o == Py_None ? nullptr : &tensor(o, what); }

int type_of(at::ScalarType t) {
  return t == at::kFloat ? BMLP_TYPE_F32 : t == at::kBFloat16 ? BMLP_TYPE_BF16 : t == at::kHalf ? BMLP_TYPE_F16 : -1;
}
int type_of(const at::Tensor &x, const char *what) {
  const int t = type_of(x.scalar_type());
  if (t < 0) refuse("%s must be float32, bfloat16 or float16", what);
  return t;
}

int32_t dim32(int64_t v, const char *what) {
  if (v > INT32_MAX) refuse("%s has more than 2^31 - 1 rows or columns", what);
  return (int32_t)v;
}

// A matrix on the GPU with contiguous rows; its row stride.
int64_t rows(const at::Tensor &x, const char *what) {
  if (x.dim() != 2 || !x.is_cuda() || (x.size(1) > 1 && x.stride(1) != 1))
    refuse("%s must be a matrix on the GPU with contiguous rows", what);
  if (x.size(0) > 1 && x.stride(0) < x.size(1)) refuse("%s's rows overlap", what);
  dim32(x.size(0), what);
  dim32(x.size(1), what);
  return x.stride(0);
}
int64_t rows_like(const at::Tensor &x, const at::Tensor &ref, const char *what) {
  const int64_t ld = rows(x, what);
  if (x.scalar_type() != ref.scalar_type() || x.sizes() != ref.sizes() || x.device() != ref.device())
    refuse("%s must have the first matrix's type, shape and device", what);
  return ld;
}
void *vector(const at::Tensor &x, const char *what, int64_t n, const at::Device &dev, at::ScalarType type) {
  if (x.scalar_type() != type || x.dim() != 1 || x.size(0) != n || x.device() != dev || !x.is_contiguous()) {
    PyErr_Format(PyExc_ValueError, "%s must be a contiguous %s vector of %lld on %s", what, c10::toString(type), (long long)n,
                 dev.str().c_str());
    throw PyError{};
  }
  return x.data_ptr();
}
float *floats(const at::Tensor *x, const char *what, int64_t n, const at::Device &dev) {
  return x == nullptr ? nullptr : static_cast<float *>(vector(*x, what, n, dev, at::kFloat));
}
// a norm's weight: of x's type or 32 bits
void *norm_weight(const at::Tensor *w, const at::Tensor &x, int64_t k, int *type) {
  *type = 0;
  if (w == nullptr) return nullptr;
  if (w->scalar_type() != x.scalar_type() && w->scalar_type() != at::kFloat)
    refuse("%s must be float32 or of x's type", "weight");
  *type = type_of(w->scalar_type());
  return vector(*w, "weight", k, x.device(), w->scalar_type());
}

// at::empty of the GPU backend, without the way there
at::Tensor make(at::IntArrayRef sizes, at::ScalarType type, const at::Device &dev) {
  return at::cuda::empty(sizes, type, at::kStrided, dev, std::nullopt, std::nullopt);
}

// Launches go to the current device: the tensors' one while this lives.
struct OnDevice {
  c10::OptionalDeviceGuard guard;
  void *stream;
  explicit OnDevice(const at::Device &dev) {
    static const c10::impl::VirtualGuardImpl impl(c10::DeviceType::CUDA);
    if (impl.getDevice() != dev) guard.reset_device(dev);
    PyObject *index = PyLong_FromLong(dev.index());
    if (index == nullptr) throw PyError{};
    PyObject *s = PyObject_CallFunctionObjArgs(g_stream, index, nullptr);
    Py_DECREF(index);
    if (s == nullptr) throw PyError{};
    stream = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (stream == nullptr && PyErr_Occurred()) throw PyError{};
  }
};

void check(int status, const char *name) {
  if (status == BMLP_OK) return;
  PyObject *r = PyObject_CallFunction(g_fail, "is", status, name);
  Py_XDECREF(r);
  if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, name);
  throw PyError{};
}

void arguments(Py_ssize_t got, Py_ssize_t want) {
  if (got != want) {
    PyErr_Format(PyExc_TypeError, "takes %zd arguments, got %zd", want, got);
    throw PyError{};
  }
}
double real(PyObject *o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PyError{};
  return v;
}
int32_t whole(PyObject *o, const char *what) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PyError{};
  if (v < 0) refuse("%s is negative", what);
  return dim32(v, what);
}
bool truth(PyObject *o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw PyError{};
  return v != 0;
}

// (tensor or None, ...) as a new tuple
template <typename... Ts>
PyObject *tuple_of(const Ts &...ts) {
  PyObject *t = PyTuple_New(sizeof...(Ts));
  if (t == nullptr) throw PyError{};
  Py_ssize_t i = 0;
  auto put = [&](const at::Tensor &x) {
    PyObject *o = x.defined() ? THPVariable_Wrap(x) : Py_None;
    if (o == Py_None) Py_INCREF(o);
    PyTuple_SET_ITEM(t, i++, o);
  };
  (put(ts), ...);
  return t;
}

// Every C++ exception ends at the entry.
template <typename F>
PyObject *guarded(F f) {
  HANDLE_TH_ERRORS
  try {
    return f();
  } catch (const PyError &) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// norm_quant(x, weight, residual, eps, values) -> (q, scale, rstd, h, y)
PyObject *norm_quant(PyObject *, PyObject *const *a, Py_ssize_t count) {
  return guarded([&]() -> PyObject * {
    arguments(count, 5);
    const at::Tensor &x = tensor(a[0], "x");
    const at::Tensor *w = tensor_or_none(a[1], "weight"), *res = tensor_or_none(a[2], "residual");
    const float eps = (float)real(a[3]);
    const int type = type_of(x, "x");
    const int64_t ldx = rows(x, "x"), n = x.size(0), k = x.size(1), ldr = res != nullptr ? rows_like(*res, x, "residual") : 0;
    const at::Device dev = x.device();
    int wtype;
    void *wp = norm_weight(w, x, k, &wtype);
    const OnDevice on(dev);
    at::Tensor q = make({n, k}, at::kChar, dev), scale = make({n}, at::kFloat, dev), rstd = make({n}, at::kFloat, dev), h, y;
    if (res != nullptr) h = make({n, k}, x.scalar_type(), dev);
    if (truth(a[4])) y = make({n, k}, x.scalar_type(), dev);
    check(bmlp_norm_quant(type, (int32_t)n, (int32_t)k, x.data_ptr(), ldx, res != nullptr ? res->data_ptr() : nullptr, ldr, wp,
                          wtype, eps, static_cast<int8_t *>(q.data_ptr()), k, static_cast<float *>(scale.data_ptr()),
                          static_cast<float *>(rstd.data_ptr()), h.defined() ? h.data_ptr() : nullptr, k,
                          y.defined() ? y.data_ptr() : nullptr, k, on.stream),
          "bmlp_norm_quant");
    return tuple_of(q, scale, rstd, h, y);
  });
}

// quantize_rows(x) -> (q, scale)
PyObject *quantize_rows(PyObject *, PyObject *const *a, Py_ssize_t count) {
  return guarded([&]() -> PyObject * {
    arguments(count, 1);
    const at::Tensor &x = tensor(a[0], "x");
    const int type = type_of(x, "x");
    const int64_t ldx = rows(x, "x"), n = x.size(0), k = x.size(1);
    const OnDevice on(x.device());
    at::Tensor q = make({n, k}, at::kChar, x.device()), scale = make({n}, at::kFloat, x.device());
    check(bmlp_quantize_rows(type, (int32_t)n, (int32_t)k, x.data_ptr(), ldx, static_cast<int8_t *>(q.data_ptr()), k,
                             static_cast<float *>(scale.data_ptr()), on.stream),
          "bmlp_quantize_rows");
    return tuple_of(q, scale);
  });
}

// norm_quant_backward(dy, h, rstd, weight, dh) -> (dx, dweight)
PyObject *norm_quant_backward(PyObject *, PyObject *const *a, Py_ssize_t count) {
  return guarded([&]() -> PyObject * {
    arguments(count, 5);
    const at::Tensor &dy = tensor(a[0], "dy"), &h = tensor(a[1], "h"), &rstd = tensor(a[2], "rstd");
    const at::Tensor *w = tensor_or_none(a[3], "weight"), *dh = tensor_or_none(a[4], "dh");
    const int type = type_of(dy, "dy");
    const int64_t lddy = rows(dy, "dy"), n = dy.size(0), k = dy.size(1), ldh = rows_like(h, dy, "h"),
                  lddh = dh != nullptr ? rows_like(*dh, dy, "dh") : 0;
    const at::Device dev = dy.device();
    int wtype;
    void *wp = norm_weight(w, dy, k, &wtype);
    float *rp = floats(&rstd, "rstd", n, dev);
    const OnDevice on(dev);
    at::Tensor dx = make({n, k}, dy.scalar_type(), dev), dw, ws;
    size_t ws_bytes = 0;
    if (w != nullptr) {
      dw = make({k}, at::kFloat, dev);
      ws_bytes = bmlp_norm_quant_backward_workspace_bytes((int32_t)n, (int32_t)k);
      ws = make({(int64_t)ws_bytes}, at::kByte, dev);
    }
    check(bmlp_norm_quant_backward(type, (int32_t)n, (int32_t)k, dy.data_ptr(), lddy, h.data_ptr(), ldh, rp, wp, wtype,
                                   dh != nullptr ? dh->data_ptr() : nullptr, lddh, dx.data_ptr(), k,
                                   dw.defined() ? static_cast<float *>(dw.data_ptr()) : nullptr,
                                   ws.defined() ? ws.data_ptr() : nullptr, ws_bytes, on.stream),
          "bmlp_norm_quant_backward");
    return tuple_of(dx, dw);
  });
}

// qlinear_pack(w, scale, bias) -> (packed,)
PyObject *qlinear_pack(PyObject *, PyObject *const *a, Py_ssize_t count) {
  return guarded([&]() -> PyObject * {
    arguments(count, 3);
    const at::Tensor &w = tensor(a[0], "w"), &scale = tensor(a[1], "scale");
    if (w.scalar_type() != at::kChar) refuse("%s must be int8", "w");
    const int64_t ldw = rows(w, "w"), n = w.size(0), k = w.size(1);
    floats(&scale, "scale", n, w.device());
    floats(tensor_or_none(a[2], "bias"), "bias", n, w.device());
    const size_t bytes = bmlp_qlinear_packed_bytes((int32_t)n, (int32_t)k);
    if (bytes == 0) refuse("%s is outside the supported sizes", "w");
    const OnDevice on(w.device());
    at::Tensor packed = make({(int64_t)bytes}, at::kByte, w.device());
    check(bmlp_qlinear_pack(static_cast<const int8_t *>(w.data_ptr()), ldw, (int32_t)n, (int32_t)k, packed.data_ptr(), on.stream),
          "bmlp_qlinear_pack");
    return tuple_of(packed);
  });
}

// qlinear(q, scale, dtype, packed, wscale, bias, n_in, n_out) -> out.  The
// layer's own tensors are attributes that a program can replace: they are checked
// against its sizes like any other argument.
PyObject *qlinear(PyObject *, PyObject *const *a, Py_ssize_t count) {
  return guarded([&]() -> PyObject * {
    arguments(count, 8);
    const at::Tensor &q = tensor(a[0], "q"), &packed = tensor(a[3], "packed"), &wscale = tensor(a[4], "wscale");
    const at::Tensor *scale = tensor_or_none(a[1], "scale"), *bias = tensor_or_none(a[5], "bias");
    if (!THPDtype_Check(a[2])) refuse("%s must be a torch dtype", "dtype");
    const at::ScalarType dtype = reinterpret_cast<THPDtype *>(a[2])->scalar_type;
    const int type = type_of(dtype);
    if (type < 0) refuse("%s must be float32, bfloat16 or float16", "dtype");
    const int32_t k = whole(a[6], "n_in"), m = whole(a[7], "n_out");
    const int64_t ldq = rows(q, "q"), n = q.size(0);
    const at::Device dev = packed.device();
    const size_t bytes = bmlp_qlinear_packed_bytes(m, k);
    if (bytes == 0 || !packed.is_cuda()) refuse("the layer's %s", "sizes are outside the supported ones, or it is not on the GPU");
    vector(packed, "the layer's packed weights", (int64_t)bytes, dev, at::kByte);
    float *wsp = floats(&wscale, "the layer's scale", m, dev), *bp = floats(bias, "the layer's bias", m, dev);
    if (q.scalar_type() != at::kChar || q.size(1) != k || q.device() != dev)
      refuse("%s must be int8 rows of the layer's width on its device", "q");
    float *sp = floats(scale, "scale", n, dev);
    const OnDevice on(dev);
    at::Tensor out = make({n, m}, dtype, dev);
    check(bmlp_qlinear(type, (int32_t)n, m, k, static_cast<const int8_t *>(q.data_ptr()), ldq, sp, packed.data_ptr(), wsp, bp,
                       out.data_ptr(), m, on.stream),
          "bmlp_qlinear");
    return THPVariable_Wrap(out);
  });
}

// distill(z, idx, t, tau, lse, weight, grad) -> (loss, dz)
PyObject *distill(PyObject *, PyObject *const *a, Py_ssize_t count) {
  return guarded([&]() -> PyObject * {
    arguments(count, 7);
    const at::Tensor &z = tensor(a[0], "z");
    const int type = type_of(z, "z");
    const at::Tensor &idx = tensor(a[1], "idx"), &t = tensor(a[2], "t");
    const float tau = (float)real(a[3]);
    const at::Tensor *lse = tensor_or_none(a[4], "lse"), *weight = tensor_or_none(a[5], "weight");
    const int t_type = type_of(t, "t");
    const int64_t ldz = rows(z, "z"), n = z.size(0), c = z.size(1);
    const at::Device dev = z.device();
    if (idx.dim() != 2 || idx.scalar_type() != at::kInt || idx.sizes() != t.sizes() || idx.size(0) != n ||
        !idx.is_contiguous() || !t.is_contiguous() || idx.device() != dev || t.device() != dev)
      refuse("%s must be contiguous int32 [n][k] and t contiguous [n][k] on z's device", "idx");
    const int32_t k = dim32(idx.size(1), "idx");
    float *lp = floats(lse, "lse", n, dev), *wp = floats(weight, "weight", n, dev);
    const OnDevice on(dev);
    at::Tensor loss = make({n}, at::kFloat, dev), dz;
    if (truth(a[6])) dz = make({n, c}, z.scalar_type(), dev);
    check(bmlp_distill(type, (int32_t)n, (int32_t)c, z.data_ptr(), ldz, k, static_cast<const int32_t *>(idx.data_ptr()),
                       t.data_ptr(), t_type, lp, wp, tau, static_cast<float *>(loss.data_ptr()),
                       dz.defined() ? dz.data_ptr() : nullptr, c, on.stream),
          "bmlp_distill");
    return tuple_of(loss, dz);
  });
}

// bind(stream, fail): the two callables above
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t count) {
  if (count != 2 || !PyCallable_Check(a[0]) || !PyCallable_Check(a[1])) {
    PyErr_SetString(PyExc_TypeError, "bind takes two callables");
    return nullptr;
  }
  Py_INCREF(a[0]);
  Py_INCREF(a[1]);
  Py_XSETREF(g_stream, a[0]);
  Py_XSETREF(g_fail, a[1]);
  Py_RETURN_NONE;
}

template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
constexpr PyMethodDef method(const char *name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {method<bind>("bind"),
                         method<norm_quant>("norm_quant"),
                         method<quantize_rows>("quantize_rows"),
                         method<norm_quant_backward>("norm_quant_backward"),
                         method<qlinear_pack>("qlinear_pack"),
                         method<qlinear>("qlinear"),
                         method<distill>("distill"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_dense_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__dense_binding() { return PyModule_Create(&module); }
