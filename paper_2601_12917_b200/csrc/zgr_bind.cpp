// Marshalling of the operators of the forward pass from torch tensors to the C ABI: checks, outputs, workspaces, the current stream.
//
// These calls last a few microseconds on the device; the same marshalling written in Python around ctypes took 4 to 7 us a call (1.4 of them for
// the conversion of the arguments) beside 2 us for the launch, this takes less than 1.  No arithmetic and no kernels here: the functions
// of libzgr.so are handed over as addresses by the module that loads it (zgr.py), which also documents the calls.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <stdexcept>
#include <string>

#include "zgr.h"

namespace {

decltype(&zgr_dropout) f_dropout;
decltype(&zgr_dropout_backward) f_dropout_backward;
decltype(&zgr_dropout_backward_workspace) f_dropout_backward_workspace;
decltype(&zgr_quantize_rows) f_quantize_rows;
decltype(&zgr_linear_i8) f_linear_i8;
decltype(&zgr_linear_i8_workspace) f_linear_i8_workspace;
decltype(&zgr_matmul_i8) f_matmul_i8;

// What becomes a ValueError.
struct Refused : std::runtime_error {
  using std::runtime_error::runtime_error;
};
// A negative code of the library, which becomes a ZgrError (raised by zgr.py).
struct Code {
  int code;
};

const at::Tensor& tensor_of(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) throw Refused(std::string(what) + " must be a tensor");
  return THPVariable_Unpack(o);
}

// The current device, and whether autograd would record a call: these record nothing, so a result would be a constant to the backward pass, and an
// output that requires gradients would keep the history of its old values.  Refused, unless the caller has switched recording off.
struct Here {
  int device;
  bool recording;
  Here() : device(c10::cuda::current_device()), recording(c10::GradMode::is_enabled()) {}
  void check(const at::Tensor& t, const char* what) const {
    dense(t, what);
    if (recording && t.requires_grad())
      throw Refused(std::string(what) + " requires gradients, which this call does not record: call it under torch.no_grad(), or pass it detached");
  }
  void dense(const at::Tensor& t, const char* what) const {
    if (!t.is_cuda() || t.get_device() != device) throw Refused(std::string(what) + " must be on the current CUDA device");
    if (t.layout() != at::kStrided) throw Refused(std::string(what) + " must be a dense tensor");
    if (t.is_neg()) throw Refused(std::string(what) + " must not be a view whose sign is still to be changed (resolve_neg)");
  }
  void* stream() const { return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream(); }
};

int storage_of(at::ScalarType t, const char* what) {
  switch (t) {
    case at::kFloat: return ZGR_F32;
    case at::kHalf: return ZGR_F16;
    case at::kBFloat16: return ZGR_BF16;
    default: throw Refused(std::string(what) + " must be float32, float16 or bfloat16");
  }
}

// Rows, columns and leading dimension of a tensor whose last dimension is contiguous, its other dimensions as rows.
struct Matrix {
  void* data;
  int64_t rows, cols, ld;
};
Matrix matrix_of(const at::Tensor& t, const char* what) {
  const int64_t d = t.dim();
  if (d == 0) throw Refused(std::string(what) + " has no dimension");
  Matrix m = {t.data_ptr(), 1, t.size(d - 1), t.size(d - 1)};
  if (m.cols > 1 && t.stride(d - 1) != 1) throw Refused(std::string(what) + ": the last dimension must be contiguous");
  bool some = false;
  int64_t below = 0;      // stride that the next dimension outwards has to have
  for (int64_t i = d - 2; i >= 0; --i) {
    const int64_t n = t.size(i);
    m.rows *= n;
    if (n == 1) continue;
    if (!some) m.ld = t.stride(i);
    else if (t.stride(i) != below && t.numel() > 0) throw Refused(std::string(what) + ": the dimensions in front of the last are not one run of rows");
    some = true;
    below = t.stride(i) * n;
  }
  return m;
}

// Address and leading dimension of a tensor that has to be of this type and shape.
Matrix same(const Here& here, PyObject* o, const char* what, at::ScalarType type, at::IntArrayRef shape) {
  const at::Tensor& t = tensor_of(o, what);
  here.check(t, what);
  if (t.scalar_type() != type || t.sizes() != shape) throw Refused(std::string(what) + " has another type or shape than the result");
  return matrix_of(t, what);
}
void* vector(const Here& here, PyObject* o, const char* what, int64_t n, at::ScalarType type) {
  const at::Tensor& t = tensor_of(o, what);
  here.check(t, what);
  if (t.scalar_type() != type || t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1))
    throw Refused(std::string(what) + " must be a contiguous vector of " + std::to_string(n) + " elements of its type");
  return t.data_ptr();
}
Matrix codes(const Here& here, PyObject* o, const char* what) {
  const at::Tensor& t = tensor_of(o, what);
  here.check(t, what);
  if (t.scalar_type() != at::kChar || t.dim() != 2) throw Refused(std::string(what) + " must be a matrix of int8 codes");
  return matrix_of(t, what);
}
// (torch's own function for this device, without the choice of it: 0.3 us)
at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, const Here& here) {
  return at::detail::empty_cuda(shape, type, at::Device(at::kCUDA, static_cast<c10::DeviceIndex>(here.device)), std::nullopt);
}
// Memory for the time of a call, from torch's allocator: given back in the order of the stream that the work runs on.
struct Workspace {
  void* data = nullptr;
  Workspace(int64_t bytes, void* stream) {
    if (bytes > 0) data = c10::cuda::CUDACachingAllocator::raw_alloc_with_stream(static_cast<size_t>(bytes), static_cast<cudaStream_t>(stream));
  }
  ~Workspace() {
    if (data) c10::cuda::CUDACachingAllocator::raw_delete(data);
  }
  Workspace(const Workspace&) = delete;
  Workspace& operator=(const Workspace&) = delete;
};

// The caller's output: written behind torch's back, so its version says it, and autograd refuses a saved tensor that is no longer itself.
PyObject* written(PyObject* o) {
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
  return Py_NewRef(o);
}

double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Code{1};
  return v;
}
uint64_t bits64(PyObject* o) {      // as ctypes takes it: any whole number, modulo 2^64
  const uint64_t v = PyLong_AsUnsignedLongLongMask(o);
  if (v == static_cast<uint64_t>(-1) && PyErr_Occurred()) throw Code{1};
  return v;
}
void check(int code) {
  if (code != ZGR_OK) throw Code{code};
}
bool given(PyObject* o) { return o != Py_None; }

// A call's body between Python and C++: exceptions become Python's; Code is returned as a whole number, which zgr.py raises as a ZgrError.
template <typename F>
PyObject* guarded(Py_ssize_t got, Py_ssize_t wanted, F&& body) {
  if (got != wanted) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return body();
  } catch (const Code& c) {
    return c.code > 0 ? nullptr : PyLong_FromLong(c.code);      // (above 0: Python's own error is set)
  } catch (const Refused& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (...) {
    torch::translate_exception_to_python(std::current_exception());      // torch's own, as its OutOfMemoryError
  }
  return nullptr;
}

// x, p, seed, tensor, bias, residual, out
PyObject* dropout(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject* {
    const Here here;
    const at::Tensor& x = tensor_of(a[0], "x");
    here.check(x, "x");
    const at::ScalarType type = x.scalar_type();
    const int storage = storage_of(type, "x");
    const Matrix m = matrix_of(x, "x");
    const void* bias = given(a[4]) ? vector(here, a[4], "bias", m.cols, type) : nullptr;
    const Matrix r = given(a[5]) ? same(here, a[5], "residual", type, x.sizes()) : Matrix{nullptr, 0, 0, 0};
    const at::Tensor made = given(a[6]) ? at::Tensor() : empty(x.sizes(), type, here);
    const Matrix y = given(a[6]) ? same(here, a[6], "out", type, x.sizes()) : matrix_of(made, "out");
    check(f_dropout(m.data, m.ld, bias, r.data, r.ld, y.data, y.ld, m.rows, m.cols, storage, number(a[1]), bits64(a[2]), static_cast<uint32_t>(bits64(a[3])),
                    here.stream()));
    return given(a[6]) ? written(a[6]) : THPVariable_Wrap(made);
  });
}

// dy, p, seed, tensor, bias_grad, out
PyObject* dropout_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    const Here here;
    const at::Tensor& dy = tensor_of(a[0], "dy");
    here.check(dy, "dy");
    const at::ScalarType type = dy.scalar_type();
    const int storage = storage_of(type, "dy");
    const Matrix m = matrix_of(dy, "dy");
    const at::Tensor made = given(a[5]) ? at::Tensor() : empty(dy.sizes(), type, here);
    const Matrix dx = given(a[5]) ? same(here, a[5], "out", type, dy.sizes()) : matrix_of(made, "out");
    const int want = PyObject_IsTrue(a[4]);
    if (want < 0) throw Code{1};
    const at::Tensor db = want ? empty({m.cols}, type, here) : at::Tensor();
    const int64_t bytes = want ? f_dropout_backward_workspace(m.rows, m.cols) : 0;
    const Workspace workspace(bytes, here.stream());
    check(f_dropout_backward(m.data, m.ld, dx.data, dx.ld, want ? db.data_ptr() : nullptr, m.rows, m.cols, storage, number(a[1]), bits64(a[2]),
                             static_cast<uint32_t>(bits64(a[3])), workspace.data, bytes, here.stream()));
    PyObject* out = given(a[5]) ? written(a[5]) : THPVariable_Wrap(made);
    if (!want || !out) return out;
    PyObject* grad = THPVariable_Wrap(db);
    PyObject* both = grad ? PyTuple_Pack(2, out, grad) : nullptr;
    Py_XDECREF(grad);
    Py_DECREF(out);
    return both;
  });
}

// x, pitch
PyObject* quantize_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 2, [&]() -> PyObject* {
    const Here here;
    const at::Tensor& x = tensor_of(a[0], "x");
    here.dense(x, "x");      // (weights that are parameters are quantised as they are: codes are whole numbers, which have no gradient)
    const int storage = storage_of(x.scalar_type(), "x");
    if (x.dim() != 2) throw Refused("x must be a matrix");
    const Matrix m = matrix_of(x, "x");
    const int64_t line = m.cols < 512 ? 16 : 128;
    int64_t pitch = (m.cols + line - 1) / line * line;
    if (given(a[1])) {
      pitch = PyLong_AsLongLong(a[1]);
      if (pitch == -1 && PyErr_Occurred()) throw Code{1};
      if (pitch < m.cols) throw Refused("pitch must not be below the number of columns");
    }
    at::Tensor q = empty({m.rows, pitch}, at::kChar, here);
    const at::Tensor scales = empty({m.rows}, at::kFloat, here);
    check(f_quantize_rows(m.data, m.ld, m.rows, m.cols, storage, static_cast<int8_t*>(q.data_ptr()), pitch, static_cast<float*>(scales.data_ptr()), here.stream()));
    if (pitch != m.cols) q = q.narrow(1, 0, m.cols);
    PyObject* first = THPVariable_Wrap(q);
    PyObject* second = THPVariable_Wrap(scales);
    PyObject* both = first && second ? PyTuple_Pack(2, first, second) : nullptr;
    Py_XDECREF(first);
    Py_XDECREF(second);
    return both;
  });
}

// What both products take beside the tokens: w, w_scale, bias, residual, p, seed, tensor, out (from a[0] on).
struct Product {
  Matrix w, residual = {nullptr, 0, 0, 0}, y;
  const float* w_scale;
  const void* bias = nullptr;
  at::Tensor made;
  double p;
  uint64_t seed;
  uint32_t tensor;
};
Product product_of(const Here& here, PyObject* const* a, at::ScalarType type, const at::Tensor& x, int64_t k) {
  Product p;
  p.w = codes(here, a[0], "w");
  if (p.w.cols != k) throw Refused("w must have rows of " + std::to_string(k) + " codes, not " + std::to_string(p.w.cols));
  at::DimVector shape(x.sizes().begin(), x.sizes().end());
  shape.back() = p.w.rows;
  if (!given(a[1])) throw Refused("w_scale is missing");
  p.w_scale = static_cast<const float*>(vector(here, a[1], "w_scale", p.w.rows, at::kFloat));
  if (given(a[2])) p.bias = vector(here, a[2], "bias", p.w.rows, type);
  if (given(a[3])) p.residual = same(here, a[3], "residual", type, shape);
  p.p = number(a[4]);
  p.seed = bits64(a[5]);
  p.tensor = static_cast<uint32_t>(bits64(a[6]));
  if (!given(a[7])) p.made = empty(shape, type, here);
  p.y = given(a[7]) ? same(here, a[7], "out", type, shape) : matrix_of(p.made, "out");
  return p;
}

// x, w, w_scale, bias, residual, p, seed, tensor, out
PyObject* linear_i8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> PyObject* {
    const Here here;
    const at::Tensor& x = tensor_of(a[0], "x");
    here.check(x, "x");
    const at::ScalarType type = x.scalar_type();
    const int storage = storage_of(type, "x");
    const Matrix m = matrix_of(x, "x");
    const Product p = product_of(here, a + 1, type, x, m.cols);
    const int64_t bytes = f_linear_i8_workspace(m.rows, p.w.rows, m.cols);      // (negative: a size that the call itself refuses)
    const Workspace workspace(bytes, here.stream());
    check(f_linear_i8(m.data, m.ld, static_cast<const int8_t*>(p.w.data), p.w.ld, p.w_scale, p.bias, p.residual.data, p.residual.ld, p.y.data, p.y.ld, m.rows, p.w.rows,
                      m.cols, storage, p.p, p.seed, p.tensor, workspace.data, bytes > 0 ? bytes : 0, here.stream()));
    return given(a[8]) ? written(a[8]) : THPVariable_Wrap(p.made);
  });
}

// x, x_scale, storage, w, w_scale, bias, residual, p, seed, tensor, out
PyObject* matmul_i8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&]() -> PyObject* {
    const Here here;
    const Matrix m = codes(here, a[0], "x");
    const long storage = PyLong_AsLong(a[2]);
    if (storage == -1 && PyErr_Occurred()) throw Code{1};
    const at::ScalarType type = storage == ZGR_F32 ? at::kFloat : (storage == ZGR_F16 ? at::kHalf : at::kBFloat16);
    if (!given(a[1])) throw Refused("x_scale is missing");
    const float* x_scale = static_cast<const float*>(vector(here, a[1], "x_scale", m.rows, at::kFloat));
    const Product p = product_of(here, a + 3, type, THPVariable_Unpack(a[0]), m.cols);
    check(f_matmul_i8(static_cast<const int8_t*>(m.data), m.ld, x_scale, static_cast<const int8_t*>(p.w.data), p.w.ld, p.w_scale, p.bias, p.residual.data, p.residual.ld,
                      p.y.data, p.y.ld, m.rows, p.w.rows, m.cols, static_cast<int32_t>(storage), p.p, p.seed, p.tensor, here.stream()));
    return given(a[10]) ? written(a[10]) : THPVariable_Wrap(p.made);
  });
}

// Addresses of the library's functions, in the order of the pointers above.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject* {
    void* f[7];
    for (int i = 0; i < 7; ++i) {
      f[i] = PyLong_AsVoidPtr(a[i]);
      if (!f[i]) throw Refused("an address is missing");
    }
    f_dropout = reinterpret_cast<decltype(f_dropout)>(f[0]);
    f_dropout_backward = reinterpret_cast<decltype(f_dropout_backward)>(f[1]);
    f_dropout_backward_workspace = reinterpret_cast<decltype(f_dropout_backward_workspace)>(f[2]);
    f_quantize_rows = reinterpret_cast<decltype(f_quantize_rows)>(f[3]);
    f_linear_i8 = reinterpret_cast<decltype(f_linear_i8)>(f[4]);
    f_linear_i8_workspace = reinterpret_cast<decltype(f_linear_i8_workspace)>(f[5]);
    f_matmul_i8 = reinterpret_cast<decltype(f_matmul_i8)>(f[6]);
    return Py_NewRef(Py_None);
  });
}

template <typename F>
PyCFunction fast(F f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}
PyMethodDef methods[] = {{"bind", fast(bind), METH_FASTCALL, nullptr},
                         {"dropout", fast(dropout), METH_FASTCALL, nullptr},
                         {"dropout_backward", fast(dropout_backward), METH_FASTCALL, nullptr},
                         {"quantize_rows", fast(quantize_rows), METH_FASTCALL, nullptr},
                         {"linear_i8", fast(linear_i8), METH_FASTCALL, nullptr},
                         {"matmul_i8", fast(matmul_i8), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_zgr_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__zgr_bind() { return PyModule_Create(&module); }
