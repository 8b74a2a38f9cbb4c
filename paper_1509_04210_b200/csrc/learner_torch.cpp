// The learner-side operators on torch tensors: argument checks, outputs from torch's allocator, the call on
// torch's current stream.  Marshalling only; the work is in librudra_ps.so.  It is native because the
// smallest of these operators take 2 us on the GPU, and the same marshalling in Python took 4 us of the
// host's time a call on top of the launch.
#include <Python.h>

#include <cstdint>
#include <memory>
#include <vector>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/AutogradState.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/forward_grad.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/rudra_learner.h"

namespace {

// A Python exception is set; unwinds to the function that returns it.
struct Raised {};

template <typename... A> [[noreturn]] void refuse(const char* format, A... a) {
  PyErr_Format(PyExc_ValueError, format, a...);
  throw Raised();
}

PyObject* g_error = nullptr;   // binding.RudraError

void check(int code) {
  if (code >= 0) return;
  if (PyObject* e = PyObject_CallFunction(g_error, "is", code, rudra_last_error())) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  throw Raised();
}

// ------------------------------------------------------------------------------- codes and scales

enum Kind { kMx4, kAct8, kFp8 };

// A matrix in blocks of 32 or 128: codes and scale bytes in one buffer, or in two tensors that the caller gave.
struct Blocks {
  PyObject_HEAD
  at::Tensor* codes;    // or the buffer
  at::Tensor* scales;   // or null
  void *codes_at, *scales_at;      // as placed() left them
  int64_t rows, cols;
  int device;
};

PyTypeObject* g_types[3] = {nullptr, nullptr, nullptr};
const char* const kNames[3] = {"MX4", "Act8", "FP8"};

int64_t codes_bytes(Kind k, int64_t rows, int64_t cols) {
  return (int64_t)(k == kMx4 ? rudra_mx4_codes_bytes(rows, cols) : k == kAct8 ? rudra_act8_codes_bytes(rows, cols) : rudra_fp8_codes_bytes(rows, cols));
}
int64_t scales_bytes(Kind k, int64_t rows, int64_t cols) {
  return (int64_t)(k == kMx4 ? rudra_mx4_scales_bytes(rows, cols) : k == kAct8 ? rudra_act8_scales_bytes(rows, cols) : rudra_fp8_scales_bytes(rows, cols));
}
int64_t codes_room(Kind k, int64_t rows, int64_t cols) { return (codes_bytes(k, rows, cols) + 511) / 512 * 512; }

Kind kind_of(PyTypeObject* t) { return PyType_IsSubtype(t, g_types[kMx4]) ? kMx4 : PyType_IsSubtype(t, g_types[kAct8]) ? kAct8 : kFp8; }
Kind kind_of(PyObject* o) { return kind_of(Py_TYPE(o)); }

at::Tensor bytes(int64_t n, int device) {
  return at::detail::empty_cuda({n}, at::kByte, c10::Device(c10::kCUDA, (c10::DeviceIndex)device), std::nullopt);
}

void check_size(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0 || rows > RUDRA_MAX_DIM || cols > RUDRA_MAX_DIM) refuse("a matrix of %lld x %lld", (long long)rows, (long long)cols);
}

// Whether the caller's codes and scales do for a matrix of this size.
void check_given(Kind k, const at::Tensor& codes, const at::Tensor& scales, int64_t rows, int64_t cols) {
  const at::Tensor* both[2] = {&codes, &scales};
  const int64_t need[2] = {codes_bytes(k, rows, cols), scales_bytes(k, rows, cols)};
  for (int i = 0; i < 2; ++i)
    if (!both[i]->is_cuda() || both[i]->element_size() != 1 || !both[i]->is_contiguous() || both[i]->numel() < need[i])
      refuse("%s of a %lld x %lld %s: %lld contiguous bytes on the GPU are wanted", i ? "scales" : "codes", (long long)rows, (long long)cols, kNames[k], (long long)need[i]);
  if (codes.get_device() != scales.get_device()) refuse("codes and scales on different devices");
}

// Codes and scales where they lie now: a tensor may have been given other memory since the last call.  written: what they share
// with lazy copies becomes their own first.
Blocks* placed(Kind k, Blocks* b, bool written) {
  const auto at = [&](const at::Tensor& t) { return written ? t.mutable_data_ptr() : const_cast<void*>(t.const_data_ptr()); };
  if (b->scales) {
    check_given(k, *b->codes, *b->scales, b->rows, b->cols);
    if (b->codes->get_device() != b->device) refuse("%s: its codes are on another device now", kNames[k]);
    b->codes_at = at(*b->codes);
    b->scales_at = at(*b->scales);
  } else {
    b->codes_at = at(*b->codes);
    b->scales_at = static_cast<char*>(b->codes_at) + codes_room(k, b->rows, b->cols);
  }
  return b;
}

Blocks* new_blocks(Kind k, int64_t rows, int64_t cols, int device) {
  check_size(rows, cols);
  at::Tensor buffer = bytes(codes_room(k, rows, cols) + scales_bytes(k, rows, cols), device);
  Blocks* b = reinterpret_cast<Blocks*>(g_types[k]->tp_alloc(g_types[k], 0));
  if (!b) throw Raised();
  b->codes = new at::Tensor(std::move(buffer));
  b->scales = nullptr;
  b->rows = rows;
  b->cols = cols;
  b->device = device;
  return placed(k, b, true);
}

template <typename F> PyObject* returning(F&& body) {
  HANDLE_TH_ERRORS
  try {
    return body();
  } catch (const Raised&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

const at::Tensor& tensor(const char* what, PyObject* o) {
  if (!THPVariable_Check(o)) refuse("%s: a tensor is wanted", what);
  return THPVariable_Unpack(o);
}

PyObject* blocks_new(PyTypeObject* type, PyObject* args, PyObject* kwargs) {
  return returning([&]() -> PyObject* {
    static const char* names[] = {"codes", "scales", "rows", "cols", nullptr};
    PyObject *c, *s;
    long long rows, cols;
    if (!PyArg_ParseTupleAndKeywords(args, kwargs, "OOLL", const_cast<char**>(names), &c, &s, &rows, &cols)) return nullptr;
    const Kind k = kind_of(type);
    check_size(rows, cols);
    const at::Tensor &codes = tensor("codes", c), &scales = tensor("scales", s);
    check_given(k, codes, scales, rows, cols);
    Blocks* b = reinterpret_cast<Blocks*>(type->tp_alloc(type, 0));
    if (!b) return nullptr;
    b->codes = new at::Tensor(codes);
    b->scales = new at::Tensor(scales);
    b->rows = rows;
    b->cols = cols;
    b->device = (int)codes.get_device();
    return reinterpret_cast<PyObject*>(b);
  });
}

void blocks_free(PyObject* o) {
  Blocks* b = reinterpret_cast<Blocks*>(o);
  delete b->codes;
  delete b->scales;
  PyTypeObject* type = Py_TYPE(o);
  type->tp_free(o);
  Py_DECREF(type);
}

PyObject* blocks_codes(PyObject* o, void*) {
  return returning([&]() -> PyObject* {
    const Blocks* b = reinterpret_cast<Blocks*>(o);
    if (b->scales) return THPVariable_Wrap(*b->codes);
    const Kind k = kind_of(o);
    const int64_t pitch = k == kMx4 ? (b->cols + 31) / 32 * 16 : k == kAct8 ? (b->cols + 31) / 32 * 32 : (b->cols + 127) / 128 * 128;
    at::Tensor t = b->codes->narrow(0, 0, codes_bytes(k, b->rows, b->cols)).view({b->rows, pitch});
    return THPVariable_Wrap(k == kAct8 ? t.view(at::kChar) : t);
  });
}
PyObject* blocks_scales(PyObject* o, void*) {
  return returning([&]() -> PyObject* {
    const Blocks* b = reinterpret_cast<Blocks*>(o);
    if (b->scales) return THPVariable_Wrap(*b->scales);
    const Kind k = kind_of(o);
    at::Tensor t = b->codes->narrow(0, codes_room(k, b->rows, b->cols), scales_bytes(k, b->rows, b->cols));
    return THPVariable_Wrap(k == kAct8 ? t.view({b->rows, (b->cols + 511) / 512 * 16}) : t);
  });
}
PyObject* blocks_rows(PyObject* o, void*) { return PyLong_FromLongLong(reinterpret_cast<Blocks*>(o)->rows); }
PyObject* blocks_cols(PyObject* o, void*) { return PyLong_FromLongLong(reinterpret_cast<Blocks*>(o)->cols); }
PyObject* blocks_device(PyObject* o, void*) { return PyLong_FromLong(reinterpret_cast<Blocks*>(o)->device); }
// For callers that write there (a pull).
PyObject* blocks_codes_at(PyObject* o, void*) {
  return returning([&]() -> PyObject* { return PyLong_FromVoidPtr(placed(kind_of(o), reinterpret_cast<Blocks*>(o), true)->codes_at); });
}
PyObject* blocks_scales_at(PyObject* o, void*) {
  return returning([&]() -> PyObject* { return PyLong_FromVoidPtr(placed(kind_of(o), reinterpret_cast<Blocks*>(o), true)->scales_at); });
}

PyGetSetDef blocks_getset[] = {{"codes", blocks_codes, nullptr, "the codes, a tensor", nullptr},
                               {"scales", blocks_scales, nullptr, "the scale bytes, a tensor", nullptr},
                               {"rows", blocks_rows, nullptr, nullptr, nullptr},
                               {"cols", blocks_cols, nullptr, nullptr, nullptr},
                               {"device", blocks_device, nullptr, "index of the GPU", nullptr},
                               {"codes_ptr", blocks_codes_at, nullptr, nullptr, nullptr},
                               {"scales_ptr", blocks_scales_at, nullptr, nullptr, nullptr},
                               {nullptr, nullptr, nullptr, nullptr, nullptr}};

// --------------------------------------------------------------------------------------- matrices

struct Matrix {
  void* p;
  int dtype;
  int64_t rows, cols, ld;
  int device;
};

int dtype_of(c10::ScalarType t) { return t == at::kFloat ? RUDRA_F32 : t == at::kBFloat16 ? RUDRA_BF16 : -1; }

// These operators record nothing for torch's differentiation: results would come out detached without a word.
void check_no_gradient(const char* what, const at::Tensor& t) {
  if (t.requires_grad() && c10::GradMode::is_enabled())
    refuse("%s requires a gradient, which these operators do not record: detach it, or call them under torch.no_grad()", what);
  if (c10::AutogradState::get_tls_state().get_fw_grad_mode() && t._fw_grad(0).defined())
    refuse("%s has a tangent, which these operators do not carry on", what);
}

Matrix matrix(const char* what, const at::Tensor& t) {
  check_no_gradient(what, t);
  const int dtype = dtype_of(t.scalar_type());
  if (dtype < 0 || !t.is_cuda() || t.dim() != 2) refuse("%s: a two-dimensional float32 or bfloat16 tensor on the GPU is wanted", what);
  Matrix m = {t.data_ptr(), dtype, t.size(0), t.size(1), t.stride(0), (int)t.get_device()};
  if (m.cols > 1 && t.stride(1) != 1) refuse("%s: rows have to be contiguous", what);
  if (m.rows <= 1) m.ld = std::max(m.ld, m.cols);
  return m;
}
Matrix matrix(const char* what, PyObject* o) { return matrix(what, tensor(what, o)); }

// A one-dimensional tensor of consecutive values.
Matrix vector(const char* what, const at::Tensor& t) {
  check_no_gradient(what, t);
  const int dtype = dtype_of(t.scalar_type());
  if (dtype < 0 || !t.is_cuda() || t.dim() != 1) refuse("%s: a one-dimensional float32 or bfloat16 tensor on the GPU is wanted", what);
  if (t.size(0) > 1 && t.stride(0) != 1) refuse("%s: its values have to be contiguous", what);
  return {t.data_ptr(), dtype, 1, t.size(0), t.size(0), (int)t.get_device()};
}
Matrix vector(const char* what, PyObject* o) { return vector(what, tensor(what, o)); }

c10::ScalarType scalar_type(PyObject* o) {
  if (!THPDtype_Check(o) || dtype_of(reinterpret_cast<THPDtype*>(o)->scalar_type) < 0) refuse("dtype: float32 or bfloat16 is wanted");
  return reinterpret_cast<THPDtype*>(o)->scalar_type;
}

// The output the caller gave (a new reference to it), or a new one of `type`.
struct Output {
  PyObject* object;
  Matrix m;
};
Output output(const char* what, PyObject* given, int64_t rows, int64_t cols, c10::ScalarType type, bool any_type, int device) {
  if (given == Py_None) {
    const at::Tensor t = at::detail::empty_cuda({rows, cols}, type, c10::Device(c10::kCUDA, (c10::DeviceIndex)device), std::nullopt);
    const Matrix m = {t.data_ptr(), dtype_of(type), rows, cols, cols, device};
    return {THPVariable_Wrap(t), m};
  }
  const Matrix m = matrix(what, given);
  if (m.rows != rows || m.cols != cols || m.device != device || (!any_type && m.dtype != dtype_of(type)))
    refuse("%s: a %lld x %lld matrix of the operator's dtype on the input's device is wanted", what, (long long)rows, (long long)cols);
  Py_INCREF(given);
  return {given, m};
}

// The caller's codes and scales (a new reference), or new ones.
Blocks* blocks(const char* what, Kind k, PyObject* given, int64_t rows, int64_t cols, int device) {
  if (given == Py_None) return new_blocks(k, rows, cols, device);
  Blocks* b = reinterpret_cast<Blocks*>(given);
  if (!PyObject_TypeCheck(given, g_types[k]) || b->rows != rows || b->cols != cols || b->device != device)
    refuse("%s: %s of %lld x %lld on the input's device is wanted", what, kNames[k], (long long)rows, (long long)cols);
  placed(k, b, true);
  Py_INCREF(given);
  return b;
}
Blocks* wanted(const char* what, Kind k, PyObject* given) {
  if (!PyObject_TypeCheck(given, g_types[k])) refuse("%s: %s is wanted", what, kNames[k]);
  return placed(k, reinterpret_cast<Blocks*>(given), false);
}

void same_device(int a, int b) {
  if (a != b) refuse("tensors on different devices (%d and %d)", a, b);
}

// Objects that go away unless they are returned.
class Held {
 public:
  explicit Held(PyObject* o) : o_(o) { if (!o) throw Raised(); }
  explicit Held(Blocks* b) : o_(reinterpret_cast<PyObject*>(b)) {}
  Held(const Held&) = delete;
  ~Held() { Py_XDECREF(o_); }
  PyObject* get() const { return o_; }
  PyObject* give() {
    PyObject* o = o_;
    o_ = nullptr;
    return o;
  }

 private:
  PyObject* o_;
};

// The device of the operands current, and torch's current stream on it.
class On {
 public:
  explicit On(int device) : guard_((c10::DeviceIndex)device), stream_(c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream()) {}
  void* stream() const { return stream_; }

 private:
  c10::cuda::CUDAGuard guard_;
  cudaStream_t stream_;
};

void count(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments instead of %zd", n, want);
    throw Raised();
  }
}
bool truth(PyObject* o) {
  const int t = PyObject_IsTrue(o);
  if (t < 0) throw Raised();
  return t != 0;
}
long long number(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return v;
}

// -------------------------------------------------------------------------------------- operators

PyObject* empty(PyObject*, PyObject* const* a, Py_ssize_t n) {   // kind, rows, cols, device
  return returning([&]() -> PyObject* {
    count(n, 4);
    const long long k = number(a[0]);
    return reinterpret_cast<PyObject*>(new_blocks(k == 2 ? kFp8 : k ? kAct8 : kMx4, number(a[1]), number(a[2]), (int)number(a[3])));
  });
}

PyObject* current_stream(PyObject*, PyObject* const* a, Py_ssize_t n) {   // device
  return returning([&]() -> PyObject* {
    count(n, 1);
    return PyLong_FromVoidPtr(c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)number(a[0])).stream());
  });
}

PyObject* mx4_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {   // x, transpose, out
  return returning([&]() -> PyObject* {
    count(n, 3);
    const Matrix x = matrix("x", a[0]);
    const bool t = truth(a[1]);
    Blocks* q = blocks("out", kMx4, a[2], t ? x.cols : x.rows, t ? x.rows : x.cols, x.device);
    Held held(q);
    const On on(x.device);
    check(rudra_mx4_quantize(x.p, x.dtype, x.rows, x.cols, x.ld, t, q->codes_at, q->scales_at, on.stream()));
    return held.give();
  });
}

PyObject* mx4_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {   // q, dtype, out
  return returning([&]() -> PyObject* {
    count(n, 3);
    const Blocks* q = wanted("q", kMx4, a[0]);
    const Output y = output("out", a[2], q->rows, q->cols, scalar_type(a[1]), true, q->device);
    Held held(y.object);
    const On on(q->device);
    check(rudra_mx4_dequantize(q->codes_at, q->scales_at, q->rows, q->cols, y.m.p, y.m.dtype, y.m.ld, on.stream()));
    return held.give();
  });
}

PyObject* mx4_matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {   // a, b, dtype, out
  return returning([&]() -> PyObject* {
    count(n, 4);
    const Blocks* b = wanted("b", kMx4, a[1]);
    const bool coded = PyObject_TypeCheck(a[0], g_types[kMx4]);
    const Blocks* left = coded ? wanted("a", kMx4, a[0]) : nullptr;
    const Matrix x = coded ? Matrix{nullptr, 0, left->rows, left->cols, 0, left->device} : matrix("a", a[0]);
    if (x.cols != b->cols) refuse("a has rows of %lld values, b of %lld", (long long)x.cols, (long long)b->cols);
    same_device(x.device, b->device);
    const Output y = output("out", a[3], x.rows, b->rows, scalar_type(a[2]), true, b->device);
    Held held(y.object);
    const On on(b->device);
    if (coded) {
      check(rudra_mx4_matmul(left->codes_at, left->scales_at, x.rows, b->codes_at, b->scales_at, b->rows, x.cols, y.m.p, y.m.dtype, y.m.ld, on.stream()));
    } else {
      const uint64_t need = rudra_mx4_linear_workspace(x.rows, x.cols);
      at::Tensor work;
      if (need) work = bytes((int64_t)need, b->device);
      check(rudra_mx4_linear(x.p, x.dtype, x.ld, x.rows, b->codes_at, b->scales_at, b->rows, x.cols, y.m.p, y.m.dtype, y.m.ld,
                             need ? work.data_ptr() : nullptr, need, on.stream()));
    }
    return held.give();
  });
}

PyObject* act8_values(PyObject*, PyObject* const* a, Py_ssize_t n) {   // saved, dtype, out
  return returning([&]() -> PyObject* {
    count(n, 3);
    const Blocks* s = wanted("saved", kAct8, a[0]);
    const Output y = output("out", a[2], s->rows, s->cols, scalar_type(a[1]), true, s->device);
    Held held(y.object);
    const On on(s->device);
    check(rudra_act8_backward(RUDRA_ACT_NONE, nullptr, y.m.dtype, s->rows, s->cols, 0, s->codes_at, s->scales_at, nullptr, nullptr, y.m.p, nullptr,
                              y.m.ld, on.stream()));
    return held.give();
  });
}

// kind, x, up, out, saved, saved_up -> saved (RUDRA_ACT_NONE), (y, saved) or (y, saved, saved_up)
PyObject* act8_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return returning([&]() -> PyObject* {
    count(n, 6);
    const int act = (int)number(a[0]);
    const Matrix x = matrix("x", a[1]);
    const bool two = act == RUDRA_ACT_SWIGLU;
    if (two != (a[2] != Py_None) || (!two && a[5] != Py_None)) refuse("\"swiglu\", and no other, has a second input");
    Matrix up = {};
    if (two) {
      up = matrix("up", a[2]);
      if (up.dtype != x.dtype || up.rows != x.rows || up.cols != x.cols || up.ld != x.ld || up.device != x.device)
        refuse("up: the dtype, shape, row distance and device of x are wanted");
    }
    Blocks* s = blocks("saved", kAct8, a[4], x.rows, x.cols, x.device);
    Held held(s);
    const On on(x.device);
    if (act == RUDRA_ACT_NONE) {
      check(rudra_act8_forward(act, x.p, nullptr, x.dtype, x.rows, x.cols, x.ld, nullptr, 0, s->codes_at, s->scales_at, nullptr, nullptr, on.stream()));
      return held.give();
    }
    const Output y = output("out", a[3], x.rows, x.cols, x.dtype == RUDRA_F32 ? at::kFloat : at::kBFloat16, false, x.device);
    Held held_y(y.object);
    if (!two) {
      check(rudra_act8_forward(act, x.p, nullptr, x.dtype, x.rows, x.cols, x.ld, y.m.p, y.m.ld, s->codes_at, s->scales_at, nullptr, nullptr, on.stream()));
      return Py_BuildValue("NN", held_y.give(), held.give());
    }
    Blocks* su = blocks("saved_up", kAct8, a[5], x.rows, x.cols, x.device);
    Held held_up(su);
    check(rudra_act8_forward(act, x.p, up.p, x.dtype, x.rows, x.cols, x.ld, y.m.p, y.m.ld, s->codes_at, s->scales_at, su->codes_at, su->scales_at,
                             on.stream()));
    return Py_BuildValue("NNN", held_y.give(), held.give(), held_up.give());
  });
}

// kind, dy, saved, saved_up, out, out_up -> dx or (dx, dup)
PyObject* act8_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return returning([&]() -> PyObject* {
    count(n, 6);
    const int act = (int)number(a[0]);
    const Matrix dy = matrix("dy", a[1]);
    const bool two = act == RUDRA_ACT_SWIGLU;
    if (two != (a[3] != Py_None) || (!two && a[5] != Py_None)) refuse("\"swiglu\", and no other, has a second checkpoint");
    const Blocks* s[2] = {wanted("saved", kAct8, a[2]), two ? wanted("saved_up", kAct8, a[3]) : nullptr};
    for (int i = 0; i < (two ? 2 : 1); ++i) {
      if (s[i]->rows != dy.rows || s[i]->cols != dy.cols) refuse("%s: a checkpoint of %lld x %lld is wanted", i ? "saved_up" : "saved", (long long)dy.rows, (long long)dy.cols);
      same_device(dy.device, s[i]->device);
    }
    const c10::ScalarType type = dy.dtype == RUDRA_F32 ? at::kFloat : at::kBFloat16;
    const Output dx = output("out", a[4], dy.rows, dy.cols, type, false, dy.device);
    Held held(dx.object);
    const On on(dy.device);
    if (!two) {
      check(rudra_act8_backward(act, dy.p, dy.dtype, dy.rows, dy.cols, dy.ld, s[0]->codes_at, s[0]->scales_at, nullptr, nullptr, dx.m.p, nullptr, dx.m.ld,
                                on.stream()));
      return held.give();
    }
    const Output du = output("out_up", a[5], dy.rows, dy.cols, type, false, dy.device);
    Held held_up(du.object);
    if (du.m.ld != dx.m.ld) refuse("out_up: the row distance of out is wanted");
    check(rudra_act8_backward(act, dy.p, dy.dtype, dy.rows, dy.cols, dy.ld, s[0]->codes_at, s[0]->scales_at, s[1]->codes_at, s[1]->scales_at, dx.m.p,
                              du.m.p, dx.m.ld, on.stream()));
    return Py_BuildValue("NN", held.give(), held_up.give());
  });
}

PyObject* act8_weight_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {   // dy, saved, dtype, out
  return returning([&]() -> PyObject* {
    count(n, 4);
    const Matrix dy = matrix("dy", a[0]);
    const Blocks* s = wanted("saved", kAct8, a[1]);
    if (s->rows != dy.rows) refuse("dy has %lld tokens, the checkpoint %lld", (long long)dy.rows, (long long)s->rows);
    same_device(dy.device, s->device);
    const Output dw = output("out", a[3], dy.cols, s->cols, scalar_type(a[2]), true, dy.device);
    Held held(dw.object);
    const On on(dy.device);
    const uint64_t need = rudra_act8_weight_grad_workspace(dy.p, dy.dtype, dy.rows, dy.cols, dy.ld);
    at::Tensor work;
    if (need) work = bytes((int64_t)need, dy.device);
    check(rudra_act8_weight_grad(dy.p, dy.dtype, dy.ld, dy.rows, dy.cols, s->codes_at, s->scales_at, s->cols, dw.m.p, dw.m.dtype, dw.m.ld,
                                 need ? work.data_ptr() : nullptr, need, on.stream()));
    return held.give();
  });
}

PyObject* fp8_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {   // x, transpose, square, out
  return returning([&]() -> PyObject* {
    count(n, 4);
    const Matrix x = matrix("x", a[0]);
    const bool t = truth(a[1]), square = truth(a[2]);
    Blocks* q = blocks("out", kFp8, a[3], t ? x.cols : x.rows, t ? x.rows : x.cols, x.device);
    Held held(q);
    const On on(x.device);
    check(rudra_fp8_quantize(x.p, x.dtype, x.rows, x.cols, x.ld, t, square, q->codes_at, q->scales_at, on.stream()));
    return held.give();
  });
}

PyObject* fp8_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {   // q, dtype, out
  return returning([&]() -> PyObject* {
    count(n, 3);
    const Blocks* q = wanted("q", kFp8, a[0]);
    const Output y = output("out", a[2], q->rows, q->cols, scalar_type(a[1]), true, q->device);
    Held held(y.object);
    const On on(q->device);
    check(rudra_fp8_dequantize(q->codes_at, q->scales_at, q->rows, q->cols, y.m.p, y.m.dtype, y.m.ld, on.stream()));
    return held.give();
  });
}

PyObject* fp8_matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {   // a, b, dtype, out
  return returning([&]() -> PyObject* {
    count(n, 4);
    const Blocks* b = wanted("b", kFp8, a[1]);
    const bool coded = PyObject_TypeCheck(a[0], g_types[kFp8]);
    const Blocks* left = coded ? wanted("a", kFp8, a[0]) : nullptr;
    const Matrix x = coded ? Matrix{nullptr, 0, left->rows, left->cols, 0, left->device} : matrix("a", a[0]);
    if (x.cols != b->cols) refuse("a has rows of %lld values, b of %lld", (long long)x.cols, (long long)b->cols);
    same_device(x.device, b->device);
    const Output y = output("out", a[3], x.rows, b->rows, scalar_type(a[2]), true, b->device);
    Held held(y.object);
    const On on(b->device);
    if (coded) {
      check(rudra_fp8_matmul(left->codes_at, left->scales_at, x.rows, b->codes_at, b->scales_at, b->rows, x.cols, y.m.p, y.m.dtype, y.m.ld, on.stream()));
    } else {
      const uint64_t need = rudra_fp8_linear_workspace(x.rows, x.cols);
      at::Tensor work;
      if (need) work = bytes((int64_t)need, b->device);
      check(rudra_fp8_linear(x.p, x.dtype, x.ld, x.rows, b->codes_at, b->scales_at, b->rows, x.cols, y.m.p, y.m.dtype, y.m.ld,
                             need ? work.data_ptr() : nullptr, need, on.stream()));
    }
    return held.give();
  });
}

// A matrix of the shape, dtype and device of x.
Matrix alike(const char* what, PyObject* o, const Matrix& x) {
  const Matrix m = matrix(what, o);
  if (m.rows != x.rows || m.cols != x.cols || m.dtype != x.dtype || m.device != x.device)
    refuse("%s: a %lld x %lld matrix of the operator's dtype on the input's device is wanted", what, (long long)x.rows, (long long)x.cols);
  return m;
}
Matrix norm_weight(PyObject* o, const Matrix& x) {
  const Matrix w = vector("weight", o);
  if (w.cols != x.cols || w.device != x.device) refuse("weight: %lld values on the input's device are wanted", (long long)x.cols);
  return w;
}
float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised();
  return (float)v;
}
c10::ScalarType type_of(const Matrix& m) { return m.dtype == RUDRA_F32 ? at::kFloat : at::kBFloat16; }

// x, weight, residual, eps, fp8, keep, out, out_sum, saved -> y, then s if there is a residual, then saved if it is kept
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return returning([&]() -> PyObject* {
    count(n, 9);
    const Matrix x = matrix("x", a[0]), w = norm_weight(a[1], x);
    const bool two = a[2] != Py_None, fp8 = truth(a[4]), keep = truth(a[5]) || a[8] != Py_None;
    const Matrix r = two ? alike("residual", a[2], x) : Matrix{};
    const float eps = real(a[3]);
    if (!two && a[7] != Py_None) refuse("out_sum: there is no residual to add");
    const Output y = fp8 ? Output{reinterpret_cast<PyObject*>(blocks("out", kFp8, a[6], x.rows, x.cols, x.device)), {}}
                         : output("out", a[6], x.rows, x.cols, type_of(x), false, x.device);
    Held held(y.object);
    const Blocks* q = fp8 ? reinterpret_cast<const Blocks*>(y.object) : nullptr;
    const Output s = two ? output("out_sum", a[7], x.rows, x.cols, type_of(x), false, x.device) : Output{Py_NewRef(Py_None), {}};
    Held held_sum(s.object);
    Blocks* kept = keep ? blocks("saved", kAct8, a[8], x.rows, x.cols, x.device) : nullptr;
    Held held_kept(kept);
    const On on(x.device);
    check(rudra_rms_norm(x.p, x.ld, two ? r.p : nullptr, r.ld, x.dtype, x.rows, x.cols, w.p, w.dtype, eps, s.m.p, s.m.ld, y.m.p, y.m.ld,
                         q ? q->codes_at : nullptr, q ? q->scales_at : nullptr, kept ? kept->codes_at : nullptr, kept ? kept->scales_at : nullptr, on.stream()));
    if (two && keep) return Py_BuildValue("NNN", held.give(), held_sum.give(), held_kept.give());
    if (two) return Py_BuildValue("NN", held.give(), held_sum.give());
    if (keep) return Py_BuildValue("NN", held.give(), held_kept.give());
    return held.give();
  });
}

// dy, s, weight, eps, dsum, dtype, out, out_weight -> (ds, dweight)
PyObject* rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return returning([&]() -> PyObject* {
    count(n, 8);
    const Matrix s = matrix("s", a[1]), dy = alike("dy", a[0], s), w = norm_weight(a[2], s);
    const float eps = real(a[3]);
    const Matrix more = a[4] != Py_None ? alike("dsum", a[4], s) : Matrix{};
    const c10::ScalarType type = scalar_type(a[5]);
    const Output ds = output("out", a[6], s.rows, s.cols, type_of(s), false, s.device);
    Held held(ds.object);
    Matrix dw;
    PyObject* dw_object;
    if (a[7] == Py_None) {
      const at::Tensor t = at::detail::empty_cuda({s.cols}, type, c10::Device(c10::kCUDA, (c10::DeviceIndex)s.device), std::nullopt);
      dw = {t.data_ptr(), dtype_of(type), 1, s.cols, s.cols, s.device};
      dw_object = THPVariable_Wrap(t);
    } else {
      dw = vector("out_weight", a[7]);
      if (dw.cols != s.cols || dw.device != s.device) refuse("out_weight: %lld values on the input's device are wanted", (long long)s.cols);
      dw_object = Py_NewRef(a[7]);
    }
    Held held_weight(dw_object);
    const On on(s.device);
    const uint64_t need = rudra_rms_norm_backward_workspace(s.rows, s.cols);
    at::Tensor work;
    if (need) work = bytes((int64_t)need, s.device);
    check(rudra_rms_norm_backward(dy.p, dy.ld, s.p, s.ld, more.p, more.ld, s.dtype, s.rows, s.cols, w.p, w.dtype, eps, ds.m.p, ds.m.ld, dw.p, dw.dtype,
                                  need ? work.data_ptr() : nullptr, need, on.stream()));
    return Py_BuildValue("NN", held.give(), held_weight.give());
  });
}

// A list of gradients, or of where they go: any shape, values one after another.  It holds the tensors until the launches are made:
// those of a generator have no other owner.
struct Gradients {
  std::unique_ptr<Held> list;
  std::vector<const void*> p;
  std::vector<int> dtypes;
  std::vector<uint64_t> sizes;
  int device = -1;
};
// written: what a tensor shares with lazy copies of it becomes its own first.
Gradients gradients(const char* what, PyObject* o, bool written) {
  Gradients g;
  g.list = std::make_unique<Held>(PySequence_Fast(o, "a list of tensors is wanted"));
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(g.list->get());
  PyObject** items = PySequence_Fast_ITEMS(g.list->get());
  if (n == 0) refuse("%s: an empty list", what);
  g.p.resize(n);
  g.dtypes.resize(n);
  g.sizes.resize(n);
  // asked once: only inside a level of forward differentiation has a tensor a tangent
  const bool recording = c10::GradMode::is_enabled();
  const bool tangents = c10::AutogradState::get_tls_state().get_fw_grad_mode() && torch::autograd::ForwardADLevel::try_get_by_idx(0) != nullptr;
  for (Py_ssize_t i = 0; i < n; ++i) {
    const at::Tensor& t = tensor(what, items[i]);
    const c10::TensorImpl& impl = *t.unsafeGetTensorImpl();
    if (tangents || (recording && t.requires_grad())) check_no_gradient(what, t);
    const int dtype = dtype_of(c10::typeMetaToScalarType(impl.dtype()));
    if (dtype < 0 || !t.is_cuda() || !impl.is_contiguous()) refuse("%s: contiguous float32 or bfloat16 tensors on the GPU are wanted", what);
    const int device = (int)impl.device().index();
    if (g.device >= 0) same_device(g.device, device);
    g.device = device;
    g.p[i] = written ? t.mutable_data_ptr() : t.const_data_ptr();
    g.dtypes[i] = dtype;
    g.sizes[i] = (uint64_t)impl.numel();
  }
  return g;
}

// A float on the device: the caller's (a new reference), or a new one of no dimensions.
Output scalar(const char* what, PyObject* given, int device) {
  if (given == Py_None) {
    const at::Tensor t = at::detail::empty_cuda({}, at::kFloat, c10::Device(c10::kCUDA, (c10::DeviceIndex)device), std::nullopt);
    return {THPVariable_Wrap(t), {t.data_ptr(), RUDRA_F32, 1, 1, 1, device}};
  }
  const at::Tensor& t = tensor(what, given);
  check_no_gradient(what, t);
  if (t.scalar_type() != at::kFloat || !t.is_cuda() || t.numel() != 1 || (int)t.get_device() != device) refuse("%s: one float32 value on the gradients' device is wanted", what);
  return {Py_NewRef(given), {t.data_ptr(), RUDRA_F32, 1, 1, 1, device}};
}

PyObject* grad_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {   // gradients, out
  return returning([&]() -> PyObject* {
    count(n, 2);
    const Gradients g = gradients("gradients", a[0], false);
    const Output norm = scalar("out", a[1], g.device);
    Held held(norm.object);
    const On on(g.device);
    const uint64_t need = rudra_grad_norm_workspace(g.p.size());
    const at::Tensor work = bytes((int64_t)need, g.device);
    check(rudra_grad_norm(g.p.data(), g.dtypes.data(), g.sizes.data(), g.p.size(), static_cast<float*>(norm.m.p), work.data_ptr(), need, on.stream()));
    return held.give();
  });
}

PyObject* clip_gradients(PyObject*, PyObject* const* a, Py_ssize_t n) {   // gradients, max_norm, out, norm -> norm
  return returning([&]() -> PyObject* {
    count(n, 4);
    const float most = real(a[1]);
    const bool in_place = a[2] == Py_None;
    const Gradients to = in_place ? Gradients() : gradients("out", a[2], true);      // first: what is read may be one of them
    const Gradients g = gradients("gradients", a[0], in_place);
    if (!in_place && (to.sizes != g.sizes || to.device != g.device)) refuse("out: as many tensors as gradients, each of its gradient's size and device, are wanted");
    const Output norm = scalar("norm", a[3], g.device);
    Held held(norm.object);
    const On on(g.device);
    const bool known = a[3] != Py_None;
    const uint64_t need = known ? 0 : rudra_grad_norm_workspace(g.p.size());
    at::Tensor work;
    if (need) work = bytes((int64_t)need, g.device);
    check(rudra_grad_clip(g.p.data(), g.dtypes.data(), g.sizes.data(), g.p.size(), static_cast<float*>(norm.m.p), known, most,
                          const_cast<void* const*>(in_place ? g.p.data() : to.p.data()), in_place ? g.dtypes.data() : to.dtypes.data(),
                          need ? work.data_ptr() : nullptr, need, on.stream()));
    return held.give();
  });
}

PyObject* synchronize(PyObject*, PyObject* const* a, Py_ssize_t n) {   // device
  return returning([&]() -> PyObject* {
    count(n, 1);
    const On on((int)number(a[0]));
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = rudra_learner_sync(on.stream());
    Py_END_ALLOW_THREADS
    check(code);
    Py_RETURN_NONE;
  });
}

PyMethodDef methods[] = {
#define RUDRA_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}
    RUDRA_METHOD(empty), RUDRA_METHOD(current_stream), RUDRA_METHOD(mx4_quantize), RUDRA_METHOD(mx4_dequantize), RUDRA_METHOD(mx4_matmul), RUDRA_METHOD(act8_values),
    RUDRA_METHOD(act8_forward), RUDRA_METHOD(act8_backward), RUDRA_METHOD(act8_weight_grad), RUDRA_METHOD(fp8_quantize), RUDRA_METHOD(fp8_dequantize),
    RUDRA_METHOD(fp8_matmul), RUDRA_METHOD(rms_norm), RUDRA_METHOD(rms_norm_backward), RUDRA_METHOD(grad_norm), RUDRA_METHOD(clip_gradients), RUDRA_METHOD(synchronize),
#undef RUDRA_METHOD
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_learner", "native marshalling of the learner-side operators", -1, methods, nullptr, nullptr, nullptr, nullptr};

PyTypeObject* new_type(const char* name, const char* doc) {
  PyType_Slot slots[] = {{Py_tp_new, reinterpret_cast<void*>(blocks_new)},
                         {Py_tp_dealloc, reinterpret_cast<void*>(blocks_free)},
                         {Py_tp_getset, blocks_getset},
                         {Py_tp_doc, const_cast<char*>(doc)},
                         {0, nullptr}};
  PyType_Spec spec = {name, sizeof(Blocks), 0, Py_TPFLAGS_DEFAULT, slots};
  return reinterpret_cast<PyTypeObject*>(PyType_FromSpec(&spec));
}

}  // namespace

PyMODINIT_FUNC PyInit__learner() {
  PyObject* binding = PyImport_ImportModule("paper_1509_04210_b200.binding");
  if (!binding) return nullptr;
  g_error = PyObject_GetAttrString(binding, "RudraError");
  Py_DECREF(binding);
  g_types[kMx4] = new_type("paper_1509_04210_b200._learner.MX4",
                           "MX4(codes, scales, rows, cols): a matrix in microscaled 4-bit floating point, uint8 tensors laid out as the header says.");
  g_types[kAct8] = new_type("paper_1509_04210_b200._learner.Act8",
                            "Act8(codes, scales, rows, cols): an 8-bit checkpoint of rows tokens x cols channels, laid out as the header says.");
  g_types[kFp8] = new_type("paper_1509_04210_b200._learner.FP8",
                           "FP8(codes, scales, rows, cols): a matrix in 8-bit floating point in blocks of 128, one-byte tensors laid out as the header says.");
  if (!g_error || !g_types[kMx4] || !g_types[kAct8] || !g_types[kFp8]) return nullptr;
  PyObject* m = PyModule_Create(&module);
  if (!m) return nullptr;
  if (PyModule_AddStringConstant(m, "build_key", RUDRA_LEARNER_KEY) < 0 ||
      PyModule_AddObjectRef(m, "MX4", reinterpret_cast<PyObject*>(g_types[kMx4])) < 0 ||
      PyModule_AddObjectRef(m, "Act8", reinterpret_cast<PyObject*>(g_types[kAct8])) < 0 ||
      PyModule_AddObjectRef(m, "FP8", reinterpret_cast<PyObject*>(g_types[kFp8])) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
