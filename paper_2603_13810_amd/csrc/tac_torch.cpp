// The dense operators' calls from Python: torch tensors are checked, outputs and scratch allocated and the C entry point called in one step.
//
// Small calls are bound by the host: a launch takes 3.5 us, and every tensor that Python itself looks at or allocates another 0.5 to 1.5.
// Functions take every argument by position and return what api.py documents, or a status (a whole number) where the library refused.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/hip/EmptyTensor.h>
#include <ATen/ops/empty_strided.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>

#include <pybind11/pybind11.h>

#include "tac.h"

namespace {

using at::ScalarType;
using at::Tensor;

struct Refused {};             // a Python error is set

[[noreturn]] void refuse(const char* format, ...) {
  va_list rest;
  va_start(rest, format);
  PyErr_FormatV(PyExc_ValueError, format, rest);
  va_end(rest);
  throw Refused();
}

// a tensor, or nullptr for None
const Tensor* maybe(PyObject* o, const char* name) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) refuse("%s must be a tensor", name);
  return &THPVariable_Unpack(o);
}
const Tensor& given(PyObject* o, const char* name) {
  const Tensor* t = maybe(o, name);
  if (!t) refuse("%s is missing", name);
  return *t;
}

int32_t float_type(const Tensor& t, const char* name) {
  if (t.scalar_type() == ScalarType::Float) return TAC_FP32;
  if (t.scalar_type() == ScalarType::BFloat16) return TAC_BF16;
  refuse("%s must be float32 or bfloat16", name);
}

// What every tensor of a call has to share with its first one.
struct Call {
  c10::Device device;
  c10::DeviceGuard guard;
  explicit Call(const Tensor& first, const char* name) : device(where(first, name)), guard(device) {}
  static c10::Device where(const Tensor& t, const char* name) {
    if (!t.is_cuda()) refuse("%s must be a device tensor", name);
    return t.device();
  }
  void* stream() const { return c10::hip::getCurrentHIPStream(device.index()).stream(); }

  void check(const Tensor& t, const char* name, ScalarType type, at::IntArrayRef shape) const {
    if (t.sizes() == shape && t.scalar_type() == type && t.device() == device) return;
    std::string want = "[";
    for (int64_t n : shape) want += (want.size() > 1 ? ", " : "") + std::to_string(n);
    refuse("%s must be a tensor %s] of %s on %s", name, want.c_str(), c10::toString(type), device.str().c_str());
  }
  // address of a contiguous tensor, or nullptr
  void* whole(const Tensor* t, const char* name, ScalarType type, at::IntArrayRef shape) const {
    if (!t) return nullptr;
    check(*t, name, type, shape);
    if (!t->is_contiguous()) refuse("%s must be contiguous", name);
    return t->data_ptr();
  }
  // address of a tensor whose last axis is contiguous, or nullptr
  void* lines(const Tensor* t, const char* name, ScalarType type, at::IntArrayRef shape) const {
    if (!t) return nullptr;
    check(*t, name, type, shape);
    if (t->strides().back() != 1 && shape.back() > 1) refuse("%s must have a contiguous last axis", name);
    return t->data_ptr();
  }
  Tensor make(at::IntArrayRef shape, ScalarType type) const {
    return Tensor(at::detail::empty_cuda(shape, type, device, std::nullopt));
  }
  // scratch: torch's again when the call has been enqueued on the current stream
  Tensor scratch(size_t bytes) const { return bytes ? make({(int64_t)bytes}, ScalarType::Byte) : Tensor(); }
};

int64_t row_stride(const Tensor* t, int64_t rows, int64_t cols) {
  return !t ? 0 : rows > 1 ? t->stride(0) : cols;             // a matrix of one row has no stride that matters
}
void* at_of(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to; }

struct Matrix8 {               // an 8-bit matrix
  Tensor codes, scales;
};
Matrix8 make_8bit(const Call& c, int64_t rows, int64_t cols) {
  return {c.make({rows, 128 * up(cols, 128)}, ScalarType::Byte), c.make({rows, 4 * up(cols, 512)}, ScalarType::Byte)};
}
struct At8 {
  const uint8_t *codes, *scales;
};
At8 at_8bit(const Call& c, const Tensor& codes, const Tensor& scales, int64_t rows, int64_t cols, const char* codes_name, const char* scales_name) {
  return {(const uint8_t*)c.whole(&codes, codes_name, ScalarType::Byte, {rows, 128 * up(cols, 128)}),
          (const uint8_t*)c.whole(&scales, scales_name, ScalarType::Byte, {rows, 4 * up(cols, 512)})};
}
void matrix_axes(const Tensor& t, const char* name) {
  if (t.dim() != 2) refuse("%s must be a matrix", name);
}

int64_t whole_number(PyObject* o) {
  const int64_t n = PyLong_AsLongLong(o);
  if (n == -1 && PyErr_Occurred()) throw Refused();
  return n;
}
// sizes are checked by the library; here only so that they can be allocated
int64_t columns_of(PyObject* o, const char* name) {
  const int64_t n = whole_number(o);
  if (n < 1 || n > INT32_MAX) refuse("%s must be a number of columns", name);
  return n;
}
ScalarType type_of(PyObject* o, ScalarType otherwise) {
  if (o == Py_None) return otherwise;
  if (!THPDtype_Check(o)) refuse("dtype must be a torch type");
  return reinterpret_cast<THPDtype*>(o)->scalar_type;
}
bool yes(PyObject* o) { return PyObject_IsTrue(o) == 1; }

// new references
PyObject* out_of(const Tensor& t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(t);
}
PyObject* out_of(const Matrix8& m) {
  if (!m.codes.defined()) Py_RETURN_NONE;
  return Py_BuildValue("(NN)", THPVariable_Wrap(m.codes), THPVariable_Wrap(m.scales));
}
PyObject* same(PyObject* o) {
  Py_INCREF(o);
  return o;
}
// the caller's tensor has been written: what autograd has kept of it is out of date (inference tensors keep no count)
void written(const Tensor* t) {
  if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}
// a dict that takes the values' references
PyObject* dict_of(std::initializer_list<std::pair<const char*, PyObject*>> items) {
  PyObject* d = PyDict_New();
  for (const auto& [key, value] : items) {
    if (!d || !value || PyDict_SetItemString(d, key, value)) Py_CLEAR(d);
    Py_XDECREF(value);
  }
  return d;
}

// a call of the library, other Python threads running on: a launch may wait for room in the queue
template <class F>
int unlocked(F f) {
  pybind11::gil_scoped_release free;
  return f();
}

#define TAC_ARGUMENTS(N) \
  if (count != N) { \
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); \
    return nullptr; \
  } \
  try {
#define TAC_END \
  } catch (const Refused&) { \
    return nullptr; \
  }

// src or codes, scales, cols, tiles, rows, columns
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  TAC_ARGUMENTS(6)
  const Tensor& src = given(a[0], "src");
  const Tensor* scales = maybe(a[1], "src scales");
  matrix_axes(src, "src");
  const Call c(src, "src");
  const int64_t R = src.size(0), C = scales ? columns_of(a[2], "cols") : src.size(1);
  tac_quantize_desc_t d = {R, C, 0, TAC_SCALED, yes(a[3]) ? TAC_BLOCK_TILE : TAC_BLOCK_ROW};
  At8 from = {nullptr, nullptr};
  if (scales) {
    from = at_8bit(c, src, *scales, R, C, "src codes", "src scales");
  } else {
    d.dtype = float_type(src, "src");
    from.codes = (const uint8_t*)c.lines(&src, "src", src.scalar_type(), src.sizes());
    d.src_stride = row_stride(&src, R, C);
  }
  Matrix8 to, turned;
  if (yes(a[4])) to = make_8bit(c, R, C);
  if (yes(a[5])) turned = make_8bit(c, C, R);
  const int status = unlocked([&] {
    return tac_quantize(&d, from.codes, from.scales, (uint8_t*)at_of(to.codes), (uint8_t*)at_of(to.scales),
                                  (uint8_t*)at_of(turned.codes), (uint8_t*)at_of(turned.scales), c.stream());
  });
  if (status) return PyLong_FromLong(status);
  return dict_of({{"rows", out_of(to)}, {"columns", out_of(turned)}});
  TAC_END
  END_HANDLE_TH_ERRORS
}

// codes, scales, cols, dtype, out
PyObject* dequantize(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  TAC_ARGUMENTS(5)
  const Tensor &codes = given(a[0], "matrix codes"), &scales = given(a[1], "matrix scales");
  matrix_axes(codes, "matrix codes");
  const Call c(codes, "matrix codes");
  const int64_t R = codes.size(0), C = columns_of(a[2], "cols");
  const At8 from = at_8bit(c, codes, scales, R, C, "matrix codes", "matrix scales");
  const Tensor* to = maybe(a[4], "out");
  const Tensor out = to ? *to : c.make({R, C}, type_of(a[3], ScalarType::Float));
  const int32_t type = float_type(out, "out");
  void* at = c.lines(&out, "out", out.scalar_type(), {R, C});
  const int status = unlocked([&] {
    return tac_dequantize(R, C, from.codes, from.scales, type, at, row_stride(&out, R, C), c.stream());
  });
  if (status) return PyLong_FromLong(status);
  written(to);
  return to ? same(a[4]) : out_of(out);
  TAC_END
  END_HANDLE_TH_ERRORS
}

// x, residual, gain, eps, h, y, want_h, want_y, want_scaled, want_rstd
PyObject* residual_norm(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  TAC_ARGUMENTS(10)
  const Tensor& x = given(a[0], "x");
  const Tensor *residual = maybe(a[1], "residual"), *gain = maybe(a[2], "gain"), *h_given = maybe(a[4], "h"), *y_given = maybe(a[5], "y");
  matrix_axes(x, "x");
  const int64_t R = x.size(0), C = x.size(1);
  const int32_t kind = float_type(x, "x");
  const ScalarType type = x.scalar_type();
  const Call c(x, "x");
  const auto shape = x.sizes();
  const void *x_at = c.lines(&x, "x", type, shape), *residual_at = c.lines(residual, "residual", type, shape);
  const float* gain_at = (const float*)c.whole(gain, "gain", ScalarType::Float, {C});
  void *h_at = c.lines(h_given, "h", type, shape), *y_at = c.lines(y_given, "y", type, shape);
  const double eps = PyFloat_AsDouble(a[3]);
  if (eps == -1.0 && PyErr_Occurred()) return nullptr;
  if (C > INT32_MAX) return PyLong_FromLong(TAC_ERR_UNSUPPORTED);
  Tensor h, y, rstd;
  Matrix8 scaled;
  if (!h_given && (a[6] == Py_None ? residual != nullptr : yes(a[6]))) h_at = (h = c.make(shape, type)).data_ptr();
  if (!y_given && yes(a[7])) y_at = (y = c.make(shape, type)).data_ptr();
  if (yes(a[8])) scaled = make_8bit(c, R, C);
  if (yes(a[9])) rstd = c.make({R}, ScalarType::Float);
  const tac_norm_desc_t d = {R, row_stride(&x, R, C), row_stride(residual, R, C), h_given ? row_stride(h_given, R, C) : C,
                             y_given ? row_stride(y_given, R, C) : C, (int32_t)C, kind, (float)eps};
  const int status = unlocked([&] {
    return tac_residual_norm(&d, x_at, residual_at, gain_at, h_at, y_at, (uint8_t*)at_of(scaled.codes), (uint8_t*)at_of(scaled.scales),
                                       (float*)at_of(rstd), c.stream());
  });
  if (status) return PyLong_FromLong(status);
  written(h_given);
  written(y_given);
  return dict_of({{"h", h_given ? same(a[4]) : out_of(h)}, {"y", y_given ? same(a[5]) : out_of(y)}, {"scaled", out_of(scaled)}, {"rstd", out_of(rstd)}});
  TAC_END
  END_HANDLE_TH_ERRORS
}

// h, gain, rstd, grad_y, grad_h, grad_x, want_grad_gain
PyObject* residual_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  TAC_ARGUMENTS(7)
  const Tensor &h = given(a[0], "h"), &rstd = given(a[2], "rstd"), &grad_y = given(a[3], "grad_y");
  const Tensor *gain = maybe(a[1], "gain"), *grad_h = maybe(a[4], "grad_h"), *to = maybe(a[5], "grad_x");
  matrix_axes(h, "h");
  const int64_t R = h.size(0), C = h.size(1);
  const int32_t kind = float_type(h, "h");
  const ScalarType type = h.scalar_type();
  const Call c(h, "h");
  const auto shape = h.sizes();
  const void *h_at = c.lines(&h, "h", type, shape), *gy_at = c.lines(&grad_y, "grad_y", type, shape), *gh_at = c.lines(grad_h, "grad_h", type, shape);
  void* gx_at = c.lines(to, "grad_x", type, shape);
  const float *gain_at = (const float*)c.whole(gain, "gain", ScalarType::Float, {C}), *rstd_at = (const float*)c.whole(&rstd, "rstd", ScalarType::Float, {R});
  if (C > INT32_MAX) return PyLong_FromLong(TAC_ERR_UNSUPPORTED);
  Tensor grad_x, grad_gain, work;
  if (!to) gx_at = (grad_x = c.make(shape, type)).data_ptr();
  const tac_norm_desc_t d = {R, to ? row_stride(to, R, C) : C, row_stride(grad_h, R, C), row_stride(&h, R, C), row_stride(&grad_y, R, C),
                             (int32_t)C, kind, 1.0f};
  if (yes(a[6])) {
    grad_gain = c.make({C}, ScalarType::Float);
    work = c.scratch(tac_residual_norm_workspace_bytes(&d));
  }
  const int status = unlocked([&] {
    return tac_residual_norm_backward(&d, h_at, gain_at, rstd_at, gy_at, gh_at, gx_at, (float*)at_of(grad_gain), at_of(work), c.stream());
  });
  if (status) return PyLong_FromLong(status);
  written(to);
  return dict_of({{"grad_x", to ? same(a[5]) : out_of(grad_x)}, {"grad_gain", out_of(grad_gain)}});
  TAC_END
  END_HANDLE_TH_ERRORS
}

// a codes, a scales, b codes, b scales, K, bias, dtype, out
PyObject* scaled_product(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  TAC_ARGUMENTS(8)
  const Tensor &ac = given(a[0], "a codes"), &as = given(a[1], "a scales"), &bc = given(a[2], "b codes"), &bs = given(a[3], "b scales");
  matrix_axes(ac, "a codes");
  matrix_axes(bc, "b codes");
  const int64_t M = ac.size(0), N = bc.size(0), K = columns_of(a[4], "K");
  const Call c(ac, "a codes");
  const At8 at = at_8bit(c, ac, as, M, K, "a codes", "a scales"), bt = at_8bit(c, bc, bs, N, K, "b codes", "b scales");
  const float* bias = (const float*)c.whole(maybe(a[5], "bias"), "bias", ScalarType::Float, {N});
  const Tensor* to = maybe(a[7], "out");
  const Tensor out = to ? *to : c.make({M, N}, type_of(a[6], ScalarType::BFloat16));
  const int32_t kind = float_type(out, "out");
  void* y = c.lines(&out, "out", out.scalar_type(), {M, N});
  const tac_product_desc_t d = {M, N, K, row_stride(&out, M, N), kind};
  const Tensor work = c.scratch(tac_scaled_product_workspace_bytes(&d));
  const int status = unlocked([&] {
    return tac_scaled_product(&d, at.codes, at.scales, bt.codes, bt.scales, bias, y, at_of(work), c.stream());
  });
  if (status) return PyLong_FromLong(status);
  written(to);
  return to ? same(a[7]) : out_of(out);
  TAC_END
  END_HANDLE_TH_ERRORS
}

// strides of the steps and sequences of a pair of tensors, which have to agree where there is more than one
struct Steps {
  int64_t t, b;
};
Steps steps_of(const Tensor& x, const Tensor& y, const char* names) {
  const Steps s = {x.stride(0), x.stride(1)};
  if ((x.size(0) > 1 && y.stride(0) != s.t) || (x.size(1) > 1 && y.stride(1) != s.b)) refuse("%s must have the same strides", names);
  return s;
}
void sequence_axes(const Tensor& t, const char* name) {
  if (t.dim() != 3) refuse("%s must be [T, B, D]", name);
  if (t.size(1) > INT32_MAX || t.size(2) > INT32_MAX) refuse("%s has too many sequences or channels", name);
}

// gate, value, lengths, h0, out, want_h_last, want_states
PyObject* gated_scan(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  TAC_ARGUMENTS(7)
  const Tensor &gate = given(a[0], "gate"), &value = given(a[1], "value");
  sequence_axes(gate, "gate");
  const int64_t T = gate.size(0), B = gate.size(1), D = gate.size(2);
  const int32_t kind = float_type(gate, "gate");
  const ScalarType type = gate.scalar_type();
  const Call c(gate, "gate");
  const auto shape = gate.sizes();
  const void *g = c.lines(&gate, "gate", type, shape), *v = c.lines(&value, "value", type, shape);
  const Steps in = steps_of(gate, value, "gate and value");
  const int32_t* lengths = (const int32_t*)c.whole(maybe(a[2], "lengths"), "lengths", ScalarType::Int, {B});
  const float* h0 = (const float*)c.whole(maybe(a[3], "h0"), "h0", ScalarType::Float, {B, D});
  const Tensor* to = maybe(a[4], "out");
  const Tensor out = to ? *to : c.make(shape, type);
  void* o = c.lines(&out, "out", type, shape);
  Tensor h_last, states;
  if (yes(a[5])) h_last = c.make({B, D}, ScalarType::Float);
  if (yes(a[6])) states = c.make({up(T, TAC_SCAN_CHUNK), B, D}, ScalarType::Float);
  const tac_scan_desc_t d = {T, (int32_t)B, (int32_t)D, in.t, in.b, out.stride(0), out.stride(1), 0, 0, kind};
  const Tensor work = c.scratch(tac_gated_scan_workspace_bytes(&d));
  const int status = unlocked([&] {
    return tac_gated_scan(&d, g, v, lengths, h0, o, (float*)at_of(h_last), (float*)at_of(states), at_of(work), c.stream());
  });
  if (status) return PyLong_FromLong(status);
  written(to);
  return dict_of({{"out", to ? same(a[4]) : out_of(out)}, {"h_last", out_of(h_last)}, {"states", out_of(states)}});
  TAC_END
  END_HANDLE_TH_ERRORS
}

// gate, value, states, grad_out, lengths, grad_h_last, grad_gate, grad_value, want_grad_h0
PyObject* gated_scan_backward(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  TAC_ARGUMENTS(9)
  const Tensor &gate = given(a[0], "gate"), &value = given(a[1], "value"), &states = given(a[2], "states"), &grad_out = given(a[3], "grad_out");
  sequence_axes(gate, "gate");
  const int64_t T = gate.size(0), B = gate.size(1), D = gate.size(2);
  const int32_t kind = float_type(gate, "gate");
  const ScalarType type = gate.scalar_type();
  const Call c(gate, "gate");
  const auto shape = gate.sizes();
  const void *g = c.lines(&gate, "gate", type, shape), *v = c.lines(&value, "value", type, shape), *go = c.lines(&grad_out, "grad_out", type, shape);
  const Steps in = steps_of(gate, value, "gate and value");
  const int32_t* lengths = (const int32_t*)c.whole(maybe(a[4], "lengths"), "lengths", ScalarType::Int, {B});
  const float* kept = (const float*)c.whole(&states, "states", ScalarType::Float, {up(T, TAC_SCAN_CHUNK), B, D});
  const float* last = (const float*)c.whole(maybe(a[5], "grad_h_last"), "grad_h_last", ScalarType::Float, {B, D});
  const Tensor *gg_given = maybe(a[6], "grad_gate"), *gv_given = maybe(a[7], "grad_value");
  c.lines(gg_given, "grad_gate", type, shape);
  c.lines(gv_given, "grad_value", type, shape);
  // the one that is not given is laid out as the other is
  auto like = [&](const Tensor* other) {
    return other && !other->is_contiguous() ? at::empty_strided(shape, other->strides(), other->options()) : c.make(shape, type);
  };
  const Tensor gg = gg_given ? *gg_given : like(gv_given), gv = gv_given ? *gv_given : like(gg_given);
  const Steps grad = steps_of(gg, gv, "grad_gate and grad_value");
  Tensor h0;
  if (yes(a[8])) h0 = c.make({B, D}, ScalarType::Float);
  const tac_scan_desc_t d = {T, (int32_t)B, (int32_t)D, in.t, in.b, grad_out.stride(0), grad_out.stride(1), grad.t, grad.b, kind};
  const Tensor work = c.scratch(tac_gated_scan_workspace_bytes(&d));
  const int status = unlocked([&] {
    return tac_gated_scan_backward(&d, g, v, lengths, kept, go, last, gg.data_ptr(), gv.data_ptr(), (float*)at_of(h0), at_of(work), c.stream());
  });
  if (status) return PyLong_FromLong(status);
  written(gg_given);
  written(gv_given);
  return dict_of({{"grad_gate", gg_given ? same(a[6]) : out_of(gg)}, {"grad_value", gv_given ? same(a[7]) : out_of(gv)}, {"grad_h0", out_of(h0)}});
  TAC_END
  END_HANDLE_TH_ERRORS
}

// gate, value, pool, slots, out
PyObject* gated_step(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  TAC_ARGUMENTS(5)
  const Tensor &gate = given(a[0], "gate"), &value = given(a[1], "value"), &pool = given(a[2], "pool");
  matrix_axes(gate, "gate");
  matrix_axes(pool, "pool");
  const int64_t B = gate.size(0), D = gate.size(1), slots = pool.size(0);
  if (B > INT32_MAX || D > INT32_MAX) refuse("gate has too many sequences or channels");
  const int32_t kind = float_type(gate, "gate");
  const ScalarType type = gate.scalar_type();
  const Call c(gate, "gate");
  const auto shape = gate.sizes();
  const void *g = c.lines(&gate, "gate", type, shape), *v = c.lines(&value, "value", type, shape);
  if (B > 1 && gate.stride(0) != value.stride(0)) refuse("gate and value must have the same strides");
  float* states = (float*)c.whole(&pool, "pool", ScalarType::Float, {slots, D});
  const int32_t* of = (const int32_t*)c.whole(maybe(a[3], "slots"), "slots", ScalarType::Int, {B});
  const Tensor* to = maybe(a[4], "out");
  const Tensor out = to ? *to : c.make(shape, type);
  void* o = c.lines(&out, "out", type, shape);
  const tac_scan_desc_t d = {1, (int32_t)B, (int32_t)D, 0, row_stride(&gate, B, D), 0, row_stride(&out, B, D), 0, 0, kind};
  const int status = unlocked([&] {
    return tac_gated_step(&d, g, v, states, slots, of, o, c.stream());
  });
  if (status) return PyLong_FromLong(status);
  written(to);
  written(&pool);
  return to ? same(a[4]) : out_of(out);
  TAC_END
  END_HANDLE_TH_ERRORS
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef entry(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}

PyMethodDef kMethods[] = {entry<quantize>("quantize"),
                          entry<dequantize>("dequantize"),
                          entry<residual_norm>("residual_norm"),
                          entry<residual_norm_backward>("residual_norm_backward"),
                          entry<scaled_product>("scaled_product"),
                          entry<gated_scan>("gated_scan"),
                          entry<gated_scan_backward>("gated_scan_backward"),
                          entry<gated_step>("gated_step"),
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_operators", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__operators() { return PyModule_Create(&kModule); }
