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

// ---- heads and the gated delta rule ----------------------------------------------------------------

double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused();
  return v;
}
void head_axes(const Tensor& t, const char* name) {
  if (t.dim() != 3) refuse("%s must be [rows, heads, features]", name);
  if (t.size(1) > INT32_MAX || t.size(2) > INT32_MAX) refuse("%s has too many heads or features", name);
}
tac_head_strides_t head_strides(const Tensor& t) { return {t.stride(0), t.stride(1)}; }

// What both directions of the head norm share: eps, positions, sections, base, interleaved from a[0] on
struct Rotation {
  tac_head_norm_desc_t d = {};
  const int32_t* positions = nullptr;
  Rotation(const Call& c, const Tensor& q, const Tensor* k, PyObject* const* a) {
    d.rows = q.size(0);
    d.query_heads = (int32_t)q.size(1);
    d.D = (int32_t)q.size(2);
    d.dtype = float_type(q, "query");
    d.query = head_strides(q);
    if (k) {
      d.key_heads = (int32_t)k->size(1);
      d.key = head_strides(*k);
    }
    if (a[0] != Py_None) {
      d.eps = (float)number(a[0]);
      if (!(d.eps > 0.0f)) refuse("eps must be more than 0 (None: no norm)");
    }
    const Tensor* at = maybe(a[1], "positions");
    if (!at) {
      if (a[2] != Py_None) refuse("sections need positions");
      if (a[0] == Py_None) refuse("neither a norm (eps) nor positions");
      return;
    }
    if (at->dim() != 1 && at->dim() != 2) refuse("positions must be [rows] or [rows, axes]");
    const int64_t axes = at->dim() == 1 ? 1 : at->size(1);
    if (axes < 1 || axes > TAC_ROTATION_AXES) refuse("positions must have 1 to %d axes", TAC_ROTATION_AXES);
    if (at->dim() == 1) positions = (const int32_t*)c.whole(at, "positions", ScalarType::Int, {d.rows});
    else positions = (const int32_t*)c.whole(at, "positions", ScalarType::Int, {d.rows, axes});
    d.axes = (int32_t)axes;
    if (a[2] == Py_None) {
      if (axes > 1) refuse("several axes need sections");
      d.pairs[0] = d.D / 2;
    } else {
      PyObject* items = PySequence_Fast(a[2], "sections must be a sequence of numbers of pairs");
      if (!items) throw Refused();
      int64_t pairs[TAC_ROTATION_AXES] = {};
      const Py_ssize_t count = PySequence_Fast_GET_SIZE(items);
      bool wrong = count != axes;
      for (Py_ssize_t i = 0; i < count && !wrong; ++i) {
        pairs[i] = PyLong_AsLongLong(PySequence_Fast_GET_ITEM(items, i));
        wrong = pairs[i] < 1 || pairs[i] > INT32_MAX;
        d.pairs[i] = (int32_t)pairs[i];
      }
      Py_DECREF(items);
      if (PyErr_Occurred()) throw Refused();
      if (wrong) refuse("sections must be one number of pairs, at least 1, for each axis");
    }
    d.base = number(a[3]);
    d.interleaved = yes(a[4]);
  }
};

// query, key, gain_query, gain_key, eps, positions, sections, base, interleaved, out_query, out_key
PyObject* head_norm(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  TAC_ARGUMENTS(11)
  const Tensor& q = given(a[0], "query");
  const Tensor *k = maybe(a[1], "key"), *gq = maybe(a[2], "gain_query"), *gk = maybe(a[3], "gain_key"), *oq_given = maybe(a[9], "out_query"), *ok_given = maybe(a[10], "out_key");
  head_axes(q, "query");
  if (k) head_axes(*k, "key");
  if (!k && (gk || ok_given)) refuse("gain_key and out_key need keys");
  const Call c(q, "query");
  Rotation r(c, q, k, a + 4);
  const ScalarType type = q.scalar_type();
  const int64_t R = q.size(0), D = q.size(2);
  const void *q_at = c.lines(&q, "query", type, q.sizes()), *k_at = k ? c.lines(k, "key", type, {R, k->size(1), D}) : nullptr;
  const float *gq_at = (const float*)c.whole(gq, "gain_query", ScalarType::Float, {D}), *gk_at = (const float*)c.whole(gk, "gain_key", ScalarType::Float, {D});
  const Tensor oq = oq_given ? *oq_given : c.make(q.sizes(), type), ok = !k ? Tensor() : ok_given ? *ok_given : c.make(k->sizes(), type);
  void *oq_at = c.lines(&oq, "out_query", type, q.sizes()), *ok_at = k ? c.lines(&ok, "out_key", type, k->sizes()) : nullptr;
  r.d.out_query = head_strides(oq);
  if (k) r.d.out_key = head_strides(ok);
  const int status = unlocked([&] { return tac_head_norm(&r.d, q_at, k_at, gq_at, gk_at, r.positions, oq_at, ok_at, c.stream()); });
  if (status) return PyLong_FromLong(status);
  written(oq_given);
  written(ok_given);
  return dict_of({{"q", oq_given ? same(a[9]) : out_of(oq)}, {"k", ok_given ? same(a[10]) : out_of(ok)}});
  TAC_END
  END_HANDLE_TH_ERRORS
}

// query, key, gain_query, gain_key, grad_out_query, grad_out_key, eps, positions, sections, base, interleaved, grad_query, grad_key, want_grad_gain
PyObject* head_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  TAC_ARGUMENTS(14)
  const Tensor &q = given(a[0], "query"), &dq = given(a[4], "grad_out_query");
  const Tensor *k = maybe(a[1], "key"), *gq = maybe(a[2], "gain_query"), *gk = maybe(a[3], "gain_key"), *dk = maybe(a[5], "grad_out_key"),
               *xq_given = maybe(a[11], "grad_query"), *xk_given = maybe(a[12], "grad_key");
  head_axes(q, "query");
  if (k) head_axes(*k, "key");
  if (!k && (gk || dk || xk_given)) refuse("gain_key, grad_out_key and grad_key need keys");
  if (k && !dk) refuse("grad_out_key is missing");
  const Call c(q, "query");
  Rotation r(c, q, k, a + 6);
  const ScalarType type = q.scalar_type();
  const int64_t R = q.size(0), D = q.size(2);
  const void *q_at = c.lines(&q, "query", type, q.sizes()), *k_at = k ? c.lines(k, "key", type, {R, k->size(1), D}) : nullptr;
  const void *dq_at = c.lines(&dq, "grad_out_query", type, q.sizes()), *dk_at = k ? c.lines(dk, "grad_out_key", type, k->sizes()) : nullptr;
  const float *gq_at = (const float*)c.whole(gq, "gain_query", ScalarType::Float, {D}), *gk_at = (const float*)c.whole(gk, "gain_key", ScalarType::Float, {D});
  const Tensor xq = xq_given ? *xq_given : c.make(q.sizes(), type), xk = !k ? Tensor() : xk_given ? *xk_given : c.make(k->sizes(), type);
  void *xq_at = c.lines(&xq, "grad_query", type, q.sizes()), *xk_at = k ? c.lines(&xk, "grad_key", type, k->sizes()) : nullptr;
  r.d.out_query = head_strides(dq);
  r.d.grad_query = head_strides(xq);
  if (k) {
    r.d.out_key = head_strides(*dk);
    r.d.grad_key = head_strides(xk);
  }
  Tensor sum_q, sum_k, work;
  if (yes(a[13])) {
    sum_q = c.make({D}, ScalarType::Float);
    if (k) sum_k = c.make({D}, ScalarType::Float);
    work = c.scratch(tac_head_norm_workspace_bytes(&r.d));
  }
  const int status = unlocked([&] {
    return tac_head_norm_backward(&r.d, q_at, k_at, gq_at, gk_at, r.positions, dq_at, dk_at, xq_at, xk_at, (float*)at_of(sum_q), (float*)at_of(sum_k), at_of(work),
                                  c.stream());
  });
  if (status) return PyLong_FromLong(status);
  written(xq_given);
  written(xk_given);
  return dict_of({{"grad_q", xq_given ? same(a[11]) : out_of(xq)}, {"grad_k", xk_given ? same(a[12]) : out_of(xk)}, {"grad_gain_q", out_of(sum_q)}, {"grad_gain_k", out_of(sum_k)}});
  TAC_END
  END_HANDLE_TH_ERRORS
}

// query, key, value, gate, write of a delta rule, [T, B, heads, ..] or (a step) [B, heads, ..]
struct Delta {
  tac_delta_desc_t d = {};
  const Tensor &q, &k, &v, &g, &w;
  bool step;
  ScalarType type;
  const void *q_at, *k_at, *v_at, *g_at, *w_at;
  static const Tensor& axes(PyObject* o, const char* name, int64_t n) {
    const Tensor& t = given(o, name);
    if (t.dim() != n) refuse("%s must have %d axes", name, (int)n);
    for (int64_t i = 0; i < n; ++i)
      if (t.size(i) > INT32_MAX) refuse("%s is too large", name);
    return t;
  }
  // a shape without an allocation
  struct Shape {
    int64_t n[5];
    size_t count;
    operator at::IntArrayRef() const { return at::IntArrayRef(n, count); }
  };
  Shape keys() const { return step ? Shape{{d.B, d.k_heads, d.Dk}, 3} : Shape{{d.T, d.B, d.k_heads, d.Dk}, 4}; }
  Shape values() const { return step ? Shape{{d.B, d.v_heads, d.Dv}, 3} : Shape{{d.T, d.B, d.v_heads, d.Dv}, 4}; }
  Shape gates() const { return step ? Shape{{d.B, d.v_heads}, 2} : Shape{{d.T, d.B, d.v_heads}, 3}; }
  Shape state() const { return Shape{{d.B, d.v_heads, d.Dk, d.Dv}, 4}; }
  tac_delta_strides_t strides(const Tensor& t) const {
    return step ? tac_delta_strides_t{0, t.stride(0), t.stride(1)} : tac_delta_strides_t{t.stride(0), t.stride(1), t.stride(2)};
  }
  Delta(PyObject* const* a, bool one)
      : q(axes(a[0], "query", one ? 3 : 4)), k(axes(a[1], "key", one ? 3 : 4)), v(axes(a[2], "value", one ? 3 : 4)), g(axes(a[3], "gate", one ? 2 : 3)),
        w(axes(a[4], "write", one ? 2 : 3)), step(one), type(q.scalar_type()) {
    const int64_t first = one ? 0 : 1;
    d.T = one ? 1 : q.size(0);
    d.B = (int32_t)q.size(first);
    d.k_heads = (int32_t)q.size(first + 1);
    d.Dk = (int32_t)q.size(first + 2);
    d.v_heads = (int32_t)v.size(first + 1);
    d.Dv = (int32_t)v.size(first + 2);
    d.dtype = float_type(q, "query");
    d.query = strides(q);
    d.key = strides(k);
    d.value = strides(v);
    d.gate = strides(g);
    d.write = strides(w);
  }
  void look(const Call& c) {
    q_at = c.lines(&q, "query", type, keys());
    k_at = c.lines(&k, "key", type, keys());
    v_at = c.lines(&v, "value", type, values());
    g_at = c.lines(&g, "gate", type, gates());
    w_at = c.lines(&w, "write", type, gates());
  }
};

// query, key, value, gate, write, lengths, h0, out, want_h_last, want_kept
PyObject* delta_scan(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  TAC_ARGUMENTS(10)
  Delta x(a, false);
  const Call c(x.q, "query");
  x.look(c);
  const auto& d = x.d;
  const int32_t* lengths = (const int32_t*)c.whole(maybe(a[5], "lengths"), "lengths", ScalarType::Int, {d.B});
  const float* h0 = (const float*)c.whole(maybe(a[6], "h0"), "h0", ScalarType::Float, x.state());
  const Tensor* to = maybe(a[7], "out");
  const Tensor out = to ? *to : c.make(x.values(), x.type);
  void* o = c.lines(&out, "out", x.type, x.values());
  x.d.out = x.strides(out);
  Tensor h_last, states, updates;
  if (yes(a[8])) h_last = c.make(x.state(), ScalarType::Float);
  if (yes(a[9])) {
    states = c.make({up(d.T, TAC_DELTA_CHUNK), d.B, d.v_heads, d.Dk, d.Dv}, ScalarType::Float);
    updates = c.make(x.values(), ScalarType::Float);
  }
  const Tensor work = c.scratch(tac_delta_scan_workspace_bytes(&x.d));
  const int status = unlocked([&] {
    return tac_delta_scan(&x.d, x.q_at, x.k_at, x.v_at, x.g_at, x.w_at, lengths, h0, o, (float*)at_of(h_last), (float*)at_of(states), (float*)at_of(updates), at_of(work),
                          c.stream());
  });
  if (status) return PyLong_FromLong(status);
  written(to);
  return dict_of({{"out", to ? same(a[7]) : out_of(out)}, {"h_last", out_of(h_last)}, {"states", out_of(states)}, {"updates", out_of(updates)}});
  TAC_END
  END_HANDLE_TH_ERRORS
}

// query, key, value, gate, write, states, updates, grad_out, lengths, grad_h_last, grad_query, grad_key, grad_value, grad_gate, grad_write, want_grad_h0
PyObject* delta_scan_backward(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  TAC_ARGUMENTS(16)
  Delta x(a, false);
  const Call c(x.q, "query");
  x.look(c);
  const auto& d = x.d;
  const float* states = (const float*)c.whole(&given(a[5], "states"), "states", ScalarType::Float, {up(d.T, TAC_DELTA_CHUNK), d.B, d.v_heads, d.Dk, d.Dv});
  const float* updates = (const float*)c.whole(&given(a[6], "updates"), "updates", ScalarType::Float, x.values());
  const Tensor& go = given(a[7], "grad_out");
  const void* go_at = c.lines(&go, "grad_out", x.type, x.values());
  x.d.out = x.strides(go);
  const int32_t* lengths = (const int32_t*)c.whole(maybe(a[8], "lengths"), "lengths", ScalarType::Int, {d.B});
  const float* last = (const float*)c.whole(maybe(a[9], "grad_h_last"), "grad_h_last", ScalarType::Float, x.state());
  const char* const names[5] = {"grad_query", "grad_key", "grad_value", "grad_gate", "grad_write"};
  const Delta::Shape shapes[5] = {x.keys(), x.keys(), x.values(), x.gates(), x.gates()};
  tac_delta_strides_t* const strides[5] = {&x.d.grad_query, &x.d.grad_key, &x.d.grad_value, &x.d.grad_gate, &x.d.grad_write};
  Tensor grads[5];
  void* at[5];
  for (int i = 0; i < 5; ++i) {
    const Tensor* t = maybe(a[10 + i], names[i]);
    grads[i] = t ? *t : c.make(shapes[i], x.type);
    at[i] = c.lines(&grads[i], names[i], x.type, shapes[i]);
    *strides[i] = x.strides(grads[i]);
  }
  Tensor h0;
  if (yes(a[15])) h0 = c.make(x.state(), ScalarType::Float);
  const Tensor work = c.scratch(tac_delta_scan_backward_workspace_bytes(&x.d));
  const int status = unlocked([&] {
    return tac_delta_scan_backward(&x.d, x.q_at, x.k_at, x.v_at, x.g_at, x.w_at, lengths, states, updates, go_at, last, at[0], at[1], at[2], at[3], at[4],
                                   (float*)at_of(h0), at_of(work), c.stream());
  });
  if (status) return PyLong_FromLong(status);
  PyObject* made[5];
  for (int i = 0; i < 5; ++i) {
    written(maybe(a[10 + i], names[i]));
    made[i] = a[10 + i] != Py_None ? same(a[10 + i]) : out_of(grads[i]);
  }
  return dict_of({{names[0], made[0]}, {names[1], made[1]}, {names[2], made[2]}, {names[3], made[3]}, {names[4], made[4]}, {"grad_h0", out_of(h0)}});
  TAC_END
  END_HANDLE_TH_ERRORS
}

// query, key, value, gate, write, pool, slots, out
PyObject* delta_step(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  TAC_ARGUMENTS(8)
  Delta x(a, true);
  const Call c(x.q, "query");
  x.look(c);
  const auto& d = x.d;
  const Tensor& pool = given(a[5], "pool");
  if (pool.dim() != 4) refuse("pool must be [slots, heads, Dk, Dv]");
  const int64_t n = pool.size(0);
  float* states = (float*)c.whole(&pool, "pool", ScalarType::Float, {n, d.v_heads, d.Dk, d.Dv});
  const int32_t* slots = (const int32_t*)c.whole(maybe(a[6], "slots"), "slots", ScalarType::Int, {d.B});
  const Tensor* to = maybe(a[7], "out");
  const Tensor out = to ? *to : c.make(x.values(), x.type);
  void* o = c.lines(&out, "out", x.type, x.values());
  x.d.out = x.strides(out);
  const int status = unlocked([&] { return tac_delta_step(&x.d, x.q_at, x.k_at, x.v_at, x.g_at, x.w_at, states, n, slots, o, c.stream()); });
  if (status) return PyLong_FromLong(status);
  written(to);
  written(&pool);
  return to ? same(a[7]) : out_of(out);
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
                          entry<head_norm>("head_norm"),
                          entry<head_norm_backward>("head_norm_backward"),
                          entry<delta_scan>("delta_scan"),
                          entry<delta_scan_backward>("delta_scan_backward"),
                          entry<delta_step>("delta_step"),
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_operators", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__operators() { return PyModule_Create(&kModule); }
