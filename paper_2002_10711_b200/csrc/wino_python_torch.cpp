// The calls a program makes once per layer and pass, WinogradConv.forward and the layers with 4-bit
// weights, on torch tensors: they allocate the output and call the library on torch's current stream.
// Argument checks and marshalling only, as in wino_python.c; being compiled against torch it reads tensor addresses
// and allocates through the caching allocator without going through Python and the dispatcher,
// which took 2.3 of the 5.5 us of a small layer's pass.
#include <Python.h>

#include <initializer_list>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/AutogradState.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "wino.h"

namespace {

bool tensor_or_none(PyObject* o) { return o == Py_None || THPVariable_Check(o); }
void* address(PyObject* o) { return o == Py_None ? nullptr : THPVariable_Unpack(o).mutable_data_ptr(); }

// (plan, x, U_q, bias, y or None, workspace, like) -> y, the (negative) return code, or None where
// an argument is not a tensor.  like: a tensor of the output's shape, type and device.
PyObject* forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 7) {
    PyErr_Format(PyExc_TypeError, "forward takes 7 arguments (%zd given)", n);
    return nullptr;
  }
  for (int i = 1; i < 6; ++i)
    if (!tensor_or_none(a[i])) Py_RETURN_NONE;
  if (!THPVariable_Check(a[6])) Py_RETURN_NONE;
  void* plan = PyLong_AsVoidPtr(a[0]);
  if (plan == nullptr && PyErr_Occurred()) return nullptr;
  PyObject* result;
  void* y;
  if (a[4] == Py_None) {
    const at::Tensor& like = THPVariable_Unpack(a[6]);
    at::Tensor out = at::detail::empty_cuda(like.sizes(), like.scalar_type(), like.device(), std::nullopt);
    y = out.mutable_data_ptr();
    result = THPVariable_Wrap(std::move(out));
    if (result == nullptr) return nullptr;
  } else {
    y = address(a[4]);
    result = Py_NewRef(a[4]);
  }
  const void* x = address(a[1]);
  const void* u = address(a[2]);
  const void* bias = address(a[3]);
  void* ws = address(a[5]);
  cudaStream_t st = c10::cuda::getCurrentCUDAStream().stream();
  int rc;
  Py_BEGIN_ALLOW_THREADS   // a launch may wait for room in the queue
  rc = wino_conv_forward(static_cast<wino_plan_t*>(plan), static_cast<const int8_t*>(x), static_cast<const int8_t*>(u),
                         static_cast<const float*>(bias), y, ws, st);
  Py_END_ALLOW_THREADS
  if (rc == WINO_OK) return result;
  Py_DECREF(result);
  return PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// ---- layers with 4-bit weights -----------------------------------------------------------
// Arguments of the wrong type raise TypeError, of the wrong shape, type of element or device ValueError.
struct Bad {};   // a Python exception is set

[[noreturn]] void refuse(PyObject* kind, const char* what) {
  PyErr_SetString(kind, what);
  throw Bad();
}
// Any tensor; one that is read or written as it lies in memory.
const at::Tensor& any_tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, what);
  return THPVariable_Unpack(o);
}
const at::Tensor& tensor(PyObject* o, const char* what) {
  const at::Tensor& t = any_tensor(o, what);
  if (t.is_neg()) refuse(PyExc_ValueError, "a view whose elements are to be negated (call resolve_neg())");
  return t;
}
long integer(PyObject* o, const char* what) {
  const long v = PyLong_Check(o) ? PyLong_AsLong(o) : (refuse(PyExc_TypeError, what), 0l);
  if ((v == -1 && PyErr_Occurred()) || v != (int32_t)v) {
    PyErr_Clear();
    refuse(PyExc_ValueError, what);
  }
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Bad();
  return v != 0;
}
// -1: not one of the library's types
int type_code(at::ScalarType t) {
  return t == at::kFloat ? WINO_FLOAT : t == at::kBFloat16 ? WINO_BF16 : t == at::kHalf ? WINO_FP16
                                                          : t == at::kChar ? WINO_INT8 : -1;
}
double number(PyObject* q, const char* name, double fallback) {
  PyObject* v;
  if (PyDict_Check(q)) {
    v = PyDict_GetItemString(q, name);
    Py_XINCREF(v);
  } else {
    v = PyObject_GetAttrString(q, name);
    if (v == nullptr && PyErr_ExceptionMatches(PyExc_AttributeError)) PyErr_Clear();
  }
  if (v == nullptr) {
    if (PyErr_Occurred()) throw Bad();
    return fallback;
  }
  const double d = PyFloat_AsDouble(v);
  Py_DECREF(v);
  if (d == -1.0 && PyErr_Occurred()) throw Bad();
  return d;
}
int32_t whole(PyObject* q, const char* name, double fallback) {
  const double d = number(q, name, fallback);
  if (!(d >= -2147483648.0 && d <= 2147483647.0)) refuse(PyExc_ValueError, "quantizer field out of range");
  if (d != (double)(int32_t)d) refuse(PyExc_ValueError, "zero point and code bounds of a quantizer must be whole numbers");
  return (int32_t)d;
}
wino_quant_t quantizer(PyObject* q) {
  wino_quant_t r = {1.0f, 0, -127, 127, 1};
  if (q == Py_None) return r;
  r.scale = (float)number(q, "scale", 1.0);
  r.zero_point = whole(q, "zero_point", 0);
  r.qmin = whole(q, "qmin", -127);
  r.qmax = whole(q, "qmax", 127);
  return r;
}
void forward_only(const at::Tensor& t) {
  if (t.requires_grad() && c10::GradMode::is_enabled())
    refuse(PyExc_ValueError, "forward only: no gradient is computed (call under torch.no_grad())");
  if (t._fw_grad(/*level=*/0).defined() && c10::AutogradState::get_tls_state().get_fw_grad_mode())
    refuse(PyExc_ValueError, "forward only: no tangent is computed (call on the primals of dual tensors)");
}

// A tuple (codes, scales, zeros or None, K, C, group) of `batch` matrices on `device`.
wino_packed_t packed(PyObject* o, long batch, const at::Device& device) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 6)
    refuse(PyExc_TypeError, "packed weights must be a W4 or a tuple (codes, scales, zeros, K, C, group)");
  const at::Tensor& codes = tensor(PyTuple_GET_ITEM(o, 0), "codes must be a tensor");
  const at::Tensor& scales = tensor(PyTuple_GET_ITEM(o, 1), "scales must be a tensor");
  PyObject* z = PyTuple_GET_ITEM(o, 2);
  wino_packed_t w;
  w.K = (int32_t)integer(PyTuple_GET_ITEM(o, 3), "K must be an int of 32 bits");
  w.C = (int32_t)integer(PyTuple_GET_ITEM(o, 4), "C must be an int of 32 bits");
  w.group = (int32_t)integer(PyTuple_GET_ITEM(o, 5), "group must be an int of 32 bits");
  const int64_t bytes = (int64_t)wino_packed_code_bytes(w.K, w.C);
  const int64_t count = (int64_t)wino_packed_scale_count(w.K, w.C, w.group);
  if (bytes == 0 || count == 0)
    refuse(PyExc_ValueError, "K and C must be positive, group 32, 64 or a multiple of 128");
  if (codes.scalar_type() != at::kByte || !codes.is_contiguous() || codes.numel() != bytes * batch)
    refuse(PyExc_ValueError, "codes must be contiguous uint8 [..., K/16, C/128, 16, 4, 16]");
  w.scale_dtype = type_code(scales.scalar_type());
  if ((w.scale_dtype != WINO_BF16 && w.scale_dtype != WINO_FP16) || !scales.is_contiguous() ||
      scales.numel() != count * batch)
    refuse(PyExc_ValueError, "scales must be contiguous bfloat16 or float16 [..., K/16, groups, 16]");
  if (codes.device() != device || scales.device() != device)
    refuse(PyExc_ValueError, "packed weights must be on the device of the input");
  forward_only(scales);
  w.codes_dev = codes.const_data_ptr();
  w.scales_dev = scales.const_data_ptr();
  w.zeros_dev = nullptr;
  if (z != Py_None) {
    const at::Tensor& zeros = tensor(z, "zeros must be a tensor or None");
    if (zeros.scalar_type() != at::kByte || !zeros.is_contiguous() || zeros.numel() != count * batch ||
        zeros.device() != device)
      refuse(PyExc_ValueError, "zeros must be contiguous uint8 [..., K/16, groups, 16] on the device of the input");
    w.zeros_dev = zeros.const_data_ptr<uint8_t>();
  }
  return w;
}
const float* float_vector(PyObject* o, int64_t n, const at::Device& device, const char* what) {
  if (o == Py_None) return nullptr;
  const at::Tensor& v = tensor(o, what);
  if (v.scalar_type() != at::kFloat || !v.is_contiguous() || v.numel() != n || v.device() != device)
    refuse(PyExc_ValueError, what);
  forward_only(v);
  return v.const_data_ptr<float>();
}
// x [..., n] as rows a constant number of elements apart; `keep` holds the copy where that takes one.
struct Rows { int64_t count, stride; const void* data; };
Rows rows_of(const at::Tensor& x, int64_t n, at::Tensor& keep) {
  if (!x.is_cuda()) refuse(PyExc_ValueError, "inputs must be on a CUDA device");
  if (x.dim() < 1 || x.size(-1) != n) refuse(PyExc_ValueError, "the last dimension of x must be the layer's input size");
  forward_only(x);
  Rows r;
  r.count = x.numel() / n;
  if (x.is_neg()) keep = x.resolve_neg().contiguous(), r.stride = n;
  else if (x.dim() == 1 && x.stride(0) == 1) r.stride = n;
  else if (x.dim() == 2 && x.stride(1) == 1 && (x.size(0) <= 1 || x.stride(0) >= n)) r.stride = x.size(0) <= 1 ? n : x.stride(0);
  else if (x.is_contiguous()) r.stride = n;
  else keep = x.contiguous(), r.stride = n;
  r.data = keep.defined() ? keep.const_data_ptr() : x.const_data_ptr();
  if (r.count > (1 << 24)) refuse(PyExc_ValueError, "more than 2^24 rows");
  return r;
}
// Whether the n bytes at p share one with the rows of ny bytes at y, `count` of them dy >= ny apart.
bool touches(uintptr_t p, int64_t n, uintptr_t y, int64_t ny, int64_t dy, int64_t count) {
  if (n < 1 || count < 1 || p + n <= y || y + (count - 1) * dy + ny <= p) return false;
  const int64_t i = p < y || count == 1 ? 0 : (int64_t)(p - y) / dy;      // the last row that begins at or in front of p
  return p < y + i * dy + ny || (i + 1 < count && y + (i + 1) * dy < p + n);
}
// The same of `count` rows of nx bytes from x, dx apart.
bool overlap(uintptr_t x, int64_t nx, int64_t dx, uintptr_t y, int64_t ny, int64_t dy, int64_t count) {
  if (count < 1 || x + (count - 1) * dx + nx <= y || y + (count - 1) * dy + ny <= x) return false;
  if (count == 1) return true;
  if (dx == dy) {
    const int64_t apart = (((int64_t)(y - x)) % dx + dx) % dx;      // columns of the same rows
    return apart < nx || apart + ny > dx;
  }
  for (int64_t i = 0; i < count; ++i)
    if (touches(x + i * dx, nx, y, ny, dy, count)) return true;
  return false;
}
// The caller's result may not lie on the other operands either, dense and null where there is none: blocks read
// them while others write.
struct Dense { const void* data; int64_t bytes; };
void apart(const at::Tensor& y, int64_t stride, int64_t count, int64_t n, std::initializer_list<Dense> operands) {
  const int64_t size = y.element_size();
  for (const Dense& o : operands)
    if (o.data != nullptr && touches(reinterpret_cast<uintptr_t>(o.data), o.bytes, reinterpret_cast<uintptr_t>(y.const_data_ptr()),
                                     n * size, stride * size, count))
      refuse(PyExc_ValueError, "out may not overlap the weights, the router or a bias");
}
int64_t code_bytes(const wino_packed_t& w) { return (int64_t)wino_packed_code_bytes(w.K, w.C); }
int64_t scale_count(const wino_packed_t& w) { return (int64_t)wino_packed_scale_count(w.K, w.C, w.group); }
// The result [..., n] like x, new or the caller's; its row stride.  Blocks read all of x while others write.
at::Tensor result_like(PyObject* out, const at::Tensor& x, const Rows& from, int64_t n, at::ScalarType type,
                       int64_t* stride) {
  c10::DimVector shape(x.sizes().begin(), x.sizes().end());
  shape.back() = n;
  *stride = n;
  if (out == Py_None) return at::detail::empty_cuda(shape, type, x.device(), std::nullopt);
  const at::Tensor& y = tensor(out, "out must be a tensor");
  if (y.sizes() != c10::IntArrayRef(shape) || y.scalar_type() != type || y.device() != x.device())
    refuse(PyExc_ValueError, "out has another shape, type or device than the result");
  forward_only(y);
  const bool rows = y.dim() == 2 && (y.size(1) <= 1 || y.stride(1) == 1) && (y.size(0) <= 1 || y.stride(0) >= n);
  if (!rows && !y.is_contiguous()) refuse(PyExc_ValueError, "out must be contiguous, or rows of contiguous elements");
  if (rows && y.size(0) > 1) *stride = y.stride(0);
  const int64_t bx = x.element_size(), by = y.element_size();
  if (overlap(reinterpret_cast<uintptr_t>(from.data), x.size(-1) * bx, from.stride * bx,
              reinterpret_cast<uintptr_t>(y.const_data_ptr()), n * by, *stride * by, from.count))
    refuse(PyExc_ValueError, "out may not overlap x");
  return y;
}
void want(const char* name, Py_ssize_t got, Py_ssize_t n) {
  if (got == n) return;
  PyErr_Format(PyExc_TypeError, "%s takes %zd arguments (%zd given)", name, n, got);
  throw Bad();
}
PyObject* tensor_or_none(const at::Tensor& t) {
  return t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None);
}

// (weight, group, symmetric, scale_dtype, values) -> (codes, scales, zeros or None, K, C, values or None) or a code
PyObject* quantize_w4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    want("quantize_w4", n, 5);
    const at::Tensor given = any_tensor(a[0], "weight must be a tensor").resolve_neg();
    const long group = integer(a[1], "group must be an int of 32 bits");
    const bool symmetric = truth(a[2]), values = truth(a[4]);
    if (!THPDtype_Check(a[3])) refuse(PyExc_TypeError, "scale_dtype must be a torch dtype");
    const at::ScalarType scale_type = reinterpret_cast<THPDtype*>(a[3])->scalar_type;
    if (scale_type != at::kBFloat16 && scale_type != at::kHalf)
      refuse(PyExc_ValueError, "scale_dtype must be bfloat16 or float16");
    const int code = type_code(given.scalar_type());
    if (!given.is_cuda() || (given.dim() != 2 && given.dim() != 3) || code < 0 || code == WINO_INT8)
      refuse(PyExc_ValueError, "weight must be [K, C] or [E, K, C], float32, bfloat16 or float16, on a CUDA device");
    const c10::cuda::CUDAGuard guard(given.device());
    const at::Tensor w = given.dim() == 2 && given.stride(1) == 1 && given.stride(0) >= given.size(1)
                             ? given : given.contiguous();
    const bool batch = w.dim() == 3;
    const int64_t E = batch ? w.size(0) : 1, K = w.size(-2), C = w.size(-1);
    if (K < 1 || C < 1 || K > (1 << 24) || C > (1 << 24) || wino_packed_scale_count((int32_t)K, (int32_t)C, (int32_t)group) == 0)
      refuse(PyExc_ValueError, "K and C must be 1 to 2^24, group 32, 64 or a multiple of 128");
    const int64_t tK = (K + 15) / 16, tC = (C + 127) / 128, groups = (C + group - 1) / group;
    const c10::DimVector code_shape = batch ? c10::DimVector{E, tK, tC, 16, 4, 16} : c10::DimVector{tK, tC, 16, 4, 16};
    const c10::DimVector scale_shape = batch ? c10::DimVector{E, tK, groups, 16} : c10::DimVector{tK, groups, 16};
    const at::Tensor codes = at::detail::empty_cuda(code_shape, at::kByte, w.device(), std::nullopt);
    const at::Tensor scales = at::detail::empty_cuda(scale_shape, scale_type, w.device(), std::nullopt);
    at::Tensor zeros, back;
    if (!symmetric) zeros = at::detail::empty_cuda(scale_shape, at::kByte, w.device(), std::nullopt);
    if (values) back = at::detail::empty_cuda(w.sizes(), w.scalar_type(), w.device(), std::nullopt);
    const cudaStream_t st = c10::cuda::getCurrentCUDAStream(w.device().index()).stream();
    const int64_t size = w.element_size(), row = K == 1 ? C : w.stride(-2), matrix = tK * tC * 1024, count = tK * groups * 16;
    uint8_t* const to_codes = codes.data_ptr<uint8_t>();
    uint8_t* const to_zeros = symmetric ? nullptr : zeros.data_ptr<uint8_t>();
    char* const to_scales = static_cast<char*>(scales.data_ptr());
    char* const to_values = values ? static_cast<char*>(back.data_ptr()) : nullptr;
    const char* const from = static_cast<const char*>(w.const_data_ptr());
    int rc = WINO_OK;
    Py_BEGIN_ALLOW_THREADS   // a launch may wait for room in the queue
    for (int64_t e = 0; e < E && rc == WINO_OK; ++e) {
      wino_packed_t p;
      p.K = (int32_t)K; p.C = (int32_t)C; p.group = (int32_t)group; p.scale_dtype = type_code(scale_type);
      p.codes_dev = to_codes + e * matrix;
      p.scales_dev = to_scales + e * count * 2;
      p.zeros_dev = symmetric ? nullptr : to_zeros + e * count;
      rc = wino_quantize_weights(&p, from + e * K * C * size, code, row, values ? to_values + e * K * C * size : nullptr, st);
    }
    Py_END_ALLOW_THREADS
    if (rc != WINO_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(NNNLLN)", THPVariable_Wrap(codes), THPVariable_Wrap(scales), tensor_or_none(zeros),
                         (long long)K, (long long)C, tensor_or_none(back));
  } catch (const Bad&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// (x, w, bias or None, q_x or None, q_Y or None, out_dtype or None, out or None) -> y or a code
PyObject* linear_w4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    want("linear_w4", n, 7);
    const at::Tensor& x = any_tensor(a[0], "x must be a tensor");
    wino_linear_desc_t d;
    d.w = packed(a[1], 1, x.device());
    at::Tensor keep;
    d.x_dtype = type_code(x.scalar_type());
    if (d.x_dtype < 0) refuse(PyExc_ValueError, "x must be float32, bfloat16, float16 or int8");
    if ((d.x_dtype == WINO_INT8) != (a[3] != Py_None))
      refuse(PyExc_ValueError, "q_x belongs to int8 inputs, and to those only");
    const c10::OptionalDeviceGuard guard(x.device());
    const Rows r = rows_of(x, d.w.C, keep);
    d.M = (int32_t)r.count; d.x_stride = r.stride;
    d.q_x = quantizer(a[3]); d.q_Y = quantizer(a[4]);
    at::ScalarType type = a[4] != Py_None ? at::kChar : d.x_dtype == WINO_INT8 ? at::kFloat : x.scalar_type();
    if (a[5] != Py_None) {
      if (!THPDtype_Check(a[5])) refuse(PyExc_TypeError, "out_dtype must be a torch dtype");
      type = reinterpret_cast<THPDtype*>(a[5])->scalar_type;
    }
    d.y_dtype = type_code(type);
    if (d.y_dtype < 0) refuse(PyExc_ValueError, "out_dtype must be float32, bfloat16, float16 or int8");
    if ((d.y_dtype == WINO_INT8) != (a[4] != Py_None))
      refuse(PyExc_ValueError, "q_Y belongs to int8 results, and to those only");
    const float* bias = float_vector(a[2], d.w.K, x.device(), "bias must be contiguous float32 [K] on the device of x");
    at::Tensor y = result_like(a[6], x, r, d.w.K, type, &d.y_stride);
    const bool given = a[6] != Py_None;
    if (given)
      apart(y, d.y_stride, r.count, d.w.K,
            {{d.w.codes_dev, code_bytes(d.w)}, {d.w.scales_dev, 2 * scale_count(d.w)}, {d.w.zeros_dev, scale_count(d.w)}, {bias, 4l * d.w.K}});
    if (given) y.unsafeGetTensorImpl()->bump_version();      // autograd sees that y was written
    void* to = y.mutable_data_ptr();
    const cudaStream_t st = c10::cuda::getCurrentCUDAStream(x.device().index()).stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS   // a launch may wait for room in the queue
    rc = wino_linear_forward(&d, r.data, bias, to, st);
    Py_END_ALLOW_THREADS
    if (rc != WINO_OK) return PyLong_FromLong(rc);
    return a[6] != Py_None ? Py_NewRef(a[6]) : THPVariable_Wrap(std::move(y));
  } catch (const Bad&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// (x, router, gate, up, down, top_k, router_bias or None, normalize, out or None) -> (y, ids, weights) or a code
PyObject* experts_w4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    want("experts_w4", n, 9);
    const at::Tensor& x = any_tensor(a[0], "x must be a tensor");
    const at::Tensor& router = tensor(a[1], "router must be a tensor");
    wino_experts_desc_t d;
    if (router.dim() != 2 || router.size(0) < 1 || router.size(1) < 1 || router.size(0) > 512 || router.size(1) > (1 << 24) ||
        !router.is_contiguous() || router.scalar_type() != x.scalar_type() || router.device() != x.device())
      refuse(PyExc_ValueError, "router must be contiguous [E, D], E at most 512, of the type and on the device of x");
    forward_only(router);
    d.E = (int32_t)router.size(0); d.D = (int32_t)router.size(1);
    d.dtype = type_code(x.scalar_type());
    if (d.dtype < 0 || d.dtype == WINO_INT8) refuse(PyExc_ValueError, "x must be float32, bfloat16 or float16");
    d.gate = packed(a[2], d.E, x.device());
    d.up = packed(a[3], d.E, x.device());
    d.down = packed(a[4], d.E, x.device());
    d.I = d.gate.K;
    if (d.gate.C != d.D || d.up.K != d.I || d.up.C != d.D || d.down.K != d.D || d.down.C != d.I)
      refuse(PyExc_ValueError, "gate and up must be [E, I, D], down [E, D, I]");
    if (d.gate.group != d.up.group || d.gate.scale_dtype != d.up.scale_dtype ||
        (d.gate.zeros_dev == nullptr) != (d.up.zeros_dev == nullptr))
      refuse(PyExc_ValueError, "gate and up must have the same group, type of scales, and both zeros or neither");
    const long top_k = integer(a[5], "top_k must be an int");
    if (top_k < 1 || top_k > d.E || top_k > 16) refuse(PyExc_ValueError, "top_k must be 1 to min(E, 16)");
    d.top_k = (int32_t)top_k;
    d.normalize = truth(a[7]) ? 1 : 0;
    const c10::OptionalDeviceGuard guard(x.device());
    at::Tensor keep;
    const Rows r = rows_of(x, d.D, keep);
    d.T = (int32_t)r.count; d.x_stride = r.stride;
    const float* bias = float_vector(a[6], d.E, x.device(), "router_bias must be contiguous float32 [E] on the device of x");
    at::Tensor y = result_like(a[8], x, r, d.D, x.scalar_type(), &d.y_stride);
    const bool given = a[8] != Py_None;
    if (given) {
      apart(y, d.y_stride, r.count, d.D, {{router.const_data_ptr(), router.numel() * router.element_size()}, {bias, 4l * d.E}});
      for (const wino_packed_t* w : {&d.gate, &d.up, &d.down})
        apart(y, d.y_stride, r.count, d.D, {{w->codes_dev, d.E * code_bytes(*w)}, {w->scales_dev, 2 * d.E * scale_count(*w)},
                                            {w->zeros_dev, d.E * scale_count(*w)}});
    }
    c10::DimVector shape(x.sizes().begin(), x.sizes().end());
    shape.back() = top_k;
    at::Tensor ids = at::detail::empty_cuda(shape, at::kInt, x.device(), std::nullopt);
    at::Tensor weights = at::detail::empty_cuda(shape, at::kFloat, x.device(), std::nullopt);
    const int64_t bytes = (int64_t)wino_experts_workspace_bytes(&d);
    const at::Tensor ws = at::detail::empty_cuda({bytes}, at::kByte, x.device(), std::nullopt);
    if (given) y.unsafeGetTensorImpl()->bump_version();      // autograd sees that y was written
    void* to = y.mutable_data_ptr();
    int32_t* to_ids = ids.mutable_data_ptr<int32_t>();
    float* to_weights = weights.mutable_data_ptr<float>();
    void* scratch = ws.mutable_data_ptr();
    const void* from = router.const_data_ptr();
    const cudaStream_t st = c10::cuda::getCurrentCUDAStream(x.device().index()).stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS   // a launch may wait for room in the queue
    rc = wino_experts_forward(&d, r.data, from, bias, to, to_ids, to_weights, scratch, st);
    Py_END_ALLOW_THREADS
    if (rc != WINO_OK) return PyLong_FromLong(rc);
    PyObject* result = a[8] != Py_None ? Py_NewRef(a[8]) : THPVariable_Wrap(std::move(y));
    return Py_BuildValue("(NNN)", result, THPVariable_Wrap(std::move(ids)), THPVariable_Wrap(std::move(weights)));
  } catch (const Bad&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(forward)), METH_FASTCALL, nullptr},
    {"quantize_w4", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(quantize_w4)), METH_FASTCALL, nullptr},
    {"linear_w4", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear_w4)), METH_FASTCALL, nullptr},
    {"experts_w4", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(experts_w4)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native_torch(void) { return PyModule_Create(&module); }
