// Calls of the operators whose small sizes the host bounds (queries and keys, the 4-bit ones): one pass over a
// call's tensors (device, type, size, strides) and the call of the C ABI on the current stream.  Nothing is refused
// here: a call that does not fit returns None, and the Python binding goes over it, which names what is wrong or
// runs what is merely unusual (a stream of the caller's, another device than the current one, strides that no
// element uses).  A call takes 3.0 to 3.2 us, of which the launch is 2.7; with the checks in Python and the call by
// ctypes it took 5.0 (quantising), 6.0 (a linear layer) and 7.8 (queries and keys).
#include <Python.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>

#include "ditmi.h"
#include "unlocked.h"

namespace {

// The loaded library's entry points and the binding's structure types, from bind().
struct Library {
  decltype(&dit_linear_fp4) linear_fp4;
  decltype(&dit_quantize_fp4) quantize_fp4;
  decltype(&dit_dequantize_fp4) dequantize_fp4;
  decltype(&dit_qk_norm_rope) qk_norm_rope;
  PyObject *linear_shape, *qk_shape;
} lib;

// What does not fit ends the function; unlocked_call() makes None of it (and of torch's own exceptions, of a tensor
// without memory).
struct Unfit {};
void need(bool ok) {
  if (!ok) throw Unfit();
}

// A call's tensors, all on the first one's device.
struct Tensors {
  int device = -1;

  const at::Tensor& get(PyObject* o) {
    need(THPVariable_CheckExact(o));
    const at::Tensor& t = THPVariable_Unpack(o);
    need(t.is_cuda() && t.layout() == at::kStrided);
    if (device < 0) device = t.get_device();
    need(t.get_device() == device);
    return t;
  }
  // of n elements, contiguous; None is NULL
  void* flat(PyObject* o, at::ScalarType type, int64_t n) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = get(o);
    need(t.scalar_type() == type && t.numel() == n && t.is_contiguous());
    return t.data_ptr();
  }
  // [rows, heads, dh] with the strides row, head, 1; None is NULL
  void* heads(PyObject* o, at::ScalarType type, int64_t rows, int64_t heads, int64_t dh, int64_t row, int64_t head) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = get(o);
    need(t.scalar_type() == type && t.dim() == 3 && t.size(0) == rows && t.size(1) == heads && t.size(2) == dh);
    need(t.stride(0) == row && t.stride(1) == head && t.stride(2) == 1);
    return t.data_ptr();
  }
  // the current stream of their device, which has to be the current one
  void* stream() const {
    need(device >= 0 && c10::hip::current_device() == device);
    return c10::hip::getCurrentHIPStream(device).stream();
  }
};

// What a ctypes structure of that type holds.
template <typename S>
S structure(PyObject* o, PyObject* type) {
  need(lib.linear_fp4 && (PyObject*)Py_TYPE(o) == type);
  Py_buffer view;
  if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) {
    PyErr_Clear();
    throw Unfit();
  }
  S s;
  std::memcpy(&s, view.buf, sizeof(S));
  PyBuffer_Release(&view);
  return s;
}
static_assert(sizeof(dit_linear_shape) == 20 && sizeof(dit_qk_shape) == 160, "the binding's structures");

int64_t panels(int64_t rows, int64_t cols) { return (cols + 255) / 256 * rows * 8; }

at::ScalarType float_type(int32_t dtype) {
  need(dtype == DIT_F32 || dtype == DIT_BF16);
  return dtype == DIT_F32 ? at::kFloat : at::kBFloat16;
}

// (shape, a, a_scale, w, w_scale, out, workspace, bias, out_scale)
auto linear_fp4(PyObject* const* v, Py_ssize_t n) {
  need(n == 9);
  const auto s = structure<dit_linear_shape>(v[0], lib.linear_shape);
  const int64_t M = s.rows, K = s.in, N = s.out;
  need(M >= 0 && K >= 0 && N >= 0);
  const bool f4 = s.dtype == DIT_MXFP4;
  const at::ScalarType type = f4 ? at::kByte : float_type(s.dtype);
  Tensors c;
  void* a = c.flat(v[1], at::kByte, M * K / 2);
  void* a_scale = c.flat(v[2], at::kByte, panels(M, K));
  void* w = c.flat(v[3], at::kByte, N * K / 2);
  void* w_scale = c.flat(v[4], at::kByte, panels(N, K));
  void* out = c.flat(v[5], type, f4 ? M * N / 2 : M * N);
  void* bias = c.flat(v[7], s.dtype == DIT_F32 ? at::kFloat : at::kBFloat16, N);
  void* out_scale = c.flat(v[8], at::kByte, panels(M, N));
  void* space = nullptr;
  size_t bytes = 0;
  if (v[6] != Py_None) {
    const at::Tensor& t = c.get(v[6]);
    need(t.is_contiguous());
    space = t.data_ptr(), bytes = t.nbytes();
  }
  void* stream = c.stream();
  return [=] { return lib.linear_fp4(&s, a, a_scale, w, w_scale, bias, out, out_scale, space, bytes, stream); };
}

// [rows, cols] fp32 or bf16 with contiguous columns
struct Rows {
  int64_t rows, cols, row;
  int32_t dtype;
  void* p;
  Rows(Tensors& c, PyObject* o) {
    const at::Tensor& t = c.get(o);
    need(t.dim() == 2 && t.stride(1) == 1 && (t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16));
    rows = t.size(0), cols = t.size(1), row = rows > 1 ? t.stride(0) : cols;
    need(rows <= INT32_MAX && cols <= INT32_MAX);
    dtype = t.scalar_type() == at::kFloat ? DIT_F32 : DIT_BF16;
    p = t.data_ptr();
  }
};

// (x, codes, scale)
auto quantize_fp4(PyObject* const* v, Py_ssize_t n) {
  need(n == 3 && lib.quantize_fp4);
  Tensors c;
  const Rows x(c, v[0]);
  void* codes = c.flat(v[1], at::kByte, x.rows * x.cols / 2);
  void* scale = c.flat(v[2], at::kByte, panels(x.rows, x.cols));
  void* stream = c.stream();
  return [=] { return lib.quantize_fp4((int32_t)x.rows, (int32_t)x.cols, x.dtype, x.p, x.row, codes, scale, stream); };
}

// (codes, scale, x)
auto dequantize_fp4(PyObject* const* v, Py_ssize_t n) {
  need(n == 3 && lib.dequantize_fp4);
  Tensors c;
  const Rows x(c, v[2]);
  void* codes = c.flat(v[0], at::kByte, x.rows * x.cols / 2);
  void* scale = c.flat(v[1], at::kByte, panels(x.rows, x.cols));
  void* stream = c.stream();
  return [=] { return lib.dequantize_fp4((int32_t)x.rows, (int32_t)x.cols, x.dtype, codes, scale, x.p, x.row, stream); };
}

// (shape, q, k, q_out, k_out, v, v_out, w_q, w_k, pos, freqs, q_dst, k_dst)
auto qk_norm_rope(PyObject* const* v, Py_ssize_t n) {
  need(n == 13);
  const auto s = structure<dit_qk_shape>(v[0], lib.qk_shape);
  const at::ScalarType type = float_type(s.dtype);
  const int64_t R = s.rows, H = s.heads, Hk = s.kv_heads, dh = s.head_dim;
  need(s.axes >= 0 && s.axes <= 4);
  int64_t pairs = 0;
  for (int i = 0; i < s.axes; ++i) pairs += s.pairs[i];
  need((v[1] != Py_None) == (H != 0) && (v[3] != Py_None) == (H != 0));
  need((v[2] != Py_None) == (Hk != 0) && (v[4] != Py_None) == (Hk != 0));
  Tensors c;
  void* q = c.heads(v[1], type, R, H, dh, s.q_row, s.q_head);
  void* k = c.heads(v[2], type, R, Hk, dh, s.k_row, s.k_head);
  void* q_out = c.heads(v[3], type, s.q_out_rows, H, dh, s.q_out_row, s.q_out_head);
  void* k_out = c.heads(v[4], type, s.k_out_rows, Hk, dh, s.k_out_row, s.k_out_head);
  void* x = c.heads(v[5], type, R, Hk, dh, s.v_row, s.v_head);
  void* x_out = c.heads(v[6], type, s.k_out_rows, Hk, dh, s.v_out_row, s.v_out_head);
  const float* w_q = (const float*)c.flat(v[7], at::kFloat, dh);
  const float* w_k = (const float*)c.flat(v[8], at::kFloat, dh);
  const int32_t* pos = (const int32_t*)c.flat(v[9], at::kInt, R * s.axes);
  const double* freqs = (const double*)c.flat(v[10], at::kDouble, pairs);
  const int32_t* q_dst = (const int32_t*)c.flat(v[11], at::kInt, R);
  const int32_t* k_dst = (const int32_t*)c.flat(v[12], at::kInt, R);
  void* stream = c.stream();
  return [=] { return lib.qk_norm_rope(&s, q, k, x, q_out, k_out, x_out, w_q, w_k, pos, freqs, q_dst, k_dst, stream); };
}

// bind(LinearShape, QkShape, addresses of dit_linear_fp4, dit_quantize_fp4, dit_dequantize_fp4, dit_qk_norm_rope)
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 6) return PyErr_Format(PyExc_TypeError, "bind takes two types and four addresses");
  void* p[4];
  for (int i = 0; i < 4; ++i) {
    p[i] = PyLong_AsVoidPtr(v[2 + i]);
    if (PyErr_Occurred()) return nullptr;
  }
  Py_INCREF(v[0]);
  Py_INCREF(v[1]);
  lib = {(decltype(lib.linear_fp4))p[0], (decltype(lib.quantize_fp4))p[1], (decltype(lib.dequantize_fp4))p[2],
         (decltype(lib.qk_norm_rope))p[3], v[0], v[1]};
  Py_RETURN_NONE;
}

#define FUNCTION(name, fn) {name, (PyCFunction)(void*)fn, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FUNCTION("bind", bind),
                         FUNCTION("linear_fp4", unlocked_call<linear_fp4>),
                         FUNCTION("quantize_fp4", unlocked_call<quantize_fp4>),
                         FUNCTION("dequantize_fp4", unlocked_call<dequantize_fp4>),
                         FUNCTION("qk_norm_rope", unlocked_call<qk_norm_rope>),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods};

}  // namespace

// BUILT_FOR: whose tensors the code above reads; the binding uses it beside no other torch or Python
PyMODINIT_FUNC PyInit__marshal(void) {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "BUILT_FOR", DITMI_BUILT_FOR) != 0) Py_CLEAR(m);
  return m;
}
