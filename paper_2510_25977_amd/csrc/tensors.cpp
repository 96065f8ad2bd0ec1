// The binding's checks of torch tensors, and the argument structures of the 8-bit operators made from them.  The smallest calls
// are bound by the host, where a launch alone takes 3.1 us: a norm of six tensors 5.0 in all, 7.8 with the checks in Python.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/svdmlp.h"

namespace {

constexpr int64_t SCALE_BLOCK = 128;
int64_t blocks(int64_t n) { return (n + SCALE_BLOCK - 1) / SCALE_BLOCK; }

struct Refused {};       // the Python error is set

const char* name_of(at::ScalarType t) {
  return t == at::kBFloat16 ? "torch.bfloat16" : t == at::kFloat ? "torch.float32" : "torch.float8_e4m3fn";
}
const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_ValueError, "%s must be a tensor, got %s", what, Py_TYPE(o)->tp_name);
    throw Refused();
  }
  return THPVariable_Unpack(o);
}
[[noreturn]] void refuse(PyObject* o, const char* of, const char* what, int64_t rows, int64_t cols, at::ScalarType type, int64_t device) {
  PyObject* shape = PyObject_GetAttrString(o, "shape");
  PyObject* strides = PyObject_CallMethod(o, "stride", nullptr);
  PyObject* dtype = PyObject_GetAttrString(o, "dtype");
  PyObject* where = PyObject_GetAttrString(o, "device");
  if (shape && strides && dtype && where) {
    char want[64];
    if (rows < 0) snprintf(want, sizeof(want), "(%lld,)", (long long)cols);
    else snprintf(want, sizeof(want), "(%lld, %lld)", (long long)rows, (long long)cols);
    PyErr_Format(PyExc_ValueError, "%s%s must be a %s %s tensor on cuda:%lld whose rows lie in one piece, got %S %S on %S with strides %S",
                 of, what, want, name_of(type), (long long)device, shape, dtype, where, strides);
  }
  Py_XDECREF(shape);
  Py_XDECREF(strides);
  Py_XDECREF(dtype);
  Py_XDECREF(where);
  throw Refused();
}

// A matrix on `device`: rows of consecutive elements, any stride between them.  The stride of a single row says nothing: it is
// taken as the row length, rounded up to `multiple`.
struct Matrix {
  void* ptr = nullptr;
  int64_t ld = 0;
};
Matrix matrix(PyObject* o, const char* what, int64_t rows, int64_t cols, at::ScalarType type, int64_t device, int64_t multiple = 1,
              const char* of = "") {
  const at::Tensor& t = tensor(o, what);
  if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols || t.scalar_type() != type || t.get_device() != device ||
      (t.stride(1) != 1 && cols != 1))
    refuse(o, of, what, rows, cols, type, device);
  return {t.data_ptr(), rows > 1 ? t.stride(0) : (cols + multiple - 1) / multiple * multiple};
}
Matrix codes(PyObject* o, const char* what, int64_t rows, int64_t cols, int64_t device) {
  return matrix(o, what, rows, cols, at::kFloat8_e4m3fn, device, 16);
}
Matrix scales(PyObject* o, const char* what, int64_t rows, int64_t cols, int64_t device) {
  return matrix(o, what, blocks(cols), rows, at::kBFloat16, device, 1, "the scales of ");
}
const float* weight_scales(PyObject* o, const char* what, int64_t rows, int64_t cols, int64_t device) {
  const Matrix m = matrix(o, what, blocks(rows), blocks(cols), at::kFloat, device, 1, "the (contiguous) scales of ");
  if (m.ld != blocks(cols)) refuse(o, "the (contiguous) scales of ", what, blocks(rows), blocks(cols), at::kFloat, device);
  return (const float*)m.ptr;
}
const void* vec(PyObject* o, const char* what, int64_t n, at::ScalarType type, int64_t device) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, what);
  if (t.dim() != 1 || t.size(0) != n || t.scalar_type() != type || t.get_device() != device || (n > 1 && t.stride(0) != 1))
    refuse(o, "", what, -1, n, type, device);
  return t.data_ptr();
}

int32_t type_code(at::ScalarType t) {
  if (t == at::kBFloat16) return SVDMLP_BF16;
  if (t == at::kFloat) return SVDMLP_F32;
  PyErr_SetString(PyExc_ValueError, "inputs must be bfloat16 or float32");
  throw Refused();
}
int64_t integer(PyObject* o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused();
  return v;
}
int32_t small(PyObject* o, const char* what) {
  const int64_t v = integer(o);
  if (v != (int32_t)v) {
    PyErr_Format(PyExc_ValueError, "%s is out of range", what);
    throw Refused();
  }
  return (int32_t)v;
}
float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused();
  return (float)v;
}

// The structure as bytes, None for a call of no rows: tensors of no rows have no address.
template <class A>
PyObject* packed(const A& a, int64_t rows) {
  if (rows == 0) Py_RETURN_NONE;
  return PyBytes_FromStringAndSize((const char*)&a, sizeof(a));
}

using Args = PyObject* const*;

PyObject* quantize_args(Args v) {
  const int64_t device = integer(v[0]);
  const at::Tensor& x = tensor(v[1], "x");
  const at::ScalarType type = x.scalar_type();
  svdmlp_quantize_args a = {};
  a.type = type_code(type);
  if (x.dim() != 2) refuse(v[1], "", "x", 0, 0, type, device);
  a.rows = x.size(0);
  a.cols = x.size(1);
  const Matrix mx = matrix(v[1], "x", a.rows, a.cols, type, device);
  a.x = mx.ptr, a.x_ld = mx.ld;
  if (v[2] != Py_None) {
    const Matrix g = matrix(v[2], "gate_with", a.rows, a.cols, type, device);
    a.gated = g.ptr, a.gated_ld = g.ld;
  }
  a.block_rows = small(v[3], "block_rows");
  const Matrix c = codes(v[4], "out", a.rows, a.cols, device);
  a.codes = c.ptr, a.codes_ld = c.ld;
  if (a.block_rows == 1) {
    const Matrix s = scales(v[5], "out", a.rows, a.cols, device);
    a.scales = s.ptr, a.scales_ld = s.ld;
  } else {
    a.scales = (void*)weight_scales(v[5], "out", a.rows, a.cols, device);
  }
  return packed(a, a.rows);
}

PyObject* norm_args(Args v) {
  const int64_t device = integer(v[0]);
  PyObject *branch = v[1], *residual = v[2], *weight = v[3], *bias = v[4], *branch_scale = v[9], *gate = v[10], *next_weight = v[13],
           *next_bias = v[14], *h = v[17], *out = v[18], *out_scales = v[19];
  const at::Tensor& x = residual != Py_None ? tensor(residual, "residual") : tensor(branch, "branch");
  const at::ScalarType stream = x.scalar_type();
  at::ScalarType type = stream;      // of everything but the residual stream
  for (PyObject* o : {branch, weight, next_weight, bias, next_bias})
    if (o != Py_None) {
      type = tensor(o, "an input").scalar_type();
      break;
    }
  svdmlp_norm_args a = {};
  a.type = a.out_type = type_code(type);
  a.stream_type = type_code(stream);
  if (x.dim() != 2) refuse(residual != Py_None ? residual : branch, "", "x", 0, 0, stream, device);
  const int64_t M = a.rows = x.size(0), d = a.d = x.size(1);
  auto put = [&](PyObject* o, const char* what, int64_t rows, at::ScalarType t, auto& ptr, int64_t& ld) {
    if (o == Py_None) return;
    const Matrix m = matrix(o, what, rows, d, t, device);
    ptr = m.ptr, ld = m.ld;
  };
  put(residual, "residual", M, stream, a.residual, a.residual_ld);
  put(branch, "branch", M, type, a.branch, a.branch_ld);
  put(h, "h", M, stream, a.h, a.h_ld);
  a.weight = vec(weight, "weight", d, type, device);
  a.bias = vec(bias, "bias", d, type, device);
  a.kind = small(v[5], "kind");
  a.eps = real(v[6]);
  a.weight_plus = real(v[7]);
  a.residual_scale = real(v[8]);
  a.branch_scale = vec(branch_scale, "branch_scale", d, type, device);
  a.gate_rows = 1;
  if (gate != Py_None) {
    a.gate_rows = integer(v[11]);
    if (a.gate_rows < 1) {
      PyErr_SetString(PyExc_ValueError, "gate_rows must be at least 1");
      throw Refused();
    }
    put(gate, "gate", M / a.gate_rows + (M % a.gate_rows != 0), type, a.gate, a.gate_ld);
  }
  a.gate_act = small(v[12], "gate_act");
  a.next_weight = vec(next_weight, "next_weight", d, type, device);
  a.next_bias = vec(next_bias, "next_bias", d, type, device);
  a.next_kind = small(v[15], "next_kind");
  a.next_eps = real(v[16]);
  if (out_scales != Py_None) {
    a.out_type = SVDMLP_F8;
    const Matrix c = codes(out, "out", M, d, device), s = scales(out_scales, "out", M, d, device);
    a.out = c.ptr, a.out_ld = c.ld, a.out_scales = s.ptr, a.out_scales_ld = s.ld;
  } else {
    put(out, "out", M, type, a.out, a.out_ld);
  }
  return packed(a, M);
}

PyObject* scaled_matmul_args(Args v) {
  const int64_t device = integer(v[0]);
  svdmlp_scaled_matmul_args a = {};
  const int64_t M = a.M = integer(v[1]), N = a.N = integer(v[2]), K = a.K = integer(v[3]);
  a.gated = small(v[11], "gated");
  const Matrix ca = codes(v[4], "a", M, K, device), sa = scales(v[5], "a", M, K, device), cw = codes(v[6], "w", N, K, device);
  a.a = ca.ptr, a.a_ld = ca.ld, a.a_scales = sa.ptr, a.a_scales_ld = sa.ld, a.w = cw.ptr, a.w_ld = cw.ld;
  a.w_scales = weight_scales(v[7], "w", N, K, device);
  Matrix c;
  if (v[9] != Py_None) {
    a.out_type = SVDMLP_F8;
    c = codes(v[8], "out", M, N, device);
    const Matrix s = scales(v[9], "out", M, N, device);
    a.c_scales = s.ptr, a.c_scales_ld = s.ld;
  } else {
    a.out_type = SVDMLP_BF16;
    c = matrix(v[8], "out", M, N, at::kBFloat16, device);
  }
  a.c = c.ptr, a.c_ld = c.ld;
  if (v[10] != Py_None) {
    const at::Tensor& w = tensor(v[10], "the workspace");
    a.workspace = w.data_ptr();
    a.workspace_bytes = w.nbytes();
  }
  return packed(a, M);
}

template <PyObject* (*F)(Args), Py_ssize_t COUNT>
PyObject* entry(PyObject*, Args v, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != COUNT) return PyErr_Format(PyExc_TypeError, "%zd arguments, expected %zd", n, COUNT);
  try {
    return F(v);
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"quantize_args", (PyCFunction)(void (*)())entry<quantize_args, 6>, METH_FASTCALL,
     "(device, x, gate_with, block_rows, codes, scales) -> svdmlp_quantize_args"},
    {"norm_args", (PyCFunction)(void (*)())entry<norm_args, 20>, METH_FASTCALL,
     "(device, branch, residual, weight, bias, kind, eps, weight_plus, residual_scale, branch_scale, gate, gate_rows, gate_act, "
     "next_weight, next_bias, next_kind, next_eps, h, out, out_scales) -> svdmlp_norm_args"},
    {"scaled_matmul_args", (PyCFunction)(void (*)())entry<scaled_matmul_args, 12>, METH_FASTCALL,
     "(device, M, N, K, a, a_scales, w, w_scales, out, out_scales, workspace, gated) -> svdmlp_scaled_matmul_args"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the Python and torch that this was compiled for, which the binding compares with those it runs on
PyMODINIT_FUNC PyInit__tensors() {
  PyObject* m = PyModule_Create(&module_def);
  if (m && PyModule_AddStringConstant(m, "built_for", BUILT_FOR) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
