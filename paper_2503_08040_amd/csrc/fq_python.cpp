// The calls of a layer's every step (quantize, multiply) without ctypes in between.
//
// A small layer is bound by the host: of the 10.8 us that fq_quantize + fq_gemm took to issue, the runtime's two
// launches are 5.4; the rest was Python reading a tensor's properties one by one, ctypes converting nine
// arguments and torch.empty parsing its own.  Here a call reads them from the tensor itself: 7.8 us.  Only the plain case is
// taken (torch.Tensor itself, the expected types, the current stream): for anything else these functions return
// None and the Python code in front of them, which is the definition of what is accepted and of every error, runs.
// What torch throws here leaves as torch's own Python functions translate it (torch.OutOfMemoryError from the
// output's allocation, a Python exception from a dispatch mode).
#include <Python.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ops/empty.h>
#include <algorithm>

#include "../../include/fq.h"

namespace {

typedef fq_status (*QuantizeFn)(const void*, int32_t, int32_t, int64_t, int32_t, fq_criterion, float, fq_qtensor*, void*);
typedef fq_status (*QuantizeSrFn)(const void*, int32_t, int32_t, int64_t, int32_t, uint64_t, fq_qtensor*, void*);
typedef fq_status (*GemmFn)(fq_op, const fq_qtensor*, const fq_qtensor*, void*, fq_out_dtype, int64_t, void*);

typedef fq_status (*MxQuantizeFn)(const void*, int32_t, int32_t, int64_t, fq_mx_rule, fq_mx_tensor*, void*);
typedef fq_status (*MxQuantizeSrFn)(const void*, int32_t, int32_t, int64_t, uint64_t, fq_mx_tensor*, void*);
typedef fq_status (*MxDequantizeFn)(const fq_mx_tensor*, int32_t, void*, fq_out_dtype, int64_t, void*);
typedef fq_status (*MxGemmFn)(fq_op, const fq_mx_tensor*, const fq_mx_tensor*, void*, fq_out_dtype, int64_t, void*);
typedef fq_status (*MxLinearFn)(const void*, int32_t, int64_t, fq_mx_rule, const fq_mx_tensor*, fq_mx_tensor*, void*,
                                fq_out_dtype, int64_t, void*);

QuantizeFn g_quantize;
QuantizeSrFn g_quantize_sr;
GemmFn g_gemm;
MxQuantizeFn g_mx_quantize;
MxQuantizeSrFn g_mx_quantize_sr;
MxDequantizeFn g_mx_dequantize;
MxGemmFn g_mx_gemm;
MxLinearFn g_mx_linear;
PyObject *g_device, *g_stream;       // torch's current device, and the raw handle of a device's current stream

// setup(address of fq_quantize, of fq_quantize_sr, of fq_gemm, current device, raw stream): the loaded library's
PyObject* setup(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 5) return PyErr_Format(PyExc_TypeError, "setup takes 5 arguments");
  void* p[3];
  for (int i = 0; i < 3; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  g_quantize = reinterpret_cast<QuantizeFn>(p[0]);
  g_quantize_sr = reinterpret_cast<QuantizeSrFn>(p[1]);
  g_gemm = reinterpret_cast<GemmFn>(p[2]);
  Py_INCREF(a[3]);
  Py_INCREF(a[4]);
  Py_XSETREF(g_device, a[3]);
  Py_XSETREF(g_stream, a[4]);
  Py_RETURN_NONE;
}

// setup_mx(addresses of fq_mx_quantize, fq_mx_quantize_sr, fq_mx_dequantize, fq_mx_gemm, fq_mx_linear), behind setup
PyObject* setup_mx(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 5) return PyErr_Format(PyExc_TypeError, "setup_mx takes 5 arguments");
  void* p[5];
  for (int i = 0; i < 5; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  g_mx_quantize = reinterpret_cast<MxQuantizeFn>(p[0]);
  g_mx_quantize_sr = reinterpret_cast<MxQuantizeSrFn>(p[1]);
  g_mx_dequantize = reinterpret_cast<MxDequantizeFn>(p[2]);
  g_mx_gemm = reinterpret_cast<MxGemmFn>(p[3]);
  g_mx_linear = reinterpret_cast<MxLinearFn>(p[4]);
  Py_RETURN_NONE;
}

bool current_stream(void** out, long* device = nullptr) {
  PyObject* dev = PyObject_CallNoArgs(g_device);
  if (!dev) return false;
  if (device) *device = PyLong_AsLong(dev);
  PyObject* s = PyObject_CallOneArg(g_stream, dev);
  Py_DECREF(dev);
  if (!s) return false;
  *out = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  return !PyErr_Occurred();
}

struct Matrix {
  void* ptr;
  int32_t rows, cols;
  int64_t ld;
  int device;
};

// A bf16 matrix on the GPU with unit column stride.
bool matrix(PyObject* o, Matrix* m) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.layout() != at::kStrided || t.dim() != 2 || t.scalar_type() != at::kBFloat16) return false;
  const int64_t rows = t.size(0), cols = t.size(1);
  if (rows > INT32_MAX || cols > INT32_MAX || (t.stride(1) != 1 && cols > 1)) return false;
  *m = {t.data_ptr(), (int32_t)rows, (int32_t)cols, rows > 1 ? t.stride(0) : std::max<int64_t>(cols, 1),
        (int)t.get_device()};
  return true;
}

bool int_arg(PyObject* o, long* v) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  *v = PyLong_AsLongAndOverflow(o, &over);
  return !over && *v >= INT32_MIN && *v <= INT32_MAX;
}

// call() while other Python threads run.
template <class F>
auto without_gil(const F& call) {
  pybind11::gil_scoped_release others;
  return call();
}

template <class F>
PyObject* launch(const F& call) {
  return PyLong_FromLong(without_gil(call));
}

// quantize(x, crit, theta, address of the fq_qtensor, block) -> status or None
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Matrix m;
  long crit, block;
  if (n != 5 || !PyFloat_CheckExact(a[2]) || !int_arg(a[1], &crit) || !int_arg(a[4], &block) || !matrix(a[0], &m))
    Py_RETURN_NONE;
  const float theta = (float)PyFloat_AS_DOUBLE(a[2]);
  fq_qtensor* const q = static_cast<fq_qtensor*>(PyLong_AsVoidPtr(a[3]));
  void* st;
  if (PyErr_Occurred() || !current_stream(&st)) return nullptr;
  return launch([&] { return g_quantize(m.ptr, m.rows, m.cols, m.ld, (int32_t)block, (fq_criterion)crit, theta, q, st); });
  END_HANDLE_TH_ERRORS
}

// quantize_sr(x, seed, address of the fq_qtensor) -> status or None
PyObject* quantize_sr(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Matrix m;
  if (n != 3 || !PyLong_CheckExact(a[1]) || !matrix(a[0], &m)) Py_RETURN_NONE;
  const uint64_t seed = PyLong_AsUnsignedLongLongMask(a[1]);
  fq_qtensor* const q = static_cast<fq_qtensor*>(PyLong_AsVoidPtr(a[2]));
  void* st;
  if (PyErr_Occurred() || !current_stream(&st)) return nullptr;
  return launch([&] { return g_quantize_sr(m.ptr, m.rows, m.cols, m.ld, FQ_BLOCK, seed, q, st); });
  END_HANDLE_TH_ERRORS
}

struct Output {
  at::Tensor t;
  fq_out_dtype type;
  int64_t ld;
};

enum Taken { kTaken, kNotTaken };

// A rows x cols output of type `type` unless dtype says another, on the device of `like`; or `given` if it fits.
Taken output(PyObject* given, PyObject* dtype, int64_t rows, int64_t cols, at::ScalarType type, const at::Tensor& like,
             Output* o) {
  o->ld = std::max<int64_t>(cols, 1);
  if (given == Py_None) {
    if (dtype != Py_None) {
      if (!THPDtype_Check(dtype)) return kNotTaken;
      type = reinterpret_cast<THPDtype*>(dtype)->scalar_type;
    }
    if (type != at::kFloat && type != at::kBFloat16) return kNotTaken;
    // a mode that sees torch's functions sees torch.empty of the Python code
    if (at::impl::torch_function_mode_enabled()) return kNotTaken;
    const at::TensorOptions options = like.options().dtype(type);
    o->t = without_gil([&] { return at::empty({rows, cols}, options); });     // may wait for the device or the driver
  } else {
    if (!THPVariable_CheckExact(given)) return kNotTaken;
    o->t = THPVariable_Unpack(given);
    type = o->t.scalar_type();
    if (!o->t.is_cuda() || (type != at::kFloat && type != at::kBFloat16) || o->t.layout() != at::kStrided ||
        o->t.dim() != 2 || o->t.size(0) != rows || o->t.size(1) != cols || (o->t.stride(1) != 1 && cols > 1))
      return kNotTaken;
    if (rows > 1) o->ld = o->t.stride(0);
  }
  o->type = type == at::kFloat ? FQ_OUT_F32 : FQ_OUT_BF16;
  return kTaken;
}

// call() -> (status, the output)
template <class F>
PyObject* launch_into(const Output& o, PyObject* given, const F& call) {
  PyObject* status = launch(call);
  if (!status) return nullptr;
  PyObject* t = given == Py_None ? THPVariable_Wrap(o.t) : Py_NewRef(given);
  if (!t) {
    Py_DECREF(status);
    return nullptr;
  }
  PyObject* r = PyTuple_Pack(2, status, t);
  Py_DECREF(status);
  Py_DECREF(t);
  return r;
}

// gemm(op, address of A's fq_qtensor, of B's, a tensor on the output's device, out or None, dtype or None)
// -> (status, out) or None
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  long op;
  if (n != 6 || !int_arg(a[0], &op) || !THPVariable_CheckExact(a[3])) Py_RETURN_NONE;
  const fq_qtensor* const A = static_cast<fq_qtensor*>(PyLong_AsVoidPtr(a[1]));
  const fq_qtensor* const B = static_cast<fq_qtensor*>(PyLong_AsVoidPtr(a[2]));
  if (PyErr_Occurred()) return nullptr;
  int64_t rows, cols;
  switch (op) {
    case FQ_OP_NT: rows = A->rows; cols = B->rows; break;
    case FQ_OP_NN: rows = A->rows; cols = B->cols; break;
    case FQ_OP_TN: rows = A->cols; cols = B->cols; break;
    default: Py_RETURN_NONE;
  }
  Output o;
  if (output(a[4], a[5], rows, cols, at::kFloat, THPVariable_Unpack(a[3]), &o) != kTaken) Py_RETURN_NONE;
  void* st;
  if (!current_stream(&st)) return nullptr;
  void* const c = o.t.data_ptr();
  return launch_into(o, a[4], [&] { return g_gemm((fq_op)op, A, B, c, o.type, o.ld, st); });
  END_HANDLE_TH_ERRORS
}

// ---- microscaled matrices.  A call whose tensors are not all on the current device is left to the Python code too,
// which refuses it.

bool on_device(PyObject* o, long device) {
  return THPVariable_CheckExact(o) && THPVariable_Unpack(o).is_cuda() && THPVariable_Unpack(o).get_device() == device;
}

// mx_quantize(x, rule, address of the fq_mx_tensor, its storage) -> status or None
PyObject* mx_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Matrix m;
  long rule, device;
  if (n != 4 || !int_arg(a[1], &rule) || !matrix(a[0], &m)) Py_RETURN_NONE;
  fq_mx_tensor* const q = static_cast<fq_mx_tensor*>(PyLong_AsVoidPtr(a[2]));
  void* st;
  if (PyErr_Occurred() || !current_stream(&st, &device)) return nullptr;
  if (m.device != device || !on_device(a[3], device)) Py_RETURN_NONE;
  return launch([&] { return g_mx_quantize(m.ptr, m.rows, m.cols, m.ld, (fq_mx_rule)rule, q, st); });
  END_HANDLE_TH_ERRORS
}

// mx_quantize_sr(x, seed, address of the fq_mx_tensor, its storage) -> status or None
PyObject* mx_quantize_sr(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Matrix m;
  long device;
  if (n != 4 || !PyLong_CheckExact(a[1]) || !matrix(a[0], &m)) Py_RETURN_NONE;
  const uint64_t seed = PyLong_AsUnsignedLongLongMask(a[1]);
  fq_mx_tensor* const q = static_cast<fq_mx_tensor*>(PyLong_AsVoidPtr(a[2]));
  void* st;
  if (PyErr_Occurred() || !current_stream(&st, &device)) return nullptr;
  if (m.device != device || !on_device(a[3], device)) Py_RETURN_NONE;
  return launch([&] { return g_mx_quantize_sr(m.ptr, m.rows, m.cols, m.ld, seed, q, st); });
  END_HANDLE_TH_ERRORS
}

// mx_dequantize(address of the fq_mx_tensor, its storage, side, out or None, dtype or None) -> (status, out) or None
PyObject* mx_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  long side, device;
  if (n != 5 || !int_arg(a[2], &side) || !THPVariable_CheckExact(a[1])) Py_RETURN_NONE;
  const fq_mx_tensor* const q = static_cast<fq_mx_tensor*>(PyLong_AsVoidPtr(a[0]));
  void* st;
  if (PyErr_Occurred() || !current_stream(&st, &device)) return nullptr;
  Output o;
  if (!on_device(a[1], device) ||
      output(a[3], a[4], q->rows, q->cols, at::kBFloat16, THPVariable_Unpack(a[1]), &o) != kTaken ||
      o.t.get_device() != device)
    Py_RETURN_NONE;
  void* const c = o.t.data_ptr();
  return launch_into(o, a[3], [&] { return g_mx_dequantize(q, (int32_t)side, c, o.type, o.ld, st); });
  END_HANDLE_TH_ERRORS
}

// mx_gemm(op, address of A's fq_mx_tensor, of B's, their storages, out or None, dtype or None) -> (status, out) or None
PyObject* mx_gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  long op, device;
  if (n != 7 || !int_arg(a[0], &op) || !THPVariable_CheckExact(a[3])) Py_RETURN_NONE;
  const fq_mx_tensor* const A = static_cast<fq_mx_tensor*>(PyLong_AsVoidPtr(a[1]));
  const fq_mx_tensor* const B = static_cast<fq_mx_tensor*>(PyLong_AsVoidPtr(a[2]));
  void* st;
  if (PyErr_Occurred() || !current_stream(&st, &device)) return nullptr;
  int64_t rows, cols;
  switch (op) {
    case FQ_OP_NT: rows = A->rows; cols = B->rows; break;
    case FQ_OP_NN: rows = A->rows; cols = B->cols; break;
    case FQ_OP_TN: rows = A->cols; cols = B->cols; break;
    default: Py_RETURN_NONE;
  }
  Output o;
  if (!on_device(a[3], device) || !on_device(a[4], device) ||
      output(a[5], a[6], rows, cols, at::kFloat, THPVariable_Unpack(a[3]), &o) != kTaken || o.t.get_device() != device)
    Py_RETURN_NONE;
  void* const c = o.t.data_ptr();
  return launch_into(o, a[5], [&] { return g_mx_gemm((fq_op)op, A, B, c, o.type, o.ld, st); });
  END_HANDLE_TH_ERRORS
}

// mx_linear(x, address of W's fq_mx_tensor, its storage, address of xq's or 0, its storage or None, rule, out or None,
// dtype or None) -> (status, out) or None
PyObject* mx_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Matrix m;
  long rule, device;
  if (n != 8 || !int_arg(a[5], &rule) || !matrix(a[0], &m)) Py_RETURN_NONE;
  const fq_mx_tensor* const W = static_cast<fq_mx_tensor*>(PyLong_AsVoidPtr(a[1]));
  fq_mx_tensor* const xq = static_cast<fq_mx_tensor*>(PyLong_AsVoidPtr(a[3]));
  void* st;
  if (PyErr_Occurred() || !current_stream(&st, &device)) return nullptr;
  Output o;
  if (m.device != device || m.cols != W->cols || (!xq && m.rows > FQ_MX_LINEAR_ROWS) || !on_device(a[2], device) ||
      (xq && !on_device(a[4], device)) ||
      output(a[6], a[7], m.rows, W->rows, at::kFloat, THPVariable_Unpack(a[0]), &o) != kTaken || o.t.get_device() != device)
    Py_RETURN_NONE;
  void* const c = o.t.data_ptr();
  return launch_into(o, a[6], [&] {
    return g_mx_linear(m.ptr, m.rows, m.ld, (fq_mx_rule)rule, W, xq, c, o.type, o.ld, st);
  });
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"setup", reinterpret_cast<PyCFunction>(setup), METH_FASTCALL, nullptr},
    {"quantize", reinterpret_cast<PyCFunction>(quantize), METH_FASTCALL, nullptr},
    {"quantize_sr", reinterpret_cast<PyCFunction>(quantize_sr), METH_FASTCALL, nullptr},
    {"gemm", reinterpret_cast<PyCFunction>(gemm), METH_FASTCALL, nullptr},
    {"setup_mx", reinterpret_cast<PyCFunction>(setup_mx), METH_FASTCALL, nullptr},
    {"mx_quantize", reinterpret_cast<PyCFunction>(mx_quantize), METH_FASTCALL, nullptr},
    {"mx_quantize_sr", reinterpret_cast<PyCFunction>(mx_quantize_sr), METH_FASTCALL, nullptr},
    {"mx_dequantize", reinterpret_cast<PyCFunction>(mx_dequantize), METH_FASTCALL, nullptr},
    {"mx_gemm", reinterpret_cast<PyCFunction>(mx_gemm), METH_FASTCALL, nullptr},
    {"mx_linear", reinterpret_cast<PyCFunction>(mx_linear), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fqnative", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fqnative() {
  PyObject* m = PyModule_Create(&module);
  if (m) {
    PyModule_AddStringConstant(m, "torch_version", FQ_TORCH_VERSION);
    PyModule_AddStringConstant(m, "header_tag", FQ_HEADER_TAG);      // of fq.h: the structs read and the entry points called
  }
  return m;
}
