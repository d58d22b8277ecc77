// The per-call part of the Python binding for the operators that run on a token or a few: argument checks, outputs from torch's
// allocator and the C call, in one extension function each.  From Python through ctypes the same takes 8 to 11 us a call, most of a
// decode step's norm, router or projection; this takes the launch and about 2 us.  Argument marshalling only: the work is libmote's.
//
// Each function returns its output tensors, or the library's status as an int where that is not MOTE_OK; a wrong type, shape, stride or
// device raises ValueError.
#include <Python.h>
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "mote.h"

namespace {

struct Refused { std::string why; };

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw Refused{std::string(name) + ": expected a tensor"};
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.requires_grad() && c10::GradMode::is_enabled())        // its gradient would be lost without a word
    throw Refused{std::string(name) + ": requires grad, and there is no backward pass; call under torch.no_grad() or with a detached tensor"};
  return t;
}

// the library works on the current device and stream
void on_current_device(int64_t device) {
  if (device < 0 || device != c10::cuda::current_device()) throw Refused{"expected tensors on the current CUDA device"};
}

// row stride of a [rows, cols] matrix with unit inner stride
int64_t row_stride(const at::Tensor& t, const char* name, at::ScalarType type, int64_t rows, int64_t cols, int64_t device) {
  if (t.scalar_type() != type || t.dim() != 2 || t.size(0) != rows || t.size(1) != cols || t.layout() != at::kStrided || !t.is_cuda() ||
      t.get_device() != device || (cols > 1 && t.stride(1) != 1))
    throw Refused{std::string(name) + ": expected " + c10::toString(type) + " [" + std::to_string(rows) + ", " + std::to_string(cols) +
                  "] with unit inner stride on cuda:" + std::to_string(device)};
  return rows > 1 ? t.stride(0) : cols;
}
int64_t rows_of(const at::Tensor& t, const char* name) {
  if (t.dim() != 2) throw Refused{std::string(name) + ": expected a matrix"};
  return t.size(0);
}
void* out_pointer(const at::Tensor& t, const char* name, at::ScalarType type, int64_t rows, int64_t cols, int64_t device) {
  if (row_stride(t, name, type, rows, cols, device) != cols) throw Refused{std::string(name) + ": expected contiguous rows"};
  return t.data_ptr();
}

bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw python_error();
  return v != 0;
}

int dtype_code(at::ScalarType t, const char* name) {
  if (t == at::kFloat) return MOTE_DTYPE_F32;
  if (t == at::kBFloat16) return MOTE_DTYPE_BF16;
  throw Refused{std::string(name) + ": expected float32 or bfloat16"};
}

at::Tensor fresh(int64_t rows, int64_t cols, at::ScalarType type, int64_t device) {
  const int64_t size[2] = {rows, cols};
  return at::Tensor(at::detail::empty_cuda(c10::IntArrayRef(size, 2), type, at::Device(at::kCUDA, (c10::DeviceIndex)device), std::nullopt));
}

void* stream_of(int64_t device) { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }

PyObject* wrap_or_none(const at::Tensor& t) {
  if (t.defined()) return THPVariable_Wrap(t);
  Py_RETURN_NONE;
}

template <typename F>
PyObject* guarded(PyObject* const* args, Py_ssize_t n, Py_ssize_t expected, F&& body) {
  HANDLE_TH_ERRORS
  if (n != expected) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return body(args);
  } catch (const Refused& r) {
    PyErr_SetString(PyExc_ValueError, r.why.c_str());
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// route_scored(router, device, x, want_logits) -> (topk_idx, topk_w, logits or None)
PyObject* route_scored(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 4, [](PyObject* const* a) -> PyObject* {
    const auto* R = static_cast<const mote_router_t*>(PyLong_AsVoidPtr(a[0]));
    const int64_t dev = PyLong_AsLongLong(a[1]);
    const at::Tensor& x = tensor(a[2], "x");
    if (const int st = mote_route_scored(R, nullptr, 0, 0, nullptr, nullptr, nullptr, nullptr)) return PyLong_FromLong(st);   // k, ahead of [T, k]
    on_current_device(dev);
    const int64_t T = rows_of(x, "x"), ldx = row_stride(x, "x", at::kBFloat16, T, R->d, dev);
    at::Tensor idx = fresh(T, R->k, at::kInt, dev), w = fresh(T, R->k, at::kFloat, dev), logits;
    if (truth(a[3])) logits = fresh(T, R->E, at::kFloat, dev);
    const int st = mote_route_scored(R, x.data_ptr(), ldx, T, static_cast<int32_t*>(idx.data_ptr()), static_cast<float*>(w.data_ptr()),
                                     logits.defined() ? static_cast<float*>(logits.data_ptr()) : nullptr, stream_of(dev));
    if (st) return PyLong_FromLong(st);
    return Py_BuildValue("(NNN)", THPVariable_Wrap(idx), THPVariable_Wrap(w), wrap_or_none(logits));
  });
}

// block_norm(norm, device of its gains or -1, y, residual, gate, res_out, normed_out, want_residual, want_normed)
//   -> (res_out or None, normed_out or None)
PyObject* block_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 9, [](PyObject* const* a) -> PyObject* {
    mote_block_norm_t N = *static_cast<const mote_block_norm_t*>(PyLong_AsVoidPtr(a[0]));
    const int64_t gains_dev = PyLong_AsLongLong(a[1]), d = N.d;
    const at::Tensor& y = tensor(a[2], "y");
    const int64_t dev = y.is_cuda() ? y.get_device() : -1;
    on_current_device(dev);
    if (gains_dev >= 0 && gains_dev != dev) throw Refused{"the gains are on another device"};
    const int64_t T = rows_of(y, "y"), ldy = row_stride(y, "y", at::kBFloat16, T, d, dev);
    at::ScalarType stream_type = at::kBFloat16;
    const void* res = nullptr;
    int64_t ldr = d;
    if (a[3] != Py_None) {
      const at::Tensor& r = tensor(a[3], "residual");
      stream_type = r.scalar_type();
      N.res_dtype = dtype_code(stream_type, "residual");
      ldr = row_stride(r, "residual", stream_type, T, d, dev);
      res = r.data_ptr();
    } else {
      if (a[5] != Py_None) stream_type = tensor(a[5], "res_out").scalar_type();
      N.res_dtype = dtype_code(stream_type, "res_out");
    }
    const void* gate = nullptr;
    N.gate_cols = 0;
    N.gate_dtype = MOTE_DTYPE_F32;
    if (a[4] != Py_None) {
      const at::Tensor& g = tensor(a[4], "gate");
      const int64_t rows = T == 0 ? 0 : N.gate_tokens == 0 ? 1 : (T - 1) / N.gate_tokens + 1;
      if (g.dim() != 2 || (g.size(1) != 1 && g.size(1) != d) || g.size(0) != rows || !g.is_contiguous() || !g.is_cuda() || g.get_device() != dev)
        throw Refused{"gate: expected contiguous [" + std::to_string(rows) + ", 1] or [" + std::to_string(rows) + ", " + std::to_string(d) + "] on cuda:" +
                      std::to_string(dev)};
      N.gate_dtype = dtype_code(g.scalar_type(), "gate");
      N.gate_cols = (int32_t)g.size(1);
      gate = g.data_ptr();
    }
    at::Tensor made_r, made_n;
    void *r_out = nullptr, *n_out = nullptr;
    if (a[5] != Py_None) r_out = out_pointer(tensor(a[5], "res_out"), "res_out", stream_type, T, d, dev);
    if (a[6] != Py_None) n_out = out_pointer(tensor(a[6], "normed_out"), "normed_out", at::kBFloat16, T, d, dev);
    if (!r_out && a[5] == Py_None && truth(a[7])) { made_r = fresh(T, d, stream_type, dev); r_out = made_r.data_ptr(); }
    if (!n_out && a[6] == Py_None && truth(a[8])) { made_n = fresh(T, d, at::kBFloat16, dev); n_out = made_n.data_ptr(); }
    const int st = mote_block_norm(&N, y.data_ptr(), ldy, res, ldr, gate, T, r_out, n_out, stream_of(dev));
    if (st) return PyLong_FromLong(st);
    auto result = [](PyObject* given, const at::Tensor& made) {
      if (given != Py_None) { Py_INCREF(given); return given; }
      return wrap_or_none(made);
    };
    return Py_BuildValue("(NN)", result(a[5], made_r), result(a[6], made_n));
  });
}

// linear(linear, device, x, residual, out, out_dtype, workspace address, workspace bytes) -> out
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded(args, n, 8, [](PyObject* const* a) -> PyObject* {
    const auto* L = static_cast<const mote_linear_t*>(PyLong_AsVoidPtr(a[0]));
    const int64_t dev = PyLong_AsLongLong(a[1]);
    const at::Tensor& x = tensor(a[2], "x");
    on_current_device(dev);
    const int64_t T = rows_of(x, "x"), ldx = row_stride(x, "x", at::kBFloat16, T, L->K, dev);
    const void* res = nullptr;
    int64_t ldr = L->N;
    if (a[3] != Py_None) {
      const at::Tensor& r = tensor(a[3], "residual");
      ldr = row_stride(r, "residual", at::kBFloat16, T, L->N, dev);
      res = r.data_ptr();
    }
    at::Tensor made;
    void* out;
    int code;
    if (a[4] != Py_None) {
      const at::Tensor& o = tensor(a[4], "out");
      code = dtype_code(o.scalar_type(), "out");
      out = out_pointer(o, "out", o.scalar_type(), T, L->N, dev);
    } else {
      if (!THPDtype_Check(a[5])) throw Refused{"out_dtype: expected a torch.dtype"};
      const at::ScalarType type = reinterpret_cast<THPDtype*>(a[5])->scalar_type;
      code = dtype_code(type, "out_dtype");
      made = fresh(T, L->N, type, dev);
      out = made.data_ptr();
    }
    const int st = mote_linear(L, x.data_ptr(), ldx, T, res, ldr, out, code, PyLong_AsVoidPtr(a[6]), PyLong_AsSize_t(a[7]), stream_of(dev));
    if (st) return PyLong_FromLong(st);
    if (a[4] != Py_None) { Py_INCREF(a[4]); return a[4]; }
    return THPVariable_Wrap(made);
  });
}

PyMethodDef kMethods[] = {
    {"route_scored", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(route_scored)), METH_FASTCALL, nullptr},
    {"block_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(block_norm)), METH_FASTCALL, nullptr},
    {"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(linear)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&kModule); }
