// Python binding of the layers (occ_linear_*, occ_gated_*; in bind_experts.hpp
// those of experts, the router, the exchange and the loss): from tensors to
// the structures of include/optcc.h and one call, in native code, since a call
// of a small layer takes the host longer than the GPU: a forward call of a
// small bf16 layer 3.8 us, a backward call (two launches) 8.1; the same checks
// in Python through ctypes 7.5 and 13.2.
//
// The functions of liboptcc.so are handed over by address (setup), so that
// this module and the rest of the binding use one loaded library.
#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>

#include "optcc.h"

namespace {

typedef occ_status_t (*fwd_fn)(const occ_linear_t*, void*, size_t, occ_stream_t);
typedef occ_status_t (*bwd_fn)(const occ_linear_grad_t*, uint32_t, void*, size_t, occ_stream_t);
typedef size_t (*fwd_size_fn)(const occ_linear_t*);
typedef size_t (*bwd_size_fn)(const occ_linear_grad_t*);

// [0]: linear, [1]: gated
struct {
  fwd_fn fwd[2];
  bwd_fn bwd[2];
  fwd_size_fn fwd_size[2];
  bwd_size_fn bwd_size[2];
  PyObject* stream_of;   // device index -> torch's current stream on it
} lib;

struct Refused {};   // the Python error is set

[[noreturn]] void refuse(PyObject* type, const char* format, const char* name) {
  PyErr_Format(type, format, name);
  throw Refused{};
}

// The tensor, or null for None.
const at::Tensor* tensor(PyObject* o, const char* name) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "%s must be a tensor", name);
  return &THPVariable_Unpack(o);
}

const at::Tensor& matrix(const at::Tensor* t, const char* name) {
  if (!t || t->dim() != 2) refuse(PyExc_ValueError, "%s must be 2-D", name);
  return *t;
}

int32_t layer_type(const at::Tensor& t, const char* name) {
  if (t.scalar_type() == at::kFloat) return OCC_F32;
  if (t.scalar_type() == at::kBFloat16) return OCC_BF16;
  refuse(PyExc_TypeError, "%s must be float32 or bfloat16", name);
}

// An activation's number; one that 32 bits do not hold is none of them.
int32_t activation(PyObject* o) {
  const long act = PyLong_AsLong(o);
  if (PyErr_Occurred()) throw Refused{};
  return act == (int32_t)act ? (int32_t)act : -1;
}

struct Call {
  at::ScalarType dtype;
  at::Device device;

  // Pointer and leading dimension of a rows x cols matrix (null: none is given).
  void* operator()(const at::Tensor* t, const char* name, int64_t rows, int64_t cols, at::ScalarType dt,
                   int64_t& ld) const {
    ld = 0;
    if (!t) return nullptr;
    if (t->scalar_type() != dt) {
      PyErr_Format(PyExc_TypeError, "%s must be %s", name, at::toString(dt));
      throw Refused{};
    }
    if (t->dim() != 2 || t->size(0) != rows || t->size(1) != cols) {
      PyErr_Format(PyExc_ValueError, "%s must be %lld x %lld", name, (long long)rows, (long long)cols);
      throw Refused{};
    }
    if (cols > 1 && t->stride(1) != 1) refuse(PyExc_ValueError, "%s must have unit column stride (row-major)", name);
    if (t->device() != device) refuse(PyExc_ValueError, "%s lies on another device", name);
    ld = rows > 1 ? t->stride(0) : cols;
    return rows ? t->data_ptr() : nullptr;
  }

  void* operator()(const at::Tensor* t, const char* name, int64_t rows, int64_t cols, int64_t& ld) const {
    return (*this)(t, name, rows, cols, dtype, ld);
  }

  float* vector(const at::Tensor* t, const char* name, int64_t n) const {
    if (!t) return nullptr;
    if (t->scalar_type() != at::kFloat) refuse(PyExc_TypeError, "%s must be float32", name);
    if (t->numel() != n || !t->is_contiguous()) {
      PyErr_Format(PyExc_ValueError, "%s must hold %lld contiguous values", name, (long long)n);
      throw Refused{};
    }
    if (t->device() != device) refuse(PyExc_ValueError, "%s lies on another device", name);
    return (float*)t->data_ptr();
  }

  // The caller's workspace: its bytes are counted, so there are no gaps in it.
  const at::Tensor* workspace(const at::Tensor* t, const char* name) const {
    if (!t) return nullptr;
    if (!t->is_contiguous()) refuse(PyExc_ValueError, "%s must be contiguous", name);
    if (t->device() != device) refuse(PyExc_ValueError, "%s lies on another device", name);
    return t;
  }

  occ_stream_t stream() const {
    if (!device.is_cuda()) refuse(PyExc_ValueError, "%s", "the tensors must lie on a GPU");
    PyObject* const index = PyLong_FromLong(device.index());
    PyObject* const s = index ? PyObject_CallOneArg(lib.stream_of, index) : nullptr;
    Py_XDECREF(index);
    if (!s) throw Refused{};
    void* const p = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (PyErr_Occurred()) throw Refused{};
    return (occ_stream_t)p;
  }
};

// The caller's workspace, or a new one that lives until the call has enqueued
// its work (torch's allocator hands it out again in the order of the stream).
struct Workspace {
  at::Tensor own;
  void* p = nullptr;
  size_t bytes = 0;
  Workspace(size_t need, const at::Tensor* given, const at::Device& device) {
    if (!need) return;
    if (given) {
      p = given->data_ptr();
      bytes = (size_t)given->numel() * given->element_size();
      return;
    }
    own = at::empty({(int64_t)need + 256}, at::TensorOptions().dtype(at::kByte).device(device));
    p = (void*)(((uintptr_t)own.data_ptr() + 255) & ~(uintptr_t)255);
    bytes = need;
  }
};

// Torch's errors and the checks' as Python errors.
template <class F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const Refused&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

bool count(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, n);
  return n == want;
}

// forward(gated, X, W, bias, act, R, Y, Z, ws) -> status
PyObject* forward(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!count(n, 9)) return nullptr;
  return guarded([&] {
    const bool gated = v[0] == Py_True;
    const at::Tensor &X = matrix(tensor(v[1], "X"), "X"), &W = matrix(tensor(v[2], "W"), "W");
    const int64_t tokens = X.size(0), in = X.size(1), rows = W.size(0), out = gated ? rows / 2 : rows;
    if (gated && rows % 2) refuse(PyExc_ValueError, "%s must hold the rows of both projections", "W");
    occ_linear_t a;
    a.dtype = layer_type(X, "X");
    a.act = activation(v[4]);
    const Call c{X.scalar_type(), X.device()};
    a.tokens = tokens;
    a.in = in;
    a.out = out;
    a.X = c(&X, "X", tokens, in, a.ldx);
    a.W = c(&W, "W", rows, in, a.ldw);
    a.Y = c(tensor(v[6], "Y"), "Y", tokens, out, a.ldy);
    a.R = c(tensor(v[5], "R"), "R", tokens, out, a.ldr);
    a.Z = c(tensor(v[7], "Z"), "Z", tokens, rows, a.ldz);
    a.bias = c.vector(tensor(v[3], "bias"), "bias", rows);
    const at::Tensor* const given = c.workspace(tensor(v[8], "ws"), "ws");
    const occ_stream_t s = c.stream();
    // a default stream's handle is null: it is the current GPU's
    const c10::DeviceGuard current(c.device);
    const Workspace ws(lib.fwd_size[gated](&a), given, c.device);
    return PyLong_FromLong(lib.fwd[gated](&a, ws.p, ws.bytes, s));
  });
}

// backward(gated, dY, X, W, Z, act, dX, dW, dbias, flags, ws) -> status
PyObject* backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!count(n, 11)) return nullptr;
  return guarded([&]() -> PyObject* {
    const bool gated = v[0] == Py_True;
    const at::Tensor& dY = matrix(tensor(v[1], "dY"), "dY");
    const at::Tensor *X = tensor(v[2], "X"), *W = tensor(v[3], "W"), *Z = tensor(v[4], "Z"), *dX = tensor(v[6], "dX"),
                     *dW = tensor(v[7], "dW"), *dbias = tensor(v[8], "dbias");
    const at::Tensor* const some = X ? X : W ? W : dX ? dX : dW;
    const int64_t tokens = dY.size(0), out = dY.size(1), rows = gated ? 2 * out : out;
    const int64_t in = some ? matrix(some, "X and W").size(1) : 1;
    if (tokens == 0 && dX && !dW && !dbias) return PyLong_FromLong(OCC_OK);   // an empty dX
    occ_linear_grad_t a;
    a.dtype = layer_type(dY, "dY");
    const Call c{dY.scalar_type(), dY.device()};
    const at::ScalarType wide = dW && dW->scalar_type() == at::kFloat ? at::kFloat : c.dtype;
    a.dw_dtype = wide == at::kFloat ? OCC_F32 : OCC_BF16;
    a.act = activation(v[5]);
    const uint32_t flags = (uint32_t)PyLong_AsUnsignedLong(v[9]);
    if (PyErr_Occurred()) throw Refused{};
    a.reserved = 0;
    a.tokens = tokens;
    a.in = in;
    a.out = out;
    a.dY = c(&dY, "dY", tokens, out, a.lddy);
    a.X = c(X, "X", tokens, in, a.ldx);
    a.W = c(W, "W", rows, in, a.ldw);
    a.Z = c(Z, "Z", tokens, rows, a.ldz);
    a.dX = c(dX, "dX", tokens, in, a.lddx);
    a.dW = c(dW, "dW", rows, in, wide, a.lddw);
    a.dbias = c.vector(dbias, "dbias", rows);
    const at::Tensor* const given = c.workspace(tensor(v[10], "ws"), "ws");
    const occ_stream_t s = c.stream();
    // a default stream's handle is null: it is the current GPU's
    const c10::DeviceGuard current(c.device);
    const Workspace ws(lib.bwd_size[gated](&a), given, c.device);
    return PyLong_FromLong(lib.bwd[gated](&a, flags, ws.p, ws.bytes, s));
  });
}

// setup(addresses, stream_of): of the forward, backward and size functions,
// linear then gated
PyObject* setup(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!count(n, 9)) return nullptr;
  void* at[8];
  for (int i = 0; i < 8; ++i) {
    at[i] = PyLong_AsVoidPtr(v[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  for (int g = 0; g < 2; ++g) {
    lib.fwd[g] = (fwd_fn)at[g];
    lib.bwd[g] = (bwd_fn)at[2 + g];
    lib.fwd_size[g] = (fwd_size_fn)at[4 + g];
    lib.bwd_size[g] = (bwd_size_fn)at[6 + g];
  }
  Py_INCREF(v[8]);
  Py_XDECREF(lib.stream_of);
  lib.stream_of = v[8];
  Py_RETURN_NONE;
}

}  // namespace

#include "bind_experts.hpp"

namespace {

#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}

PyMethodDef methods[] = {
    {"forward", (PyCFunction)(void (*)(void))forward, METH_FASTCALL, nullptr},
    {"backward", (PyCFunction)(void (*)(void))backward, METH_FASTCALL, nullptr},
    {"setup", (PyCFunction)(void (*)(void))setup, METH_FASTCALL, nullptr},
    FAST(experts_forward),
    FAST(experts_backward),
    FAST(route_forward),
    FAST(route_backward),
    FAST(dispatch),
    FAST(combine),
    FAST(combine_backward),
    FAST(distill),
    FAST(setup_experts),
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_layers", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layers() { return PyModule_Create(&module); }
