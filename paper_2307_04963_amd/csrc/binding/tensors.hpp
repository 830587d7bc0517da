// What the Python entry points share: arguments taken one after the other, checks
// of tensors, outputs and workspaces on the current stream, errors.
#pragma once

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/AutogradState.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <string>

#include "../../../include/dycl_decode.h"

// the decoding operators' functions (decode.cpp), ended by a null entry
PyMethodDef* decode_methods();

namespace binding {

struct Refused {                       // a Python exception is set
};

[[noreturn]] inline void refuse(const std::string& what) {
  PyErr_SetString(PyExc_ValueError, what.c_str());
  throw Refused{};
}

inline PyObject*& error_type() {        // DyclError(code, message)
  static PyObject* type = nullptr;
  return type;
}

inline void check(int rc) {
  if (rc >= 0) return;
  PyObject* e = error_type() ? PyObject_CallFunction(error_type(), "is", rc, dycl_last_error()) : nullptr;
  if (e) {
    PyErr_SetObject(error_type(), e);
    Py_DECREF(e);
  } else if (!PyErr_Occurred()) {
    PyErr_SetString(PyExc_RuntimeError, dycl_last_error());
  }
  throw Refused{};
}

// The arguments of one call, taken one after the other.
struct Args {
  PyObject* const* a;
  Py_ssize_t left;
  Args(PyObject* const* args, Py_ssize_t n, Py_ssize_t want) : a(args), left(n) {
    if (n != want) {
      PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
      throw Refused{};
    }
  }
  PyObject* next() {
    --left;
    return *a++;
  }
  // a tensor or (if allowed) None
  const at::Tensor* tensor(const char* what, bool optional = true) {
    PyObject* o = next();
    if (optional && o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) refuse(std::string(what) + " must be a tensor" + (optional ? " or None" : ""));
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.requires_grad() && c10::GradMode::is_enabled())
      refuse(std::string(what) + " requires grad, and these operators record no gradients: call them under torch.no_grad(), or detach it");
    if (c10::AutogradState::get_tls_state().get_fw_grad_mode() && t._fw_grad(0).defined())
      refuse(std::string(what) + " carries a forward-mode tangent, which these operators would drop: give them forward_ad.unpack_dual(...).primal");
    return &t;
  }
  long integer() {
    const long v = PyLong_AsLong(next());
    if (v == -1 && PyErr_Occurred()) throw Refused{};
    return v;
  }
  int small(const char* what) {
    const long v = integer();
    if (v < INT32_MIN || v > INT32_MAX) refuse(std::string(what) + " out of range");
    return static_cast<int>(v);
  }
  float real() {
    const double v = PyFloat_AsDouble(next());
    if (v == -1.0 && PyErr_Occurred()) throw Refused{};
    return static_cast<float>(v);
  }
};

inline std::string sizes(int64_t rows, int64_t cols) { return "[" + std::to_string(rows) + ", " + std::to_string(cols) + "]"; }

inline bool either(const at::Tensor& t) { return t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kFloat; }
inline int type_of(const at::Tensor& t) { return t.scalar_type() == at::kFloat ? DYCL_F32 : DYCL_BF16; }

inline void input(const at::Tensor& t, const char* what) {
  if (t.dim() != 2) refuse(std::string(what) + " must be a 2-D tensor");
  if (!t.is_cuda()) refuse(std::string(what) + " must be on a GPU");
}

// a matrix's row pitch; rows may be strided, their values not
inline int64_t matrix(const at::Tensor& t, const char* what, int64_t rows, int64_t cols, const at::Device& dev) {
  if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols) refuse(std::string(what) + " must be " + sizes(rows, cols));
  if (!either(t)) refuse(std::string(what) + " must be bfloat16 or float32");
  if (t.device() != dev) refuse(std::string(what) + " is on another device");
  if (cols > 1 && t.stride(1) != 1) refuse(std::string(what) + ": the last dimension must be contiguous");
  if (rows <= 1) return std::max<int64_t>(cols, t.stride(0));
  if (t.stride(0) < cols) refuse(std::string(what) + ": rows overlap");
  return t.stride(0);
}

inline int64_t bf16_matrix(const at::Tensor& t, const char* what, int64_t rows, int64_t cols, const at::Device& dev) {
  const int64_t ld = matrix(t, what, rows, cols, dev);
  if (t.scalar_type() != at::kBFloat16) refuse(std::string(what) + " must be bfloat16");
  return ld;
}

template <class T>
T* vector(const at::Tensor* t, const char* what, at::IntArrayRef shape, at::ScalarType dtype, const at::Device& dev) {
  if (!t) return nullptr;
  if (t->sizes() != shape || t->scalar_type() != dtype || !t->is_contiguous() || t->device() != dev)
    refuse(std::string(what) + ": wrong shape, type or device, or not contiguous");
  return static_cast<T*>(t->data_ptr());
}

inline const float* floats(const at::Tensor* t, const char* what, at::IntArrayRef shape, const at::Device& dev) {
  return vector<float>(t, what, shape, at::kFloat, dev);
}

inline at::Tensor make(at::IntArrayRef shape, at::ScalarType dtype, const at::Device& dev) {
  return at::detail::empty_cuda(shape, dtype, dev, std::nullopt);
}

// the caller's workspace, or one of `bytes` in `own`; null where none is needed
inline void* workspace_of(const at::Tensor* given, bool automatic, size_t bytes, const at::Device& dev, at::Tensor& own, size_t& have) {
  have = 0;
  if (!bytes) return nullptr;
  if (automatic) {
    own = make({static_cast<int64_t>(bytes)}, at::kByte, dev);
    have = bytes;
    return own.data_ptr();
  }
  if (!given || given->device() != dev || !given->is_contiguous())
    refuse("needs a contiguous workspace of " + std::to_string(bytes) + " bytes on the inputs' device");
  have = given->nbytes();
  return given->data_ptr();
}

inline void* stream_of(const at::Device& dev) { return c10::hip::getCurrentHIPStream(dev.index()).stream(); }

inline void* pointer(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

inline PyObject* wrap(const at::Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None); }

inline PyObject* tuple(std::initializer_list<at::Tensor> ts) {
  PyObject* r = PyTuple_New(static_cast<Py_ssize_t>(ts.size()));
  Py_ssize_t i = 0;
  for (const at::Tensor& t : ts) PyTuple_SET_ITEM(r, i++, wrap(t));
  return r;
}

template <class F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const Refused&) {
    return nullptr;
  } catch (const c10::OutOfMemoryError& e) {
    PyErr_SetString(PyExc_MemoryError, e.what_without_backtrace());
  } catch (const c10::Error& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown failure");
  }
  return nullptr;
}

inline uint16_t* bits(const at::Tensor* t) { return t ? static_cast<uint16_t*>(t->data_ptr()) : nullptr; }

}  // namespace binding
