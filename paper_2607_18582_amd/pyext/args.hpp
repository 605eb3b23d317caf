// What the marshalling of a call's tensors needs, whichever operator it is:
// checks of torch tensors, outputs, Python's errors.
#pragma once

#include <ATen/EmptyTensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/AutogradState.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <string>

#include "../../include/mure_attn.h"

namespace margs {

struct Raised {};                              // a Python exception is set

[[noreturn]] inline void raise(PyObject* type, const std::string& msg) {
  PyErr_SetString(type, msg.c_str());
  throw Raised();
}

inline std::string text(c10::IntArrayRef shape) {
  std::string s = "(";
  for (size_t i = 0; i < shape.size(); ++i) s += (i ? ", " : "") + std::to_string(shape[i]);
  return s + (shape.size() == 1 ? ",)" : ")");
}

inline std::string type_and_place(const at::Tensor& t) { return std::string(c10::toString(t.scalar_type())) + " on " + t.device().str(); }

inline const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) raise(PyExc_TypeError, std::string(what) + " must be a torch tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.requires_grad() && at::GradMode::is_enabled())
    raise(PyExc_ValueError, std::string(what) + " requires a gradient, which no operator here has: call under torch.no_grad()");
  if (c10::AutogradState::get_tls_state().get_fw_grad_mode() && t._fw_grad(/*level=*/0).defined())
    raise(PyExc_ValueError, std::string(what) + " has a forward tangent, which no operator here carries on");
  if (t.is_neg()) raise(PyExc_ValueError, std::string(what) + " has the negative bit, its memory the other sign: call its resolve_neg()");
  if (t._is_zerotensor()) raise(PyExc_ValueError, std::string(what) + " has no memory (a tensor of zeros of autograd)");
  return t;
}

inline int64_t whole(PyObject* o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return v;
}

inline int32_t whole32(PyObject* o, const char* what) {
  const int64_t v = whole(o);
  if (v != (int32_t)v) raise(PyExc_ValueError, std::string(what) + " is " + std::to_string(v));
  return (int32_t)v;
}

inline double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised();
  return v;
}

inline bool contiguous_from(const at::Tensor& t, int64_t dim) {       // its axes from dim on
  if (t.numel() == 0) return true;
  int64_t n = 1;
  for (int64_t i = t.dim() - 1; i >= dim; --i) {
    if (t.size(i) != 1 && t.stride(i) != n) return false;
    n *= t.size(i);
  }
  return true;
}

// The tensors of one call: their types and places, and the number of mutants.
struct Call {
  const at::Tensor& first;
  at::ScalarType type;
  int32_t code;
  int64_t rows, width, mutants = 1;
  bool axis = false;                           // the results have a mutant axis

  Call(const at::Tensor& t, const char* what, int64_t device) : first(t), type(t.scalar_type()) {
    if (t.is_cuda() ? t.get_device() != device : device >= 0 || !t.is_cpu())
      raise(PyExc_ValueError, std::string(what) + " is on " + t.device().str() + ", the context on device " + std::to_string(device));
    if (type != at::kFloat && type != at::kBFloat16)
      raise(PyExc_TypeError, std::string(what) + " is " + c10::toString(type) + "; float32 or bfloat16 is needed");
    code = type == at::kFloat ? MURE_F32 : MURE_BF16;
    if (t.dim() < 2 || t.dim() > 3 || t.size(-1) > INT32_MAX)
      raise(PyExc_ValueError, std::string(what) + " has shape " + text(t.sizes()) + "; [rows][channels] is needed, or that of each mutant");
    rows = t.size(-2);
    width = t.size(-1);
  }

  const at::Tensor& same_place(PyObject* o, const char* what, at::ScalarType dtype) const {
    const at::Tensor& t = tensor(o, what);
    if (t.scalar_type() != dtype || t.device() != first.device())
      raise(PyExc_TypeError, std::string(what) + " is " + type_and_place(t) + "; " + c10::toString(dtype) + " on " + first.device().str() + " is needed");
    return t;
  }

  int64_t mutant_axis(int64_t n, int64_t stride, const char* what) {
    axis = true;
    if (n == 1) return 0;
    if (n == 0 || n > INT32_MAX || (mutants != 1 && mutants != n))
      raise(PyExc_ValueError, std::string(what) + " has " + std::to_string(n) + " mutants, another argument " + std::to_string(mutants));
    mutants = n;
    return stride;
  }

  [[noreturn]] void wrong_shape(const at::Tensor& t, c10::IntArrayRef shape, const char* what) const {
    raise(PyExc_ValueError, std::string(what) + " has shape " + text(t.sizes()) + "; " + text(shape) + " is needed, or that of each mutant");
  }

  // [n][w] with contiguous rows, or that of each mutant
  mure_seq_in in(PyObject* o, const char* what, int64_t n, int64_t w, at::ScalarType dtype) {
    if (o == Py_None) return {nullptr, 0, 0};
    const at::Tensor& t = same_place(o, what, dtype);
    const int64_t d = t.dim();
    if (d < 2 || d > 3 || t.size(-2) != n || t.size(-1) != w) wrong_shape(t, {n, w}, what);
    if (w > 1 && t.stride(-1) != 1) raise(PyExc_ValueError, std::string("the last axis of ") + what + " must be contiguous");
    const int64_t m = d == 3 ? mutant_axis(t.size(0), t.stride(0), what) : 0;
    return {t.const_data_ptr(), m, t.stride(-2)};
  }

  // contiguous, or that of each mutant: (address, mutant stride)
  std::pair<const void*, int64_t> dense(PyObject* o, const char* what, c10::IntArrayRef shape, at::ScalarType dtype) {
    if (o == Py_None) return {nullptr, 0};
    const at::Tensor& t = same_place(o, what, dtype);
    const int64_t extra = t.dim() - (int64_t)shape.size();
    if (extra < 0 || extra > 1 || t.sizes().slice(extra) != shape) wrong_shape(t, shape, what);
    if (!contiguous_from(t, extra))
      raise(PyExc_ValueError, std::string(what) + " must be contiguous" + (extra ? " for each mutant" : ""));
    const int64_t m = extra ? mutant_axis(t.size(0), t.stride(0), what) : 0;
    return {t.const_data_ptr(), m};
  }

  mure_seq_param param(PyObject* o, const char* what) {
    const auto p = dense(o, what, {width}, at::kFloat);
    return {static_cast<const float*>(p.first), p.second};
  }

  // The result given, checked, or a new one of `shape` for every mutant: from the device's allocator, ahead of the
  // dispatcher, which would add a tenth to a call on single tokens (two results each).
  at::Tensor result(PyObject* o, const char* what, c10::IntArrayRef shape, at::ScalarType dtype) const {
    c10::SmallVector<int64_t, 4> full;
    if (axis) full.push_back(mutants);
    full.append(shape.begin(), shape.end());
    if (o == Py_None)
      return at::Tensor(first.is_cuda() ? at::detail::empty_cuda(full, dtype, first.device(), std::nullopt) : at::detail::empty_cpu(full, dtype));
    const at::Tensor& t = same_place(o, what, dtype);
    if (t.sizes() != c10::IntArrayRef(full))
      raise(PyExc_ValueError, std::string(what) + " has shape " + text(t.sizes()) + "; " + text(full) + " is needed");
    return t;
  }

  mure_seq_out out(const at::Tensor& t, const char* what) const {
    if (t.size(-1) > 1 && t.stride(-1) != 1) raise(PyExc_ValueError, std::string("the last axis of ") + what + " must be contiguous");
    return {t.mutable_data_ptr(), axis ? t.stride(0) : 0, t.stride(-2)};
  }

  std::pair<void*, int64_t> out_dense(const at::Tensor& t, const char* what) const {
    if (!contiguous_from(t, axis)) raise(PyExc_ValueError, std::string(what) + " must be contiguous" + (axis ? " for each mutant" : ""));
    return {t.mutable_data_ptr(), axis ? t.stride(0) : 0};
  }
};

template <typename F> mure_status without_gil(F&& f) {
  mure_status st;
  Py_BEGIN_ALLOW_THREADS st = f();
  Py_END_ALLOW_THREADS return st;
}

// A result's tensor that the caller gave counts as changed, where it keeps count.
inline void written(mure_status st, PyObject* given, const at::Tensor& t) {
  if (st == MURE_OK && THPVariable_Check(given) && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// (status, the first result, the second)
inline PyObject* answer(mure_status st, PyObject* a, PyObject* b) {
  PyObject* r = Py_BuildValue("(iNN)", (int)st, a, b);
  if (!r) throw Raised();
  return r;
}

inline PyObject* none() {
  Py_INCREF(Py_None);
  return Py_None;
}

template <PyObject* (*F)(PyObject* const*), int N> PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  try {
    if (n != N) raise(PyExc_TypeError, "wrong number of arguments");
    return F(args);
  } catch (const Raised&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unexpected error");
  }
  return nullptr;
}

template <typename T> T address(PyObject* o) { return reinterpret_cast<T>((intptr_t)whole(o)); }

#define FAST(F, N) {#F, (PyCFunction)(void (*)(void))entry<F, N>, METH_FASTCALL, nullptr}

// the calls of mure_attn.h (attn_args.cpp), for the module's table
PyObject* bind_attn(PyObject* const* p);
PyObject* rotate(PyObject* const* p);
PyObject* attend(PyObject* const* p);
PyObject* gated(PyObject* const* p);

}  // namespace margs
