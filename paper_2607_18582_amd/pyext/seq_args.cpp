// Argument marshalling of the sequence operators (include/mure_seq.h) for
// Python: checks torch tensors, allocates outputs, fills the argument blocks
// and makes the call.  A call on single tokens runs for some 5 us on the GPU;
// the same work done by ctypes takes 14 us on the host, this 5.6.
//
// The library stays free of torch: its entry points come in as addresses
// (bind), and only this module, used by seq.py, knows tensors.
#include <ATen/EmptyTensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/AutogradState.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <string>

#include "../../include/mure_seq.h"

namespace {

decltype(&mure_seq_conv) g_conv = nullptr;
decltype(&mure_seq_scan) g_scan = nullptr;
decltype(&mure_seq_norm) g_norm = nullptr;

struct Raised {};                              // a Python exception is set

[[noreturn]] void raise(PyObject* type, const std::string& msg) {
  PyErr_SetString(type, msg.c_str());
  throw Raised();
}

std::string text(c10::IntArrayRef shape) {
  std::string s = "(";
  for (size_t i = 0; i < shape.size(); ++i) s += (i ? ", " : "") + std::to_string(shape[i]);
  return s + (shape.size() == 1 ? ",)" : ")");
}

std::string type_and_place(const at::Tensor& t) { return std::string(c10::toString(t.scalar_type())) + " on " + t.device().str(); }

const at::Tensor& tensor(PyObject* o, const char* what) {
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

int64_t whole(PyObject* o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return v;
}

int32_t whole32(PyObject* o, const char* what) {
  const int64_t v = whole(o);
  if (v != (int32_t)v) raise(PyExc_ValueError, std::string(what) + " is " + std::to_string(v));
  return (int32_t)v;
}

double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised();
  return v;
}

bool contiguous_from(const at::Tensor& t, int64_t dim) {       // its axes from dim on
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
void written(mure_status st, PyObject* given, const at::Tensor& t) {
  if (st == MURE_OK && THPVariable_Check(given) && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// (status, the first result, the second)
PyObject* answer(mure_status st, PyObject* a, PyObject* b) {
  PyObject* r = Py_BuildValue("(iNN)", (int)st, a, b);
  if (!r) throw Raised();
  return r;
}

PyObject* none() {
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

PyObject* bind(PyObject* const* p) {
  g_conv = address<decltype(g_conv)>(p[0]);
  g_scan = address<decltype(g_scan)>(p[1]);
  g_norm = address<decltype(g_norm)>(p[2]);
  return none();
}

// handle, device, sequences, tokens, x, taps, bias, activation, state, state_out, out
PyObject* conv(PyObject* const* p) {
  mure_seq* seq = address<mure_seq*>(p[0]);
  const int64_t count = whole(p[2]), tokens = whole(p[3]);
  Call c(tensor(p[4], "x"), "x", whole(p[1]));
  mure_seq_conv_args a{};
  a.x = c.in(p[4], "x", tokens, c.width, c.type);
  const at::Tensor& w = tensor(p[5], "taps");
  const int64_t K = w.dim() ? w.size(-1) : 0;
  if (K < 1 || K > INT32_MAX) raise(PyExc_ValueError, "taps has shape " + text(w.sizes()) + "; [channels][taps] is needed");
  std::tie(a.taps, a.taps_mutant_stride) = c.dense(p[5], "taps", {c.width, K}, c.type);
  a.bias = c.param(p[6], "bias");
  a.activation = whole32(p[7], "activation");
  const int64_t held[3] = {count, K - 1, c.width};
  std::tie(a.state, a.state_mutant_stride) = c.dense(p[8], "state", held, c.type);
  const at::Tensor out = c.result(p[10], "out", {tokens, c.width}, c.type), state = c.result(p[9], "state_out", held, c.type);
  std::tie(a.state_out, a.state_out_mutant_stride) = c.out_dense(state, "state_out");
  a.out = c.out(out, "out");
  a.dtype = c.code;
  a.n_mutants = (int32_t)c.mutants;
  a.channels = (int32_t)c.width;
  a.n_taps = (int32_t)K;
  const mure_status st = without_gil([&] { return g_conv(seq, &a); });
  written(st, p[10], out);
  written(st, p[9], state);
  return answer(st, THPVariable_Wrap(out), THPVariable_Wrap(state));
}

// handle, device, sequences, tokens, u, dt, A, B, C, skip, dt_bias, gate, softplus, state, state_out, out
PyObject* scan(PyObject* const* p) {
  mure_seq* seq = address<mure_seq*>(p[0]);
  const int64_t count = whole(p[2]), tokens = whole(p[3]);
  Call c(tensor(p[4], "u"), "u", whole(p[1]));
  const at::Tensor &A = tensor(p[6], "A"), &B = tensor(p[7], "B");
  const int64_t N = A.dim() ? A.size(-1) : 0, cols = B.dim() ? B.size(-1) : 0;
  if (N < 1 || cols % N || cols > INT32_MAX)
    raise(PyExc_ValueError, "B has " + std::to_string(cols) + " columns, no multiple of the " + std::to_string(N) + " states of A");
  mure_seq_scan_args a{};
  a.u = c.in(p[4], "u", tokens, c.width, c.type);
  a.dt = c.in(p[5], "dt", tokens, c.width, c.type);
  a.b = c.in(p[7], "B", tokens, cols, c.type);
  a.c = c.in(p[8], "C", tokens, cols, c.type);
  a.gate = c.in(p[11], "gate", tokens, c.width, c.type);
  const auto ap = c.dense(p[6], "A", {c.width, N}, at::kFloat);
  a.a = {static_cast<const float*>(ap.first), ap.second};
  a.skip = c.param(p[9], "skip");
  a.dt_bias = c.param(p[10], "dt_bias");
  a.softplus = whole32(p[12], "softplus");
  const int64_t held[3] = {count, c.width, N};
  const auto st0 = c.dense(p[13], "state", held, at::kFloat);
  a.state = static_cast<const float*>(st0.first);
  a.state_mutant_stride = st0.second;
  const at::Tensor out = c.result(p[15], "out", {tokens, c.width}, c.type), state = c.result(p[14], "state_out", held, at::kFloat);
  const auto st1 = c.out_dense(state, "state_out");
  a.state_out = static_cast<float*>(st1.first);
  a.state_out_mutant_stride = st1.second;
  a.out = c.out(out, "out");
  a.dtype = c.code;
  a.n_mutants = (int32_t)c.mutants;
  a.channels = (int32_t)c.width;
  a.states = (int32_t)N;
  a.groups = (int32_t)(cols / N);
  const mure_status st = without_gil([&] { return g_scan(seq, &a); });
  written(st, p[15], out);
  written(st, p[14], state);
  return answer(st, THPVariable_Wrap(out), THPVariable_Wrap(state));
}

// context, device, y, residual, gate, gate_at, gate_activation, after, after_weight, after_bias, scale (a tensor, or a
// number), before, before_weight, before_bias, eps, residual_out (False: none), out
PyObject* norm(PyObject* const* p) {
  mure_ctx* ctx = address<mure_ctx*>(p[0]);
  Call c(tensor(p[2], "y"), "y", whole(p[1]));
  mure_seq_norm_args a{};
  at::ScalarType rtype = c.type;
  if (p[3] != Py_None) {
    rtype = tensor(p[3], "residual").scalar_type();
    if (rtype != c.type && rtype != at::kFloat)
      raise(PyExc_TypeError, std::string("residual is ") + c10::toString(rtype) + "; " + c10::toString(c.type) + " or float32 is needed");
  }
  a.y = c.in(p[2], "y", c.rows, c.width, c.type);
  a.residual = c.in(p[3], "residual", c.rows, c.width, rtype);
  a.gate = c.in(p[4], "gate", c.rows, c.width, c.type);
  a.gate_at = p[4] == Py_None ? 0 : whole32(p[5], "gate_at");
  a.gate_activation = whole32(p[6], "gate_activation");
  a.after = whole32(p[7], "after");
  a.after_weight = c.param(p[8], "after_weight");
  a.after_bias = c.param(p[9], "after_bias");
  a.scale_all = 1.f;
  if (THPVariable_Check(p[10])) a.scale = c.param(p[10], "scale");
  else a.scale_all = (float)real(p[10]);
  a.before = whole32(p[11], "before");
  a.before_weight = c.param(p[12], "before_weight");
  a.before_bias = c.param(p[13], "before_bias");
  a.eps = (float)real(p[14]);
  at::Tensor res, out;
  if (p[15] != Py_False) {
    res = c.result(p[15], "residual_out", {c.rows, c.width}, rtype);
    a.residual_out = c.out(res, "residual_out");
  }
  if (a.before) {
    out = c.result(p[16], "out", {c.rows, c.width}, c.type);
    a.out = c.out(out, "out");
  } else if (p[16] != Py_None) {
    raise(PyExc_ValueError, "out needs a `before` norm");
  }
  a.dtype = c.code;
  a.residual_dtype = rtype == at::kFloat ? MURE_F32 : MURE_BF16;
  a.n_mutants = (int32_t)c.mutants;
  a.channels = (int32_t)c.width;
  a.rows = c.rows;
  const mure_status st = without_gil([&] { return g_norm(ctx, &a); });
  written(st, p[16], out);
  written(st, p[15], res);
  return answer(st, res.defined() ? THPVariable_Wrap(res) : none(), out.defined() ? THPVariable_Wrap(out) : none());
}

#define FAST(F, N) {#F, (PyCFunction)(void (*)(void))entry<F, N>, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {FAST(bind, 3), FAST(conv, 11), FAST(scan, 16), FAST(norm, 17), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_seq_args", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__seq_args(void) { return PyModule_Create(&g_module); }
