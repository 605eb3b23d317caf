// Argument marshalling of the sequence operators (include/mure_seq.h) for
// Python: checks torch tensors, allocates outputs, fills the argument blocks
// and makes the call.  A call on single tokens runs for some 5 us on the GPU;
// the same work done by ctypes takes 14 us on the host, this 5.6.
//
// The library stays free of torch: its entry points come in as addresses
// (bind), and only this module, used by seq.py, knows tensors.
#include "args.hpp"

using namespace margs;

namespace {

decltype(&mure_seq_conv) g_conv = nullptr;
decltype(&mure_seq_scan) g_scan = nullptr;
decltype(&mure_seq_norm) g_norm = nullptr;

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

PyMethodDef g_methods[] = {FAST(bind, 3), FAST(conv, 11), FAST(scan, 16), FAST(norm, 17), FAST(bind_attn, 3), FAST(rotate, 18), FAST(attend, 14), FAST(gated, 9),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_seq_args", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__seq_args(void) { return PyModule_Create(&g_module); }
