// Argument marshalling of the operators of an attention block
// (include/mure_attn.h) for Python, as in seq_args.cpp.
#include "args.hpp"

#include <cmath>

namespace margs {

namespace {

decltype(&mure_attn_rotate) g_rotate = nullptr;
decltype(&mure_attn_attend) g_attend = nullptr;
decltype(&mure_attn_gated) g_gated = nullptr;

// The heads of a tensor of rows of heads of `dim` channels.
int32_t heads_of(const at::Tensor& t, int64_t dim, const char* what) {
  const int64_t w = t.dim() ? t.size(-1) : 0;
  if (dim < 1 || w < 1 || w % dim) raise(PyExc_ValueError, std::string(what) + " has " + std::to_string(w) + " channels, no multiple of head_dim " + std::to_string(dim));
  return (int32_t)(w / dim);
}

// A contiguous int32 tensor of `shape`, that all mutants share.
const int32_t* counts(const Call& c, PyObject* o, const char* what, c10::IntArrayRef shape) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = c.same_place(o, what, at::kInt);
  if (t.sizes() != shape) raise(PyExc_ValueError, std::string(what) + " has shape " + text(t.sizes()) + "; " + text(shape) + " is needed");
  if (!contiguous_from(t, 0)) raise(PyExc_ValueError, std::string(what) + " must be contiguous");
  return static_cast<const int32_t*>(t.const_data_ptr());
}

mure_seq_param param(Call& c, PyObject* o, const char* what, int64_t n) {
  const auto p = c.dense(o, what, {n}, at::kFloat);
  return {static_cast<const float*>(p.first), p.second};
}

}  // namespace

PyObject* bind_attn(PyObject* const* p) {
  g_rotate = address<decltype(g_rotate)>(p[0]);
  g_attend = address<decltype(g_attend)>(p[1]);
  g_gated = address<decltype(g_gated)>(p[2]);
  return none();
}

// handle, device, sequences, tokens, q, k, frequencies, head_dim, norm, q_weight, k_weight, eps, positions, past, sections (a tuple), interleaved,
// q_out, k_out
PyObject* rotate(PyObject* const* p) {
  mure_seq* seq = address<mure_seq*>(p[0]);
  const int64_t count = whole(p[2]), tokens = whole(p[3]), dim = whole32(p[7], "head_dim");
  Call c(tensor(p[4], "q"), "q", whole(p[1]));
  mure_attn_rotate_args a{};
  a.q_heads = heads_of(c.first, dim, "q");
  a.q = c.in(p[4], "q", tokens, c.width, c.type);
  const bool keys = p[5] != Py_None;
  int64_t kw = 0;
  if (keys) {
    const at::Tensor& k = tensor(p[5], "k");
    a.k_heads = heads_of(k, dim, "k");
    kw = k.size(-1);
    a.k = c.in(p[5], "k", tokens, kw, c.type);
  } else if (p[10] != Py_None || p[17] != Py_None) {
    raise(PyExc_ValueError, "k_weight and k_out need k");
  }
  const at::Tensor& f = tensor(p[6], "frequencies");
  const int64_t pairs = f.dim() ? f.size(-1) : 0;
  if (2 * pairs > dim) raise(PyExc_ValueError, "frequencies are " + std::to_string(pairs) + ", more than the " + std::to_string(dim / 2) + " pairs of a head");
  a.frequencies = param(c, p[6], "frequencies", pairs);
  a.q_weight = param(c, p[9], "q_weight", dim);
  a.k_weight = param(c, p[10], "k_weight", dim);
  if (!PyTuple_Check(p[14])) raise(PyExc_TypeError, "sections must be a list of whole numbers");
  const int64_t axes = PyTuple_GET_SIZE(p[14]);
  if (p[12] != Py_None) {
    if (axes < 1 || axes > MURE_ATTN_MAX_AXES) raise(PyExc_ValueError, "positions have " + std::to_string(axes) + " sections; 1 to " + std::to_string(MURE_ATTN_MAX_AXES) + " are needed");
    a.positions = counts(c, p[12], "positions", {axes, tokens});
    // no tensor memory, but no absence either: a position of nothing
    if (!a.positions && tokens) raise(PyExc_ValueError, "positions have no memory");
    a.axes = (int32_t)axes;
    for (int64_t x = 0; x < axes; ++x) a.section[x] = whole32(PyTuple_GET_ITEM(p[14], x), "a section");
  } else if (axes) {
    raise(PyExc_ValueError, "sections without positions");
  }
  a.past = counts(c, p[13], "past", {count});
  const at::Tensor qo = c.result(p[16], "q_out", {tokens, c.width}, c.type);
  a.q_out = c.out(qo, "q_out");
  at::Tensor ko;
  if (keys) {
    ko = c.result(p[17], "k_out", {tokens, kw}, c.type);
    a.k_out = c.out(ko, "k_out");
  }
  a.dtype = c.code;
  a.n_mutants = (int32_t)c.mutants;
  a.head_dim = (int32_t)dim;
  a.rotated = (int32_t)(2 * pairs);
  a.norm = whole32(p[8], "norm");
  a.interleaved = whole32(p[15], "interleaved");
  a.eps = (float)real(p[11]);
  const mure_status st = without_gil([&] { return g_rotate(seq, &a); });
  written(st, p[16], qo);
  if (keys) written(st, p[17], ko);
  return answer(st, THPVariable_Wrap(qo), keys ? THPVariable_Wrap(ko) : none());
}

// handle, device, sequences, tokens, q, k, v, head_dim, scale, causal, window, (k_cache, v_cache) or None, past, out
PyObject* attend(PyObject* const* p) {
  mure_seq* seq = address<mure_seq*>(p[0]);
  const int64_t count = whole(p[2]), tokens = whole(p[3]), dim = whole32(p[7], "head_dim");
  Call c(tensor(p[4], "q"), "q", whole(p[1]));
  mure_attn_attend_args a{};
  a.heads = heads_of(c.first, dim, "q");
  a.q = c.in(p[4], "q", tokens, c.width, c.type);
  const at::Tensor& k = tensor(p[5], "k");
  a.kv_heads = heads_of(k, dim, "k");
  const int64_t kw = k.size(-1);
  a.k = c.in(p[5], "k", tokens, kw, c.type);
  a.v = c.in(p[6], "v", tokens, kw, c.type);
  const at::Tensor* held[2] = {};
  mure_attn_cache* to[2] = {&a.k_cache, &a.v_cache};
  const char* names[2] = {"the cache of keys", "the cache of values"};
  if (p[11] != Py_None) {
    if (!PyTuple_Check(p[11]) || PyTuple_GET_SIZE(p[11]) != 2) raise(PyExc_TypeError, "cache must be a pair of tensors, of keys and of values");
    for (int i = 0; i < 2; ++i) {
      const at::Tensor& t = c.same_place(PyTuple_GET_ITEM(p[11], i), names[i], c.type);
      if (t.dim() < 3 || t.dim() > 4 || t.size(-3) != count || t.size(-1) != kw || t.size(-2) < 1 || (i && t.size(-2) != held[0]->size(-2)))
        raise(PyExc_ValueError, std::string(names[i]) + " has shape " + text(t.sizes()) + "; [" + std::to_string(count) + " sequences][rows][" + std::to_string(kw) +
                                    "] is needed, or that of each mutant, of keys and values alike");
      if (kw > 1 && t.stride(-1) != 1) raise(PyExc_ValueError, std::string("the last axis of ") + names[i] + " must be contiguous");
      held[i] = &t;
      *to[i] = {t.mutable_data_ptr(), t.dim() == 4 ? c.mutant_axis(t.size(0), t.stride(0), names[i]) : 0, t.stride(-3), t.stride(-2)};
    }
    a.capacity = held[0]->size(-2);
  }
  a.past = counts(c, p[12], "past", {count});
  const at::Tensor out = c.result(p[13], "out", {tokens, c.width}, c.type);
  a.out = c.out(out, "out");
  a.dtype = c.code;
  a.n_mutants = (int32_t)c.mutants;
  a.head_dim = (int32_t)dim;
  a.causal = whole32(p[9], "causal");
  if (p[10] != Py_None) {
    a.window = whole(p[10]);
    if (a.window < 1) raise(PyExc_ValueError, "window is " + std::to_string(a.window) + "; None, or 1 and more is needed");
  }
  a.scale = (float)(p[8] == Py_None ? 1.0 / std::sqrt((double)dim) : real(p[8]));
  const mure_status st = without_gil([&] { return g_attend(seq, &a); });
  written(st, p[13], out);
  for (int i = 0; i < 2 && held[0]; ++i) written(st, PyTuple_GET_ITEM(p[11], i), *held[i]);
  return answer(st, THPVariable_Wrap(out), none());
}

// context, device, x, gate, up, gate_bias, up_bias, activation, out
PyObject* gated(PyObject* const* p) {
  mure_ctx* ctx = address<mure_ctx*>(p[0]);
  Call c(tensor(p[2], "x"), "x", whole(p[1]));
  mure_attn_gated_args a{};
  a.x = c.in(p[2], "x", c.rows, c.width, c.type);
  const at::Tensor& g = tensor(p[3], "gate");
  const int64_t n = g.dim() >= 2 ? g.size(-2) : 0;
  if (n < 1 || n > INT32_MAX) raise(PyExc_ValueError, "gate has shape " + text(g.sizes()) + "; [outputs][inputs] is needed, or that of each mutant");
  a.gate = c.in(p[3], "gate", n, c.width, c.type);
  if (p[4] == Py_None) raise(PyExc_TypeError, "up must be a torch tensor");
  a.up = c.in(p[4], "up", n, c.width, c.type);
  a.gate_bias = param(c, p[5], "gate_bias", n);
  a.up_bias = param(c, p[6], "up_bias", n);
  const at::Tensor out = c.result(p[8], "out", {c.rows, n}, c.type);
  a.out = c.out(out, "out");
  a.dtype = c.code;
  a.n_mutants = (int32_t)c.mutants;
  a.inner = (int32_t)c.width;
  a.outer = (int32_t)n;
  a.rows = c.rows;
  a.activation = whole32(p[7], "activation");
  const mure_status st = without_gil([&] { return g_gated(ctx, &a); });
  written(st, p[8], out);
  return answer(st, THPVariable_Wrap(out), none());
}

}  // namespace margs
