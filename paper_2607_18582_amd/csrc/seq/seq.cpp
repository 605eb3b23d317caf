// C ABI of the sequence operators (mure_seq.h): batches, checks of arguments,
// workspaces and launches.
#include "seq.hpp"
#include "workspace.hpp"

#include <algorithm>
#include <cmath>
#include <exception>
#include <memory>
#include <new>
#include <vector>

using namespace mure;

namespace {

typedef __int128 wide;

struct Fail {
  mure_status st;
  std::string msg;
};

[[noreturn]] void invalid(const std::string& m) { throw Fail{MURE_E_INVALID, m}; }

void check(hipError_t e, const char* what) {
  if (e == hipSuccess) return;
  (void)hipGetLastError();                     // reported here: not again by a later launch
  throw Fail{e == hipErrorOutOfMemory ? MURE_E_NOMEM : MURE_E_DEVICE, std::string(what) + ": " + hipGetErrorString(e)};
}

// Allocations and frees are no part of a capture, of this stream or another one.
struct Relaxed {
  hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;
  Relaxed() { (void)hipThreadExchangeStreamCaptureMode(&mode); }
  ~Relaxed() { (void)hipThreadExchangeStreamCaptureMode(&mode); }
};

struct Api {
  static hipError_t alloc(void** p, size_t n) {
    Relaxed relaxed;
    const hipError_t e = hipMalloc(p, n);
    if (e != hipSuccess) (void)hipGetLastError();        // less may be asked for next
    return e;
  }
  static void free(void* p) {
    Relaxed relaxed;
    (void)hipFree(p);
  }
  static hipError_t synchronize(hipStream_t s) { return hipStreamSynchronize(s); }
  static hipError_t capture(hipStream_t s, bool* on, unsigned long long* id) {
    if (!s) return hipSuccess;                 // the null stream cannot be captured
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    const hipError_t e = hipStreamGetCaptureInfo(s, &status, id);
    *on = status != hipStreamCaptureStatusNone;
    return e;
  }
};
using Mem = SeqMem<Api>;

}  // namespace

struct mure_seq {
  mure_ctx* ctx = nullptr;
  int device = -1;
  hipStream_t stream = nullptr;
  int64_t n_seq = 0, tokens = 0, longest = 0;
  // work lists, in device memory
  Mem lists;
  const SeqItem* conv[N_RUNS] = {};            // runs of at most CONV_RUNS tokens
  int n_conv[N_RUNS] = {};
  const SeqItem* scan = nullptr;               // whole sequences and chunks, longest first
  int n_scan = 0;
  const SeqItem* ends = nullptr;               // the chunks but each sequence's last
  int n_ends = 0;
  const SeqChunks* chunked = nullptr;
  int n_chunked = 0;
  int64_t n_slots = 0;
  SeqWorkspace<Api> work;                      // the chunks' states
};

namespace {

template <typename F>
mure_status guarded(mure_ctx* ctx, F&& f) noexcept {
  mure_status st = MURE_E_INVALID;
  try {
    std::string msg;
    try {
      f();
      return MURE_OK;
    } catch (const Fail& e) {
      st = e.st;
      msg = e.msg;
    } catch (const std::bad_alloc&) {
      st = MURE_E_NOMEM;
      msg = "host memory exhausted";
    } catch (const std::exception& e) {
      msg = e.what();
    }
    if (ctx) *ctx_view(ctx).err = msg;
  } catch (...) {
  }
  return st;
}

// ---- checks of arguments

constexpr wide MOST = (wide)1 << 60;           // elements of a tensor, from its first to its last

// The elements that an output writes or an input reads: rows of `width`
// elements, `rows` of them `row_stride` apart, `mutants` times.
struct Span {
  const char* name;
  const char* p;
  int64_t esize, width, rows, row_stride, mutants, mutant_stride;
  wide extent() const {                        // bytes from the first element past the last
    if (rows == 0 || width == 0) return 0;
    return ((wide)(mutants - 1) * mutant_stride + (wide)(rows - 1) * row_stride + width) * esize;
  }
};

Span span(const char* name, const void* p, int64_t esize, int64_t width, int64_t rows, int64_t row_stride, int64_t mutants,
          int64_t mutant_stride) {
  if (!p && rows > 0) invalid(std::string(name) + " is NULL");
  if (row_stride < 0 || mutant_stride < 0) invalid(std::string(name) + ": a stride is negative");
  Span s{name, static_cast<const char*>(p), esize, width, rows, rows > 1 ? row_stride : 0, mutants, mutants > 1 ? mutant_stride : 0};
  if (s.extent() > MOST) invalid(std::string(name) + ": its strides pass the address space");
  if (reinterpret_cast<uintptr_t>(p) % esize) invalid(std::string(name) + " is not aligned to its elements");
  return s;
}

// An output's elements are apart from each other.
void check_output(const Span& s) {
  if (s.extent() == 0) return;
  const wide rows = (wide)(s.rows - 1) * s.row_stride + s.width, muts = (wide)(s.mutants - 1) * s.mutant_stride + s.width;
  const bool rows_inside = (s.rows == 1 || s.row_stride >= s.width) && (s.mutants == 1 || s.mutant_stride >= rows);
  const bool muts_inside = (s.mutants == 1 || s.mutant_stride >= s.width) && (s.rows == 1 || s.row_stride >= muts);
  if (!rows_inside && !muts_inside) invalid(std::string(s.name) + ": its rows overlap");
}

// Whether two tensors may share memory.  Rows side by side in one buffer (the
// same pitch, at different columns) do not.
bool meet(const Span& a, const Span& b) {
  if (a.extent() == 0 || b.extent() == 0) return false;
  const wide pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
  if (pa + a.extent() <= pb || pb + b.extent() <= pa) return false;
  // The pitch in bytes of a tensor of several rows, and of one with one row
  // per mutant, or none.
  auto pitch = [](const Span& s) { return (s.rows > 1 ? s.row_stride : s.mutant_stride) * (wide)s.esize; };
  const wide q = pitch(a);
  if (q == 0 || pitch(b) != q) return true;
  for (const Span* s : {&a, &b})
    if ((wide)s->mutant_stride * s->esize % q || (wide)s->width * s->esize > q) return true;
  const wide d = ((pb - pa) % q + q) % q;      // b's first column, as a's rows see it
  return d < (wide)a.width * a.esize || d + (wide)b.width * b.esize > q;
}

bool same(const Span& a, const Span& b) {
  return a.p == b.p && a.esize == b.esize && a.row_stride == b.row_stride && a.mutant_stride == b.mutant_stride &&
         (a.mutants == 1 || a.mutant_stride > 0);
}

// The tensors of a call (a norm has the most, 10).
struct Spans {
  Span v[10];
  int n = 0;
  void push_back(const Span& s) { v[n++] = s; }
  const Span* begin() const { return v; }
  const Span* end() const { return v + n; }
};

// `out` may be one of `allowed`, element by element, and may meet nothing else.
void check_apart(const Span& out, const Spans& others, std::initializer_list<const Span*> allowed = {}) {
  for (const Span& o : others) {
    if (!meet(out, o)) continue;
    bool ok = false;
    for (const Span* s : allowed) ok = ok || (s && s->p == o.p && s->name == o.name && same(out, o));
    if (!ok) invalid(std::string(out.name) + " overlaps " + o.name);
  }
}

int64_t esize_of(int32_t dtype, const char* what) {
  if (dtype != MURE_F32 && dtype != MURE_BF16) invalid(std::string(what) + ": unknown type");
  return dtype == MURE_F32 ? 4 : 2;
}

void check_range(int64_t v, int64_t lo, int64_t hi, const char* what) {
  if (v < lo || v > hi)
    invalid(std::string(what) + " is " + std::to_string(v) + ", outside " + std::to_string(lo) + " ... " + std::to_string(hi));
}

// An optional float32 parameter of n values a mutant.
void add_param(Spans& in, const char* name, const mure_seq_param& p, int64_t n, int64_t mutants) {
  if (p.p) in.push_back(span(name, p.p, 4, n, 1, 0, mutants, p.mutant_stride));
}

void check_device(int device) {
  if (device < 0) throw Fail{MURE_E_UNSUPPORTED, "planning-only context"};
  check(hipSetDevice(device), "hipSetDevice");
}

// ---- batches

// Sequence i's runs of at most `run` tokens, its chunks in the workspace from
// `slot` on (or -1); a sequence without tokens has one empty run.
void add_runs(std::vector<SeqItem>& to, int32_t i, int64_t row, int64_t length, int64_t run, int64_t slot) {
  for (int64_t t = 0; t == 0 || t < length; t += run)
    to.push_back({i, (int32_t)(row + t), (int32_t)std::min(run, length - t), (int32_t)t, (int32_t)length,
                  slot < 0 ? -1 : (int32_t)(slot + t / run)});
}

void create(mure_ctx* ctx, int64_t n_seq, const int64_t* lengths, mure_seq** out) {
  if (!out) invalid("out is NULL");
  *out = nullptr;
  if (!lengths) invalid("lengths is NULL");
  check_range(n_seq, 1, 1 << 20, "n_seq");
  const CtxView cv = ctx_view(ctx);
  std::unique_ptr<mure_seq> s(new mure_seq());
  s->ctx = ctx;
  s->device = cv.device;
  s->stream = cv.stream;
  s->n_seq = n_seq;
  for (int64_t i = 0; i < n_seq; ++i) {
    check_range(lengths[i], 0, INT32_MAX, "a length");
    s->tokens += lengths[i];
    if (s->tokens > INT32_MAX) invalid("the batch has 2^31 tokens or more");
    s->longest = std::max(s->longest, lengths[i]);
  }
  const bool ones = std::all_of(lengths, lengths + n_seq, [](int64_t n) { return n == 1; });
  std::vector<SeqItem> conv[N_RUNS], scan, ends;
  std::vector<SeqChunks> chunked;
  int64_t row = 0, slots = 0;
  for (int32_t i = 0; i < (int32_t)n_seq; ++i) {
    const int64_t L = lengths[i];
    if (L <= MURE_SEQ_SPLIT_TOKENS) {
      add_runs(scan, i, row, L, MURE_SEQ_SPLIT_TOKENS, -1);
    } else {
      const int64_t n = (L + SCAN_CHUNK - 1) / SCAN_CHUNK;
      const size_t first = scan.size();
      add_runs(scan, i, row, L, SCAN_CHUNK, slots);
      ends.insert(ends.end(), scan.begin() + first, scan.end() - 1);
      chunked.push_back({i, (int32_t)slots, (int32_t)n, (int32_t)row});
      slots += n;
    }
    row += L;
  }
  // the convolution's runs: shorter ones only where a layer may take them (conv below)
  for (int k = 0; k < N_RUNS; ++k) {
    if (k && conv[k - 1].size() >= (k == 1 ? 1u << 17 : 1u << 15)) break;
    row = 0;
    for (int32_t i = 0; i < (int32_t)n_seq; row += lengths[i++]) add_runs(conv[k], i, row, lengths[i], CONV_RUNS[k], -1);
  }
  // the longest first, so that a launch does not end with one long run
  std::stable_sort(scan.begin(), scan.end(), [](const SeqItem& a, const SeqItem& b) { return a.len > b.len; });
  s->n_slots = slots;
  std::vector<char> host;
  size_t at[N_RUNS + 3];
  int k = 0;
  auto put = [&](const void* p, size_t bytes) {
    at[k++] = host.size();
    host.insert(host.end(), static_cast<const char*>(p), static_cast<const char*>(p) + bytes);
    host.resize((host.size() + 15) / 16 * 16);
  };
  for (const auto& v : conv) put(v.data(), v.size() * sizeof(SeqItem));
  for (const auto* v : {&scan, &ends}) put(v->data(), v->size() * sizeof(SeqItem));
  put(chunked.data(), chunked.size() * sizeof(SeqChunks));
  for (int i = 0; i < N_RUNS; ++i) s->n_conv[i] = (int)conv[i].size();
  s->n_scan = (int)scan.size();
  s->n_ends = (int)ends.size();
  s->n_chunked = (int)chunked.size();
  if (s->device >= 0) {
    check_device(s->device);
    check(s->lists.alloc(host.size()), "work lists");
    check(hipMemcpyAsync(s->lists.p, host.data(), host.size(), hipMemcpyHostToDevice, s->stream), "upload of the work lists");
    check(hipStreamSynchronize(s->stream), "upload of the work lists");
    const char* d = static_cast<const char*>(s->lists.p);
    if (!ones)
      for (int i = 0; i < N_RUNS; ++i) s->conv[i] = reinterpret_cast<const SeqItem*>(d + at[i]);
    if (!ones) s->scan = reinterpret_cast<const SeqItem*>(d + at[N_RUNS]);
    s->ends = reinterpret_cast<const SeqItem*>(d + at[N_RUNS + 1]);
    s->chunked = reinterpret_cast<const SeqChunks*>(d + at[N_RUNS + 2]);
  }
  *out = s.release();
}

// ---- the operators

void conv(mure_seq* s, const mure_seq_conv_args* args) {
  if (!args) invalid("args is NULL");
  SeqConvArgs k;
  k.a = *args;
  mure_seq_conv_args& a = k.a;
  const int64_t es = esize_of(a.dtype, "dtype");
  check_range(a.n_mutants, 1, MURE_SEQ_MAX_MUTANTS, "n_mutants");
  check_range(a.channels, 1, MURE_SEQ_MAX_CHANNELS, "channels");
  check_range(a.n_taps, 1, MURE_SEQ_MAX_TAPS, "n_taps");
  if (a.activation != MURE_SEQ_LINEAR && a.activation != MURE_SEQ_SILU) invalid("unknown activation");
  if (a.reserved) invalid("reserved must be 0");
  const int64_t M = a.n_mutants, C = a.channels, K = a.n_taps;
  if (K == 1) a.state = nullptr, a.state_out = nullptr;
  Spans in;
  in.push_back(span("x", a.x.p, es, C, s->tokens, a.x.row_stride, M, a.x.mutant_stride));
  in.push_back(span("taps", a.taps, es, C * K, 1, 0, M, a.taps_mutant_stride));
  add_param(in, "bias", a.bias, C, M);
  const int64_t held = s->n_seq * (K - 1) * C;
  Span state{};
  if (a.state) {
    state = span("state", a.state, es, held, 1, 0, M, a.state_mutant_stride);
    in.push_back(state);
  }
  const Span out = span("out", a.out.p, es, C, s->tokens, a.out.row_stride, M, a.out.mutant_stride);
  check_output(out);
  check_apart(out, in);
  if (a.state_out) {
    const Span so = span("state_out", a.state_out, es, held, 1, 0, M, a.state_out_mutant_stride);
    check_output(so);
    check_apart(so, in, {a.state ? &state : nullptr});
    if (meet(so, out)) invalid("state_out overlaps out");
  }
  check_device(s->device);
  // Long runs read fewer rows twice (at 4 taps 3 of 36, 15 and 6), short ones give more threads (of 16 bytes of
  // channels): the longest is taken that fills the chip, or the next that comes near it.  24 prompts of 18865 tokens
  // and 1536 bfloat16 channels take 25.0 us in runs of 12 and 26.9 in runs of 32; 65536 tokens of 4096 channels 203 us
  // in runs of 33 and 209 in runs of 16.
  const int64_t vecs = (C * es + 15) / 16 * M;
  // A run reads the state for rows before the sequence, and the sequence's first run may overwrite it: every other
  // run starts n_taps - 1 rows in, or later.
  static_assert(CONV_RUNS[1] >= MURE_SEQ_MAX_TAPS - 1, "");
  const bool shortest = s->n_conv[2] && s->n_conv[1] * vecs < 1 << 15 && CONV_RUNS[2] >= K - 1;
  const int w = !s->n_conv[1] || s->n_conv[0] * vecs >= 1 << 17 ? 0 : shortest ? 2 : 1;
  k.items = s->conv[w];
  k.n_items = s->n_conv[w];
  check(launch_seq_conv(k, s->stream), "mure_seq_conv");
}

void scan(mure_seq* s, const mure_seq_scan_args* args) {
  if (!args) invalid("args is NULL");
  SeqScanArgs k;
  k.a = *args;
  const mure_seq_scan_args& a = k.a;
  const int64_t es = esize_of(a.dtype, "dtype");
  check_range(a.n_mutants, 1, MURE_SEQ_MAX_MUTANTS, "n_mutants");
  check_range(a.channels, 1, MURE_SEQ_MAX_CHANNELS, "channels");
  check_range(a.states, 1, MURE_SEQ_MAX_STATES, "states");
  check_range(a.groups, 1, a.channels, "groups");
  if (a.channels % a.groups) invalid("channels is no multiple of groups");
  check_range(a.softplus, 0, 1, "softplus");
  if (seq_scan_blocks(a) > SCAN_GRID) throw Fail{MURE_E_UNSUPPORTED, "too many channels times mutants for one scan"};
  const int64_t M = a.n_mutants, D = a.channels, N = a.states, T = s->tokens;
  Spans in;
  in.push_back(span("u", a.u.p, es, D, T, a.u.row_stride, M, a.u.mutant_stride));
  in.push_back(span("dt", a.dt.p, es, D, T, a.dt.row_stride, M, a.dt.mutant_stride));
  in.push_back(span("b", a.b.p, es, a.groups * N, T, a.b.row_stride, M, a.b.mutant_stride));
  in.push_back(span("c", a.c.p, es, a.groups * N, T, a.c.row_stride, M, a.c.mutant_stride));
  if (a.gate.p) in.push_back(span("gate", a.gate.p, es, D, T, a.gate.row_stride, M, a.gate.mutant_stride));
  in.push_back(span("a", a.a.p, 4, D * N, 1, 0, M, a.a.mutant_stride));
  add_param(in, "skip", a.skip, D, M);
  add_param(in, "dt_bias", a.dt_bias, D, M);
  const int64_t held = s->n_seq * D * N;
  Span state{};
  if (a.state) {
    state = span("state", a.state, 4, held, 1, 0, M, a.state_mutant_stride);
    in.push_back(state);
  }
  const Span out = span("out", a.out.p, es, D, T, a.out.row_stride, M, a.out.mutant_stride);
  check_output(out);
  check_apart(out, in);
  if (a.state_out) {
    const Span so = span("state_out", a.state_out, 4, held, 1, 0, M, a.state_out_mutant_stride);
    check_output(so);
    check_apart(so, in, {a.state ? &state : nullptr});
    if (meet(so, out)) invalid("state_out overlaps out");
  }
  check_device(s->device);
  k.n_slots = s->n_slots;
  k.longest = s->longest;
  if (s->n_chunked) {
    const wide need = (wide)M * s->n_slots * D * (N + 1) * 4;
    if (need > MOST) throw Fail{MURE_E_NOMEM, "sequence workspace"};
    void* work = nullptr;
    check(s->work.get(s->stream, (size_t)need, &work), "sequence workspace");
    k.ws_h = static_cast<float*>(work);
    k.ws_d = k.ws_h + M * s->n_slots * D * N;
    k.chunks = s->chunked;
    k.n_chunked = s->n_chunked;
    k.items = s->ends;
    k.n_items = s->n_ends;
    check(launch_seq_scan_ends(k, s->stream), "mure_seq_scan");
    check(launch_seq_scan_join(k, s->stream), "mure_seq_scan");
  }
  k.items = s->scan;
  k.n_items = s->n_scan;
  check(launch_seq_scan(k, s->stream), "mure_seq_scan");
}

void norm(mure_ctx* ctx, const mure_seq_norm_args* args) {
  if (!args) invalid("args is NULL");
  mure_seq_norm_args a = *args;
  const int64_t es = esize_of(a.dtype, "dtype"), rs = esize_of(a.residual_dtype, "residual_dtype");
  if (rs < es) invalid("a float32 y needs a float32 residual");
  check_range(a.n_mutants, 1, MURE_SEQ_MAX_MUTANTS, "n_mutants");
  check_range(a.channels, 1, MURE_SEQ_MAX_WIDTH, "channels");
  check_range(a.rows, 0, INT32_MAX, "rows");
  check_range(a.gate_at, 0, 2, "gate_at");
  check_range(a.gate_activation, 0, MURE_SEQ_SIGMOID, "gate_activation");
  check_range(a.after, 0, MURE_SEQ_LAYER, "after");
  check_range(a.before, 0, MURE_SEQ_LAYER, "before");
  if (!(a.eps >= 0.f) || !std::isfinite(a.eps)) invalid("eps is no finite value >= 0");
  if (!a.after && (a.after_weight.p || a.after_bias.p)) invalid("a weight or bias of `after` without its norm");
  if (!a.before && (a.before_weight.p || a.before_bias.p)) invalid("a weight or bias of `before` without its norm");
  if ((a.gate_at != 0) != (a.gate.p != nullptr) && a.rows > 0) invalid("gate and gate_at go together");
  if (a.rows > 0 && !a.out.p && !a.residual_out.p) invalid("neither out nor residual_out is given");
  if (a.out.p && !a.before) invalid("out needs a `before`");
  const int64_t M = a.n_mutants, C = a.channels, R = a.rows;
  Spans in;
  const Span y = span("y", a.y.p, es, C, R, a.y.row_stride, M, a.y.mutant_stride);
  in.push_back(y);
  Span gate{}, res{};
  if (a.gate.p) in.push_back(gate = span("gate", a.gate.p, es, C, R, a.gate.row_stride, M, a.gate.mutant_stride));
  if (a.residual.p) in.push_back(res = span("residual", a.residual.p, rs, C, R, a.residual.row_stride, M, a.residual.mutant_stride));
  add_param(in, "after_weight", a.after_weight, C, M);
  add_param(in, "after_bias", a.after_bias, C, M);
  add_param(in, "scale", a.scale, C, M);
  add_param(in, "before_weight", a.before_weight, C, M);
  add_param(in, "before_bias", a.before_bias, C, M);
  Span ro{};
  if (a.residual_out.p) {
    ro = span("residual_out", a.residual_out.p, rs, C, R, a.residual_out.row_stride, M, a.residual_out.mutant_stride);
    check_output(ro);
    check_apart(ro, in, {a.residual.p ? &res : nullptr});
  }
  if (a.out.p) {
    const Span o = span("out", a.out.p, es, C, R, a.out.row_stride, M, a.out.mutant_stride);
    check_output(o);
    check_apart(o, in, {&y, a.gate.p ? &gate : nullptr});
    if (a.residual_out.p && meet(o, ro)) invalid("out overlaps residual_out");
  }
  const CtxView cv = ctx_view(ctx);
  check_device(cv.device);
  if (R == 0) return;
  check(launch_seq_norm(a, cv.stream), "mure_seq_norm");
}

}  // namespace

// =========================================================================
extern "C" {

int32_t mure_seq_version(void) { return MURE_SEQ_VERSION; }

mure_status mure_seq_create(mure_ctx* ctx, int64_t n_seq, const int64_t* lengths, mure_seq** out) {
  if (!ctx) return MURE_E_INVALID;
  return guarded(ctx, [&] { create(ctx, n_seq, lengths, out); });
}

mure_status mure_seq_conv(mure_seq* seq, const mure_seq_conv_args* args) {
  if (!seq) return MURE_E_INVALID;
  return guarded(seq->ctx, [&] { conv(seq, args); });
}

mure_status mure_seq_scan(mure_seq* seq, const mure_seq_scan_args* args) {
  if (!seq) return MURE_E_INVALID;
  return guarded(seq->ctx, [&] { scan(seq, args); });
}

mure_status mure_seq_norm(mure_ctx* ctx, const mure_seq_norm_args* args) {
  if (!ctx) return MURE_E_INVALID;
  return guarded(ctx, [&] { norm(ctx, args); });
}

void mure_seq_destroy(mure_seq* seq) {
  if (!seq) return;
  if (seq->device >= 0) {
    (void)hipSetDevice(seq->device);
    bool on = false;
    unsigned long long id = 0;
    // A wait would end a capture of the stream; what it had before is waited for by the frees.
    if (Api::capture(seq->stream, &on, &id) != hipSuccess || !on) (void)hipStreamSynchronize(seq->stream);
  }
  delete seq;
}

}  // extern "C"
