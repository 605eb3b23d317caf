// What the calls on batches of sequences share (mure_seq.h, mure_attn.h): the
// batch, checks of arguments, errors.
#pragma once

#include "seq.hpp"
#include "workspace.hpp"

#include <algorithm>
#include <exception>
#include <initializer_list>
#include <new>
#include <string>

namespace mure {

typedef __int128 wide;

struct Fail {
  mure_status st;
  std::string msg;
};

[[noreturn]] inline void invalid(const std::string& m) { throw Fail{MURE_E_INVALID, m}; }

inline void check(hipError_t e, const char* what) {
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

struct SeqApi {
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

}  // namespace mure

struct mure_seq {
  mure_ctx* ctx = nullptr;
  int device = -1;
  hipStream_t stream = nullptr;
  int64_t n_seq = 0, tokens = 0, longest = 0;
  // work lists, in device memory
  mure::SeqMem<mure::SeqApi> lists;
  const mure::SeqItem* conv[mure::N_RUNS] = {};            // runs of at most CONV_RUNS tokens
  int n_conv[mure::N_RUNS] = {};
  const mure::SeqItem* scan = nullptr;               // whole sequences and chunks, longest first
  int n_scan = 0;
  const mure::SeqItem* ends = nullptr;               // the chunks but each sequence's last
  int n_ends = 0;
  const mure::SeqChunks* chunked = nullptr;
  int n_chunked = 0;
  int64_t n_slots = 0;
  // attention: sequences of at most ATTN_WHOLE tokens, the longest first (the last n_short have at most ATTN_SHORT, the first of
  // those longest_short); runs of
  // ATTN_ROWS tokens of those above ATTN_SHORT: of sequences above ATTN_MID (n_long_runs), above ATTN_WHOLE, the others
  // (n_small_runs), and in each the last runs of the longest first
  const mure::SeqItem* brief = nullptr;
  int n_brief = 0, n_short = 0, longest_brief = 0, longest_short = 0;
  const mure::SeqItem* runs = nullptr;
  int n_runs = 0, n_long_runs = 0, n_small_runs = 0, longest_mid_run = 0;      // the last: tokens, of sequences up to ATTN_MID
  mure::SeqWorkspace<mure::SeqApi> work;          // the chunks' states, attention over parts of the keys
};

namespace mure {

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
// elements, `rows` of them `row_stride` apart, `mutants` times (of a cache: for
// each of `outers` sequences).
struct Span {
  const char* name;
  const char* p;
  int64_t esize, width, rows, row_stride, mutants, mutant_stride, outers = 1, outer_stride = 0;
  wide extent() const {                        // bytes from the first element past the last
    if (rows == 0 || width == 0) return 0;
    return ((wide)(mutants - 1) * mutant_stride + (wide)(outers - 1) * outer_stride + (wide)(rows - 1) * row_stride + width) * esize;
  }
};

inline Span span(const char* name, const void* p, int64_t esize, int64_t width, int64_t rows, int64_t row_stride, int64_t mutants,
          int64_t mutant_stride) {
  if (!p && rows > 0) invalid(std::string(name) + " is NULL");
  if (row_stride < 0 || mutant_stride < 0) invalid(std::string(name) + ": a stride is negative");
  Span s{name, static_cast<const char*>(p), esize, width, rows, rows > 1 ? row_stride : 0, mutants, mutants > 1 ? mutant_stride : 0};
  if (s.extent() > MOST) invalid(std::string(name) + ": its strides pass the address space");
  if (reinterpret_cast<uintptr_t>(p) % esize) invalid(std::string(name) + " is not aligned to its elements");
  return s;
}

// An output's elements are apart from each other.
inline void check_output(const Span& s) {
  if (s.extent() == 0) return;
  const wide rows = (wide)(s.rows - 1) * s.row_stride + s.width, muts = (wide)(s.mutants - 1) * s.mutant_stride + s.width;
  const bool rows_inside = (s.rows == 1 || s.row_stride >= s.width) && (s.mutants == 1 || s.mutant_stride >= rows);
  const bool muts_inside = (s.mutants == 1 || s.mutant_stride >= s.width) && (s.rows == 1 || s.row_stride >= muts);
  if (!rows_inside && !muts_inside) invalid(std::string(s.name) + ": its rows overlap");
}

// Whether two tensors may share memory.  Blocks side by side in one buffer (rows at different columns, caches as an axis of
// one tensor, whichever axis goes around which) do not.
inline bool meet(const Span& a, const Span& b) {
  if (a.extent() == 0 || b.extent() == 0) return false;
  const wide pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
  if (pa + a.extent() <= pb || pb + b.extent() <= pa) return false;
  struct Axis { wide stride, n; };
  const Axis axes[2][3] = {{{a.row_stride, a.rows}, {a.outer_stride, a.outers}, {a.mutant_stride, a.mutants}},
                           {{b.row_stride, b.rows}, {b.outer_stride, b.outers}, {b.mutant_stride, b.mutants}}};
  const Span* const spans[2] = {&a, &b};
  // With any stride as the border: the axes of smaller ones make a block, and what divides the others, in bytes, is the
  // length of pieces in each of which a tensor has its blocks in the same place.
  for (int which = 0; which < 6; ++which) {
    const wide border = axes[which / 3][which % 3].stride * spans[which / 3]->esize;
    if (border == 0) continue;
    wide q = 0, block[2];
    for (int s = 0; s < 2; ++s) {
      block[s] = (wide)spans[s]->width * spans[s]->esize;
      for (const Axis& x : axes[s]) {
        wide stride = x.stride * spans[s]->esize;
        if (stride < border) {
          block[s] += (x.n - 1) * stride;
          continue;
        }
        while (stride) {
          const wide rest = q % stride;
          q = stride;
          stride = rest;
        }
      }
    }
    const wide d = ((pb - pa) % q + q) % q;    // b's first block, as a's pieces see it
    if (block[0] <= q && block[1] <= q && d >= block[0] && d + block[1] <= q) return false;
  }
  return true;
}

inline bool same(const Span& a, const Span& b) {
  return a.p == b.p && a.esize == b.esize && a.row_stride == b.row_stride && a.mutant_stride == b.mutant_stride &&
         (a.mutants == 1 || a.mutant_stride > 0);
}

// The tensors of a call (a norm has the most, 10).
struct Spans {
  Span v[12];
  int n = 0;
  void push_back(const Span& s) { v[n++] = s; }
  const Span* begin() const { return v; }
  const Span* end() const { return v + n; }
};

// `out` may be one of `allowed`, element by element, and may meet nothing else.
inline void check_apart(const Span& out, const Spans& others, std::initializer_list<const Span*> allowed = {}) {
  for (const Span& o : others) {
    if (!meet(out, o)) continue;
    bool ok = false;
    for (const Span* s : allowed) ok = ok || (s && s->p == o.p && s->name == o.name && same(out, o));
    if (!ok) invalid(std::string(out.name) + " overlaps " + o.name);
  }
}

inline int64_t esize_of(int32_t dtype, const char* what) {
  if (dtype != MURE_F32 && dtype != MURE_BF16) invalid(std::string(what) + ": unknown type");
  return dtype == MURE_F32 ? 4 : 2;
}

inline void check_range(int64_t v, int64_t lo, int64_t hi, const char* what) {
  if (v < lo || v > hi)
    invalid(std::string(what) + " is " + std::to_string(v) + ", outside " + std::to_string(lo) + " ... " + std::to_string(hi));
}

// An optional float32 parameter of n values a mutant.
inline void add_param(Spans& in, const char* name, const mure_seq_param& p, int64_t n, int64_t mutants) {
  if (p.p) in.push_back(span(name, p.p, 4, n, 1, 0, mutants, p.mutant_stride));
}

inline void check_device(int device) {
  if (device < 0) throw Fail{MURE_E_UNSUPPORTED, "planning-only context"};
  check(hipSetDevice(device), "hipSetDevice");
}

}  // namespace mure
