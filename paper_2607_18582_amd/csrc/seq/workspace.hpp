// Device memory of a batch's scans of long sequences: the chunks' states.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstddef>
#include <utility>
#include <vector>

namespace mure {

// Api: hipError_t alloc(void** p, size_t bytes), void free(void* p), hipError_t synchronize(hipStream_t) and
// hipError_t capture(hipStream_t, bool* on, unsigned long long* id), static.

// Device memory held until it is destroyed.
template <typename Api> struct SeqMem {
  void* p = nullptr;
  size_t bytes = 0;
  SeqMem() = default;
  SeqMem(SeqMem&& o) noexcept : p(o.p), bytes(o.bytes) { o.p = nullptr, o.bytes = 0; }
  SeqMem(const SeqMem&) = delete;
  SeqMem& operator=(SeqMem&& o) noexcept {
    std::swap(p, o.p);
    std::swap(bytes, o.bytes);
    return *this;
  }
  ~SeqMem() {
    if (p) Api::free(p);
  }
  hipError_t alloc(size_t n) {
    const hipError_t e = Api::alloc(&p, n);
    if (e == hipSuccess) bytes = n;
    else p = nullptr;
    return e;
  }
};

// Calls made directly take one block, as they run one after the other on the context's stream.  A captured graph may be
// replayed at any time beside them and beside other graphs, so every capture has blocks of its own, kept until the
// batch is destroyed; the calls of one capture share them, as they follow each other in its graph.
template <typename Api> class SeqWorkspace {
  SeqMem<Api> direct_;
  struct Capture {
    unsigned long long id;
    std::vector<SeqMem<Api>> held;             // the last is the largest; the graph's earlier calls hold the others
  };
  std::vector<Capture> captures_;

 public:
  // *p: at least `need` bytes for a call on `stream`.
  hipError_t get(hipStream_t stream, size_t need, void** p) {
    bool on = false;
    unsigned long long id = 0;
    if (const hipError_t e = Api::capture(stream, &on, &id); e != hipSuccess) return e;
    if (!on) {
      if (direct_.bytes < need) {
        // Twice the last, so that growing calls allocate seldom, or what is needed where there is no memory for that.
        const size_t twice = 2 * direct_.bytes;
        if (const hipError_t e = Api::synchronize(stream); e != hipSuccess) return e;
        direct_ = SeqMem<Api>();
        hipError_t e = direct_.alloc(std::max(need, twice));
        if (e == hipErrorOutOfMemory && twice > need) e = direct_.alloc(need);
        if (e != hipSuccess) return e;
      }
      *p = direct_.p;
      return hipSuccess;
    }
    auto c = std::find_if(captures_.begin(), captures_.end(), [&](const Capture& c) { return c.id == id; });
    if (c == captures_.end() || c->held.back().bytes < need) {
      SeqMem<Api> m;
      if (const hipError_t e = m.alloc(need); e != hipSuccess) return e;
      if (c == captures_.end()) c = captures_.insert(c, Capture{id, {}});
      c->held.push_back(std::move(m));
    }
    *p = c->held.back().p;
    return hipSuccess;
  }
};

}  // namespace mure
