// Device memory of a batch's scans of long sequences: the chunks' states.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstddef>
#include <utility>
#include <vector>

namespace mure {

// Api: hipError_t alloc(void** p, size_t bytes) and void free(void* p), static.
// Device memory held until it is destroyed.
template <typename Api> struct SeqMem {
  void* p = nullptr;
  size_t bytes = 0;
  SeqMem() = default;
  SeqMem(SeqMem&& o) noexcept : p(o.p), bytes(o.bytes) { o.p = nullptr, o.bytes = 0; }
  SeqMem(const SeqMem&) = delete;
  SeqMem& operator=(const SeqMem&) = delete;
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

template <typename Api> class SeqWorkspace {
  // The last is the largest.  Smaller ones stay: a captured graph may hold them.
  std::vector<SeqMem<Api>> held_;

 public:
  // *p: at least `need` bytes.  A new one has twice the last one's bytes, so that those that stay are no more than
  // the largest, or what is needed where there is no memory for that.
  hipError_t get(size_t need, void** p) {
    if (held_.empty() || held_.back().bytes < need) {
      SeqMem<Api> m;
      const size_t twice = held_.empty() ? 0 : 2 * held_.back().bytes;
      hipError_t e = m.alloc(std::max(need, twice));
      if (e == hipErrorOutOfMemory && twice > need) e = m.alloc(need);
      if (e != hipSuccess) return e;
      held_.push_back(std::move(m));
    }
    *p = held_.back().p;
    return hipSuccess;
  }
};

}  // namespace mure
