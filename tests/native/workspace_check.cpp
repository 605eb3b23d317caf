// Host-only check of the memory that a batch's scans hold (csrc/seq/workspace.hpp),
// on a device of 100 bytes, built with AddressSanitizer and
// UndefinedBehaviorSanitizer by tests/test_seq_workspace.py.
#include <cstdio>
#include <cstdlib>
#include <map>

#include "../../paper_2607_18582_amd/csrc/seq/workspace.hpp"

namespace {

struct Fake {
  static inline std::map<void*, size_t> held;
  static inline size_t most = 100;
  static size_t used() {
    size_t n = 0;
    for (const auto& h : held) n += h.second;
    return n;
  }
  static hipError_t alloc(void** p, size_t n) {
    if (used() + n > most) return hipErrorOutOfMemory;
    *p = malloc(n);
    held[*p] = n;
    return hipSuccess;
  }
  static void free(void* p) {
    held.erase(p);
    ::free(p);
  }
};

int failures = 0;
void expect(bool ok, const char* what) {
  if (ok) return;
  ++failures;
  printf("FAILED: %s\n", what);
}

// What is needed is given where it fits, also where twice as much does not.
void growth() {
  {
    mure::SeqWorkspace<Fake> w;
    void *a = nullptr, *b = nullptr;
    expect(w.get(40, &a) == hipSuccess && Fake::held.at(a) >= 40, "the first");
    expect(w.get(30, &b) == hipSuccess && b == a, "a smaller one is the same");
    expect(w.get(50, &b) == hipSuccess && Fake::held.at(b) >= 50, "50 of 100 bytes, 40 of them held");
    expect(w.get(101, &a) == hipErrorOutOfMemory, "more than there is");
    expect(w.get(50, &a) == hipSuccess && a == b, "and the last is still there");
  }
  expect(Fake::held.empty(), "nothing stays");
}

}  // namespace

int main() {
  growth();
  printf("failures %d\n", failures);
  return failures != 0;
}
