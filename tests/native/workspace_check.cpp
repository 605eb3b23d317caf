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
  static inline unsigned long long captured = 0;     // the running capture's id, or 0
  static inline int waits = 0;
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
  static hipError_t synchronize(hipStream_t) {
    ++waits;
    return hipSuccess;
  }
  static hipError_t capture(hipStream_t, bool* on, unsigned long long* id) {
    *on = captured != 0;
    *id = captured;
    return hipSuccess;
  }
};

int failures = 0;
void expect(bool ok, const char* what) {
  if (ok) return;
  ++failures;
  printf("FAILED: %s\n", what);
}

struct Batch {
  mure::SeqWorkspace<Fake> w;
  // the block that a call gets, nullptr where there is no memory; captured: the capture that the call is part of
  void* call(size_t need, unsigned long long captured = 0) {
    Fake::captured = captured;
    void* p = nullptr;
    const hipError_t e = w.get(nullptr, need, &p);
    Fake::captured = 0;
    if (e != hipSuccess) expect(e == hipErrorOutOfMemory && !p, "out of memory is said");
    else expect(Fake::held.at(p) >= need, "a block is large enough");
    return p;
  }
};

// What is needed is given where it fits, also where twice as much does not; a smaller block does not stay beside a
// larger one, and goes only when the stream's work on it is done.
void growth() {
  {
    Batch b;
    void* first = b.call(30);
    expect(first && b.call(20) == first, "a smaller one is the same");
    const int waits = Fake::waits;
    expect(b.call(31) && Fake::used() >= 60, "growing calls allocate seldom");
    expect(Fake::waits == waits + 1, "the stream's work is waited for");
    expect(Fake::held.size() == 1, "one block");
    expect(b.call(61) && Fake::used() == 61, "61 of 100 bytes, of which 60 were held");
    expect(b.call(100) && Fake::used() == 100, "all there is");
    expect(!b.call(101), "more than there is");
    expect(b.call(40) && Fake::used() >= 40, "and it goes on");
  }
  expect(Fake::held.empty(), "nothing stays");
}

// A capture's blocks are its own.
void captures() {
  {
    Batch b;
    void* direct = b.call(10);
    void* one = b.call(10, 1);
    expect(one && one != direct, "a capture has a block of its own");
    expect(b.call(8, 1) == one, "the calls of one capture share it");
    void* two = b.call(10, 2);
    expect(two && two != one && two != direct, "another capture has another");
    expect(b.call(10) == direct, "direct calls keep theirs");
    void* larger = b.call(15, 1);
    expect(larger && larger != one && Fake::held.count(one), "the earlier calls of a graph keep their block");
    expect(b.call(10, 1) == larger, "the later ones take the larger");
    expect(b.call(20) && Fake::held.count(one) && Fake::held.count(two) && Fake::held.count(larger), "a larger direct one frees none of them");
    expect(!b.call(90, 3), "more than there is");
    expect(b.call(5, 3), "and less after it");
  }
  expect(Fake::held.empty(), "nothing stays");
  Batch b;
  void* first = b.call(10, 7);                       // no call before the capture
  expect(first && b.call(10) != first, "a direct call after a capture");
}

}  // namespace

int main() {
  growth();
  captures();
  printf("failures %d\n", failures);
  return failures != 0;
}
