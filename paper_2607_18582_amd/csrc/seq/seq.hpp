// Sequence operators (mure_seq.h): argument blocks and launchers of their
// kernels, and what they need of a context.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>
#include <string>

#include "../../../include/mure_seq.h"
#include "../kernels.hpp"

namespace mure {

// One run of consecutive tokens of a sequence: rows row0 .. row0 + len - 1 of
// the packed batch, positions pos0 .. of a sequence of `total` tokens.
// slot >= 0: the run is a chunk of a sequence scanned in chunks, and slot is
// its place in the workspace (a sequence's chunks are consecutive).
struct SeqItem {
  int32_t seq, row0, len, pos0, total, slot;
};

// Item i of a list; a list that is not there (nullptr) is that of sequences of
// one token each, which a decoding step need not wait for.
__device__ __forceinline__ SeqItem seq_item(const SeqItem* items, int i) { return items ? items[i] : SeqItem{i, i, 1, 0, 1, -1}; }

// A sequence scanned in chunks: its slots slot0 .. slot0 + n - 1, its first row.
struct SeqChunks {
  int32_t seq, slot0, n, row0;
};

constexpr int SCAN_CHUNK = 128;                // tokens of a chunk
constexpr int CONV_RUNS[] = {33, 12, 3};       // tokens of a convolution's runs
constexpr int N_RUNS = 3;

struct SeqConvArgs {
  mure_seq_conv_args a;
  const SeqItem* items = nullptr;
  int n_items = 0, item0 = 0;
};

struct SeqScanArgs {
  mure_seq_scan_args a;
  const SeqItem* items = nullptr;              // of this launch
  int n_items = 0, item0 = 0;
  int64_t longest = 0;                         // tokens of the longest sequence
  const SeqChunks* chunks = nullptr;
  int n_chunked = 0;
  int64_t n_slots = 0;
  float* ws_h = nullptr;                       // [mutants][slots][channels][states]
  float* ws_d = nullptr;                       // [mutants][slots][channels]
};

// Blocks of a scan per work item: channel blocks times mutants.  A launch has
// at most SCAN_GRID blocks (a grid has fewer than 2^32 threads).
int64_t seq_scan_blocks(const mure_seq_scan_args& a);
constexpr int64_t SCAN_GRID = (1 << 24) - 1;

// launchers (return the launch status)
hipError_t launch_seq_conv(const SeqConvArgs& a, hipStream_t s);
hipError_t launch_seq_scan(const SeqScanArgs& a, hipStream_t s);         // the outputs and final states
hipError_t launch_seq_scan_ends(const SeqScanArgs& a, hipStream_t s);    // the chunks' states from zero
hipError_t launch_seq_scan_join(const SeqScanArgs& a, hipStream_t s);    // ... to their first states
hipError_t launch_seq_norm(const mure_seq_norm_args& a, hipStream_t s);

// What the operators use of a context (defined beside it).
struct CtxView {
  int device;                                  // -1: planning only
  hipStream_t stream;
  std::string* err;
};
CtxView ctx_view(mure_ctx* ctx);

}  // namespace mure
