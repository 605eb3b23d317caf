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
// Tokens of sequences that attention takes in other ways than by runs of ATTN_ROWS over all of their keys.  Heads of 128
// channels, us:
// at most ATTN_SHORT over a cache, by waves of 16 rows over parts of the keys: 16 sequences of 2, 16 and 32 tokens over 4000
//   rows, 16 heads of 4, bfloat16, take 35, 70 and 109 so and 84, 91 and 99 in runs over parts of the keys;
// at most ATTN_WHOLE without a cache, by waves of 16 rows: 200 sequences of 64, 96 and 128 tokens, 8 heads of 2, take 32, 46
//   and 80 so and 37, 52 and 59 in runs (float32: 77, 116 and 236, in runs 96 tokens 128, 128 tokens 162);
// at most ATTN_MID over a cache, in runs over parts of the keys: one sequence of 512 tokens over 16000 rows takes 124 so and
//   334 in one piece; 16 of 64 over 4000 rows, enough to fill the chip, 122 and 90.  Longer ones have runs enough, and
//   their parts' results would be many bytes: 2048 tokens over 16000 rows 409 and 364.
constexpr int ATTN_SHORT = 16, ATTN_WHOLE = 96, ATTN_MID = 512;
constexpr int ATTN_ROWS = 128;                 // tokens of a run of the others

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
