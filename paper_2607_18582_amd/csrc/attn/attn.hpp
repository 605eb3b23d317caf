// Operators of an attention block (mure_attn.h): argument blocks and launchers
// of their kernels.
#pragma once

#include "../../../include/mure_attn.h"
#include "../seq/seq.hpp"

namespace mure {

struct AttnRotateArgs {
  mure_attn_rotate_args a;
  const SeqItem* items = nullptr;              // runs of tokens
  int n_items = 0, item0 = 0, longest = 0;     // longest: tokens of a run
  int64_t tokens = 0;
};

// Keys of a part, where they are worked on side by side: over a cache, for sequences of at most ATTN_SHORT tokens and of at most
// ATTN_MID.  Heads of 128 bfloat16 channels, parts of 256, 512 and 1024 keys, us: 64 tokens over 4000 rows each 129, 122 and
// 123; one over 100000 rows 115, 104 and 103; 8 over 1000 rows 13, 17 and 26.  512 tokens over 16000 rows, parts of 1024 and
// 2048: 124 and 110; 64 tokens 40 and 57.
constexpr int ATTN_KEYS_SHORT = 512, ATTN_KEYS_MID = 1024;

// How rows are read: element by element, or copied to LDS in pieces of 16 bytes, of which they are a whole number, aligned, or
// in which they are whole words of 4 bytes.
enum AttnReads : int { ELEMENTS, WORDS, PIECES };

struct AttnArgs {
  mure_attn_attend_args a;
  const SeqItem* items = nullptr;              // a list (nullptr: all sequences, one token each), of which items first ... first + n_items - 1
  int first = 0, n_items = 0, item0 = 0;       // item0: of a launch, counted from `first` as the workspace's rows are
  int longest = 0;                             // tokens of an item, at most
  int rows_each = 0;                           // rows of the workspace that an item has
  int parts = 1;                               // of the keys
  float* ws_o = nullptr;                       // [mutants][items][rows_each][heads][parts][head_dim], before the division
  float* ws_ml = nullptr;                      // ... [2]: the largest exponent (of 2), the sum
  int fast = 0;                                // of k, v and the caches
};

// launchers (return the launch status)
hipError_t launch_attn_rotate(const AttnRotateArgs& a, hipStream_t s);
// short sequences (over a cache those of at most ATTN_SHORT tokens), runs of ATTN_ROWS tokens, and the results of parts of `keys` keys
hipError_t attn_short_f32(const AttnArgs& a, hipStream_t s);
hipError_t attn_short_bf16(const AttnArgs& a, hipStream_t s);
hipError_t attn_runs_f32(const AttnArgs& a, hipStream_t s);
hipError_t attn_runs_bf16(const AttnArgs& a, hipStream_t s);
hipError_t attn_join_f32(const AttnArgs& a, int keys, hipStream_t s);
hipError_t attn_join_bf16(const AttnArgs& a, int keys, hipStream_t s);
hipError_t launch_attn_gated(const mure_attn_gated_args& a, bool fast, hipStream_t s);     // fast: rows of x, gate and up are whole aligned 16-byte pieces

}  // namespace mure
