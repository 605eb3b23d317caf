/*
 * mure_attn.h -- the operators of an attention block, over many mutants at
 * once, on one AMD Instinct MI355X (gfx950).
 *
 * Between plain projections and the norms of mure_seq.h, such a block norms
 * and rotates the queries and keys of every head (mure_attn_rotate), weighs
 * the values of a sequence's tokens (mure_attn_attend) and has a gated
 * feed-forward layer (mure_attn_gated).  These calls compute them for a whole
 * test set and many mutants in one go: for whole sequences, and for further
 * tokens over a cache of the earlier ones' keys and values.
 *
 *   mure_create -> mure_seq_create (the test set's lengths)
 *     -> mure_attn_rotate, mure_attn_attend, mure_attn_gated, and the calls
 *        of mure_seq.h (any number of times)
 *     -> mure_seq_destroy -> mure_destroy
 *
 * The conventions are those of mure_seq.h: packed sequences, the mutant axis,
 * strides, overlap, streams, planning-only contexts, captures.  In particular
 *   - a sequence's results (a row's, of mure_attn_gated) depend on its own
 *     tokens, past and parameters only, bit for bit.  Attention's sums follow
 *     from the sequence's lengths in this call and before it, and from whether
 *     there is a cache, so that a token may round differently when the same
 *     tokens come in other calls;
 *   - arithmetic is float32.  Values are rounded to the tensors' type once,
 *     when they are stored; in bfloat16 so is the weight of every key and
 *     value before it meets the value.
 */
#ifndef MURE_ATTN_H
#define MURE_ATTN_H

#include "mure_seq.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MURE_ATTN_VERSION 1
#define MURE_ATTN_MAX_HEAD 256     /* channels of a head */
#define MURE_ATTN_MAX_HEADS 1024
#define MURE_ATTN_MAX_AXES 4       /* axes of a position */
#define MURE_ATTN_MAX_ROWS (1 << 30)   /* rows of a sequence's cache */

/* Norm and rotation of queries and keys.  For every token and head, with
 * v = norm(head's channels) (norm: MURE_SEQ_NO_NORM, MURE_SEQ_RMS or
 * MURE_SEQ_LAYER of mure_seq.h over head_dim channels, times the weight where
 * given), pair i < rotated / 2 of channels turns by the angle
 * f = position * frequencies[i]:
 *   (a, b) -> (a cos f - b sin f, a sin f + b cos f);
 * the pair is channels (i, i + rotated / 2), or (2 i, 2 i + 1) where
 * interleaved.  Channels from `rotated` on stay as they are in v.
 * Without `positions` a token's position is past[its sequence] (NULL: 0) plus
 * its place in the sequence.  positions: int32 [axes][tokens]; section[x] pairs
 * turn by axis x's position, in order (their sum is rotated / 2).
 * Angles are products in float64; they are good to float32 up to 2^33.
 * dtype: of q, k and their outputs; rows of q_heads * head_dim and
 * k_heads * head_dim channels.  k_heads = 0: no keys, no k_weight.  frequencies: float32
 * [rotated / 2], rotated even, <= head_dim (0: none turns).  q_weight, k_weight: [head_dim],
 * optional.  q_out may be q and k_out may be k (same pointer and strides, not
 * shared by several mutants). */
typedef struct {
  int32_t dtype, n_mutants, q_heads, k_heads, head_dim, rotated, norm, interleaved;
  int32_t axes, section[MURE_ATTN_MAX_AXES];
  float eps;
  mure_seq_in q, k;
  mure_seq_param q_weight, k_weight, frequencies;
  const int32_t* positions;          /* [axes][tokens], optional; all mutants' */
  const int32_t* past;               /* [n_seq], optional; all mutants' */
  mure_seq_out q_out, k_out;
} mure_attn_rotate_args;
mure_status mure_attn_rotate(mure_seq* seq, const mure_attn_rotate_args* args);

/* The keys (or values) of earlier tokens: row r of sequence i for mutant m is
 * at p + m * mutant_stride + i * seq_stride + r * row_stride (in elements),
 * kv_heads * head_dim elements. */
typedef struct {
  void* p;
  int64_t mutant_stride, seq_stride, row_stride;
} mure_attn_cache;

/* Attention.  For every token t and head h, of group g = h / (heads / kv_heads):
 *   out[t][h] = sum_j w_j v[j][g] / sum_j w_j,   w_j = exp(scale q[t][h] . k[j][g])
 * over the keys j of t's sequence that t sees: all of them, or those up to t
 * itself (causal), and with window > 0 those fewer than `window` places away.
 * With a cache (k_cache.p not NULL) a sequence's first past[i] keys and values
 * are its cache's first rows (past NULL: none), the call's own follow, and the
 * call writes those to the rows past[i] .. of the caches.  Where past[i] < 0 or
 * past[i] + length(i) > capacity, the sequence's results are NaN and its
 * caches are left alone.  Rows of a cache that hold no key are not read.
 * What is NaN or infinite goes on by the arithmetic of the formula to those
 * tokens that see it, and to no other: an infinite value makes a token's result
 * infinite (or NaN, beside one of the other sign) however small its weight is.
 * Over caches of more than 512 rows parts of the keys meet in the batch's
 * workspace (mure_seq.h).  A call takes 1 GiB of it at most (more only where
 * one head of one sequence needs it): where it would need more, it takes
 * sequences, mutants or heads in rounds.
 * dtype: of q, k, v, the caches and out.  All mutants may share a cache
 * (mutant stride 0) where they share k and v too.  k_cache and v_cache overlap
 * no other tensor and no row of their own. */
typedef struct {
  int32_t dtype, n_mutants, heads, kv_heads, head_dim, causal;
  int64_t window;
  float scale;
  int32_t reserved;
  mure_seq_in q, k, v;
  mure_attn_cache k_cache, v_cache;
  int64_t capacity;                  /* rows of a sequence's cache, 1 .. 2^31 - 1; more than
                                        MURE_ATTN_MAX_ROWS: MURE_E_UNSUPPORTED */
  const int32_t* past;               /* [n_seq], device memory, optional */
  mure_seq_out out;
} mure_attn_attend_args;
mure_status mure_attn_attend(mure_seq* seq, const mure_attn_attend_args* args);

typedef enum {
  MURE_ATTN_LINEAR = 0, MURE_ATTN_SILU = 1, MURE_ATTN_SIGMOID = 2,   /* as MURE_SEQ_... */
  MURE_ATTN_RELU = 3,
  MURE_ATTN_GELU = 4,                /* a (1 + erf(a / sqrt 2)) / 2 */
  MURE_ATTN_GELU_TANH = 5            /* a (1 + tanh(sqrt(2 / pi) (a + 0.044715 a^3))) / 2 */
} mure_attn_activation;

/* Gated feed-forward layer, row by row over `rows` rows:
 *   out[r][n] = act(sum_k x[r][k] gate[n][k] + gate_bias[n]) (sum_k x[r][k] up[n][k] + up_bias[n])
 * dtype: of x, gate, up and out.  gate, up: [outer][inner], rows at any stride.
 * gate_bias, up_bias: [outer], each optional. */
typedef struct {
  int32_t dtype, n_mutants, inner, outer, activation, reserved;
  int64_t rows;
  mure_seq_in x, gate, up;
  mure_seq_param gate_bias, up_bias;
  mure_seq_out out;
} mure_attn_gated_args;
mure_status mure_attn_gated(mure_ctx* ctx, const mure_attn_gated_args* args);

int32_t mure_attn_version(void);

#ifdef __cplusplus
}
#endif

#endif /* MURE_ATTN_H */
