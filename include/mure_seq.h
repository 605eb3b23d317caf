/*
 * mure_seq.h -- the operators of a selective state space block, over many
 * mutants at once, on one AMD Instinct MI355X (gfx950).
 *
 * The recurrent networks of today's language models consist of blocks that
 * are, between plain projections, a short causal convolution of every channel
 * along its sequence (mure_seq_conv), a selective scan (mure_seq_scan) and
 * the norms after the block and before the next one, fused with the gate and
 * the scaled residual sum (mure_seq_norm).  These calls compute them for a
 * whole test set and many mutants in one go: for prompts, and for single
 * tokens on states that an earlier call returned.
 *
 *   mure_create -> mure_seq_create (the test set's lengths)
 *     -> mure_seq_conv, mure_seq_scan, mure_seq_norm (any number of times)
 *     -> mure_seq_destroy -> mure_destroy
 *
 * Conventions (those of mure.h, and)
 *   - A batch of n_seq sequences is packed: sequence i's tokens are the rows
 *     start(i) .. start(i) + length(i) - 1 of every [tokens][channels] tensor,
 *     start(i) = the sum of the lengths before i.  A length may be 0: such a
 *     sequence has no rows and keeps its states.
 *   - The mutant axis.  Every tensor and parameter has a mutant stride, in
 *     elements: mutant m reads or writes at p + m * mutant_stride.  0: all
 *     mutants read the same values (a memoized activation of the original
 *     model, unmutated parameters).  Outputs hold every mutant's values.
 *   - A sequence's results depend on its own tokens, states and parameters
 *     only, bit for bit: not on the other sequences or mutants of the call,
 *     and not on alignment or strides.  So a mutant that is evaluated alone,
 *     or without memoization, gets the same results.
 *   - Arithmetic is float32; values are rounded to the tensors' type once,
 *     when they are stored.
 *   - Calls enqueue on the context's stream and return: device outputs are
 *     complete when the stream has got there.  Tensors that other streams
 *     write or read are ordered by the caller.
 *   - Inputs may overlap each other.  An output may overlap neither an input
 *     nor another output, but where a call says so.
 *   - On a planning-only context the calls check their arguments and return
 *     MURE_E_UNSUPPORTED where they would launch.
 *   - Every call but mure_seq_create may be captured into a HIP graph, which
 *     holds until the batch is destroyed.  Scans of sequences of more than
 *     MURE_SEQ_SPLIT_TOKENS tokens need a workspace: a batch has one for the
 *     calls made directly, which grows with them, and one for each capture, kept
 *     until the batch is destroyed.  So graphs may be replayed beside each other
 *     and beside other calls, as far as their tensors allow it.
 */
#ifndef MURE_SEQ_H
#define MURE_SEQ_H

#include "mure.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MURE_SEQ_VERSION 1
#define MURE_SEQ_MAX_TAPS 8        /* taps of a convolution */
#define MURE_SEQ_MAX_STATES 64     /* states per channel of a scan */
#define MURE_SEQ_MAX_WIDTH 16384   /* channels of a norm */
#define MURE_SEQ_MAX_CHANNELS (1 << 20)   /* channels of a convolution, of a scan */
#define MURE_SEQ_MAX_MUTANTS 65535
/* A sequence of more tokens than this is scanned in chunks that run side by
 * side (by its own length alone, so that its results do not depend on the
 * batch); 16 384 tokens are 128 chunks. */
#define MURE_SEQ_SPLIT_TOKENS 512

/* A batch of sequences: their lengths and work lists, on the context's GPU. */
typedef struct mure_seq mure_seq;

/* A tensor of rows: element (mutant m, row r, channel c) is
 * p[m * mutant_stride + r * row_stride + c].  Strides are in elements, >= 0;
 * an output's rows are apart from each other (row_stride >= channels, and the
 * mutants' rows do not meet). */
typedef struct {
  const void* p;
  int64_t mutant_stride, row_stride;
} mure_seq_in;

typedef struct {
  void* p;
  int64_t mutant_stride, row_stride;
} mure_seq_out;

/* A float32 parameter array, dense for one mutant; p = NULL where optional. */
typedef struct {
  const float* p;
  int64_t mutant_stride;
} mure_seq_param;

typedef enum { MURE_SEQ_LINEAR = 0, MURE_SEQ_SILU = 1, MURE_SEQ_SIGMOID = 2 } mure_seq_activation;

/* Register n_seq (1 .. 2^20) sequences of lengths[i] >= 0 tokens (host array,
 * fewer than 2^31 in all).  *out receives the batch, owned by the caller until
 * mure_seq_destroy; it must be destroyed before its context.  Synchronises the
 * context's stream.  Errors: MURE_E_INVALID, MURE_E_NOMEM. */
mure_status mure_seq_create(mure_ctx* ctx, int64_t n_seq, const int64_t* lengths, mure_seq** out);

/* Causal depthwise convolution of K = taps taps along every sequence:
 *   out[t][c] = act(bias[c] + sum_{k < K} taps[c][k] x[t - K + 1 + k][c]),
 * t the position in the sequence; x at position p < 0 is row K - 1 + p of the
 * sequence's state, or 0 without one.  state_out receives the last K - 1 rows
 * of (state, x): the state for the sequence's next tokens.
 * dtype: of x, taps, state, out and state_out.  activation: LINEAR or SILU.
 * taps: [channels][K]; state, state_out: [n_seq][K - 1][channels], dense for
 * one mutant, each may be NULL.  state_out may be the state (same pointer and
 * mutant stride, not shared by several mutants): it is updated in place.
 * K = 1 has no state: both are ignored. */
typedef struct {
  int32_t dtype, n_mutants, channels, n_taps, activation, reserved;
  mure_seq_in x;
  const void* taps;
  int64_t taps_mutant_stride;
  mure_seq_param bias;               /* [channels], optional */
  const void* state;
  int64_t state_mutant_stride;
  void* state_out;
  int64_t state_out_mutant_stride;
  mure_seq_out out;
} mure_seq_conv_args;
mure_status mure_seq_conv(mure_seq* seq, const mure_seq_conv_args* args);

/* Selective scan: per channel d of group g(d) = d / (channels / groups) and
 * state n < N = states, along every sequence, with
 *   D    = softplus(dt[t][d] + dt_bias[d])    (softplus = 0: without softplus)
 *   h[n] = exp(D a[d][n]) h[n] + D u[t][d] b[t][g(d)][n]
 *   out[t][d] = (sum_n c[t][g(d)][n] h[n] + skip[d] u[t][d]) silu(gate[t][d])
 * from the sequence's state (or 0), whose last value goes to state_out.
 * The rates a and the steps may have either sign.  A state past float32's
 * range is infinite.  What is or becomes infinite goes on by the arithmetic of
 * infinities: NaN after a decay that underflows to 0 or with an infinite term
 * of the other sign (in a long sequence also one summed up over a chunk).
 * dtype: of u, dt, b, c, gate and out.  b, c: rows of groups * states.
 * a: float32 [channels][states]; skip, dt_bias, gate (p = NULL) optional.
 * state, state_out: float32 [n_seq][channels][states], dense for one mutant,
 * each may be NULL.  state_out may be the state, as in mure_seq_conv.
 * MURE_E_UNSUPPORTED where channels (rounded up to 64 in each group) times
 * n_mutants is 2^30 or more. */
typedef struct {
  int32_t dtype, n_mutants, channels, states, groups, softplus;
  mure_seq_in u, dt, b, c, gate;
  mure_seq_param a, skip, dt_bias;
  const float* state;
  int64_t state_mutant_stride;
  float* state_out;
  int64_t state_out_mutant_stride;
  mure_seq_out out;
} mure_seq_scan_args;
mure_status mure_seq_scan(mure_seq* seq, const mure_seq_scan_args* args);

typedef enum { MURE_SEQ_NO_NORM = 0, MURE_SEQ_RMS = 1, MURE_SEQ_LAYER = 2 } mure_seq_norm_kind;

/* The norms after a block and before the next, with the block's gate and the
 * scaled residual sum, row by row over `rows` rows:
 *   v = y, times act(gate) where gate_at = 1
 *   v = after(v)                              (after: kind, weight, bias)
 *   v = v times act(gate) where gate_at = 2
 *   r = residual + scale v                    (scale: scalar times scale[c])
 *   residual_out = r,   out = before(r)       (before: kind, weight, bias)
 * with RMS(v) = v / sqrt(mean(v^2) + eps) and LAYER(v) the same of v - mean(v),
 * times the weight, plus the bias, where given.  `before` reads r before it is
 * rounded.  residual (p = NULL) counts as 0.  residual_out and out are each
 * optional (p = NULL), not both; out needs a `before`.
 * dtype: of y, gate and out; residual_dtype: of residual and residual_out.
 * residual_out may be the residual, and out may be y or the gate (same
 * pointer, type and strides, not shared by several mutants). */
typedef struct {
  int32_t dtype, residual_dtype, n_mutants, channels;
  int64_t rows;
  int32_t gate_at, gate_activation, after, before;
  float eps, scale_all;
  mure_seq_in y, gate, residual;
  mure_seq_param after_weight, after_bias, scale, before_weight, before_bias;
  mure_seq_out residual_out, out;
} mure_seq_norm_args;
mure_status mure_seq_norm(mure_ctx* ctx, const mure_seq_norm_args* args);

/* Release the batch.  NULL is ignored.  Waits for the context's stream; one that
 * is being captured stays so. */
void mure_seq_destroy(mure_seq* seq);

int32_t mure_seq_version(void);

#ifdef __cplusplus
}
#endif

#endif /* MURE_SEQ_H */
