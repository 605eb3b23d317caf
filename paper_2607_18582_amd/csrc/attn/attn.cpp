// C ABI of the operators of an attention block (mure_attn.h): checks of a
// call's arguments, workspaces and launches.
#include "attn.hpp"

#include "../seq/batch.hpp"

#include <algorithm>
#include <cmath>

using namespace mure;

namespace {

constexpr int64_t GRID = (1 << 24) - 1;        // blocks of a launch: a grid has fewer than 2^32 threads
constexpr int64_t PARTS_BYTES = 1 << 30;       // of a workspace for parts of keys, or as many as one head's run needs

// ---- norm and rotation

void rotate(mure_seq* s, const mure_attn_rotate_args* args) {
  if (!args) invalid("args is NULL");
  AttnRotateArgs k;
  k.a = *args;
  mure_attn_rotate_args& a = k.a;
  const int64_t es = esize_of(a.dtype, "dtype");
  check_range(a.n_mutants, 1, MURE_SEQ_MAX_MUTANTS, "n_mutants");
  check_range(a.q_heads, 1, MURE_ATTN_MAX_HEADS, "q_heads");
  check_range(a.k_heads, 0, MURE_ATTN_MAX_HEADS, "k_heads");
  check_range(a.head_dim, 1, MURE_ATTN_MAX_HEAD, "head_dim");
  check_range(a.rotated, 0, a.head_dim, "rotated");
  if (a.rotated % 2) invalid("rotated is odd");
  check_range(a.norm, 0, MURE_SEQ_LAYER, "norm");
  check_range(a.interleaved, 0, 1, "interleaved");
  if (!(a.eps >= 0.f) || !std::isfinite(a.eps)) invalid("eps is no finite value >= 0");
  if (!a.norm && (a.q_weight.p || a.k_weight.p)) invalid("a weight without a norm");
  if (!a.k_heads && a.k_weight.p) invalid("k_weight without keys");
  const int64_t M = a.n_mutants, D = a.head_dim, T = s->tokens;
  if (a.positions) {
    check_range(a.axes, 1, MURE_ATTN_MAX_AXES, "axes");
    int64_t sum = 0;
    for (int x = 0; x < a.axes; ++x) {
      check_range(a.section[x], 0, a.rotated / 2, "a section");
      sum += a.section[x];
    }
    if (sum != a.rotated / 2) invalid("the sections are " + std::to_string(sum) + " pairs, rotated / 2 is " + std::to_string(a.rotated / 2));
    if (a.past) invalid("positions and past exclude each other");
  } else {
    a.axes = 1;
    a.section[0] = a.rotated / 2;
  }
  Spans in;
  const Span q = span("q", a.q.p, es, a.q_heads * D, T, a.q.row_stride, M, a.q.mutant_stride);
  in.push_back(q);
  Span key{};
  if (a.k_heads) in.push_back(key = span("k", a.k.p, es, a.k_heads * D, T, a.k.row_stride, M, a.k.mutant_stride));
  add_param(in, "q_weight", a.q_weight, D, M);
  if (a.k_heads) add_param(in, "k_weight", a.k_weight, D, M);
  if (a.rotated) in.push_back(span("frequencies", a.frequencies.p, 4, a.rotated / 2, 1, 0, M, a.frequencies.mutant_stride));
  if (a.positions) in.push_back(span("positions", a.positions, 4, a.axes * T, 1, 0, 1, 0));
  if (a.past) in.push_back(span("past", a.past, 4, s->n_seq, 1, 0, 1, 0));
  const Span qo = span("q_out", a.q_out.p, es, a.q_heads * D, T, a.q_out.row_stride, M, a.q_out.mutant_stride);
  check_output(qo);
  check_apart(qo, in, {&q});
  if (a.k_heads) {
    const Span ko = span("k_out", a.k_out.p, es, a.k_heads * D, T, a.k_out.row_stride, M, a.k_out.mutant_stride);
    check_output(ko);
    check_apart(ko, in, {&key});
    if (meet(ko, qo)) invalid("k_out overlaps q_out");
  }
  check_device(s->device);
  if (T == 0) return;
  // Runs of 12 tokens, or of 3 where those are few: a run's angles are computed once for all heads.  16 and 4 heads of 128
  // bfloat16 channels, norm: 40 sequences of 24 tokens take 10.9 us in runs of 12 and 6.4 in runs of 3, 8 of 500 12.9 and
  // 12.6, 12 of 1000 23.9 and 26.8; 65536 tokens 102 and 130.
  const int w = s->n_conv[2] && s->n_conv[1] * M < 512 ? 2 : s->n_conv[1] ? 1 : 0;
  k.items = s->conv[w];
  k.n_items = s->n_conv[w];
  k.longest = CONV_RUNS[w];
  k.tokens = T;
  check(launch_attn_rotate(k, s->stream), "mure_attn_rotate");
}

// ---- attention

// The rows of a cache, of every sequence and mutant.
Span cache_span(const char* name, const mure_attn_cache& c, int64_t es, int64_t width, int64_t capacity, int64_t n_seq, int64_t M) {
  if (c.seq_stride < 0) invalid(std::string(name) + ": a stride is negative");
  Span s = span(name, c.p, es, width, capacity, c.row_stride, M, c.mutant_stride);
  s.outers = n_seq;
  s.outer_stride = n_seq > 1 ? c.seq_stride : 0;
  if (s.extent() > MOST) invalid(std::string(name) + ": its strides pass the address space");
  // every row apart from the others, whichever axis goes around which
  struct Axis { wide stride, n; } axes[3] = {{s.row_stride, s.rows}, {s.outer_stride, s.outers}, {s.mutant_stride, c.mutant_stride ? s.mutants : 1}};
  std::sort(axes, axes + 3, [](const Axis& a, const Axis& b) { return a.stride < b.stride; });
  wide extent = width;
  for (const Axis& x : axes) {
    if (x.n <= 1) continue;
    if (x.stride < extent) invalid(std::string(name) + ": its rows overlap");
    extent += (x.n - 1) * x.stride;
  }
  return s;
}

// Whether `bytes` divides the address and strides (the first between rows) of rows, 64 of which lie within 2^31 bytes.
bool aligned(int64_t bytes, const void* p, int64_t es, std::initializer_list<int64_t> strides) {
  bool ok = reinterpret_cast<uintptr_t>(p) % bytes == 0 && *strides.begin() * es < 1 << 24;
  for (int64_t v : strides) ok = ok && v * es % bytes == 0;
  return ok;
}

// The call's mutants m0 ... m0 + ms - 1 and heads h0 ... h0 + hs - 1 of them: whole groups, or some of one.
AttnArgs some_of(const AttnArgs& k, int64_t es, int64_t m0, int64_t ms, int64_t h0, int64_t hs) {
  AttnArgs p = k;
  const mure_attn_attend_args& a = k.a;
  const int64_t group = a.heads / a.kv_heads, g0 = h0 / group, D = a.head_dim;
  const auto move = [&](auto& rows, int64_t head) {
    if (rows.p) rows.p = const_cast<char*>(static_cast<const char*>(rows.p)) + (m0 * rows.mutant_stride + head * D) * es;
  };
  move(p.a.q, h0);
  move(p.a.out, h0);
  for (mure_seq_in* t : {&p.a.k, &p.a.v}) move(*t, g0);
  for (mure_attn_cache* t : {&p.a.k_cache, &p.a.v_cache}) move(*t, g0);
  p.a.n_mutants = (int32_t)ms;
  p.a.heads = (int32_t)hs;
  p.a.kv_heads = (int32_t)std::max<int64_t>(1, hs / group);
  return p;
}

void attend(mure_seq* s, const mure_attn_attend_args* args) {
  if (!args) invalid("args is NULL");
  AttnArgs k;
  k.a = *args;
  mure_attn_attend_args& a = k.a;
  const int64_t es = esize_of(a.dtype, "dtype");
  check_range(a.n_mutants, 1, MURE_SEQ_MAX_MUTANTS, "n_mutants");
  check_range(a.heads, 1, MURE_ATTN_MAX_HEADS, "heads");
  check_range(a.kv_heads, 1, a.heads, "kv_heads");
  if (a.heads % a.kv_heads) invalid("heads is no multiple of kv_heads");
  check_range(a.head_dim, 1, MURE_ATTN_MAX_HEAD, "head_dim");
  check_range(a.causal, 0, 1, "causal");
  if (a.window < 0) invalid("window is negative");
  a.window = std::min(a.window, (int64_t)1 << 32);             // further than any key
  if (!std::isfinite(a.scale)) invalid("scale is not finite");
  if (a.reserved) invalid("reserved must be 0");
  const int64_t M = a.n_mutants, D = a.head_dim, T = s->tokens, W = a.kv_heads * D;
  const bool held = a.k_cache.p || a.v_cache.p;
  Spans in;
  in.push_back(span("q", a.q.p, es, a.heads * D, T, a.q.row_stride, M, a.q.mutant_stride));
  in.push_back(span("k", a.k.p, es, W, T, a.k.row_stride, M, a.k.mutant_stride));
  in.push_back(span("v", a.v.p, es, W, T, a.v.row_stride, M, a.v.mutant_stride));
  if (!held && a.past) invalid("past without caches");
  if (a.past) in.push_back(span("past", a.past, 4, s->n_seq, 1, 0, 1, 0));
  const Span out = span("out", a.out.p, es, a.heads * D, T, a.out.row_stride, M, a.out.mutant_stride);
  check_output(out);
  check_apart(out, in);
  if (held) {
    if (!a.k_cache.p || !a.v_cache.p) invalid("k_cache and v_cache go together");
    check_range(a.capacity, 1, INT32_MAX, "capacity");
    const Span kc = cache_span("k_cache", a.k_cache, es, W, a.capacity, s->n_seq, M);
    const Span vc = cache_span("v_cache", a.v_cache, es, W, a.capacity, s->n_seq, M);
    if (M > 1 && ((a.k_cache.mutant_stride == 0 && a.k.mutant_stride) || (a.v_cache.mutant_stride == 0 && a.v.mutant_stride)))
      invalid("a cache that all mutants share needs k and v that they share");
    check_apart(kc, in);
    check_apart(vc, in);
    if (meet(kc, vc)) invalid("v_cache overlaps k_cache");
    if (meet(kc, out) || meet(vc, out)) invalid("out overlaps a cache");
  } else {
    a.capacity = 0;
  }
  const int64_t parts_short = held ? (a.capacity + ATTN_KEYS_SHORT - 1) / ATTN_KEYS_SHORT : 1;
  const int64_t parts_mid = held ? (a.capacity + ATTN_KEYS_MID - 1) / ATTN_KEYS_MID : 1;
  // the kernels count keys, and the blocks of one head's parts, in 32 bits
  if (a.capacity > MURE_ATTN_MAX_ROWS) throw Fail{MURE_E_UNSUPPORTED, "too many rows of a cache: 2^30 at most"};
  check_device(s->device);
  if (T == 0) return;
  if (T == 1) a.k.row_stride = a.v.row_stride = W;             // one row has no stride
  // A copied tile's buffer ends with its last row, and what lies behind a row reads as zeros: rows that begin inside the one
  // before them go element by element.
  const auto reads = [&](int64_t bytes) {
    return D * es % bytes == 0 && a.k.row_stride >= D && a.v.row_stride >= D && aligned(bytes, a.k.p, es, {a.k.row_stride, a.k.mutant_stride}) && aligned(bytes, a.v.p, es, {a.v.row_stride, a.v.mutant_stride}) &&
           (!held || (aligned(bytes, a.k_cache.p, es, {a.k_cache.row_stride, a.k_cache.seq_stride, a.k_cache.mutant_stride}) &&
                      aligned(bytes, a.v_cache.p, es, {a.v_cache.row_stride, a.v_cache.seq_stride, a.v_cache.mutant_stride})));
  };
  k.fast = reads(16) ? PIECES : D * es >= 16 && reads(4) ? WORDS : ELEMENTS;
  const bool f32 = a.dtype == MURE_F32;
  const auto launch_short = f32 ? attn_short_f32 : attn_short_bf16;
  const auto launch_runs = f32 ? attn_runs_f32 : attn_runs_bf16;
  const auto launch_join = f32 ? attn_join_f32 : attn_join_bf16;
  // Items of at most `longest` tokens, their keys in parts of `keys`: as many mutants and heads a round as one item may have
  // blocks for; with several parts, which are joined from the workspace, as many items as it has room for, or of one
  // item as many mutants, or heads.  `blocks`: of an item, mutants and heads.
  auto rounds = [&](const SeqItem* items, int first, int n, int64_t parts, int64_t longest, int keys, auto run, auto blocks) {
    const int64_t group = a.heads / a.kv_heads;
    int64_t most = n, mutants = M, heads = a.heads;            // a round's
    if (n == 0) return;
    float* work = nullptr;
    int64_t slots = 0;
    if (parts > 1) {
      const int64_t each = longest * parts * (D + 2) * 4;      // of an item, mutant and head
      const int64_t fit = std::max<int64_t>(1, PARTS_BYTES / each);
      if (fit < heads) heads = fit < group ? fit : fit / group * group, mutants = most = 1;
      else if (fit < heads * M) mutants = fit / heads, most = 1;
      else most = std::min(most, fit / (heads * M));
    }
    if (blocks(mutants, heads) > GRID) {
      while (blocks(1, heads) > GRID) heads = heads > group ? (heads / group + 1) / 2 * group : (heads + 1) / 2;
      mutants = std::min(mutants, GRID / blocks(1, heads));
    }
    if (parts > 1) {
      slots = most * mutants * heads * longest * parts;
      void* p = nullptr;
      check(s->work.get(s->stream, (size_t)(slots * (D + 2) * 4), &p), "attention workspace");
      work = static_cast<float*>(p);
    }
    for (int64_t h0 = 0, hs; h0 < a.heads; h0 += hs) {
      hs = heads < group ? std::min(heads, group - h0 % group) : std::min(heads, a.heads - h0);
      for (int64_t m0 = 0; m0 < M; m0 += mutants)
        for (int64_t i = 0; i < n; i += most) {
          AttnArgs p = some_of(k, es, m0, std::min(mutants, M - m0), h0, hs);
          p.items = items;
          p.parts = (int)parts;
          p.rows_each = p.longest = (int)longest;
          p.ws_ml = work;
          p.ws_o = work + 2 * slots;
          p.first = (int)(first + i);
          p.n_items = (int)std::min(most, n - i);
          check(run(p, s->stream), "mure_attn_attend");
          if (parts > 1) check(launch_join(p, keys, s->stream), "mure_attn_attend");
        }
    }
  };
  const int64_t group = a.heads / a.kv_heads;
  const auto run_blocks = [](int64_t parts) { return [=](int64_t mutants, int64_t heads) { return mutants * heads * parts; }; };
  const auto short_blocks = [&](int64_t longest, int64_t parts) {
    return [=](int64_t mutants, int64_t heads) {
      const int64_t shared = std::min(group, heads);
      return mutants * (heads / shared) * ((longest * shared + 15) / 16) * parts;
    };
  };
  if (!held) {
    rounds(s->brief, 0, s->n_brief, 1, s->longest_brief, 0, launch_short, short_blocks(s->longest_brief, 1));
    rounds(s->runs, 0, s->n_runs - s->n_small_runs, 1, ATTN_ROWS, 0, launch_runs, run_blocks(1));
    return;
  }
  // one after the other: the workspace serves all
  rounds(s->brief, s->n_brief - s->n_short, s->n_short, parts_short, s->longest_short, ATTN_KEYS_SHORT, launch_short, short_blocks(s->longest_short, parts_short));
  // without parts the longer sequences' runs and the others' go in one launch
  const int n_mid = s->n_runs - s->n_long_runs;
  const bool split = parts_mid > 1 && n_mid;
  rounds(s->runs, 0, split ? s->n_long_runs : s->n_runs, 1, ATTN_ROWS, 0, launch_runs, run_blocks(1));
  if (split) rounds(s->runs, s->n_long_runs, n_mid, parts_mid, s->longest_mid_run, ATTN_KEYS_MID, launch_runs, run_blocks(parts_mid));
}

// ---- gated feed-forward layer

void gated(mure_ctx* ctx, const mure_attn_gated_args* args) {
  if (!args) invalid("args is NULL");
  mure_attn_gated_args a = *args;
  const int64_t es = esize_of(a.dtype, "dtype");
  check_range(a.n_mutants, 1, MURE_SEQ_MAX_MUTANTS, "n_mutants");
  check_range(a.inner, 1, MURE_SEQ_MAX_CHANNELS, "inner");
  check_range(a.outer, 1, MURE_SEQ_MAX_CHANNELS, "outer");
  check_range(a.rows, 0, INT32_MAX, "rows");
  check_range(a.activation, 0, MURE_ATTN_GELU_TANH, "activation");
  if (a.reserved) invalid("reserved must be 0");
  const int64_t M = a.n_mutants, K = a.inner, N = a.outer, R = a.rows;
  Spans in;
  in.push_back(span("x", a.x.p, es, K, R, a.x.row_stride, M, a.x.mutant_stride));
  in.push_back(span("gate", a.gate.p, es, K, N, a.gate.row_stride, M, a.gate.mutant_stride));
  in.push_back(span("up", a.up.p, es, K, N, a.up.row_stride, M, a.up.mutant_stride));
  add_param(in, "gate_bias", a.gate_bias, N, M);
  add_param(in, "up_bias", a.up_bias, N, M);
  const Span out = span("out", a.out.p, es, N, R, a.out.row_stride, M, a.out.mutant_stride);
  check_output(out);
  check_apart(out, in);
  const CtxView cv = ctx_view(ctx);
  check_device(cv.device);
  if (R == 0) return;
  const bool fast = K * es % 16 == 0 && aligned(16, a.x.p, es, {a.x.row_stride, a.x.mutant_stride}) &&
                    aligned(16, a.gate.p, es, {a.gate.row_stride, a.gate.mutant_stride}) && aligned(16, a.up.p, es, {a.up.row_stride, a.up.mutant_stride});
  check(launch_attn_gated(a, fast, cv.stream), "mure_attn_gated");
}

}  // namespace

// =========================================================================
extern "C" {

int32_t mure_attn_version(void) { return MURE_ATTN_VERSION; }

mure_status mure_attn_rotate(mure_seq* seq, const mure_attn_rotate_args* args) {
  if (!seq) return MURE_E_INVALID;
  return guarded(seq->ctx, [&] { rotate(seq, args); });
}

mure_status mure_attn_attend(mure_seq* seq, const mure_attn_attend_args* args) {
  if (!seq) return MURE_E_INVALID;
  return guarded(seq->ctx, [&] { attend(seq, args); });
}

mure_status mure_attn_gated(mure_ctx* ctx, const mure_attn_gated_args* args) {
  if (!ctx) return MURE_E_INVALID;
  return guarded(ctx, [&] { gated(ctx, args); });
}

}  // extern "C"
