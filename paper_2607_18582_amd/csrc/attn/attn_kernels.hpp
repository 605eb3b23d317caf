// Kernels of attention (mure_attn_attend) and their launches, for one type of
// tensors (compiled in a source of its own each).
#pragma once

#include "attn_dev.hpp"

#include <algorithm>

namespace mure {

// One sequence's rows of keys and values of a head of one mutant.
template <typename T> struct Source {
  Rows<T> k, v;
  int past, total;
  bool bad;                                    // its past does not fit the cache
  __device__ __forceinline__ Source(const AttnArgs& k_, const SeqItem& it, int m, int g) {
    const mure_attn_attend_args& a = k_.a;
    const bool held = a.k_cache.p;
    past = uniform(held && a.past ? a.past[it.seq] : 0);
    bad = held && (past < 0 || past > a.capacity - it.total);
    total = past + it.total;
    const int64_t row = it.row0 - it.pos0, c = (int64_t)g * a.head_dim;
    k.past = v.past = past;
    k.own = static_cast<const T*>(a.k.p) + m * a.k.mutant_stride + row * a.k.row_stride + c;
    v.own = static_cast<const T*>(a.v.p) + m * a.v.mutant_stride + row * a.v.row_stride + c;
    k.own_stride = a.k.row_stride;
    v.own_stride = a.v.row_stride;
    k.held = static_cast<const T*>(a.k_cache.p) + m * a.k_cache.mutant_stride + it.seq * a.k_cache.seq_stride + c;
    v.held = static_cast<const T*>(a.v_cache.p) + m * a.v_cache.mutant_stride + it.seq * a.v_cache.seq_stride + c;
    k.held_stride = a.k_cache.row_stride;
    v.held_stride = a.v_cache.row_stride;
  }
  // The run's own keys and values into the cache; the call reads them from where they come from.
  __device__ __forceinline__ void keep(const mure_attn_attend_args& a, const SeqItem& it, int m, int tid, int threads) const {
    if (m && !a.k_cache.mutant_stride && !a.v_cache.mutant_stride) return;
    const bool keep_k = !m || a.k_cache.mutant_stride, keep_v = !m || a.v_cache.mutant_stride;
    constexpr int E = 16 / sizeof(T);
    const int per = (a.head_dim + E - 1) / E;
    for (int i = tid; i < it.len * per; i += threads) {
      const int t = i / per, e = i % per * E, j = past + it.pos0 + t;
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        if (!(which ? keep_v : keep_k)) continue;
        const Rows<T>& r = which ? v : k;
        const T* from = r.at(j);
        T* to = const_cast<T*>(r.held) + j * r.held_stride;
        if (e + E <= a.head_dim) {
          *reinterpret_cast<v4u_any*>(to + e) = *reinterpret_cast<const v4u_any*>(from + e);
        } else {
          for (int x = e; x < a.head_dim; ++x) to[x] = from[x];
        }
      }
    }
  }
};

// A wave's own reads and writes of LDS before this are done.
__device__ __forceinline__ void settle() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

__device__ __forceinline__ SeqItem item_of(const AttnArgs& k, int i) {
  const SeqItem it = seq_item(k.items, k.first + i);
  return {uniform(it.seq), uniform(it.row0), uniform(it.len), uniform(it.pos0), uniform(it.total), it.slot};
}

// Head and mutant number i of n: neighbouring blocks go to the chip's eight dies in turn, so each die gets neighbouring
// heads, which share keys and values in its L2.
__device__ __forceinline__ int spread(int i, int n) { return n % 8 ? i : i % 8 * (n / 8) + i / 8; }

// ---- runs of tokens: one head, 128 tokens, 32 of them a wave; tiles of keys and values in LDS, two at a time
//
// Every 32 keys cost a wave as many cycles of matrix instructions as of others (an exponential, a multiply-add, a sum and
// half a maximum and a conversion per score).  Two waves on a SIMD overlap them by a fifth only, so a wave does it itself:
// the softmax of one block goes between the products of the next and of the last one.  16384 tokens, 16 heads of 4, 128
// bfloat16 channels, causal: 1.08 to 1.12 ms, about 1000 TFLOP/s, at which the chip lowers its clock to 1.7 GHz (one after the other,
// with the same tiles: 1.20 ms); on a card that is held to 1.6 GHz 1.23 to 1.27.  A batch of prompts is bound by its longest
// run, 1.5 us a tile of 64 keys.
//
// Heads of more than 128 channels leave one wave a SIMD, and their sums fill the accumulation registers: 4096 tokens of the
// same heads take 112 us with 128 channels, 294 with 192 and 409 with 256; in float32 809, 1184 and 4739, the last with 1.5 KB
// of scratch a lane.  Rows of whole words (126 channels: 309 us) and of elements (127: 761) have about 0.6 KB of it up to
// 128 bfloat16 channels.

template <typename T, int DB> struct Run {
  using H = Head<T, DB>;
  static constexpr int KT = H::ROW <= 256 ? 64 : 32;           // keys of a tile
  static constexpr int TILE = KT * H::ROW;
  static constexpr int LDS = 4 * TILE;         // keys twice, values twice
  static constexpr bool MIXED = sizeof(T) == 2 && DB <= 4;     // float32 is bound by its matrix instructions anyway
};

template <typename T, int DB, int FAST> __global__ __launch_bounds__(256, DB <= 4 ? 2 : 1) void run_kernel(AttnArgs k) {
  using R = Run<T, DB>;
  constexpr int KT = R::KT, KB = KT / 32;
  extern __shared__ char lds[];
  const mure_attn_attend_args& a = k.a;
  const int n = a.heads * a.n_mutants, at = uniform(blockIdx.x / n), hm = spread(blockIdx.x - at * n, n), m = uniform(hm / a.heads), h = hm - m * a.heads;
  const int group = uniform(a.heads / a.kv_heads), g = uniform(h / group), part = uniform(at % k.parts), i = k.item0 + uniform(at / k.parts);
  const SeqItem it = item_of(k, i);
  const Source<T> src(k, it, m, g);
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, half = lane >> 5;
  T* out = static_cast<T*>(a.out.p) + m * a.out.mutant_stride + it.row0 * a.out.row_stride + (int64_t)h * a.head_dim;
  if (src.bad) {
    if (part == 0)
      for (int x = tid; x < it.len * a.head_dim; x += 256) out[x / a.head_dim * a.out.row_stride + x % a.head_dim] = from_f<T>(__builtin_nanf(""));
    return;
  }
  if (a.k_cache.p && part == 0 && h % group == 0) src.keep(a, it, m, tid, 256);
  // keys that any row of the block sees, in this part
  const int first = src.past + it.pos0, last = first + it.len - 1;
  int from, to, block_lo, block_hi, none;      // ... and that all rows see
  sees(a, first, src.total, from, block_hi);
  sees(a, last, src.total, block_lo, to);
  if (k.parts > 1) {
    from = max(from, part * ATTN_KEYS_MID);
    to = (int)min((int64_t)to, (int64_t)(part + 1) * ATTN_KEYS_MID);
    if (from >= to) return;
  }
  const int row = wave * 32 + (lane & 31), pos = min(first + row, last);
  int lo, hi;
  sees(a, pos, src.total, lo, hi);
  // ... that any row of the wave sees, and that all of them see
  int any_lo, any_hi, wave_lo, wave_hi;
  sees(a, min(first + wave * 32, last), src.total, any_lo, wave_hi);
  sees(a, min(first + wave * 32 + 31, last), src.total, wave_lo, any_hi);
  wave_lo = max(wave_lo, from);
  wave_hi = min(wave_hi, to);
  Query<T, DB> q;
  load_query<T, Head<T, DB>::STEPS, 2>(q, static_cast<const T*>(a.q.p) + m * a.q.mutant_stride + (it.row0 + (int64_t)(pos - first)) * a.q.row_stride + (int64_t)h * a.head_dim,
                    a.head_dim, half, a.scale);
  const float c = factor(a.scale);
  Running<DB> run;
  run.start();
  const Reader<T, DB> read(lane);
  using Keys = Copy<T, DB, KT, 4, KEYS>;
  using Values = Copy<T, DB, KT, 4, VALUES32>;
  const int t0 = from / KT * KT, tiles = (to - t0 + KT - 1) / KT;
  const auto k_tile = [&](int i) { return lds + (i & 1) * R::TILE; };
  const auto v_tile = [&](int i) { return lds + (2 + (i & 1)) * R::TILE; };
  const auto load_k = [&](int i) { Keys::template run<FAST>(k_tile(i), src.k, t0 + i * KT, src.total, a.head_dim, wave, lane); };
  const auto load_v = [&](int i) { Values::template run<FAST>(v_tile(i), src.v, t0 + i * KT, src.total, a.head_dim, wave, lane); };
  const auto trim_k = [&](int i) {
    if constexpr (FAST == WORDS) Keys::trim(k_tile(i), a.head_dim, wave, lane);
  };
  const auto trim_v = [&](int i) {
    if constexpr (FAST == WORDS) Values::trim(v_tile(i), a.head_dim, wave, lane);
  };
  // Blocks of 32 keys, numbered from t0 on, of which the wave's rows see any: begin ... end - 1.
  const int begin = wave * 32 >= it.len ? 0 : (max(any_lo, from) - t0) / 32, end = wave * 32 >= it.len ? 0 : (min(any_hi, to) - t0 + 31) / 32;
  const auto seen = [&](int j) { return j >= begin && j < end; };
  // Scores of the block that is next and weights of the one before it, for even blocks and odd ones.
  v16f s[2] = {};
  Weights<T> w[2];
  // One step: the last block's values, the softmax of block j, the next block's scores.
  const auto step = [&](int j, v16f& mine, v16f& after, Weights<T>& before, Weights<T>& weights, const char* next, int next_at, const char* last, int last_at) {
    const int t = t0 + 32 * j;
    if (seen(j - 1)) run.template add<T>(read, last, last_at, before);
    if (seen(j)) {
      if (t < wave_lo || t + 32 > wave_hi) hide(mine, max(lo, from) - t, min(hi, to) - t, half);
      float old;
      if (__any(run.base_for(mine, c, old))) run.rescale(old);
      weights = run.template weigh<T>(mine, c);
    }
    if (seen(j + 1)) after = read.scores(next, next_at, q);
  };
  // The same with the products between the parts of the softmax, so that the matrix units and the others are busy at once,
  // where all rows of the wave see the three blocks.
  const auto mixed = [&](const v16f& mine, v16f& after, const Weights<T>& before, Weights<T>& weights, const char* next, int next_at, const char* last, int last_at) {
    float old;
    const bool grows = run.base_for(mine, c, old);
    if constexpr (R::MIXED) run.template mixed<T>(mine, c, weights, read, next, next_at, q, after, last, last_at, before);
    if (__any(grows)) run.rescale(old);
  };
  const auto aside = [&](int i) {              // whether values of tile i are hidden from some row of the block
    const int t = t0 + i * KT;
    return max(block_lo, from) > t || min(block_hi, to) < min(t + KT, src.total);
  };
  // Values of tile i that are not finite in places hidden from some row are put aside; its other rows get them at the end.
  int found = 0;
  const auto put_aside = [&](int i) {
    if (!aside(i)) return;
    const int t = t0 + i * KT, see_from = max(block_lo, from) - t, see_to = min(block_hi, to) - t, there = min(KT, src.total - t);
    char* tile = v_tile(i);
    const bool before = clean<T, DB>(tile, 0, min(see_from, there), tid, 256), behind = clean<T, DB>(tile, max(0, see_to), there, tid, 256);
    found |= __syncthreads_or(before || behind);
  };
  load_k(0);
  if (KB == 2) load_v(0);
  if (tiles > 1) load_k(1);
  wait_copies();
  trim_k(0);
  if (KB == 2) trim_v(0);
  if (tiles > 1) trim_k(1);
  __syncthreads();
  if (seen(0)) s[0] = read.scores(k_tile(0), 0, q);
  if constexpr (KB == 2) {
    // Tile i's first block reads the second one's keys and the last tile's second values; its second block the next
    // tile's first keys and its own first values.  In between, the places of this tile's keys and the last one's values
    // are free.
    const auto middle = [&](int i) {
      wait_copies();
      if (i) {
        if (i + 1 < tiles) trim_k(i + 1);
        trim_v(i);
      }
      __syncthreads();
      if (i + 2 < tiles) load_k(i + 2);
      if (i + 1 < tiles) load_v(i + 1);
    };
    const auto careful = [&](int i) {
      step(2 * i, s[0], s[1], w[1], w[0], k_tile(i), 32, v_tile(i - 1), 32);
      middle(i);
      put_aside(i);
      step(2 * i + 1, s[1], s[0], w[0], w[1], k_tile(i + 1), 0, v_tile(i), 0);
    };
    // Tiles in which all rows of the wave see all keys, and so in the blocks beside them, and none of whose values is to be
    // put aside: clear ... cloudy - 1.
    const int see_from = max(block_lo, from), see_to = min(block_hi, to);
    int clear = max(begin / 2 + 1, (max(wave_lo, see_from) - t0 + KT - 1) / KT);
    int cloudy = min(min((end - 1) / 2, (wave_hi - t0) / KT), see_to >= src.total ? tiles : (see_to - t0) / KT);
    if (!R::MIXED || begin >= end || clear >= cloudy) clear = cloudy = tiles;
    int i = 0;
    for (; i < clear; ++i) careful(i);
    if constexpr (R::MIXED) {
      for (; i < cloudy; ++i) {
        mixed(s[0], s[1], w[1], w[0], k_tile(i), 32, v_tile(i - 1), 32);
        middle(i);
        mixed(s[1], s[0], w[0], w[1], k_tile(i + 1), 0, v_tile(i), 0);
      }
      for (; i < tiles; ++i) careful(i);
    }
    if (seen(2 * tiles - 1)) run.template add<T>(read, v_tile(tiles - 1), 32, w[1]);
  } else {
    // Block i reads the next tile's keys and the last one's values; this tile's keys and the values before are done with.
    for (int i = 0; i < tiles; ++i) {
      wait_copies();
      if (i) {
        if (i + 1 < tiles) trim_k(i + 1);
        trim_v(i - 1);
      }
      __syncthreads();
      if (i + 2 < tiles) load_k(i + 2);
      load_v(i);
      if (i) put_aside(i - 1);
      step(i, s[0], s[1], w[0], w[1], k_tile(i + 1), 0, v_tile(i - 1), 0);
      s[0] = s[1];
      w[0] = w[1];
    }
    wait_copies();
    trim_v(tiles - 1);
    __syncthreads();
    put_aside(tiles - 1);
    if (seen(tiles - 1)) run.template add<T>(read, v_tile(tiles - 1), 0, w[0]);
  }
  if (wave * 32 >= it.len) return;
  const Halves both(run.l);
  const float l = both.a + both.b;
  bool lost = false;                           // a sum is NaN
#pragma unroll
  for (int x = 0; x < 16 * DB; ++x) lost |= run.o[x / 16][x % 16] != run.o[x / 16][x % 16];
  const bool numbers = row < it.len && l == l;
  const auto rest = [&](auto* to_row) {
    if (__builtin_expect(found || __any(lost && numbers), false))
      add_nonfinite<16 * DB>(numbers, l, found, to_row, src.k, src.v, a.head_dim, max(any_lo, from), 64, 64, min(any_hi, to), lo, hi, max(block_lo, from), min(block_hi, to), lane,
                             Running<DB>::channel);
  };
  if (k.parts > 1) {
    const int64_t at_row = (((int64_t)m * k.n_items + i) * k.rows_each + row) * a.heads + h, slot = at_row * k.parts + part;
    if (row < it.len) {
      store_row<float, DB>(k.ws_o + slot * a.head_dim, a.head_dim, run.o, 1.f, half);
      if (!half) k.ws_ml[2 * slot] = run.m, k.ws_ml[2 * slot + 1] = l;
    }
    rest(k.ws_o + slot * a.head_dim);
  } else {
    if (row < it.len) store_row<T, DB>(out + row * a.out.row_stride, a.head_dim, run.o, 1.f / l, half);
    rest(out + row * a.out.row_stride);
  }
}

// ---- short sequences: 16 rows (token, head of a group) a wave
//
// As above in 16x16 products: a lane has row l % 16 of the queries and of every 16 keys those numbered 4 (l / 16) + i.
// Little is used twice here, so keys go straight into registers, values through a small tile of the wave's own, and
// nobody waits for another wave: what counts is how many loads are on their way.  64 tokens over caches of 500 to 8000
// rows, 16 heads of 4, 128 bfloat16 channels: 91 to 95 us, 3.8 TB/s (32 rows a wave, tiles in LDS: 160).

template <typename T, int DB> struct Short {
  using H = Head<T, DB>;
  static constexpr int KT = 32, WAVES = 4, TILE = KT * H::ROW;
  static constexpr int PITCH = 32 * DB + 4;                    // floats of a row of sums
  static constexpr int EACH = TILE > 16 * PITCH * 4 ? TILE : 16 * PITCH * 4;
  static constexpr int LDS = WAVES * EACH + WAVES * 16 * 2 * 4;
  static constexpr int OCCUPANCY = DB * sizeof(T) <= 8 ? 4 : DB * sizeof(T) <= 24 ? 2 : 1;
};

// 16 rows of a sequence's queries: rows 16 unit ..., row r being token r / group, head g group + r % group.
struct Unit {
  int rows, token, head;                       // rows there are; the lane's row's
  __device__ __forceinline__ Unit(const SeqItem& it, int unit, int group, int g, int lane) {
    const int r = min(unit * 16 + (lane & 15), it.len * group - 1);
    rows = min(16, it.len * group - unit * 16);
    token = r / group;
    head = g * group + r - token * group;
  }
};

template <typename T, int DB, int FAST> struct ShortWave {
  using S = Short<T, DB>;
  using H = Head<T, DB>;
  static constexpr int STEPS = H::BYTES / 64, E = 16 / (int)sizeof(T);
  v4f o[2 * DB];
  float top = -__builtin_inff(), l = 0.f;
  bool apart = false;                          // values that are not finite were taken out of some tile

  __device__ __forceinline__ ShortWave() {
#pragma unroll
    for (int d = 0; d < 2 * DB; ++d) o[d] = v4f{};
  }

  static __device__ __forceinline__ int channel(int x, int lane) { return x / 4 * 16 + (lane >> 4) * 4 + x % 4; }

  // Whether add_nonfinite has something to do: for rows whose weights are numbers.
  __device__ __forceinline__ bool rest(bool numbers) const {
    bool nan = false;
#pragma unroll
    for (int x = 0; x < 8 * DB; ++x) nan |= o[x / 4][x % 4] != o[x / 4][x % 4];
    return apart || __any(nan && numbers);
  }

  // Of keys from ... to - 1 the tiles at `first`, `step` further and so on, of which the lane's row sees keys lo ... hi - 1 and
  // all of the sequence's rows all_lo ... all_hi - 1.
  __device__ __forceinline__ void run(const Source<T>& src, const T* query, int n, float scale, int first, int step, int from, int to, int lo, int hi, int all_lo, int all_hi, char* tile, int lane) {
    constexpr float LOWEST = -__builtin_inff();
    const int quarter = lane >> 4;
    v4u q[STEPS];
    load_query<T, STEPS, 4>(q, query, n, quarter, scale);
    const float c = factor(scale);
    for (int t = first; t < to; t += step) {
      const bool two = t + 16 < to;            // keys in the tile's second half
      // keys 16 b + l % 16; those behind the sequence's are hidden
      v4u keys[2][STEPS];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const T* p = src.k.at(min(t + 16 * b + (lane & 15), src.total - 1));
        if (b == 0 || two)
#pragma unroll
          for (int s = 0; s < STEPS; ++s) {
            const int e = (4 * s + quarter) * E;
            if constexpr (FAST == PIECES) keys[b][s] = e < n ? *reinterpret_cast<const v4u*>(p + e) : v4u{0, 0, 0, 0};
            else if constexpr (FAST == WORDS) keys[b][s] = load_words<T>(p, e, n);
            else keys[b][s] = e < n ? load_piece<T>(p, e, n) : v4u{0, 0, 0, 0};
          }
      }
      Copy<T, DB, S::KT, 1, VALUES16>::template run<FAST>(tile, src.v, t, src.total, n, 0, lane);
      v4f s[2] = {};
#pragma unroll
      for (int b = 0; b < 2; ++b)
        if (b == 0 || two)
#pragma unroll
          for (int x = 0; x < STEPS; ++x) s[b] = mma16<T>(keys[b][x], q[x], s[b]);
      const int row_lo = max(lo, from) - t, row_hi = min(hi, to) - t;
      float most = LOWEST;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int key = 16 * b + 4 * quarter + x;
          s[b][x] = key >= row_lo && key < row_hi ? s[b][x] : LOWEST;
          most = fmaxf(most, s[b][x]);
        }
      most = fmaxf(most, __shfl_xor(most, 16));
      most = fmaxf(most, __shfl_xor(most, 32)) * c;
      const bool grows = most > top + 8.f;
      if (__any(grows)) {
        const float old = grows ? __builtin_amdgcn_exp2f(top - most) : 1.f;    // 0 of an infinite sum is NaN, which add_nonfinite mends
        top = grows ? most : top;
        l *= old;
#pragma unroll
        for (int d = 0; d < 2 * DB; ++d) o[d] *= old;
      }
      const float base = top == LOWEST ? 0.f : top;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          s[b][x] = __builtin_amdgcn_exp2f(fmaf(s[b][x], c, -base));
          l += s[b][x];
        }
      wait_copies();
      if constexpr (FAST == WORDS) Copy<T, DB, S::KT, 1, VALUES16>::trim(tile, n, 0, lane);
      settle();
      const int see_from = max(all_lo, from) - t, see_to = min(all_hi, to) - t, there = min(S::KT, src.total - t);
      if (see_from > 0 || see_to < there) {
        const bool before = clean<T, DB>(tile, 0, min(see_from, there), lane, 64), behind = clean<T, DB>(tile, max(0, see_to), there, lane, 64);
        apart |= __any(before || behind);
        settle();
      }
      if constexpr (sizeof(T) == 2) {
        v4u w;
#pragma unroll
        for (int x = 0; x < 4; ++x) w[x] = pack2(s[x / 2][2 * (x & 1)], s[x / 2][2 * (x & 1) + 1]);
        const v8bf p = __builtin_bit_cast(v8bf, w);
        const int key = 4 * quarter + (lane & 15) / 4, twist = Twist<T, H::PIECES, VALUES16>::of(key);       // and key + 16
        const int v = key * H::ROW + ((((lane & 3) >> 1) ^ twist) << 4) + (lane & 1) * 8;
#pragma unroll
        for (int d = 0; d < 2 * DB; ++d) {
          v4s x[2];
#pragma unroll
          for (int b = 0; b < 2; ++b) x[b] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(tile + (v ^ (d << 5)) + 16 * b * H::ROW));
          o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7)), p, o[d], 0, 0, 0);
        }
      } else {
        const int key = 4 * quarter, twist = Twist<T, H::PIECES, VALUES16>::of(key), v = key * H::ROW + ((((lane & 15) >> 2) ^ twist) << 4) + (lane & 3) * 4;
#pragma unroll
        for (int b = 0; b < 2; ++b)
          if (b == 0 || two)
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
              for (int d = 0; d < 2 * DB; ++d)
                o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(*reinterpret_cast<const float*>(tile + (v ^ (d << 6)) + (16 * b + x) * H::ROW), s[b][x], o[d], 0, 0, 0);
      }
      settle();
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
  }
};

// Without a cache: a unit a wave, all of the sequence's keys.
template <typename T, int DB, int FAST> __global__ __launch_bounds__(256, (Short<T, DB>::OCCUPANCY)) void whole_kernel(AttnArgs k, int each) {
  using S = Short<T, DB>;
  extern __shared__ char lds[];
  const mure_attn_attend_args& a = k.a;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, quarter = lane >> 4;
  const int at = uniform(blockIdx.x / each), i = k.item0 + at, w = (blockIdx.x - at * each) * S::WAVES + wave;       // unit, group and mutant
  const SeqItem it = item_of(k, i);
  const int group = uniform(a.heads / a.kv_heads), units = (it.len * group + 15) / 16, gm = uniform(w / units), unit = w - gm * units;
  if (gm >= a.kv_heads * a.n_mutants) return;
  const int m = uniform(gm / a.kv_heads), g = gm - m * a.kv_heads;
  const Source<T> src(k, it, m, g);
  const Unit u(it, unit, group, g, lane);
  int lo, hi, from, to, all_lo, all_hi;        // keys that the row sees, that any of the unit's tokens sees, that all do
  sees(a, u.token, src.total, lo, hi);
  sees(a, unit * 16 / group, src.total, from, all_hi);
  sees(a, (unit * 16 + u.rows - 1) / group, src.total, all_lo, to);
  ShortWave<T, DB, FAST> sw;
  sw.run(src, static_cast<const T*>(a.q.p) + m * a.q.mutant_stride + (it.row0 + (int64_t)u.token) * a.q.row_stride + (int64_t)u.head * a.head_dim, a.head_dim, a.scale,
         from / S::KT * S::KT, S::KT, from, to, lo, hi, all_lo, all_hi, lds + wave * S::TILE, lane);
  T* out = static_cast<T*>(a.out.p) + m * a.out.mutant_stride + (it.row0 + (int64_t)u.token) * a.out.row_stride + (int64_t)u.head * a.head_dim;
  const bool there = (lane & 15) < u.rows;
  if (there) {
    const float f = 1.f / sw.l;
#pragma unroll
    for (int d = 0; d < 2 * DB; ++d) store4<T>(out, 16 * d + 4 * quarter, a.head_dim, sw.o[d][0] * f, sw.o[d][1] * f, sw.o[d][2] * f, sw.o[d][3] * f);
  }
  const bool numbers = there && sw.l == sw.l;
  if (__builtin_expect(sw.rest(numbers), false)) {
    int l = lane, lo, hi;
    asm volatile("" : "+v"(l));                // the row's numbers anew, out of registers until here
    const Unit u(it, unit, group, g, l);
    sees(a, u.token, src.total, lo, hi);
    add_nonfinite<8 * DB>(numbers, sw.l, sw.apart, out, src.k, src.v, a.head_dim, from, 64, 64, to, lo, hi, all_lo, all_hi, l, sw.channel);
  }
}

// Over a cache: a unit a block, the part's keys spread over its waves.
template <typename T, int DB, int FAST> __global__ __launch_bounds__(256, (Short<T, DB>::OCCUPANCY)) void short_kernel(AttnArgs k, int units) {
  using S = Short<T, DB>;
  constexpr float LOWEST = -__builtin_inff();
  extern __shared__ char lds[];
  const mure_attn_attend_args& a = k.a;
  const int n = a.kv_heads * a.n_mutants, at = uniform(blockIdx.x / n), gm = spread(blockIdx.x - at * n, n), m = uniform(gm / a.kv_heads), g = gm - m * a.kv_heads;
  const int group = uniform(a.heads / a.kv_heads), ip = uniform(at / units), unit = at - ip * units, part = uniform(ip % k.parts), i = k.item0 + uniform(ip / k.parts);
  const SeqItem it = item_of(k, i);
  if (unit * 16 >= it.len * group) return;
  const Source<T> src(k, it, m, g);
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, quarter = lane >> 4;
  const Unit u(it, unit, group, g, lane);
  T* out = static_cast<T*>(a.out.p) + m * a.out.mutant_stride + it.row0 * a.out.row_stride;
  if (src.bad) {
    if (part == 0)
      for (int x = tid; x < u.rows * a.head_dim; x += 256) {
        const int y = unit * 16 + x / a.head_dim;
        out[y / group * a.out.row_stride + (int64_t)(g * group + y % group) * a.head_dim + x % a.head_dim] = from_f<T>(__builtin_nanf(""));
      }
    return;
  }
  if (part == 0 && unit == 0) src.keep(a, it, m, tid, 256);
  int lo, hi, from, to, all_lo, all_hi;        // keys that the row sees, that any token sees, that all do
  sees(a, src.past + u.token, src.total, lo, hi);
  sees(a, src.past, src.total, from, all_hi);
  sees(a, src.total - 1, src.total, all_lo, to);
  const int64_t part0 = (int64_t)part * ATTN_KEYS_SHORT;
  if (max((int64_t)from, part0) >= min((int64_t)to, part0 + ATTN_KEYS_SHORT)) return;
  from = (int)max((int64_t)from, part0);
  to = (int)min((int64_t)to, part0 + ATTN_KEYS_SHORT);
  // the tiles go to the waves in turn, so that few keys are spread too
  const int tile0 = from / S::KT, first = (tile0 + ((wave - tile0) & (S::WAVES - 1))) * S::KT;
  char* tile = lds + wave * S::EACH;
  ShortWave<T, DB, FAST> sw;
  if (first < to)
    sw.run(src, static_cast<const T*>(a.q.p) + m * a.q.mutant_stride + (it.row0 + (int64_t)u.token) * a.q.row_stride + (int64_t)u.head * a.head_dim, a.head_dim, a.scale, first,
           S::WAVES * S::KT, from, to, lo, hi, all_lo, all_hi, tile, lane);
  // the waves' sums, added in order
  float* sums = reinterpret_cast<float*>(tile);
  float* ml = reinterpret_cast<float*>(lds + S::WAVES * S::EACH);              // [4][16][2]
#pragma unroll
  for (int d = 0; d < 2 * DB; ++d) *reinterpret_cast<v4f*>(sums + (lane & 15) * S::PITCH + 16 * d + 4 * quarter) = sw.o[d];
  if (!quarter) ml[(wave * 16 + lane) * 2] = sw.top, ml[(wave * 16 + lane) * 2 + 1] = sw.l;
  const bool numbers = sw.l == sw.l;
  if (__builtin_expect(sw.rest(numbers), false)) {
    int l = lane, lo, hi;
    asm volatile("" : "+v"(l));                // the row's numbers anew, out of registers until here
    const Unit u(it, unit, group, g, l);
    sees(a, src.past + u.token, src.total, lo, hi);
    add_nonfinite<8 * DB>(numbers, sw.l, sw.apart, sums + (l & 15) * S::PITCH, src.k, src.v, a.head_dim, first, S::WAVES * S::KT, S::KT, to, max(lo, from), hi, all_lo, all_hi, l,
                          sw.channel);
  }
  __syncthreads();
  for (int x = tid; x < u.rows * a.head_dim; x += 256) {
    const int y = x / a.head_dim, e = x - y * a.head_dim, all = unit * 16 + y, tk = all / group, hd = g * group + all % group;
    float most = LOWEST;
#pragma unroll
    for (int w = 0; w < S::WAVES; ++w) most = fmaxf(most, ml[(w * 16 + y) * 2]);
    const float base = most == LOWEST ? 0.f : most;
    float v = 0.f, size = 0.f;
#pragma unroll
    for (int w = 0; w < S::WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml[(w * 16 + y) * 2] - base);
      size = fmaf(ml[(w * 16 + y) * 2 + 1], f, size);
      v = join_sum(reinterpret_cast<const float*>(lds + w * S::EACH)[y * S::PITCH + e], f, v);
    }
    if (k.parts > 1) {
      const int64_t slot = ((((int64_t)m * k.n_items + i) * k.rows_each + tk) * a.heads + hd) * k.parts + part;
      k.ws_o[slot * a.head_dim + e] = v;
      if (e == 0) k.ws_ml[2 * slot] = most, k.ws_ml[2 * slot + 1] = size;
    } else {
      out[tk * a.out.row_stride + (int64_t)hd * a.head_dim + e] = from_f<T>(v * (1.f / size));
    }
  }
}

// ---- the parts' results of one token and head: every 16th part in order, then the 16 sums in order
//
// Bound by latency: 16 parts of 1024 rows take 7 us, 196 parts of 32 rows 12.

template <typename T> __global__ __launch_bounds__(1024) void join_kernel(AttnArgs k, int keys, int64_t first_row) {
  __shared__ float sums[16][MURE_ATTN_MAX_HEAD], sizes[16];
  const mure_attn_attend_args& a = k.a;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int64_t at = first_row + blockIdx.x;
  const int rows = a.heads * k.rows_each, im = uniform((int)(at / rows)), x = (int)(at - (int64_t)im * rows), row = uniform(x / a.heads), h = x - row * a.heads;
  const int m = uniform(im / k.n_items), i = im - m * k.n_items;
  const SeqItem it = item_of(k, i);
  if (row >= it.len) return;
  const int past = uniform(a.past ? a.past[it.seq] : 0);
  if (past < 0 || past > a.capacity - it.total) return;        // NaN already
  int lo, hi;
  sees(a, past + it.pos0 + row, past + it.total, lo, hi);
  const int first = lo / keys, last = (hi - 1) / keys;         // the parts with keys that the row sees
  const float* ml = k.ws_ml + 2 * at * k.parts;
  const float* o = k.ws_o + at * k.parts * a.head_dim;
  float top = -__builtin_inff();
  for (int p = first + lane; p <= last; p += 64) top = fmaxf(top, ml[2 * p]);
  for (int w = 1; w < 64; w *= 2) top = fmaxf(top, __shfl_xor(top, w));
  const float base = top == -__builtin_inff() ? 0.f : top;
  for (int slot = wave; slot < 16; slot += waves) {
    float l = 0.f, v[4] = {};
#pragma unroll 4
    for (int p = first + slot; p <= last; p += 16) {
      const float f = __builtin_amdgcn_exp2f(ml[2 * p] - base);
      l = fmaf(ml[2 * p + 1], f, l);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (lane + 64 * j < a.head_dim) v[j] = join_sum(o[(int64_t)p * a.head_dim + lane + 64 * j], f, v[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) sums[slot][lane + 64 * j] = v[j];
    if (lane == 0) sizes[slot] = l;
  }
  __syncthreads();
  const int c = threadIdx.x;
  if (c >= a.head_dim) return;
  float l = 0.f, v = 0.f;
  for (int s = 0; s < 16; ++s) l += sizes[s], v += sums[s][c];
  T* out = static_cast<T*>(a.out.p) + m * a.out.mutant_stride + (it.row0 + (int64_t)row) * a.out.row_stride + (int64_t)h * a.head_dim;
  out[c] = from_f<T>(v * (1.f / l));
}

// ---- launches

constexpr int64_t BLOCKS = (1 << 24) - 1;

// `each` blocks an item, as many items a launch as fit
template <typename F> hipError_t over_items(AttnArgs& k, int64_t each, F&& f) {
  const int n = k.n_items;
  const int most = (int)std::min<int64_t>(n, BLOCKS / each);
  for (k.item0 = 0; k.item0 < n; k.item0 += most)
    if (const hipError_t e = f((unsigned)(each * std::min(most, n - k.item0))); e != hipSuccess) return e;
  return hipSuccess;
}

template <typename... P, typename... A> hipError_t launch_lds(void (*kernel)(P...), unsigned grid, unsigned lds, hipStream_t s, A&&... a) {
  if (lds > 65536)                             // more than the default limit has to be asked for
    if (const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds); e != hipSuccess) return e;
  std::tuple<P...> params(std::forward<A>(a)...);
  return std::apply(
      [&](auto&... p) {
        void* at[] = {&p...};
        return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(grid), dim3(256), at, lds, s);
      },
      params);
}

template <typename T, int DB, int FAST> hipError_t short_f(AttnArgs k, hipStream_t s) {
  const int units = (k.longest * (k.a.heads / k.a.kv_heads) + 15) / 16;
  if (!k.a.k_cache.p) {
    const int each = (int)(((int64_t)k.a.kv_heads * k.a.n_mutants * units + 3) / 4);
    return over_items(k, each, [&](unsigned grid) { return launch_lds(whole_kernel<T, DB, FAST>, grid, Short<T, DB>::WAVES * Short<T, DB>::TILE, s, k, each); });
  }
  return over_items(k, (int64_t)k.a.kv_heads * k.a.n_mutants * units * k.parts,
                    [&](unsigned grid) { return launch_lds(short_kernel<T, DB, FAST>, grid, Short<T, DB>::LDS, s, k, units); });
}

template <typename T, int DB, int FAST> hipError_t runs_f(AttnArgs k, hipStream_t s) {
  return over_items(k, (int64_t)k.a.heads * k.a.n_mutants * k.parts,
                    [&](unsigned grid) { return launch_lds(run_kernel<T, DB, FAST>, grid, Run<T, DB>::LDS, s, k); });
}

template <typename T, int DB> hipError_t with_speed(const AttnArgs& k, bool brief, hipStream_t s) {
  if (k.fast == PIECES) return brief ? short_f<T, DB, PIECES>(k, s) : runs_f<T, DB, PIECES>(k, s);
  if (k.fast == WORDS) return brief ? short_f<T, DB, WORDS>(k, s) : runs_f<T, DB, WORDS>(k, s);
  return brief ? short_f<T, DB, ELEMENTS>(k, s) : runs_f<T, DB, ELEMENTS>(k, s);
}

template <typename T> hipError_t with_head(const AttnArgs& k, bool brief, hipStream_t s) {
  const int d = k.a.head_dim;
  if (d <= 32) return with_speed<T, 1>(k, brief, s);
  if (d <= 64) return with_speed<T, 2>(k, brief, s);
  if (d <= 96) return with_speed<T, 3>(k, brief, s);
  if (d <= 128) return with_speed<T, 4>(k, brief, s);
  if (d <= 192) return with_speed<T, 6>(k, brief, s);
  return with_speed<T, 8>(k, brief, s);
}

template <typename T> hipError_t join(AttnArgs k, int keys, hipStream_t s) {
  const int64_t rows = (int64_t)k.rows_each * k.a.heads, blocks = (int64_t)k.a.n_mutants * k.n_items * rows;
  // few rows get a wave for every 16th part; otherwise the waves take several each
  const unsigned threads = blocks < 512 && k.parts > 16 ? 1024 : 256;
  const int64_t most = ((int64_t)1 << 32) / threads - 1;
  for (int64_t first = 0; first < blocks; first += most)
    if (const hipError_t e = launch(join_kernel<T>, dim3((unsigned)std::min(most, blocks - first)), threads, s, k, keys, first); e != hipSuccess) return e;
  return hipSuccess;
}

}  // namespace mure
