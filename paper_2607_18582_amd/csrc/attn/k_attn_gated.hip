// Gated feed-forward layer (mure_attn_gated): both projections as one tiled
// matrix product, with biases, activation and product behind it.
//
// A block computes MT rows by NT outputs: for every 128 bytes of the summed
// axis, MT rows of x and NT rows of each projection's weights are copied to
// LDS, two stages in turn.  A wave's instructions are 16 x 16 results of 64
// bytes of the summed axis, weights first, so that a lane ends with four
// neighbouring outputs of a row, gate and up alike.  Every result adds its
// terms in the same order in any tile, so that it does not depend on the
// number of rows.  16384 rows, 4096 inputs to 11008 outputs, bfloat16: 2.44 to
// 2.52 ms, 1.2 PFLOP/s: LDS delivers and takes what the tiles need in as many
// cycles as the matrix instructions last.
#include "attn_dev.hpp"

#include <algorithm>

namespace mure {
namespace {

__device__ __forceinline__ float activated(float v, int act) {
  switch (act) {
    case MURE_ATTN_SILU: return seq_silu(v);
    case MURE_ATTN_SIGMOID: return seq_sigmoid(v);
    case MURE_ATTN_RELU: return v < 0.f ? 0.f : v;
    case MURE_ATTN_GELU: return 0.5f * v * (1.f + erff(v * 0.70710678118654752440f));
    case MURE_ATTN_GELU_TANH: return v * seq_sigmoid(1.59576912160573071176f * (v + 0.044715f * v * v * v));   // (1 + tanh u) / 2 = sigmoid(2 u)
  }
  return v;
}

// A block's tile: consecutive blocks go to the chip's eight dies in turn; each die gets a run of neighbouring tiles, and
// within it bands of 8 row tiles, so that what its blocks read together stays in its L2.
__device__ __forceinline__ void place_of(int block, int n_tiles, int m_tiles, int& mt, int& nt, int& m) {
  const int each = n_tiles * m_tiles, all = gridDim.x;
  int b = all % 8 ? block : block % 8 * (all / 8) + block / 8;
  m = uniform(b / each);
  b -= m * each;
  const int band = uniform(b / (8 * n_tiles)), tall = min(8, m_tiles - band * 8);
  b -= band * 8 * n_tiles;
  nt = uniform(b / tall);
  mt = band * 8 + b - nt * tall;
}

// A row's piece from element e on, zeros from element n on.  `end` is the end of the tensor: a piece that reaches over
// its row's end lies before it, but in the tensor's last rows.
template <typename T> __device__ __forceinline__ v4u piece_of(const T* row, int e, int n, const T* end) {
  constexpr int E = 16 / (int)sizeof(T);
  if (e >= n) return v4u{0, 0, 0, 0};
  if (row + e + E > end) return load_piece<T>(row, e, n);
  v4u v = *reinterpret_cast<const v4u_any*>(row + e);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int left = (n - e) * (int)sizeof(T) - 4 * i;         // bytes of the word that are the row's
    v[i] &= left >= 4 ? ~0u : left <= 0 ? 0u : 0xffffu;
  }
  return v;
}

// Where a block's rows are read: rows of x and of both weights, those behind the last one in its place (their results
// are not kept).
template <typename T> struct Operands {
  const T *x, *gate, *up, *x_end, *gate_end, *up_end;
  __device__ __forceinline__ Operands(const mure_attn_gated_args& a, int m)
      : x(static_cast<const T*>(a.x.p) + m * a.x.mutant_stride), gate(static_cast<const T*>(a.gate.p) + m * a.gate.mutant_stride),
        up(static_cast<const T*>(a.up.p) + m * a.up.mutant_stride), x_end(x + (a.rows - 1) * a.x.row_stride + a.inner),
        gate_end(gate + (int64_t)(a.outer - 1) * a.gate.row_stride + a.inner), up_end(up + (int64_t)(a.outer - 1) * a.up.row_stride + a.inner) {}
  __device__ __forceinline__ const T* x_row(const mure_attn_gated_args& a, int64_t r) const { return x + min(r, a.rows - 1) * a.x.row_stride; }
  __device__ __forceinline__ const T* gate_row(const mure_attn_gated_args& a, int n) const { return gate + (int64_t)min(n, a.outer - 1) * a.gate.row_stride; }
  __device__ __forceinline__ const T* up_row(const mure_attn_gated_args& a, int n) const { return up + (int64_t)min(n, a.outer - 1) * a.up.row_stride; }
};

// Four neighbouring values of a bias from n on
__device__ __forceinline__ v4f bias_at(const mure_seq_param& b, int m, int n, int outer) {
  v4f v = {};
  if (b.p)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = b.p[m * b.mutant_stride + min(n + e, outer - 1)];
  return v;
}

// Four neighbouring outputs from n on of one row, from their sums and biases.
template <typename T> __device__ __forceinline__ void finish(const mure_attn_gated_args& a, int m, int64_t row, int n, v4f g, v4f u, v4f gb, v4f ub) {
  if (row >= a.rows) return;
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = activated(g[e] + gb[e], a.activation) * (u[e] + ub[e]);
  store4<T>(static_cast<T*>(a.out.p) + m * a.out.mutant_stride + row * a.out.row_stride, n, a.outer, v[0], v[1], v[2], v[3]);
}

// Few outputs over a long summed axis make few tiles, each with a long chain of products.  Their axis is summed in
// eighths, which are added in order: in one block after the other, or side by side (gated_split_kernel).  This follows from
// the weights' sizes alone, as a row's results do.
constexpr int SPLIT = 8, SPLIT_OUTPUTS = 512, SPLIT_BYTES = 2048;

template <typename T> __host__ __device__ __forceinline__ bool splits(const mure_attn_gated_args& a) {
  return a.outer <= SPLIT_OUTPUTS && a.inner * (int)sizeof(T) >= SPLIT_BYTES;
}

// Elements of an eighth: pieces of 256 bytes
template <typename T> __device__ __forceinline__ int eighth(int inner) {
  constexpr int KS = 256 / (int)sizeof(T);
  return ((inner + KS - 1) / KS + SPLIT - 1) / SPLIT * KS;
}

// WM x WN waves; BYTES of the summed axis a stage (64 or 128); PARTS: the axis in eighths
template <typename T, int MT, int NT, int WM, int WN, int BYTES, bool FAST, bool PARTS>
__global__ __launch_bounds__(64 * WM * WN, 2) void gated_kernel(mure_attn_gated_args a, int n_tiles, int m_tiles) {
  constexpr int WAVES = WM * WN, ROWS = MT + 2 * NT, STAGE = ROWS * BYTES, E = 16 / (int)sizeof(T), PIECES = BYTES / 16, KS = PIECES * E;
  constexpr int TM = MT / WM / 16, TN = NT / WN / 16, EACH = 64 / PIECES;      // rows of a copy of 1024 bytes
  // 16 rows' pieces of one place in distinct banks
  const auto twist = [](int row) { return PIECES == 8 ? (row >> 1) & 7 : (row >> 2) & 3; };
  extern __shared__ char lds[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  int mt, nt, m;
  place_of(blockIdx.x, n_tiles, m_tiles, mt, nt, m);
  const int64_t row0 = (int64_t)mt * MT;
  const int col0 = nt * NT;
  const Operands<T> op(a, m);
  constexpr int COPIES = ROWS / EACH / WAVES;
  static_assert(ROWS / EACH % WAVES == 0 && MT % EACH == 0 && NT % EACH == 0, "");
  const T* from[COPIES];                       // the lane's row of each, at its piece of a stage
#pragma unroll
  for (int c = 0; c < COPIES; ++c) {
    const int r = (wave * COPIES + c) * EACH + lane / PIECES;
    from[c] = r < MT ? op.x_row(a, row0 + r) : r < MT + NT ? op.gate_row(a, col0 + r - MT) : op.up_row(a, col0 + r - MT - NT);
    from[c] += (lane % PIECES ^ twist(r)) * E;
  }
  // FAST: straight to LDS.  Otherwise through registers: on their way while the last stage is worked on.
  v4u held[FAST ? 1 : COPIES];
  auto load = [&](int k0, int stage) {
    const bool whole = k0 + KS <= a.inner;     // nothing of the stage lies behind the rows
#pragma unroll
    for (int c = 0; c < COPIES; ++c) {
      const int q = wave * COPIES + c, r = q * EACH + lane / PIECES, at = (lane % PIECES ^ twist(r)) * E;
      if constexpr (FAST) {
        const void* p = whole || k0 + at < a.inner ? static_cast<const void*>(from[c] + k0) : ZEROS;
        __builtin_amdgcn_global_load_lds(p, (lds_void*)(lds + stage * STAGE + q * 1024), 16, 0, 0);
      } else if (whole) {
        held[c] = *reinterpret_cast<const v4u_any*>(from[c] + k0);
      } else {
        held[c] = piece_of<T>(from[c] - at, k0 + at, a.inner, r < MT ? op.x_end : r < MT + NT ? op.gate_end : op.up_end);
      }
    }
  };
  auto put = [&](int stage) {
    if constexpr (!FAST)
#pragma unroll
      for (int c = 0; c < COPIES; ++c) *reinterpret_cast<v4u*>(lds + stage * STAGE + (wave * COPIES + c) * 1024 + lane * 16) = held[c];
  };
  const int wm = wave % WM, wn = wave / WM;
  v4f g[TN][TM], u[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) g[i][j] = v4f{}, u[i][j] = v4f{};
  v4f all_g[PARTS ? TN : 1][PARTS ? TM : 1] = {}, all_u[PARTS ? TN : 1][PARTS ? TM : 1] = {};
  const int part = PARTS ? eighth<T>(a.inner) : 0;
  int left = part;                             // of the eighth
  load(0, 0);
  put(0);
  int stage = 0;
  for (int k0 = 0; k0 < a.inner; k0 += KS, stage ^= 1) {
    if constexpr (FAST) wait_copies();
    __syncthreads();
    if (k0 + KS < a.inner) load(k0 + KS, stage ^ 1);
    const char* base = lds + stage * STAGE;
    auto piece = [&](int r, int s) { return *reinterpret_cast<const v4u*>(base + r * BYTES + ((s * 4 + (lane >> 4)) ^ twist(r)) * 16); };
#pragma unroll
    for (int s = 0; s < BYTES / 64; ++s) {
      v4u xs[TM], gs[TN], us[TN];
#pragma unroll
      for (int j = 0; j < TM; ++j) xs[j] = piece(wm * (MT / WM) + j * 16 + (lane & 15), s);
#pragma unroll
      for (int i = 0; i < TN; ++i) {
        const int r = wn * (NT / WN) + i * 16 + (lane & 15);
        gs[i] = piece(MT + r, s);
        us[i] = piece(MT + NT + r, s);
      }
      // instructions that follow each other add to different results
#pragma unroll
      for (int e = 0; e < (sizeof(T) == 2 ? 1 : 4); ++e)
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int j = 0; j < TM; ++j) {
            g[i][j] = mma16_part<T>(gs[i], xs[j], e, g[i][j]);
            u[i][j] = mma16_part<T>(us[i], xs[j], e, u[i][j]);
          }
    }
    if (k0 + KS < a.inner) put(stage ^ 1);
    if constexpr (PARTS)
      if ((left -= KS) == 0 || k0 + KS >= a.inner) {
        left = part;
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int j = 0; j < TM; ++j) {
            all_g[i][j] += g[i][j], all_u[i][j] += u[i][j];
            g[i][j] = v4f{}, u[i][j] = v4f{};
          }
      }
  }
#pragma unroll
  for (int i = 0; i < TN; ++i) {
    const int n = col0 + wn * (NT / WN) + i * 16 + (lane >> 4) * 4;
    const v4f gb = bias_at(a.gate_bias, m, n, a.outer), ub = bias_at(a.up_bias, m, n, a.outer);
#pragma unroll
    for (int j = 0; j < TM; ++j)
      finish<T>(a, m, row0 + wm * (MT / WM) + j * 16 + (lane & 15), n, PARTS ? all_g[PARTS ? i : 0][PARTS ? j : 0] : g[i][j],
                PARTS ? all_u[PARTS ? i : 0][PARTS ? j : 0] : u[i][j], gb, ub);
  }
}

// ---- the eighths side by side: a wave each, of 16 TM rows by 16 outputs, from memory to registers; their sums meet in LDS.
// Bound by the loads, 8 (float32) or 16 operations a byte: 50 and 120 TFLOP/s, 156 rows of 2764 to 180 float32 27 us.

template <typename T, int TM> __global__ __launch_bounds__(64 * SPLIT, 2) void gated_split_kernel(mure_attn_gated_args a, int n_tiles, int m_tiles) {
  constexpr int E = 16 / (int)sizeof(T), KS = 256 / (int)sizeof(T), PITCH = 36;
  __shared__ float sums[SPLIT][16 * TM][PITCH];                // a row: 16 of the gate, 16 of the other projection
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, quarter = lane >> 4;
  int mt, nt, m;
  place_of(blockIdx.x, n_tiles, m_tiles, mt, nt, m);
  const int64_t row0 = (int64_t)mt * 16 * TM;
  const int col0 = nt * 16;
  const Operands<T> op(a, m);
  const T *xr[TM], *wr[2] = {op.gate_row(a, col0 + (lane & 15)), op.up_row(a, col0 + (lane & 15))};
#pragma unroll
  for (int j = 0; j < TM; ++j) xr[j] = op.x_row(a, row0 + 16 * j + (lane & 15));
  struct Pieces {
    v4u x[4][TM], w[4][2];
  };
  auto load = [&](int k0, Pieces& p) {
    const bool whole = k0 + KS <= a.inner;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = k0 + (4 * i + quarter) * E;
#pragma unroll
      for (int j = 0; j < TM; ++j) p.x[i][j] = whole ? *reinterpret_cast<const v4u_any*>(xr[j] + e) : piece_of<T>(xr[j], e, a.inner, op.x_end);
#pragma unroll
      for (int w = 0; w < 2; ++w) p.w[i][w] = whole ? *reinterpret_cast<const v4u_any*>(wr[w] + e) : piece_of<T>(wr[w], e, a.inner, w ? op.up_end : op.gate_end);
    }
  };
  v4f acc[2][TM] = {};
  auto add = [&](const Pieces& p) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < (sizeof(T) == 2 ? 1 : 4); ++e)
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int j = 0; j < TM; ++j) acc[w][j] = mma16_part<T>(p.w[i][w], p.x[i][j], e, acc[w][j]);
  };
  const int part = eighth<T>(a.inner), from = wave * part, to = min(a.inner, from + part);
  Pieces one, other;
  if (from < to) load(from, one);
  for (int k0 = from; k0 < to; k0 += 2 * KS) {
    if (k0 + KS < to) load(k0 + KS, other);
    add(one);
    if (k0 + KS >= to) break;
    if (k0 + 2 * KS < to) load(k0 + 2 * KS, one);
    add(other);
  }
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int j = 0; j < TM; ++j) *reinterpret_cast<v4f*>(&sums[wave][16 * j + (lane & 15)][16 * w + 4 * quarter]) = acc[w][j];
  __syncthreads();
  const int r = tid / 16, n = col0 + tid % 16;
  const int64_t row = row0 + r;
  if (r >= 16 * TM || row >= a.rows || n >= a.outer) return;
  float g = 0.f, u = 0.f;
#pragma unroll
  for (int w = 0; w < SPLIT; ++w) g += sums[w][r][tid % 16], u += sums[w][r][16 + tid % 16];
  if (a.gate_bias.p) g += a.gate_bias.p[m * a.gate_bias.mutant_stride + n];
  if (a.up_bias.p) u += a.up_bias.p[m * a.up_bias.mutant_stride + n];
  static_cast<T*>(a.out.p)[m * a.out.mutant_stride + row * a.out.row_stride + n] = from_f<T>(activated(g, a.activation) * u);
}

// ---- few rows: bound by the weights' bytes.  W waves have 16 rows of x each; NT = 8: the gate's 8 rows of weights and the
// other projection's share an operand of 16, so that even few outputs make many blocks; NT = 16: an operand each, as 64
// rows of x would be read too often otherwise.  A block of one wave has all but one of the stages of 256 bytes of the summed
// axis on their way; with more waves the barrier waits for all copies, so that it has those issued since the last one.
// 64 rows, 2048 to 5632, bfloat16: 14 us, 3.3 TB/s.

template <typename T, int W, int NT, int STAGES, bool FAST> __global__ __launch_bounds__(64 * W) void gated_few_kernel(mure_attn_gated_args a, int n_tiles, int m_tiles) {
  constexpr int ROWS = 16 * W + 2 * NT, STAGE = ROWS * 256, E = 16 / (int)sizeof(T), KS = 16 * E, COPIES = ROWS / 4 / W, N = NT / 8;
  static_assert(ROWS / 4 % W == 0 && (NT == 8 || NT == 16), "");
  extern __shared__ char lds[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int nt = uniform(blockIdx.x % n_tiles), rest = uniform(blockIdx.x / n_tiles), mt = uniform(rest % m_tiles), m = uniform(rest / m_tiles);
  const int64_t row0 = (int64_t)mt * 16 * W;
  const int col0 = nt * NT;
  const Operands<T> op(a, m);
  // rows of x, then NT of each projection's weights; 4 rows of 16 pieces a copy, pieces xored with the row
  const T* from[COPIES];
#pragma unroll
  for (int c = 0; c < COPIES; ++c) {
    const int r = (wave * COPIES + c) * 4 + lane / 16, w = r - 16 * W;
    from[c] = w < 0 ? op.x_row(a, row0 + r) : w < NT ? op.gate_row(a, col0 + w) : op.up_row(a, col0 + w - NT);
  }
  // FAST: straight to LDS.  Otherwise through registers, which hold as many stages.
  v4u held[FAST ? 1 : STAGES - 1][COPIES];
  auto load = [&](int k0, int stage, int slot) {
    const bool whole = k0 + KS <= a.inner;
#pragma unroll
    for (int c = 0; c < COPIES; ++c) {
      const int q = wave * COPIES + c, r = q * 4 + lane / 16, e = k0 + ((lane & 15) ^ (r & 15)) * E;
      if constexpr (FAST) {
        const void* p = e < a.inner ? static_cast<const void*>(from[c] + e) : ZEROS;
        __builtin_amdgcn_global_load_lds(p, (lds_void*)(lds + stage * STAGE + q * 1024), 16, 0, 0);
      } else {
        held[slot][c] = whole ? *reinterpret_cast<const v4u_any*>(from[c] + e)
                              : piece_of<T>(from[c], e, a.inner, r < 16 * W ? op.x_end : r < 16 * W + NT ? op.gate_end : op.up_end);
      }
    }
  };
  v4f acc[N] = {};                             // outputs 4 (l / 16) ... of row l % 16: NT = 8: the gate's, from l = 32 on the other's
  const int stages = (a.inner + KS - 1) / KS;
  auto products = [&](const char* base) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = (i * 4 + (lane >> 4)) ^ (lane & 15);
      const v4u xs = *reinterpret_cast<const v4u*>(base + (16 * wave + (lane & 15)) * 256 + p * 16);
#pragma unroll
      for (int w = 0; w < N; ++w) acc[w] = mma16<T>(*reinterpret_cast<const v4u*>(base + (16 * (W + w) + (lane & 15)) * 256 + p * 16), xs, acc[w]);
    }
  };
  if constexpr (FAST) {
    for (int s = 0; s < STAGES - 1 && s < stages; ++s) load(s * KS, s, 0);
    int at = 0;
    for (int s = 0; s < stages; ++s) {         // this stage's copies are there, the next ones' may be on their way
      const int next = min(STAGES - 2, stages - 1 - s);
      if (next == 2) wait_copies<2 * COPIES>();
      else if (next == 1) wait_copies<COPIES>();
      else wait_copies();
      __syncthreads();
      if (s + STAGES - 1 < stages) load((s + STAGES - 1) * KS, at ? at - 1 : STAGES - 1, 0);
      products(lds + at * STAGE);
      at = at + 1 == STAGES ? 0 : at + 1;
    }
  } else {
    constexpr int D = STAGES - 1;
#pragma unroll
    for (int s = 0; s < D; ++s)
      if (s < stages) load(s * KS, 0, s);
    for (int s0 = 0; s0 < stages; s0 += D)
#pragma unroll
      for (int d = 0; d < D; ++d) {
        const int s = s0 + d;
        if (s >= stages) break;
        char* base = lds + s % 2 * STAGE;      // whose readers have passed the last barrier
#pragma unroll
        for (int c = 0; c < COPIES; ++c) *reinterpret_cast<v4u*>(base + (wave * COPIES + c) * 1024 + lane * 16) = held[d][c];
        __syncthreads();
        if (s + D < stages) load((s + D) * KS, 0, d);
        products(base);
      }
  }
  const int64_t row = row0 + 16 * wave + (lane & 15);
  const int n = col0 + (lane >> 4) * 4;
  const v4f gb = bias_at(a.gate_bias, m, n, a.outer), ub = bias_at(a.up_bias, m, n, a.outer);
  if constexpr (N == 1) {
    v4f up;
#pragma unroll
    for (int e = 0; e < 4; ++e) up[e] = __shfl_xor(acc[0][e], 32);
    if (lane < 32) finish<T>(a, m, row, n, acc[0], up, gb, ub);
  } else {
    finish<T>(a, m, row, n, acc[0], acc[1], gb, ub);
  }
}

// Launches over tiles of MT rows and NT outputs: as many mutants a launch as fit, or rows.
hipError_t over_tiles(const void* kernel, const mure_attn_gated_args& a, int64_t es, int MT, int NT, unsigned threads, unsigned lds, hipStream_t s) {
  if (lds > 65536)                             // more than the default limit has to be asked for
    if (const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds); e != hipSuccess) return e;
  const int64_t m_tiles = (a.rows + MT - 1) / MT;
  const int n_tiles = (a.outer + NT - 1) / NT;
  const int64_t blocks = ((int64_t)1 << 32) / threads - 1;
  const int64_t rows_most = std::min(m_tiles, blocks / n_tiles), mutants_most = std::max<int64_t>(1, blocks / (n_tiles * rows_most));
  for (int64_t m0 = 0; m0 < a.n_mutants; m0 += mutants_most)
    for (int64_t r0 = 0; r0 < m_tiles; r0 += rows_most) {
      mure_attn_gated_args b = a;
      const int64_t ms = std::min(mutants_most, a.n_mutants - m0);
      auto moved = [&](const void* p, int64_t e) { return static_cast<const void*>(static_cast<const char*>(p) + e * es); };
      b.x.p = moved(a.x.p, m0 * a.x.mutant_stride + r0 * MT * a.x.row_stride);
      b.gate.p = moved(a.gate.p, m0 * a.gate.mutant_stride);
      b.up.p = moved(a.up.p, m0 * a.up.mutant_stride);
      b.out.p = const_cast<void*>(moved(a.out.p, m0 * a.out.mutant_stride + r0 * MT * a.out.row_stride));
      if (b.gate_bias.p) b.gate_bias.p += m0 * a.gate_bias.mutant_stride;
      if (b.up_bias.p) b.up_bias.p += m0 * a.up_bias.mutant_stride;
      int tiles = (int)std::min(rows_most, m_tiles - r0), nt = n_tiles;
      b.rows = std::min(a.rows - r0 * MT, (int64_t)tiles * MT);
      void* at[] = {&b, &nt, &tiles};
      if (const hipError_t e = hipLaunchKernel(kernel, dim3((unsigned)(ms * tiles * n_tiles)), dim3(threads), at, lds, s); e != hipSuccess) return e;
    }
  return hipSuccess;
}

template <typename T, int MT, int NT, int WM, int WN, int BYTES, bool PARTS> hipError_t gated_f(const mure_attn_gated_args& a, bool fast, hipStream_t s) {
  return over_tiles(fast ? reinterpret_cast<const void*>(gated_kernel<T, MT, NT, WM, WN, BYTES, true, PARTS>)
                         : reinterpret_cast<const void*>(gated_kernel<T, MT, NT, WM, WN, BYTES, false, PARTS>),
                    a, sizeof(T), MT, NT, 64 * WM * WN, 2 * (MT + 2 * NT) * BYTES, s);
}

template <typename T, int W, int NT, int STAGES> hipError_t gated_few(const mure_attn_gated_args& a, bool fast, hipStream_t s) {
  return over_tiles(fast ? reinterpret_cast<const void*>(gated_few_kernel<T, W, NT, STAGES, true>) : reinterpret_cast<const void*>(gated_few_kernel<T, W, NT, STAGES, false>), a,
                    sizeof(T), 16 * W, NT, 64 * W, STAGES * (16 * W + 2 * NT) * 256, s);
}

template <typename T, int TM> hipError_t gated_split(const mure_attn_gated_args& a, hipStream_t s) {
  return over_tiles(reinterpret_cast<const void*>(gated_split_kernel<T, TM>), a, sizeof(T), 16 * TM, 16, 64 * SPLIT, 0, s);
}

constexpr int64_t CUS = 256;

// Whether the last round of blocks is nearly full, counted as if a compute unit worked on one at a time.  Two and more of the
// smaller tiles fit, so that a launch just past a round of either counts as worse than it is: 4 mutants' weights over 2724 shared
// float32 rows, 2667 inputs to 175 outputs, 264 tiles of 128 rows or 516 of 64, take 332 us.
bool fills(int64_t blocks) { return 6 * blocks >= 5 * ((blocks + CUS - 1) / CUS * CUS); }

// Tiles of 128 rows by 64 outputs, in float32 of 64 rows where those leave the last round half empty: 2048 inputs to 1024
// outputs, 3000 rows (384 tiles) 217 us so and 264 in tiles of 128; 512 to 1024, 2600 rows (336 tiles) 58 and 71.
template <typename T, bool PARTS> hipError_t gated_tiles(const mure_attn_gated_args& a, bool fast, hipStream_t s) {
  constexpr int BYTES = sizeof(T) == 4 ? 64 : 128;             // 12500 rows of 16 mutants, 128 to 341 float32: 330 us, with 128 bytes 380
  if constexpr (sizeof(T) == 4)
    if (!fills((a.rows + 127) / 128 * ((a.outer + 63) / 64) * a.n_mutants)) return gated_f<T, 64, 64, 2, 2, BYTES, PARTS>(a, fast, s);
  return gated_f<T, 128, 64, 2, 2, BYTES, PARTS>(a, fast, s);
}

// Which form, from the sizes (times in us).
// Sums in eighths (`splits`), 2048 inputs to 512 outputs: side by side, or one after the other in tiles.  bfloat16: 64 rows 10
//   side by side (26 in tiles), 1000 rows 35 (27), 4000 rows 119 (30).  float32: 64 rows 21 (139), 1000 rows 81 (88), 1200
//   rows 100 (88), 2000 rows 160 (89).  Without the eighths 16000 rows take 71 in place of 74 (float32: 520, 548).
// Otherwise, 2048 inputs to 5632 outputs: few rows with 8 or 16 outputs a block.  bfloat16: 64 rows 14 (tiles 26), 128 rows
//   25 (26).  float32: 128 rows 73 (tiles 140), 170 rows 115 (147, two rounds of tiles); 1000 rows to 1024 outputs 90 (89).
// A round of float32 tiles of 64 x 64 takes as long as these forms for 64 and 108 tiles' results of 128 x 64.
// Larger tiles, of 256 rows by 128 outputs and bfloat16, take half the loads for a product, but one is all that a compute
//   unit holds: where their last round is nearly full.  4096 inputs to 4096 outputs, 1024 rows (half a round) 99 (smaller
//   tiles 69), 2048 rows (one round) 114 (137), 4096 rows 220 (260), 8192 rows 432 (511).
template <typename T> hipError_t gated_t(const mure_attn_gated_args& a, bool fast, hipStream_t s) {
  const int64_t results = a.rows * a.outer * a.n_mutants / (128 * 64), small = (a.rows + 63) / 64 * ((a.outer + 63) / 64) * a.n_mutants, rounds = (small + CUS - 1) / CUS;
  if (splits<T>(a)) {
    if (results >= (sizeof(T) == 4 ? 64 * rounds : 40)) return gated_tiles<T, true>(a, fast, s);
    return a.rows <= 16 ? gated_split<T, 1>(a, s) : gated_split<T, 2>(a, s);
  }
  if (a.rows <= 16) return gated_few<T, 1, 8, 4>(a, fast, s);
  if (a.rows <= 32) return gated_few<T, 2, 8, 4>(a, fast, s);
  if (a.rows <= 64 || (sizeof(T) == 4 && results < 108 * rounds)) return gated_few<T, 4, 16, 3>(a, fast, s);
  if constexpr (sizeof(T) == 2)
    if (fills((a.rows + 255) / 256 * ((a.outer + 127) / 128) * a.n_mutants)) return gated_f<T, 256, 128, 2, 4, 128, false>(a, fast, s);
  return gated_tiles<T, false>(a, fast, s);
}

}  // namespace

hipError_t launch_attn_gated(const mure_attn_gated_args& args, bool fast, hipStream_t s) {
  mure_attn_gated_args a = args;
  // Rows of all mutants of a layer that they share are one matrix.
  if (a.n_mutants > 1 && !a.gate.mutant_stride && !a.up.mutant_stride && !(a.gate_bias.p && a.gate_bias.mutant_stride) && !(a.up_bias.p && a.up_bias.mutant_stride) &&
      a.x.mutant_stride == a.rows * a.x.row_stride && a.out.mutant_stride == a.rows * a.out.row_stride && a.x.mutant_stride) {
    a.rows *= a.n_mutants;
    a.n_mutants = 1;
  }
  return a.dtype == MURE_F32 ? gated_t<float>(a, fast, s) : gated_t<bf16_t>(a, fast, s);
}

}  // namespace mure
