// Gated feed-forward layer (mure_attn_gated): both projections as one tiled
// matrix product, with biases, activation and product behind it.
//
// A block computes MT rows by NT outputs: for every 128 bytes of the summed
// axis, MT rows of x and NT rows of each projection's weights are copied to
// LDS, two stages in turn.  A wave's instructions are 16 x 16 results of 64
// bytes of the summed axis, weights first, so that a lane ends with four
// neighbouring outputs of a row, gate and up alike.  Every result adds its
// terms in the same order in any tile, so that it does not depend on the
// number of rows.
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

__device__ __forceinline__ int twist(int row) { return (row >> 1) & 7; }

// WM x WN waves
template <typename T, int MT, int NT, int WM, int WN, bool FAST>
__global__ __launch_bounds__(64 * WM * WN, 2) void gated_kernel(mure_attn_gated_args a, int n_tiles, int m_tiles) {
  constexpr int WAVES = WM * WN, ROWS = MT + 2 * NT, STAGE = ROWS * 128, E = 16 / (int)sizeof(T), KS = 8 * E;
  constexpr int TM = MT / WM / 16, TN = NT / WN / 16;
  extern __shared__ char lds[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int mt = blockIdx.x / n_tiles % m_tiles, nt = blockIdx.x % n_tiles, m = blockIdx.x / n_tiles / m_tiles;
  const int64_t row0 = (int64_t)mt * MT;
  const int col0 = nt * NT;
  const T* x = static_cast<const T*>(a.x.p) + m * a.x.mutant_stride;
  const T* wg = static_cast<const T*>(a.gate.p) + m * a.gate.mutant_stride;
  const T* wu = static_cast<const T*>(a.up.p) + m * a.up.mutant_stride;
  // copies of 1024 bytes: 8 rows of 8 pieces
  constexpr int COPIES = ROWS / 8 / WAVES;
  static_assert(ROWS / 8 % WAVES == 0, "");
  const T* from[COPIES];                       // the lane's row of each, or nothing
#pragma unroll
  for (int c = 0; c < COPIES; ++c) {
    const int r = (wave * COPIES + c) * 8 + lane / 8;
    if (r < MT) from[c] = row0 + r < a.rows ? x + (row0 + r) * a.x.row_stride : nullptr;
    else if (r < MT + NT) from[c] = col0 + r - MT < a.outer ? wg + (int64_t)(col0 + r - MT) * a.gate.row_stride : nullptr;
    else from[c] = col0 + r - MT - NT < a.outer ? wu + (int64_t)(col0 + r - MT - NT) * a.up.row_stride : nullptr;
  }
  auto load = [&](int k0, int stage) {
#pragma unroll
    for (int c = 0; c < COPIES; ++c) {
      const int q = wave * COPIES + c, r = q * 8 + lane / 8, e = k0 + ((lane & 7) ^ twist(r)) * E;
      char* to = lds + stage * STAGE + q * 1024;
      if constexpr (FAST) {
        const void* p = from[c] && e < a.inner ? static_cast<const void*>(from[c] + e) : ZEROS;
        __builtin_amdgcn_global_load_lds(p, (lds_void*)to, 16, 0, 0);
      } else {
        *reinterpret_cast<v4u*>(to + lane * 16) = from[c] && e < a.inner ? load_piece<T>(from[c], e, a.inner) : v4u{0, 0, 0, 0};
      }
    }
  };
  const int wm = wave % WM, wn = wave / WM;
  v4f g[TN][TM], u[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) g[i][j] = v4f{}, u[i][j] = v4f{};
  load(0, 0);
  int stage = 0;
  for (int k0 = 0; k0 < a.inner; k0 += KS, stage ^= 1) {
    wait_copies();
    __syncthreads();
    if (k0 + KS < a.inner) load(k0 + KS, stage ^ 1);
    const char* base = lds + stage * STAGE;
    auto piece = [&](int r, int s) { return *reinterpret_cast<const v4u*>(base + r * 128 + ((s * 4 + (lane >> 4)) ^ twist(r)) * 16); };
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      v4u xs[TM];
#pragma unroll
      for (int j = 0; j < TM; ++j) xs[j] = piece(wm * (MT / WM) + j * 16 + (lane & 15), s);
#pragma unroll
      for (int i = 0; i < TN; ++i) {
        const int r = wn * (NT / WN) + i * 16 + (lane & 15);
        const v4u gs = piece(MT + r, s), us = piece(MT + NT + r, s);
#pragma unroll
        for (int j = 0; j < TM; ++j) {
          g[i][j] = mma16<T>(gs, xs[j], g[i][j]);
          u[i][j] = mma16<T>(us, xs[j], u[i][j]);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < TN; ++i) {
    const int n = col0 + wn * (NT / WN) + i * 16 + (lane >> 4) * 4;
    float gb[4] = {}, ub[4] = {};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (a.gate_bias.p && n + j < a.outer) gb[j] = a.gate_bias.p[m * a.gate_bias.mutant_stride + n + j];
      if (a.up_bias.p && n + j < a.outer) ub[j] = a.up_bias.p[m * a.up_bias.mutant_stride + n + j];
    }
#pragma unroll
    for (int j = 0; j < TM; ++j) {
      const int64_t row = row0 + wm * (MT / WM) + j * 16 + (lane & 15);
      if (row >= a.rows) continue;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = activated(g[i][j][e] + gb[e], a.activation) * (u[i][j][e] + ub[e]);
      store4<T>(static_cast<T*>(a.out.p) + m * a.out.mutant_stride + row * a.out.row_stride, n, a.outer, v[0], v[1], v[2], v[3]);
    }
  }
}

template <typename T, int MT, int NT, int WM, int WN, bool FAST> hipError_t gated_f(const mure_attn_gated_args& a, hipStream_t s) {
  constexpr unsigned LDS = 2 * (MT + 2 * NT) * 128;
  const void* kernel = reinterpret_cast<const void*>(gated_kernel<T, MT, NT, WM, WN, FAST>);
  if (LDS > 65536)
    if (const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)LDS); e != hipSuccess) return e;
  const int64_t m_tiles = (a.rows + MT - 1) / MT;
  const int n_tiles = (a.outer + NT - 1) / NT;
  // as many mutants a launch as fit, or rows
  constexpr int64_t BLOCKS = ((int64_t)1 << 32) / (64 * WM * WN) - 1;
  const int64_t rows_most = std::min(m_tiles, BLOCKS / n_tiles), mutants_most = std::max<int64_t>(1, BLOCKS / (n_tiles * rows_most));
  const int64_t es = sizeof(T);
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
      if (const hipError_t e = hipLaunchKernel(kernel, dim3((unsigned)(ms * tiles * n_tiles)), dim3(64 * WM * WN), at, LDS, s); e != hipSuccess) return e;
    }
  return hipSuccess;
}

template <typename T> hipError_t gated_t(const mure_attn_gated_args& a, bool fast, hipStream_t s) {
  return fast ? gated_f<T, 128, 64, 2, 2, true>(a, s) : gated_f<T, 128, 64, 2, 2, false>(a, s);
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
