// The norms around a block, row by row:
//   v = after(y act(gate)),  r = residual + scale v,  out = before(r).
//
// A few operations per element moved: bound by HBM (65536 rows of 4096, gate,
// bfloat16: 517 us, 5.2 TB/s, a copy of as much takes 465).  L lanes own a row (16 to
// a whole wave up to 2 vectors a lane, a block above) and keep it in registers
// through both norms, so that every tensor is read or written once (above 8192
// channels 92 to 132 bytes a lane are in scratch: 4096 rows of 16384 run at 2.8
// to 4.6 TB/s); means are
// taken over the lanes by cross-lane adds, over waves through LDS.  A block
// goes from row to row and keeps the weights in registers; a row's inputs are
// loaded before the row before it is computed, so that the loads are in flight
// during the sums.  Variances are of the centred values (two passes over the
// registers).  A row's last vector may start early (its first `dup` channels
// are another lane's and count for nothing here).
#include <algorithm>

#include "seq_dev.hpp"

namespace mure {

template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}

// Sum over the L lanes of a row: the same in all of them.  Within 16 lanes
// through DPP: lane ^ 1, lane ^ 2, the mirror of 8 and of 16 lanes; across
// rows of 16 and halves of 32 through gfx950's swaps.
template <int L> __device__ __forceinline__ float row_sum(float v, float (*lds)[16], int& turn) {
  v += dpp<0xb1>(v);                                   // quad_perm 1 0 3 2
  v += dpp<0x4e>(v);                                   // quad_perm 2 3 0 1
  v += dpp<0x141>(v);                                  // row_half_mirror
  v += dpp<0x140>(v);                                  // row_mirror
  if constexpr (L > 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (L > 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (L > 64) {
    float* at = lds[turn ^= 1];                        // the other turn's sums may still be read
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
    __syncthreads();
    v = at[0];
#pragma unroll
    for (int w = 1; w < L / 64; ++w) v += at[w];
  }
  return v;
}

// A vector of N elements of R as it comes from memory, and as floats.
template <typename R, int N> struct Raw {
  typedef R one __attribute__((ext_vector_type(N)));
  typedef one __attribute__((aligned(sizeof(R)))) any;
  one r;
  __device__ __forceinline__ void load(const R* p) { r = *reinterpret_cast<const any*>(p); }
  __device__ __forceinline__ float operator[](int j) const { return to_f<R>(r[j]); }
};
template <typename R> struct Raw<R, 1> {
  R r;
  __device__ __forceinline__ void load(const R* p) { r = *p; }
  __device__ __forceinline__ float operator[](int) const { return to_f<R>(r); }
};

template <typename R, int N> __device__ __forceinline__ void store_row(R* p, const float (&v)[N], int first) {
  if constexpr (sizeof(R) == 4 && N == 8) {            // a float32 residual beside 8 bfloat16
    if (first == 0) {
      const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
      store_n<R, 4>(p, lo);
      store_n<R, 4>(p + 4, hi);
      return;
    }
#pragma unroll
    for (int j = 1; j < N; ++j)
      if (j >= first) p[j] = v[j];
  } else {
    store_from<R, N>(p, v, first);
  }
}

// T: y, gate, out; R: residual; L: lanes of a row; V: vectors of a lane
template <typename T, typename R, int L, int V, int N>
__global__ __launch_bounds__(L > 256 ? L : 256) void seq_norm_kernel(mure_seq_norm_args a, int vecs) {
  constexpr int BLOCK = L > 256 ? L : 256, PER = BLOCK / L;
  constexpr bool AHEAD = BLOCK == 256 || V * N < 16;   // else a block of 1024 has no registers for it
  __shared__ float lds[2][16];
  int turn = 0;
  const int64_t m = blockIdx.y;
  const int lane = threadIdx.x % L, C = a.channels;
  const float inv_width = 1.f / (float)C;
  int at[V], dup[V];                                   // dup = N: no vector here
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int v = lane + i * L;
    at[i] = min(v * N, C - N);
    dup[i] = v >= vecs ? N : v * N - at[i];
  }
  const T* yp = static_cast<const T*>(a.y.p) + m * a.y.mutant_stride;
  const T* zp = static_cast<const T*>(a.gate.p) + m * a.gate.mutant_stride;
  const R* rp = static_cast<const R*>(a.residual.p) + m * a.residual.mutant_stride;
  R* ro = static_cast<R*>(a.residual_out.p) + m * a.residual_out.mutant_stride;
  T* op = static_cast<T*>(a.out.p) + m * a.out.mutant_stride;
  const bool gated = a.gate_at != 0, summed = a.residual.p != nullptr;

  Raw<T, N> ny[V], nz[V];                              // the next row
  Raw<R, N> nr[V];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      ny[i].load(yp + row * a.y.row_stride + at[i]);
      if (gated) nz[i].load(zp + row * a.gate.row_stride + at[i]);
      if (summed) nr[i].load(rp + row * a.residual.row_stride + at[i]);
    }
  };
  int64_t row = (int64_t)blockIdx.x * PER + threadIdx.x / L;
  if (AHEAD && row < a.rows) fetch(row);

  // the weights: of `after` with the scale, of `before`; their biases are read where they are used
  float aw[V][N], bw[V][N];
  {
    const float* w1 = a.after_weight.p ? a.after_weight.p + m * a.after_weight.mutant_stride : nullptr;
    const float* sc = a.scale.p ? a.scale.p + m * a.scale.mutant_stride : nullptr;
    const float* w2 = a.before_weight.p ? a.before_weight.p + m * a.before_weight.mutant_stride : nullptr;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      Raw<float, N> r1, rs, r2;
      if (w1) r1.load(w1 + at[i]);
      if (sc) rs.load(sc + at[i]);
      if (w2) r2.load(w2 + at[i]);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        aw[i][j] = (sc ? rs[j] * a.scale_all : a.scale_all) * (w1 ? r1[j] : 1.f);
        bw[i][j] = w2 ? r2[j] : 1.f;
      }
    }
  }
  const float* ab = a.after_bias.p ? a.after_bias.p + m * a.after_bias.mutant_stride : nullptr;
  const float* as = a.scale.p ? a.scale.p + m * a.scale.mutant_stride : nullptr;
  const float* bb = a.before_bias.p ? a.before_bias.p + m * a.before_bias.mutant_stride : nullptr;

  // v to its norm, without weight and bias
  auto norm = [&](float (&v)[V][N], int kind) {
    if (kind == MURE_SEQ_LAYER) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) s += j >= dup[i] ? v[i][j] : 0.f;
      const float mean = row_sum<L>(s, lds, turn) * inv_width;
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) v[i][j] -= mean;
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) s = j >= dup[i] ? fmaf(v[i][j], v[i][j], s) : s;
    const float f = rsqrtf(fmaf(row_sum<L>(s, lds, turn), inv_width, a.eps));
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) v[i][j] *= f;
  };

  while (row < a.rows) {
    const int64_t next = row + (int64_t)gridDim.x * PER;
    if (!AHEAD) fetch(row);
    Raw<T, N> cy[V], cz[V];
    Raw<R, N> cr[V];
#pragma unroll
    for (int i = 0; i < V; ++i) cy[i] = ny[i], cz[i] = nz[i], cr[i] = nr[i];
    if (AHEAD && next < a.rows) fetch(next);
    float v[V][N], g[V][N];
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) v[i][j] = cy[i][j];
    if (gated) {
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float z = cz[i][j];
          g[i][j] = a.gate_activation == MURE_SEQ_LINEAR ? z : seq_sigmoid(z) * (a.gate_activation == MURE_SEQ_SILU ? z : 1.f);
          if (a.gate_at == 1) v[i][j] *= g[i][j];
        }
    }
    if (a.after) norm(v, a.after);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      Raw<float, N> rb, rs;
      if (ab) rb.load(ab + at[i]);
      if (ab && as) rs.load(as + at[i]);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        v[i][j] *= aw[i][j];
        if (ab) v[i][j] = fmaf(rb[j], as ? rs[j] * a.scale_all : a.scale_all, v[i][j]);
        if (a.gate_at == 2) v[i][j] *= g[i][j];
        if (summed) v[i][j] += cr[i][j];
      }
      if (a.residual_out.p && dup[i] < N) store_row<R, N>(ro + row * a.residual_out.row_stride + at[i], v[i], dup[i]);
    }
    if (a.out.p) {
      norm(v, a.before);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        Raw<float, N> rb;
        if (bb) rb.load(bb + at[i]);
#pragma unroll
        for (int j = 0; j < N; ++j) v[i][j] = bb ? fmaf(v[i][j], bw[i][j], rb[j]) : v[i][j] * bw[i][j];
        if (dup[i] < N) store_row<T, N>(op + row * a.out.row_stride + at[i], v[i], dup[i]);
      }
    }
    row = next;
  }
}

template <typename T, typename R, int L, int V, int N>
static hipError_t norm_l(const mure_seq_norm_args& a, hipStream_t s) {
  constexpr int BLOCK = L > 256 ? L : 256, PER = BLOCK / L;
  const int vecs = (a.channels + N - 1) / N;
  // Blocks that the chip holds at once where a SIMD has 3 waves (a lane of 16 channels) or 4, shared out over the
  // mutants.  Times of 65536 rows of 4096 bfloat16 with 512, 768, 1024 and 2048 blocks: 511, 516, 546 and 532 us; with
  // a float32 residual, of which a SIMD has 2 waves: 751, 771, 758 and 787; 16384 channels of which with 128, 192, 256
  // and 512 blocks, one of them a CU, 4096 rows: 369, 292, 243 and 249.
  constexpr int FULL = (V * N == 16 ? 768 : 1024) * 256 / BLOCK;
  const int64_t most = std::max<int64_t>(1, FULL / a.n_mutants);
  const int64_t blocks = std::min<int64_t>((a.rows + PER - 1) / PER, most);
  return launch(seq_norm_kernel<T, R, L, V, N>, dim3((unsigned)blocks, (unsigned)a.n_mutants), BLOCK, s, a, vecs);
}

// Lanes and vectors by the width alone: the order of the sums is part of the
// result.
template <typename T, typename R>
static hipError_t norm_r(const mure_seq_norm_args& a, hipStream_t s) {
  constexpr int N = Vec<T>::N;
  if (a.channels < N) return norm_l<T, R, 16, 1, 1>(a, s);
  const int vecs = (a.channels + N - 1) / N;
  if (vecs <= 16) return norm_l<T, R, 16, 1, N>(a, s);
  if (vecs <= 32) return norm_l<T, R, 32, 1, N>(a, s);
  if (vecs <= 64) return norm_l<T, R, 64, 1, N>(a, s);
  if (vecs <= 128) return norm_l<T, R, 64, 2, N>(a, s);
  if (vecs <= 256) return norm_l<T, R, 256, 1, N>(a, s);
  if (vecs <= 512) return norm_l<T, R, 256, 2, N>(a, s);
  if (vecs <= 1024) return norm_l<T, R, 1024, 1, N>(a, s);
  if (vecs <= 2048) return norm_l<T, R, 1024, 2, N>(a, s);
  if constexpr (N == 4) return norm_l<T, R, 1024, 4, N>(a, s);
  return hipErrorInvalidValue;                         // 8 channels a vector: 16384 channels are 2048
}

hipError_t launch_seq_norm(const mure_seq_norm_args& a, hipStream_t s) {
  if (a.dtype == MURE_F32) return norm_r<float, float>(a, s);
  return a.residual_dtype == MURE_F32 ? norm_r<bf16_t, float>(a, s) : norm_r<bf16_t, bf16_t>(a, s);
}

}  // namespace mure
