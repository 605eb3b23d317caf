// The norms around a block, row by row:
//   v = after(y act(gate)),  r = residual + scale v,  out = before(r).
//
// A few operations per element moved: bound by HBM.  L lanes own a row (16 or
// more; a whole wave up to 4 vectors a lane, a block above) and keep it in
// registers through both norms, so that every tensor is read or written once;
// means are taken over the lanes by cross-lane adds, over waves through LDS.
// Variances are of the centred values (two passes over the registers).  A
// row's last vector may start early (its first `dup` channels are another
// lane's and count for nothing here).
#include <algorithm>

#include "seq_dev.hpp"

namespace mure {

// Sum over the L lanes of a row: the same in all of them.
template <int L> __device__ __forceinline__ float row_sum(float v, float* lds) {
#pragma unroll
  for (int s = 1; s < (L < 64 ? L : 64); s *= 2) v += __shfl_xor(v, s);
  if constexpr (L > 64) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();                                   // the last sum is read
    if ((threadIdx.x & 63) == 0) lds[wave] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < L / 64; ++w) v += lds[w];
  }
  return v;
}

// v to its norm, times w plus b where given.
template <int L, int V, int N>
__device__ __forceinline__ void norm_row(float (&v)[V][N], const int (&dup)[V], int kind, float inv_width, float eps, float* lds) {
  if (kind == MURE_SEQ_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) s += j >= dup[i] ? v[i][j] : 0.f;
    const float mean = row_sum<L>(s, lds) * inv_width;
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
  const float f = rsqrtf(fmaf(row_sum<L>(s, lds), inv_width, eps));
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) v[i][j] *= f;
}

template <typename R, int N> __device__ __forceinline__ void load_row(const R* p, float (&v)[N]) {
  if constexpr (sizeof(R) == 4 && N == 8) {            // a float32 residual beside 8 bfloat16
    float t[4];
    load_n<R, 4>(p, t);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = t[j];
    load_n<R, 4>(p + 4, t);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[4 + j] = t[j];
  } else {
    load_n<R, N>(p, v);
  }
}

template <typename R, int N> __device__ __forceinline__ void store_row(R* p, const float (&v)[N], int first) {
  if constexpr (sizeof(R) == 4 && N == 8) {
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
  __shared__ float lds[16];
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
  const float* aw = a.after_weight.p ? a.after_weight.p + m * a.after_weight.mutant_stride : nullptr;
  const float* ab = a.after_bias.p ? a.after_bias.p + m * a.after_bias.mutant_stride : nullptr;
  const float* sc = a.scale.p ? a.scale.p + m * a.scale.mutant_stride : nullptr;
  const float* bw = a.before_weight.p ? a.before_weight.p + m * a.before_weight.mutant_stride : nullptr;
  const float* bb = a.before_bias.p ? a.before_bias.p + m * a.before_bias.mutant_stride : nullptr;
  const T* yp = static_cast<const T*>(a.y.p) + m * a.y.mutant_stride;
  const T* zp = a.gate_at ? static_cast<const T*>(a.gate.p) + m * a.gate.mutant_stride : nullptr;
  const R* rp = a.residual.p ? static_cast<const R*>(a.residual.p) + m * a.residual.mutant_stride : nullptr;
  R* ro = a.residual_out.p ? static_cast<R*>(a.residual_out.p) + m * a.residual_out.mutant_stride : nullptr;
  T* op = a.out.p ? static_cast<T*>(a.out.p) + m * a.out.mutant_stride : nullptr;
  for (int64_t row = (int64_t)blockIdx.x * PER + threadIdx.x / L; row < a.rows; row += (int64_t)gridDim.x * PER) {
    float v[V][N], g[V][N], res[V][N];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      load_row<T, N>(yp + row * a.y.row_stride + at[i], v[i]);
      if (zp) load_row<T, N>(zp + row * a.gate.row_stride + at[i], g[i]);
      if (rp) load_row<R, N>(rp + row * a.residual.row_stride + at[i], res[i]);
    }
    if (zp)
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
          g[i][j] = a.gate_activation == MURE_SEQ_SILU      ? seq_silu(g[i][j])
                    : a.gate_activation == MURE_SEQ_SIGMOID ? seq_sigmoid(g[i][j])
                                                            : g[i][j];
    if (a.gate_at == 1)
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) v[i][j] *= g[i][j];
    if (a.after) norm_row<L, V, N>(v, dup, a.after, inv_width, a.eps, lds);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float t[N];
      if (aw) {
        load_row<float, N>(aw + at[i], t);
#pragma unroll
        for (int j = 0; j < N; ++j) v[i][j] *= t[j];
      }
      if (ab) {
        load_row<float, N>(ab + at[i], t);
#pragma unroll
        for (int j = 0; j < N; ++j) v[i][j] += t[j];
      }
      if (a.gate_at == 2)
#pragma unroll
        for (int j = 0; j < N; ++j) v[i][j] *= g[i][j];
#pragma unroll
      for (int j = 0; j < N; ++j) t[j] = 1.f;
      if (sc) load_row<float, N>(sc + at[i], t);
#pragma unroll
      for (int j = 0; j < N; ++j) v[i][j] = fmaf(t[j] * a.scale_all, v[i][j], rp ? res[i][j] : 0.f);
      if (ro && dup[i] < N) store_row<R, N>(ro + row * a.residual_out.row_stride + at[i], v[i], dup[i]);
    }
    if (!op) continue;
    norm_row<L, V, N>(v, dup, a.before, inv_width, a.eps, lds);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float t[N];
      if (bw) {
        load_row<float, N>(bw + at[i], t);
#pragma unroll
        for (int j = 0; j < N; ++j) v[i][j] *= t[j];
      }
      if (bb) {
        load_row<float, N>(bb + at[i], t);
#pragma unroll
        for (int j = 0; j < N; ++j) v[i][j] += t[j];
      }
      if (dup[i] < N) store_row<T, N>(op + row * a.out.row_stride + at[i], v[i], dup[i]);
    }
  }
}

template <typename T, typename R, int L, int V, int N>
static hipError_t norm_l(const mure_seq_norm_args& a, hipStream_t s) {
  constexpr int BLOCK = L > 256 ? L : 256, PER = BLOCK / L;
  const int vecs = (a.channels + N - 1) / N;
  const int64_t blocks = std::min<int64_t>((a.rows + PER - 1) / PER, 1 << 20);
  seq_norm_kernel<T, R, L, V, N><<<dim3((unsigned)blocks, (unsigned)a.n_mutants), BLOCK, 0, s>>>(a, vecs);
  return hipGetLastError();
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
  return norm_l<T, R, 1024, 4, N>(a, s);
}

hipError_t launch_seq_norm(const mure_seq_norm_args& a, hipStream_t s) {
  if (a.dtype == MURE_F32) return norm_r<float, float>(a, s);
  return a.residual_dtype == MURE_F32 ? norm_r<bf16_t, float>(a, s) : norm_r<bf16_t, bf16_t>(a, s);
}

}  // namespace mure
