// Causal depthwise convolution along the sequences of a batch:
//   y[t][c] = act(b[c] + sum_k w[c][k] x[t - K + 1 + k][c]).
//
// 2 K operations for 2 elements moved: bound by HBM (65536 x 4096 bfloat16, 4
// taps: 203 us, 5.3 TB/s; a copy of as much takes 181).  A thread owns 16 bytes
// of channels (8 bfloat16, 4 float32) of one run of consecutive tokens; the
// last K - 1 rows stay in its registers, so that a row is read once, but for
// the K - 1 rows before the run, which the run before reads too.  Rows are
// taken ROWS at a time: three keep 3 waves a SIMD at 4 taps of bfloat16, with
// four the float32 kernel waits longer (250 sequences of 16 mutants 24.7 us,
// now 21.3).  The activation and odd widths are instances of their own: as
// branches in the row they cost a quarter of the smallest calls' time.
// Widths that fill no whole vector: the last vector of a row starts early (its
// first `dup` channels are the neighbour's and are not stored); vectors then
// stand at any address, which costs up to a fifth of the bandwidth.
#include <algorithm>

#include "seq_dev.hpp"

namespace mure {

// N elements copied as they are
template <typename T, int N> struct Bits {
  typedef T one __attribute__((ext_vector_type(N)));
  typedef one __attribute__((aligned(sizeof(T)))) any;
  static __device__ __forceinline__ one load(const T* p) { return *reinterpret_cast<const any*>(p); }
  static __device__ __forceinline__ void store_from(T* p, one v, int first) {
    if (first == 0) {
      *reinterpret_cast<any*>(p) = v;
      return;
    }
#pragma unroll
    for (int j = 1; j < N; ++j)
      if (j >= first) p[j] = v[j];
  }
};
template <typename T> struct Bits<T, 1> {
  typedef T one;
  static __device__ __forceinline__ one load(const T* p) { return *p; }
  static __device__ __forceinline__ void store_from(T* p, one v, int) { *p = v; }
};

// SILU: the activation; ODD: the last vector of a row starts early
template <typename T, int K, int N, bool SILU, bool ODD>
__global__ __launch_bounds__(256) void seq_conv_kernel(SeqConvArgs k, DivU32 dvec, uint32_t total) {
  constexpr int ROWS = 3, H = K - 1;
  const mure_seq_conv_args& a = k.a;
  const uint32_t id = blockIdx.x * 256u + threadIdx.x;
  if (id >= total) return;
  int item, v;
  divmodu(dvec, id, item, v);
  const SeqItem it = seq_item(k.items, k.item0 + item);
  const int64_t m = blockIdx.y;
  const int C = a.channels;
  int c = v * N, dup = 0;
  if (ODD && c + N > C) dup = c + N - C, c = C - N;    // N == 1 where C < the vector
  const T* x = static_cast<const T*>(a.x.p) + m * a.x.mutant_stride + (int64_t)it.row0 * a.x.row_stride + c;
  T* y = static_cast<T*>(a.out.p) + m * a.out.mutant_stride + (int64_t)it.row0 * a.out.row_stride + c;
  const int64_t held = (int64_t)it.seq * H * C + c;    // of this sequence's state
  const T* st = a.state ? static_cast<const T*>(a.state) + m * a.state_mutant_stride + held : nullptr;

  float w[K][N], b[N];
  {
    const T* wp = static_cast<const T*>(a.taps) + m * a.taps_mutant_stride + (int64_t)c * K;
#pragma unroll
    for (int i = 0; i < K; ++i) {                      // K vectors hold the channels' K taps each
      float t[N];
      load_n<T, N>(wp + i * N, t);
#pragma unroll
      for (int j = 0; j < N; ++j) w[(i * N + j) % K][(i * N + j) / K] = t[j];
    }
#pragma unroll
    for (int j = 0; j < N; ++j) b[j] = a.bias.p ? a.bias.p[m * a.bias.mutant_stride + c + j] : 0.f;
  }
  float r[H + ROWS][N];                                // rows t - H ... t + ROWS - 1
#pragma unroll
  for (int i = 0; i < H; ++i) {
    const int pos = it.pos0 - H + i;
    if (pos >= 0) load_n<T, N>(x - (int64_t)(H - i) * a.x.row_stride, r[i]);
    else if (st) load_n<T, N>(st + (int64_t)(H + pos) * C, r[i]);
    else
#pragma unroll
      for (int j = 0; j < N; ++j) r[i][j] = 0.f;
  }
  // The new state, by the sequence's first run: it has read the old one, which
  // may lie in the same place.  Row j comes from position total - H + j: from
  // the old state's row total + j, which is not before row j, or from x.
  const bool carry = H > 0 && it.pos0 == 0 && a.state_out;
  typename Bits<T, N>::one keep[H + 1];
  if (carry)
#pragma unroll
    for (int j = 0; j < H; ++j) {
      const int pos = it.total - H + j;
      keep[j] = typename Bits<T, N>::one(0);
      if (pos >= 0) keep[j] = Bits<T, N>::load(x + (int64_t)pos * a.x.row_stride);
      else if (st) keep[j] = Bits<T, N>::load(st + (int64_t)(H + pos) * C);
    }
  auto rows = [&](int t, auto whole) {                 // ROWS of them, or what is left
    constexpr bool WHOLE = decltype(whole)::value;
    const T* from = x + (int64_t)t * a.x.row_stride;
#pragma unroll
    for (int u = 0; u < ROWS; ++u)
      if (WHOLE || t + u < it.len) load_n<T, N>(from + u * a.x.row_stride, r[H + u]);
    T* to = y + (int64_t)t * a.out.row_stride;
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
      if (!WHOLE && t + u >= it.len) break;
      float s[N];
#pragma unroll
      for (int j = 0; j < N; ++j) {
        s[j] = b[j];
#pragma unroll
        for (int i = 0; i < K; ++i) s[j] = fmaf(w[i][j], r[u + i][j], s[j]);
        if (SILU) s[j] = seq_silu(s[j]);
      }
      store_from<T, N>(to + u * a.out.row_stride, s, ODD ? dup : 0);
    }
#pragma unroll
    for (int i = 0; i < H; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) r[i][j] = r[ROWS + i][j];
  };
  int t = 0;
  for (; t + ROWS <= it.len; t += ROWS) rows(t, std::true_type());
  if (t < it.len) rows(t, std::false_type());
  if (carry) {
    T* so = static_cast<T*>(a.state_out) + m * a.state_out_mutant_stride + held;
#pragma unroll
    for (int j = 0; j < H; ++j) Bits<T, N>::store_from(so + (int64_t)j * C, keep[j], ODD ? dup : 0);
  }
}

template <typename T, int K, int N, bool SILU, bool ODD>
static hipError_t conv_n(SeqConvArgs k, hipStream_t s) {
  const int vecs = (k.a.channels + N - 1) / N;
  const int most = (1 << 30) / vecs;                   // items of a launch: its grid has fewer than 2^32 threads
  for (int left = k.n_items; left > 0; left -= most, k.item0 += most) {
    const uint32_t total = (uint32_t)std::min(left, most) * (uint32_t)vecs;
    if (hipError_t e = launch(seq_conv_kernel<T, K, N, SILU, ODD>, dim3((total + 255) / 256, (unsigned)k.a.n_mutants), 256, s, k,
                              make_divu32((uint32_t)vecs), total);
        e != hipSuccess)
      return e;
  }
  return hipSuccess;
}

template <typename T, int K, bool SILU>
static hipError_t conv_v(const SeqConvArgs& k, hipStream_t s) {
  constexpr int N = Vec<T>::N;
  if (k.a.channels < N) return conv_n<T, K, 1, SILU, false>(k, s);
  return k.a.channels % N ? conv_n<T, K, N, SILU, true>(k, s) : conv_n<T, K, N, SILU, false>(k, s);
}

template <typename T, int K>
static hipError_t conv_k(const SeqConvArgs& k, hipStream_t s) {
  return k.a.activation == MURE_SEQ_SILU ? conv_v<T, K, true>(k, s) : conv_v<T, K, false>(k, s);
}

template <typename T>
static hipError_t conv_t(const SeqConvArgs& k, hipStream_t s) {
  switch (k.a.n_taps) {
    case 1: return conv_k<T, 1>(k, s);
    case 2: return conv_k<T, 2>(k, s);
    case 3: return conv_k<T, 3>(k, s);
    case 4: return conv_k<T, 4>(k, s);
    case 5: return conv_k<T, 5>(k, s);
    case 6: return conv_k<T, 6>(k, s);
    case 7: return conv_k<T, 7>(k, s);
    case 8: return conv_k<T, 8>(k, s);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_seq_conv(const SeqConvArgs& k, hipStream_t s) {
  return k.a.dtype == MURE_F32 ? conv_t<float>(k, s) : conv_t<bf16_t>(k, s);
}

}  // namespace mure
