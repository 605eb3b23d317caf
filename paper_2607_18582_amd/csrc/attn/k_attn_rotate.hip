// Norm of queries and keys for each head and rotation of their pairs
// (mure_attn_rotate).
//
// Bound by memory: each element is read and written once.  A block takes a run
// of tokens and computes their angles once, for all heads: the product of
// position and frequency and its remainder by pi/2 in float64, sine and cosine
// of that in float32.  Then a team of lanes takes a head at a time, each lane
// both halves of the pairs it turns, in vectors: nothing is exchanged but the
// norm's sums.
#include "../seq/seq_dev.hpp"
#include "attn.hpp"

#include <algorithm>

namespace mure {
namespace {

constexpr int THREADS = 256;

// Cosine and sine of x: x = n pi/2 + r with |r| <= pi/4 (pi/2 in two parts: r is good to 2^-24 for |x| < 2^33, where x
// has 20 bits behind the point itself), then their series, whose next terms are below 2^-27.
__device__ __forceinline__ float2 cos_sin(double x) {
  const double n = __builtin_rint(x * 0.63661977236758134308);
  const double rd = __builtin_fma(-n, 6.123233995736766036e-17, __builtin_fma(-n, 1.5707963267948965580, x));
  const float r = (float)rd, z = r * r;
  const float s = r + r * z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880))));
  const float c = 1.f + z * (-0.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320 + z * (-1.f / 3628800)))));
  const int q = (int)(long long)n & 3;
  const float a = q & 1 ? s : c, b = q & 1 ? c : s;
  return {q == 1 || q == 2 ? -a : a, q >= 2 ? -b : b};
}

template <typename T, int V> struct Raw {
  typedef T raw __attribute__((ext_vector_type(V)));
  typedef raw __attribute__((aligned(sizeof(T)))) any;
};

template <typename T, int V> __device__ __forceinline__ void get(const T* p, float (&v)[V]) {
  if constexpr (V == 1) v[0] = to_f<T>(*p);
  else {
    const auto r = *reinterpret_cast<const typename Raw<T, V>::any*>(p);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = to_f<T>(r[j]);
  }
}

template <typename T, int V> __device__ __forceinline__ void put(T* p, const float (&v)[V]) {
  if constexpr (V == 1) *p = from_f<T>(v[0]);
  else {
    typename Raw<T, V>::raw r;
#pragma unroll
    for (int j = 0; j < V; ++j) r[j] = from_f<T>(v[j]);
    *reinterpret_cast<typename Raw<T, V>::any*>(p) = r;
  }
}

// V pairs a unit, U units a lane.
template <typename T, int V, int U>
__global__ __launch_bounds__(THREADS) void rotate_kernel(AttnRotateArgs k, int team) {
  extern __shared__ float2 turn[];             // [tokens][pairs]
  const mure_attn_rotate_args& a = k.a;
  const int m = blockIdx.x % a.n_mutants, item = k.item0 + blockIdx.x / a.n_mutants, tid = threadIdx.x;
  const SeqItem it = seq_item(k.items, item);
  const int pairs = a.rotated / 2, D = a.head_dim;
  const float* freq = a.frequencies.p + m * a.frequencies.mutant_stride;
  const int64_t at = (a.past ? a.past[it.seq] : 0) + (int64_t)it.pos0;
  for (int x = tid; x < it.len * pairs; x += THREADS) {
    const int t = x / pairs, i = x % pairs;
    double position = (double)(at + t);
    if (a.positions) {
      int axis = 0, end = a.section[0];
      while (i >= end && axis + 1 < a.axes) end += a.section[++axis];
      position = a.positions[axis * k.tokens + it.row0 + t];
    }
    turn[x] = cos_sin(position * (double)freq[i]);
  }
  __syncthreads();
  const int heads = a.q_heads + a.k_heads, lane = tid & (team - 1), units = (D + 2 * V - 1) / (2 * V), turning = pairs / V;
  for (int x = tid / team; x < it.len * heads; x += THREADS / team) {
    const int t = x / heads, h = x % heads;
    const bool key = h >= a.q_heads;
    const mure_seq_in& src = key ? a.k : a.q;
    const mure_seq_out& dst = key ? a.k_out : a.q_out;
    const int64_t row = it.row0 + t, col = (int64_t)(key ? h - a.q_heads : h) * D;
    const T* p = static_cast<const T*>(src.p) + m * src.mutant_stride + row * src.row_stride + col;
    T* o = static_cast<T*>(dst.p) + m * dst.mutant_stride + row * dst.row_stride + col;
    const mure_seq_param& wp = key ? a.k_weight : a.q_weight;
    float v[U][2][V];
    int e[U][2];
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int unit = lane + u * team;
      const bool turns = unit < turning;
      e[u][0] = a.interleaved || !turns ? unit * 2 * V : unit * V;     // channels behind the pairs are 2 V a unit too
      e[u][1] = a.interleaved || !turns ? e[u][0] + V : pairs + unit * V;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (unit < units && e[u][s] < D) get<T, V>(p + e[u][s], v[u][s]);
        else {
#pragma unroll
          for (int j = 0; j < V; ++j) v[u][s][j] = 0.f;
          e[u][s] = -1;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) sum += v[u][s][j];
      }
    }
    if (a.norm) {
      float mean = 0.f;
      if (a.norm == MURE_SEQ_LAYER) {
        for (int w = 1; w < team; w *= 2) sum += __shfl_xor(sum, w);
        mean = sum / (float)D;
      }
      float sq = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            if (e[u][s] >= 0) v[u][s][j] -= mean;
            sq = fmaf(v[u][s][j], v[u][s][j], sq);
          }
      for (int w = 1; w < team; w *= 2) sq += __shfl_xor(sq, w);
      const float f = 1.f / sqrtf(sq / (float)D + a.eps);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          float w[V];
#pragma unroll
          for (int j = 0; j < V; ++j) w[j] = 1.f;
          if (wp.p && e[u][s] >= 0) get<float, V>(wp.p + m * wp.mutant_stride + e[u][s], w);
#pragma unroll
          for (int j = 0; j < V; ++j) v[u][s][j] = v[u][s][j] * f * w[j];
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int unit = lane + u * team;
      if (unit < turning) {
        const float2* cs = turn + t * pairs + unit * V;
        if (a.interleaved) {
          if constexpr (V > 1) {
#pragma unroll
            for (int j = 0; j < V; ++j) {      // pair j: channels 2 j, 2 j + 1 of the unit's 2 V
              float& x0 = v[u][2 * j / V][2 * j % V];
              float& x1 = v[u][2 * j / V][2 * j % V + 1];
              const float2 f = cs[j];
              const float y = x0 * f.x - x1 * f.y;
              x1 = x0 * f.y + x1 * f.x;
              x0 = y;
            }
          } else {
            const float2 f = cs[0];
            const float y = v[u][0][0] * f.x - v[u][1][0] * f.y;
            v[u][1][0] = v[u][0][0] * f.y + v[u][1][0] * f.x;
            v[u][0][0] = y;
          }
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float2 f = cs[j];
            const float y = v[u][0][j] * f.x - v[u][1][j] * f.y;
            v[u][1][j] = v[u][0][j] * f.y + v[u][1][j] * f.x;
            v[u][0][j] = y;
          }
        }
      }
#pragma unroll
      for (int s = 0; s < 2; ++s)
        if (e[u][s] >= 0) put<T, V>(o + e[u][s], v[u][s]);
    }
  }
}

template <typename T, int V, int U> hipError_t rotate_u(AttnRotateArgs k, int team, hipStream_t s) {
  const int n = k.n_items, M = k.a.n_mutants, most = std::min(n, (int)(((1 << 24) - 1) / M));
  const unsigned lds = (unsigned)(k.longest * (k.a.rotated / 2) * sizeof(float2));
  for (k.item0 = 0; k.item0 < n; k.item0 += most) {
    std::tuple<AttnRotateArgs, int> params(k, team);
    void* at[] = {&std::get<0>(params), &std::get<1>(params)};
    if (const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(rotate_kernel<T, V, U>), dim3((unsigned)(std::min(most, n - k.item0) * M)), dim3(THREADS), at, lds, s);
        e != hipSuccess)
      return e;
  }
  return hipSuccess;
}

// units of V pairs over teams of at most a wave
template <typename T, int V> hipError_t rotate_v(const AttnRotateArgs& k, hipStream_t s) {
  const int units = (k.a.head_dim + 2 * V - 1) / (2 * V);
  int team = 1;
  while (team < units && team < 64) team *= 2;
  if constexpr (V == 1)
    if (units > 64) return rotate_u<T, V, 2>(k, team, s);
  return rotate_u<T, V, 1>(k, team, s);
}

template <typename T> hipError_t rotate_t(const AttnRotateArgs& k, hipStream_t s) {
  // the widest vectors of which the pairs and the channels behind them are made
  auto made = [&](int v) { return k.a.rotated / 2 % v == 0 && (k.a.head_dim - k.a.rotated) % (2 * v) == 0; };
  if (sizeof(T) == 2 && made(8)) return rotate_v<T, 16 / sizeof(T)>(k, s);
  if (made(4)) return rotate_v<T, 4>(k, s);
  if (made(2)) return rotate_v<T, 2>(k, s);
  return rotate_v<T, 1>(k, s);
}

}  // namespace

hipError_t launch_attn_rotate(const AttnRotateArgs& k, hipStream_t s) {
  return k.a.dtype == MURE_F32 ? rotate_t<float>(k, s) : rotate_t<bf16_t>(k, s);
}

}  // namespace mure
