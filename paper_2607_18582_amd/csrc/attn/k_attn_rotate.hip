// Norm of queries and keys for each head and rotation of their pairs
// (mure_attn_rotate).
//
// Bound by memory: each element is read and written once.  A block takes a run
// of tokens and computes their angles once, for all heads: the product of
// position and frequency and its remainder by pi/2 in float64, sine and cosine
// of that in float32.  Then a team of lanes takes a head at a time, each lane
// both halves of the pairs it turns, in vectors: nothing is exchanged but the
// norm's sums.  65536 tokens, 20 heads of 96 bfloat16 channels, three axes: 114
// us, 4.4 TB/s, the vector ALU busy for 79 % of it; 64 tokens 4.5 us.
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
template <typename T> struct Raw<T, 1> {
  typedef T raw;
  typedef T any;
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
    __builtin_nontemporal_store(r, reinterpret_cast<typename Raw<T, V>::any*>(p));
  }
}

template <typename T, int V> __device__ __forceinline__ T element(const typename Raw<T, V>::raw& r, int j) {
  if constexpr (V == 1) return r;
  else return r[j];
}

// V pairs a unit, U units a lane.
template <typename T, int V, int U, bool INTERLEAVED>
__global__ __launch_bounds__(THREADS) void rotate_kernel(AttnRotateArgs k, int team) {
  extern __shared__ float2 turn[];             // [tokens][pairs]
  const mure_attn_rotate_args& a = k.a;
  const int m = blockIdx.x % a.n_mutants, item = k.item0 + blockIdx.x / a.n_mutants, tid = threadIdx.x;
  const int begin = gridDim.y == 1 ? 0 : blockIdx.y, end = gridDim.y > 1 ? begin + 1 : a.k_heads ? 2 : 1;     // of queries and keys
  const SeqItem it = seq_item(k.items, item);
  const int pairs = a.rotated / 2, D = a.head_dim;
  const float* freq = a.frequencies.p + m * a.frequencies.mutant_stride;
  const int64_t at = (a.past ? a.past[it.seq] : 0) + (int64_t)it.pos0;
  for (int x = tid; x < it.len * pairs; x += THREADS) {
    const int t = x / pairs, i = x % pairs;
    double position = (double)(at + t);
    if (a.positions) {
      int axis = 0, behind = a.section[0];
      while (i >= behind && axis + 1 < a.axes) behind += a.section[++axis];
      position = a.positions[axis * k.tokens + it.row0 + t];
    }
    turn[x] = cos_sin(position * (double)freq[i]);
  }
  __syncthreads();
  // a team's lanes have the same channels of every head: their weights stay in registers, and the next head's
  // channels are on their way while this one's are worked on
  const int lane = tid & (team - 1), units = (D + 2 * V - 1) / (2 * V), turning = pairs / V, teams = THREADS / team;
  int e[U][2];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int unit = lane + u * team;
    const bool apart = !INTERLEAVED && unit < turning;                 // channels behind the pairs are 2 V a unit too
    e[u][0] = apart ? unit * V : unit * 2 * V;
    e[u][1] = apart ? pairs + unit * V : e[u][0] + V;
#pragma unroll
    for (int s = 0; s < 2; ++s)
      if (unit >= units || e[u][s] >= D) e[u][s] = -1;
  }
#pragma unroll 1
  for (int which = begin; which < end; ++which) {
    const int heads = which ? a.k_heads : a.q_heads, count = it.len * heads;
    const mure_seq_in& src = which ? a.k : a.q;
    const mure_seq_out& dst = which ? a.k_out : a.q_out;
    const mure_seq_param& wp = which ? a.k_weight : a.q_weight;
    const T* in = static_cast<const T*>(src.p) + m * src.mutant_stride + it.row0 * src.row_stride;
    T* out = static_cast<T*>(dst.p) + m * dst.mutant_stride + it.row0 * dst.row_stride;
    float w[U][2][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int j = 0; j < V; ++j) w[u][s][j] = 1.f;
        if (wp.p && e[u][s] >= 0) get<float, V>(wp.p + m * wp.mutant_stride + e[u][s], w[u][s]);
      }
    typename Raw<T, V>::raw next[U][2];
    const auto fetch = [&](int x) {
      const int t = x / heads, h = x - t * heads;
      const T* p = in + t * src.row_stride + (int64_t)h * D;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int s = 0; s < 2; ++s)
          if (e[u][s] >= 0) next[u][s] = *reinterpret_cast<const typename Raw<T, V>::any*>(p + e[u][s]);
    };
    int x = tid / team;
    if (x < count) fetch(x);
    for (; x < count; x += teams) {
      const int t = x / heads, h = x - t * heads;
      float v[U][2][V], sum = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            v[u][s][j] = e[u][s] >= 0 ? to_f<T>(element<T, V>(next[u][s], j)) : 0.f;
            sum += v[u][s][j];
          }
      if (x + teams < count) fetch(x + teams);
      if (a.norm) {
        float mean = 0.f;
        if (a.norm == MURE_SEQ_LAYER) {
          for (int d = 1; d < team; d *= 2) sum += __shfl_xor(sum, d);
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
        for (int d = 1; d < team; d *= 2) sq += __shfl_xor(sq, d);
        const float f = 1.f / sqrtf(sq / (float)D + a.eps);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < V; ++j) v[u][s][j] *= f * w[u][s][j];
      }
      T* o = out + t * dst.row_stride + (int64_t)h * D;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int unit = lane + u * team;
        if (unit < turning) {
          const float2* cs = turn + t * pairs + unit * V;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            // interleaved: channels 2 j, 2 j + 1 of the unit's 2 V
            const float2 f = cs[j];
            float& x0 = INTERLEAVED && V > 1 ? v[u][2 * j / V][2 * j % V] : v[u][0][j];
            float& x1 = INTERLEAVED && V > 1 ? v[u][2 * j / V][(2 * j + 1) % V] : v[u][1][j];
            const float y = x0 * f.x - x1 * f.y;
            x1 = x0 * f.y + x1 * f.x;
            x0 = y;
          }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
          if (e[u][s] >= 0) put<T, V>(o + e[u][s], v[u][s]);
      }
    }
  }
}

template <typename T, int V, int U> hipError_t rotate_u(AttnRotateArgs k, int team, hipStream_t s) {
  const int n = k.n_items, M = k.a.n_mutants, most = std::min(n, (int)(((1 << 24) - 1) / M));
  const unsigned lds = (unsigned)(k.longest * (k.a.rotated / 2) * sizeof(float2));
  // where blocks are few, queries and keys get their own: 64 sequences of one token take 4.6 us so and 6.0 one after the other
  const unsigned y = k.a.k_heads && (int64_t)n * M < 1024 ? 2 : 1;
  for (k.item0 = 0; k.item0 < n; k.item0 += most) {
    std::tuple<AttnRotateArgs, int> params(k, team);
    void* at[] = {&std::get<0>(params), &std::get<1>(params)};
    if (const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(k.a.interleaved ? rotate_kernel<T, V, U, true> : rotate_kernel<T, V, U, false>), dim3((unsigned)(std::min(most, n - k.item0) * M), y), dim3(THREADS), at, lds, s);
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
