// Selective scan of the sequences of a batch:
//   D = softplus(dt + dt_bias),  h[n] = exp(D a[n]) h[n] + D u b[n],
//   y = (sum_n c[n] h[n] + skip u) silu(gate).
//
// Per token, channel and state: an exponential, two products and two fused
// multiply-adds, so from some 8 states on the vector ALU bounds it, and HBM
// below that.  Four lanes (a quad) own a channel; each keeps a quarter of its
// states in registers for the whole run, a wave has 16 channels, a block 64
// of one group.  Four tokens at a time, lane q of the quad loads and prepares
// token q (softplus, D u, gate), so no lane repeats another's work; the quad
// then steps through the four tokens, each lane broadcasting its token's D
// and D u to the quad, and the partial sums over n go back to the token's
// lane, which stores y.  b and c of TILE tokens stand in LDS as floats, shared
// by the block; the next tile's loads are issued before a tile is computed.
//
// A sequence of at most MURE_SEQ_SPLIT_TOKENS tokens is one run.  A longer
// one is scanned in chunks: the scan is linear in h, so a chunk's last state
// is its last state from zero plus exp(a sum D) times its first.  One launch
// computes the chunks' states from zero and their sums of D (seq_scan_kernel,
// ENDS), one walks the chunks of every channel and state (seq_scan_join_kernel)
// and one computes the outputs from the chunks' first states.
#include <algorithm>

#include "seq_dev.hpp"

namespace mure {

constexpr int TILE = 32;                               // tokens whose b and c stand in LDS
constexpr float LOG2E = 1.44269504088896340736f;

// log(1 + e^s) = max(s, 0) + log1p(e^-|s|), and with e = e^-|s| and w = 1 + e
// rounded, log1p(e) = log(w) e / (w - 1), or e where w = 1 (D. Goldberg, "What
// every computer scientist should know about floating-point arithmetic", ACM
// Computing Surveys 23 (1991), Theorem 4): the error in w cancels.
__device__ __forceinline__ float softplus(float s) {
  const float e = __expf(-fabsf(s));
  const float w = 1.f + e, d = w - 1.f;
  const float l = __builtin_amdgcn_logf(w) * (1.f / LOG2E);
  const float p = d == 0.f ? e : l * (e / d);
  return fmaxf(s, 0.f) + p;
}

// Lane j's value of every quad, in all its lanes.
template <int J> __device__ __forceinline__ float quad_bcast(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), J * 0x55, 0xf, 0xf, true));
}
__device__ __forceinline__ float quad_xor1(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0xb1, 0xf, 0xf, true));
}
__device__ __forceinline__ float quad_xor2(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x4e, 0xf, 0xf, true));
}

// Q: states per lane (4 Q in all); PAD: some of them are past N; ENDS: only
// the state that the run reaches from zero.
template <typename T, int Q, bool PAD, bool ENDS>
__global__ __launch_bounds__(256) void seq_scan_kernel(SeqScanArgs k, DivU32 dcb, DivU32 dm, DivU32 dtile) {
  constexpr int NP = 4 * Q;
  typedef float vq __attribute__((ext_vector_type(Q)));
  __shared__ __attribute__((aligned(16))) float sb[TILE][NP];
  __shared__ __attribute__((aligned(16))) float sc[ENDS ? 1 : TILE][NP];
  const mure_seq_scan_args& a = k.a;
  const int tid = threadIdx.x, q = tid & 3, nthr = blockDim.x;
  int rest, cb, item, mi, group, tile;
  divmodu(dcb, blockIdx.x, rest, cb);                  // channel block fastest, then the mutant
  divmodu(dm, (uint32_t)rest, item, mi);
  divmodu(dtile, (uint32_t)cb, group, tile);
  const SeqItem it = k.items[item];
  const int64_t m = mi;
  const int D = a.channels, N = a.states, width = D / a.groups;
  const int dg = tile * 64 + (tid >> 2);               // in the group
  const bool live = dg < width;
  const int d = group * width + min(dg, width - 1);

  float al[Q], h[Q];                                   // a log2(e): exp(D a) is one hardware exp2
  const float* ap = a.a.p + m * a.a.mutant_stride + (int64_t)d * N;
  const int64_t state = ((int64_t)it.seq * D + d) * N;
  const float* hp = nullptr;                           // the first state
  if (!ENDS) {
    if (it.slot >= 0) hp = k.ws_h + ((m * k.n_slots + it.slot) * D + d) * N;
    else if (a.state) hp = a.state + m * a.state_mutant_stride + state;
  }
#pragma unroll
  for (int i = 0; i < Q; ++i) {
    const int n = q * Q + i;
    const bool in = !PAD || n < N;
    al[i] = in ? ap[n] * LOG2E : 0.f;
    h[i] = in && hp ? hp[n] : 0.f;
  }
  const float bias = a.dt_bias.p ? a.dt_bias.p[m * a.dt_bias.mutant_stride + d] : 0.f;
  const float skip = !ENDS && a.skip.p ? a.skip.p[m * a.skip.mutant_stride + d] : 0.f;
  const T* u = static_cast<const T*>(a.u.p) + m * a.u.mutant_stride + (int64_t)it.row0 * a.u.row_stride + d;
  const T* dt = static_cast<const T*>(a.dt.p) + m * a.dt.mutant_stride + (int64_t)it.row0 * a.dt.row_stride + d;
  const T* z = !ENDS && a.gate.p ? static_cast<const T*>(a.gate.p) + m * a.gate.mutant_stride + (int64_t)it.row0 * a.gate.row_stride + d
                                 : nullptr;
  const T* b = static_cast<const T*>(a.b.p) + m * a.b.mutant_stride + (int64_t)it.row0 * a.b.row_stride + group * N;
  const T* c = static_cast<const T*>(a.c.p) + m * a.c.mutant_stride + (int64_t)it.row0 * a.c.row_stride + group * N;
  T* y = ENDS ? nullptr
              : static_cast<T*>(a.out.p) + m * a.out.mutant_stride + (int64_t)it.row0 * a.out.row_stride + d;

  float sum_d = 0.f;                                   // of this lane's tokens
  for (int t0 = 0; t0 < it.len; t0 += TILE) {
    const int count = min(TILE, it.len - t0);
    __syncthreads();                                   // the last tile is read
    for (int e = tid; e < TILE * NP; e += nthr) {
      const int t = e / NP, n = e % NP;
      const bool in = t < count && (!PAD || n < N);
      sb[t][n] = in ? to_f<T>(b[(int64_t)(t0 + t) * a.b.row_stride + n]) : 0.f;
      if (!ENDS) sc[t][n] = in ? to_f<T>(c[(int64_t)(t0 + t) * a.c.row_stride + n]) : 0.f;
    }
    __syncthreads();
    for (int tq = 0; tq < count; tq += 4) {
      const int left = count - tq, t = t0 + tq + min(q, left - 1);     // past the run: its last token again
      const float uv = to_f<T>(u[(int64_t)t * a.u.row_stride]);
      float dv = to_f<T>(dt[(int64_t)t * a.dt.row_stride]) + bias;
      const float zv = z ? to_f<T>(z[(int64_t)t * a.gate.row_stride]) : 0.f;
      if (a.softplus) dv = softplus(dv);
      const float du = dv * uv;
      if (ENDS && q < left) sum_d += dv;
      float yq = 0.f;
      auto step = [&](auto jc) {
        constexpr int J = decltype(jc)::value;
        if (J >= left) return;
        const float dj = quad_bcast<J>(dv), duj = quad_bcast<J>(du);
        const vq bv = *reinterpret_cast<const vq*>(&sb[tq + J][q * Q]);
        float p = 0.f;
        vq cv;
        if (!ENDS) cv = *reinterpret_cast<const vq*>(&sc[ENDS ? 0 : tq + J][q * Q]);
#pragma unroll
        for (int i = 0; i < Q; ++i) {
          h[i] = fmaf(__builtin_amdgcn_exp2f(dj * al[i]), h[i], duj * bv[i]);
          if (!ENDS) p = fmaf(cv[i], PAD && q * Q + i >= N ? 0.f : h[i], p);
        }
        if (!ENDS) {
          p += quad_xor1(p);
          p += quad_xor2(p);
          yq = q == J ? p : yq;
        }
      };
      step(std::integral_constant<int, 0>());
      step(std::integral_constant<int, 1>());
      step(std::integral_constant<int, 2>());
      step(std::integral_constant<int, 3>());
      if (!ENDS && q < left && live) {
        float v = fmaf(skip, uv, yq);
        if (z) v *= seq_silu(zv);
        y[(int64_t)t * a.out.row_stride] = from_f<T>(v);
      }
    }
  }
  if (!live) return;
  float* to = nullptr;
  if (ENDS) {
    to = k.ws_h + ((m * k.n_slots + it.slot) * D + d) * N;
    sum_d += quad_xor1(sum_d);
    sum_d += quad_xor2(sum_d);
    if (q == 0) k.ws_d[(m * k.n_slots + it.slot) * D + d] = sum_d;
  } else if (a.state_out && it.pos0 + it.len == it.total) {
    to = a.state_out + m * a.state_out_mutant_stride + state;
  }
  if (to)
#pragma unroll
    for (int i = 0; i < Q; ++i)
      if (!PAD || q * Q + i < N) to[q * Q + i] = h[i];
}

// The chunks' first states from their states from zero, in place.
__global__ __launch_bounds__(256) void seq_scan_join_kernel(SeqScanArgs k, DivU32 dn) {
  const mure_seq_scan_args& a = k.a;
  const uint32_t e = blockIdx.x * 256u + threadIdx.x;
  const int D = a.channels, N = a.states;
  if (e >= (uint32_t)D * (uint32_t)N) return;
  const int64_t m = blockIdx.z, d = divu(dn, e), DN = (int64_t)D * N;
  const float al = a.a.p[m * a.a.mutant_stride + e] * LOG2E;
  for (int i = blockIdx.y; i < k.n_chunked; i += gridDim.y) {
    const SeqChunks ch = k.chunks[i];
    float h = a.state ? a.state[m * a.state_mutant_stride + ch.seq * DN + e] : 0.f;
    float* ws = k.ws_h + (m * k.n_slots + ch.slot0) * DN + e;
    const float* sd = k.ws_d + (m * k.n_slots + ch.slot0) * D + d;
    int j = 0;
    for (; j + 8 < ch.n; j += 8) {                     // eight chunks' loads at a time
      float end[8], s[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) end[i] = ws[(j + i) * DN], s[i] = sd[(int64_t)(j + i) * D];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ws[(j + i) * DN] = h;
        h = fmaf(__builtin_amdgcn_exp2f(s[i] * al), h, end[i]);
      }
    }
    for (; j + 1 < ch.n; ++j) {
      const float end = ws[j * DN];
      ws[j * DN] = h;
      h = fmaf(__builtin_amdgcn_exp2f(sd[(int64_t)j * D] * al), h, end);
    }
    ws[j * DN] = h;
  }
}

int64_t seq_scan_blocks(const mure_seq_scan_args& a) {
  return (int64_t)((a.channels / a.groups + 63) / 64) * a.groups * a.n_mutants;
}

template <typename T, int Q, bool PAD, bool ENDS>
static hipError_t scan_q(SeqScanArgs k, hipStream_t s) {
  const int width = k.a.channels / k.a.groups, tiles = (width + 63) / 64;
  const int threads = 64 * std::min(4, (width + 15) / 16);
  const int64_t blocks = seq_scan_blocks(k.a);         // of an item: at most SCAN_GRID (checked by the caller)
  const int most = (int)(SCAN_GRID / blocks);
  for (int left = k.n_items; left > 0; left -= most, k.items += most) {
    seq_scan_kernel<T, Q, PAD, ENDS><<<(unsigned)(blocks * std::min(left, most)), threads, 0, s>>>(
        k, make_divu32((uint32_t)(tiles * k.a.groups)), make_divu32((uint32_t)k.a.n_mutants), make_divu32((uint32_t)tiles));
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T, int Q, bool ENDS>
static hipError_t scan_p(const SeqScanArgs& k, hipStream_t s) {
  return k.a.states == 4 * Q ? scan_q<T, Q, false, ENDS>(k, s) : scan_q<T, Q, true, ENDS>(k, s);
}

template <typename T, bool ENDS>
static hipError_t scan_t(const SeqScanArgs& k, hipStream_t s) {
  const int N = k.a.states;
  if (N <= 4) return scan_p<T, 1, ENDS>(k, s);
  if (N <= 8) return scan_p<T, 2, ENDS>(k, s);
  if (N <= 16) return scan_p<T, 4, ENDS>(k, s);
  if (N <= 32) return scan_p<T, 8, ENDS>(k, s);
  return scan_p<T, 16, ENDS>(k, s);
}

hipError_t launch_seq_scan(const SeqScanArgs& k, hipStream_t s) {
  return k.a.dtype == MURE_F32 ? scan_t<float, false>(k, s) : scan_t<bf16_t, false>(k, s);
}

hipError_t launch_seq_scan_ends(const SeqScanArgs& k, hipStream_t s) {
  return k.a.dtype == MURE_F32 ? scan_t<float, true>(k, s) : scan_t<bf16_t, true>(k, s);
}

hipError_t launch_seq_scan_join(const SeqScanArgs& k, hipStream_t s) {
  const int64_t DN = (int64_t)k.a.channels * k.a.states;
  seq_scan_join_kernel<<<dim3((unsigned)((DN + 255) / 256), (unsigned)std::min(k.n_chunked, 65535), (unsigned)k.a.n_mutants), 256, 0,
                         s>>>(k, make_divu32((uint32_t)k.a.states));
  return hipGetLastError();
}

}  // namespace mure
