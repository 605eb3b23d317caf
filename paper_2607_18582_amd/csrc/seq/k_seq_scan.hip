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
// by the block, twice: the next tile's loads (of all inputs) are issued before
// a tile is computed.  Runs of fewer than four tokens read b and c from memory:
// a single token needs neither LDS nor a barrier.
//
// A sequence of at most MURE_SEQ_SPLIT_TOKENS tokens is one run.  A longer
// one is scanned in chunks: the scan is linear in h, so a chunk's last state
// is its last state from zero plus exp(a sum D) times its first.  One launch
// computes the chunks' states from zero and their sums of D (seq_scan_kernel,
// ENDS), one walks the chunks of every channel and state (seq_scan_join_kernel)
// and one computes the outputs from the chunks' first states.
//
// 32768 tokens of 2048 channels and 16 states, bfloat16: 427 to 435 us a call
// (its launches one by one under the profiler 193, 22 and 261, more than they
// take in a call).  The two scans keep the vector ALU busy
// all the time: of the second one's 113 instructions per quad and four tokens 80
// are the recurrence, and the 20 transcendental ones take two slots.
#include <algorithm>

#include "seq_dev.hpp"

namespace mure {

constexpr int TILE = 16;                               // tokens whose b and c stand in LDS
constexpr float LOG2E = 1.44269504088896340736f;

// log(1 + e^s) = max(s, 0) + log(1 + e) with e = e^-|s|.  Of a small e the sum
// w = 1 + e keeps only some bits; what it loses is r = e - (w - 1), exactly,
// and log(1 + e) = log(w) + log(1 + r / w) = log(w) + r to the float's
// precision: r is below 2^-24, and w is near 1 wherever r counts.
__device__ __forceinline__ float softplus(float s) {
  const float e = __builtin_amdgcn_exp2f(-LOG2E * fabsf(s));
  const float w = 1.f + e, r = e - (w - 1.f);
  float m;                                             // of fmaxf the compiler makes two instructions; of a NaN e is one
  asm("v_max_f32 %0, 0, %1" : "=v"(m) : "v"(s));
  return m + fmaf(1.f / LOG2E, __builtin_amdgcn_logf(w), r);
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

// Lane j of each quad receives the quad's sum of its p[j].
__device__ __forceinline__ float quad_sums(float p0, float p1, float p2, float p3, int q) {
  const bool odd = q & 1, high = q & 2;
  const float a = (odd ? p1 : p0) + quad_xor1(odd ? p0 : p1);
  const float b = (odd ? p3 : p2) + quad_xor1(odd ? p2 : p3);
  return (high ? b : a) + quad_xor2(high ? a : b);
}

// The state h after tokens that take a state of zero to `end`, and whose steps times the state's rate sum to
// 2 half / log2(e): 2^(2 half) h + end.  In two products: the result may be in float's range where the factor is not.
__device__ __forceinline__ float carried(float half, float h, float end) {
  const float f = __builtin_amdgcn_exp2f(half);
  return fmaf(f, f * h, end);
}

// An element `off` bytes past p, which is the same in all lanes: with 32 bits through a buffer at p, whose loads and
// stores take p from scalar registers and need no 64-bit addition in every lane.
template <typename T> __device__ __forceinline__ T lane_load(const T* p, uint64_t off) {
  return *reinterpret_cast<const T*>(reinterpret_cast<const char*>(p) + off);
}
template <typename T> __device__ __forceinline__ void lane_store(T* p, uint64_t off, T v) {
  *reinterpret_cast<T*>(reinterpret_cast<char*>(p) + off) = v;
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const void* p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, -1, 0x00027000);       // raw, 2^32 - 1 bytes
}
template <typename T> __device__ __forceinline__ T lane_load(const T* p, uint32_t off) {
  if constexpr (sizeof(T) == 2) return __builtin_amdgcn_raw_buffer_load_b16(buffer_at(p), off, 0, 0);
  else return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buffer_at(p), off, 0, 0));
}
template <typename T> __device__ __forceinline__ void lane_store(T* p, uint32_t off, T v) {
  if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(v, buffer_at(p), off, 0, 0);
  else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), buffer_at(p), off, 0, 0);
}

// Q: states per lane (4 Q in all); PAD: some of them are past N.
// KIND: RUNS; ENDS, only the state that a run reaches from zero; STEPS, runs of
// fewer than four tokens all, which need no LDS and half the registers.
enum { RUNS = 0, ENDS_ONLY = 1, STEPS = 2 };
template <typename T, int Q, bool PAD, int KIND>
__global__ __launch_bounds__(256) void seq_scan_kernel(SeqScanArgs k, DivU32 dcb, DivU32 dm, DivU32 dtile) {
  constexpr bool ENDS = KIND == ENDS_ONLY;
  constexpr int NP = 4 * Q, GROUPS = TILE / 4;
  constexpr int BC = TILE * NP * (ENDS ? 1 : 2), PER = (BC + 255) / 256;       // b and c of a tile; of a thread
  typedef float vq __attribute__((ext_vector_type(Q)));
  typedef vq __attribute__((aligned(4))) vq_any;
  __shared__ __attribute__((aligned(16))) float lds[2][KIND == STEPS ? 4 : BC];   // [b, c][TILE][NP]
  const mure_seq_scan_args& a = k.a;
  const int tid = threadIdx.x, q = tid & 3;
  int rest, cb, item, mi, group, tile;
  divmodu(dcb, blockIdx.x, rest, cb);                  // channel block fastest, then the mutant
  divmodu(dm, (uint32_t)rest, item, mi);
  divmodu(dtile, (uint32_t)cb, group, tile);
  const SeqItem it = seq_item(k.items, k.item0 + item);
  const int64_t m = mi;
  const int D = a.channels, N = a.states, width = D / a.groups;
  const int dg = tile * 64 + (tid >> 2);               // in the group
  const bool live = dg < width;                        // else the last channel again, not stored
  const bool wave_live = tile * 64 + 16 * __builtin_amdgcn_readfirstlane(tid >> 6) < width;
  const int d0 = group * width + tile * 64, d = group * width + min(dg, width - 1);
  const int64_t su = a.u.row_stride, sd = a.dt.row_stride, sz = a.gate.row_stride, sy = a.out.row_stride;
  // The next rows to be loaded, and stored: the same address in all lanes, and a lane's distance from it.
  const bool gated = !ENDS && a.gate.p;
  const T* u = static_cast<const T*>(a.u.p) + m * a.u.mutant_stride + it.row0 * su + d0;
  const T* dt = static_cast<const T*>(a.dt.p) + m * a.dt.mutant_stride + it.row0 * sd + d0;
  const T* z = static_cast<const T*>(a.gate.p) + m * a.gate.mutant_stride + it.row0 * sz + d0;
  using Off = std::conditional_t<PAD, uint64_t, uint32_t>;
  auto lane_off = [&](int64_t stride) { return Off((q * stride + (d - d0)) * sizeof(T)); };
  const Off ou = lane_off(su), od = lane_off(sd), oz = lane_off(sz), oy = lane_off(sy);
  const int64_t sb = a.b.row_stride, sc = a.c.row_stride;
  const T* b = static_cast<const T*>(a.b.p) + m * a.b.mutant_stride + it.row0 * sb + group * N;
  const T* c = static_cast<const T*>(a.c.p) + m * a.c.mutant_stride + it.row0 * sc + group * N;
  T* y = static_cast<T*>(a.out.p) + m * a.out.mutant_stride + it.row0 * sy + d0;

  // A tile's inputs, as they come from memory: b and c; u, dt and gate of its whole groups of four tokens, and of
  // the one to three tokens after them, where the run ends.
  T bc[PER], ru[GROUPS + 1], rd[GROUPS + 1], rz[GROUPS + 1] = {};
  auto fetch_rows = [&](T& fu, T& fd, T& fz) {         // four tokens
    fu = lane_load(u, ou);
    fd = lane_load(dt, od);
    if (gated) fz = lane_load(z, oz);
    u += 4 * su, dt += 4 * sd, z += 4 * sz;
  };
  auto fetch_last = [&](int left, T& fu, T& fd, T& fz) {       // one to three tokens
    const int64_t t = min(q, left - 1), c = d - d0;
    fu = u[t * su + c], fd = dt[t * sd + c];
    if (gated) fz = z[t * sz + c];
  };
  // Element tid + 256 i of a tile's b and c, of the next tile to be loaded: from 16 states on a block's threads take
  // STEP whole rows at a time, of b and then of c; below that all of them at once.
  constexpr bool ROWWISE = TILE * NP >= 256;
  constexpr int STEP = 256 / NP, OF_B = ROWWISE ? TILE / STEP : 1;
  const int br = tid / NP % TILE, bn = tid % NP;
  const bool of_c = !ROWWISE && !ENDS && tid / NP >= TILE;
  const int64_t s0 = of_c ? sc : sb;
  const T *b0 = (of_c ? c : b) + br * s0 + bn, *c0 = c + br * sc + bn;
  auto fetch_bc = [&](int count) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const bool is_c = i >= OF_B;
      const int step = i % OF_B * STEP;                // rows on from this thread's first
      const T* p = is_c ? c0 + step * sc : b0 + step * s0;
      if (count < TILE) p += (min(br + step, count - 1) - br - step) * (is_c ? sc : s0);       // rows past the run are not used
      bc[i] = T(0);
      if ((BC % 256 == 0 || tid + 256 * i < BC) && (!PAD || bn < N)) bc[i] = *p;
    }
    b0 += TILE * s0;
    if (ROWWISE && !ENDS) c0 += TILE * sc;
  };
  auto fetch_group = [&](int count, int g) {           // of a tile of `count` tokens; g = GROUPS: after the whole groups
    if (g < GROUPS && 4 * g + 4 <= count) fetch_rows(ru[g], rd[g], rz[g]);
    if (g == GROUPS && count % 4) fetch_last(count % 4, ru[g], rd[g], rz[g]);
  };
  const bool tiled = KIND != STEPS && it.len >= 4;
  if (tiled) {
    const int count = min(TILE, it.len);
    fetch_bc(count);
#pragma unroll
    for (int g = 0; g <= GROUPS; ++g) fetch_group(count, g);
  } else if (it.len) {
    fetch_last(it.len, ru[GROUPS], rd[GROUPS], rz[GROUPS]);
  }

  float al[Q], h[Q];                                   // a log2(e): exp(D a) is one hardware exp2
  const float* ap = a.a.p + m * a.a.mutant_stride + (int64_t)d * N + q * Q;
  const int64_t state = ((int64_t)it.seq * D + d) * N + q * Q;
  const int64_t slot = ((m * k.n_slots + it.slot) * D + d) * N + q * Q;
  const float* hp = nullptr;                           // the first state
  if (!ENDS) {
    if (it.slot >= 0) hp = k.ws_h + slot;
    else if (a.state) hp = a.state + m * a.state_mutant_stride + state;
  }
  if constexpr (PAD) {
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      const bool in = q * Q + i < N;
      al[i] = in ? ap[i] * LOG2E : 0.f;
      h[i] = in && hp ? hp[i] : 0.f;
    }
  } else {
    const vq av = *reinterpret_cast<const vq_any*>(ap);
    vq hv = {};
    if (hp) hv = *reinterpret_cast<const vq_any*>(hp);
#pragma unroll
    for (int i = 0; i < Q; ++i) al[i] = av[i] * LOG2E, h[i] = hv[i];
  }
  const float bias = a.dt_bias.p ? a.dt_bias.p[m * a.dt_bias.mutant_stride + d] : 0.f;
  const float skip = !ENDS && a.skip.p ? a.skip.p[m * a.skip.mutant_stride + d] : 0.f;

  float sum_d = 0.f;                                   // of this lane's tokens
  // token J of the quad's four, with D in dv's lane J and D u in du's
  auto step = [&](auto jc, float dv, float du, vq bv, vq cv) {
    constexpr int J = decltype(jc)::value;
    const float dj = quad_bcast<J>(dv), duj = quad_bcast<J>(du);
    float p = 0.f;
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      h[i] = fmaf(__builtin_amdgcn_exp2f(dj * al[i]), h[i], duj * bv[i]);
      const float hi = PAD && q * Q + i >= N ? 0.f : h[i];
      if (!ENDS) p = i ? fmaf(cv[i], hi, p) : cv[i] * hi;
    }
    return p;
  };
  auto prepare = [&](float dv, float uv, float& du) {
    dv += bias;
    if (a.softplus) dv = softplus(dv);
    du = dv * uv;
    return dv;
  };
  auto finish = [&](float yq, float uv, float zv) {
    const float v = fmaf(skip, uv, yq);
    return gated ? v * seq_silu(zv) : v;
  };
  using J0 = std::integral_constant<int, 0>;
  using J1 = std::integral_constant<int, 1>;
  using J2 = std::integral_constant<int, 2>;
  using J3 = std::integral_constant<int, 3>;
  // the run's last one to three tokens, with their rows of b and c
  auto last = [&](int left, T fu, T fd, T fz, auto brow, auto crow) {
    const float uv = to_f<T>(fu);
    float du;
    const float dv = prepare(to_f<T>(fd), uv, du);
    const vq b0 = brow(0), c0 = ENDS ? b0 : crow(0), b1 = brow(min(1, left - 1)), c1 = ENDS ? b1 : crow(min(1, left - 1)),
             b2 = brow(left - 1), c2 = ENDS ? b2 : crow(left - 1);
    const float p0 = step(J0(), dv, du, b0, c0);
    float p1 = 0.f, p2 = 0.f;
    if (left > 1) p1 = step(J1(), dv, du, b1, c1);
    if (left > 2) p2 = step(J2(), dv, du, b2, c2);
    const float yq = ENDS ? 0.f : quad_sums(p0, p1, p2, 0.f, q);
    if (q >= left) return;
    if (ENDS) sum_d += dv;
    else if (live) lane_store(y, oy, from_f<T>(finish(yq, uv, to_f<T>(fz))));
  };
  if (tiled) {
    for (int t0 = 0, i = 0; t0 < it.len; t0 += TILE, i ^= 1) {
      const int count = min(TILE, it.len - t0);
      float* now = lds[i];
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (BC % 256 == 0 || tid + 256 * j < BC) now[tid + 256 * j] = to_f<T>(bc[j]);
      __syncthreads();                                 // this tile is there, and the one before last is read
      const int t1 = t0 + TILE, more = min(TILE, it.len - t1);     // the next tile: its inputs take the registers of
      if (more > 0) fetch_bc(more);                                // this one's as they are used
      if (!wave_live) continue;
      const float *bt = now + q * Q, *ct = ENDS ? bt : bt + TILE * NP;
      auto row = [&](const float* p, int t) { return *reinterpret_cast<const vq*>(p + t * NP); };
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        if (4 * g + 4 > count) break;
        float uv = to_f<T>(ru[g]), zv = to_f<T>(rz[g]), du;
        asm("" : "+v"(uv), "+v"(zv));                  // converted here: the registers are free for the next tile's
        const float dv = prepare(to_f<T>(rd[g]), uv, du);
        fetch_group(more, g);
        const float p0 = step(J0(), dv, du, row(bt, 4 * g), row(ct, 4 * g));
        const float p1 = step(J1(), dv, du, row(bt, 4 * g + 1), row(ct, 4 * g + 1));
        const float p2 = step(J2(), dv, du, row(bt, 4 * g + 2), row(ct, 4 * g + 2));
        const float p3 = step(J3(), dv, du, row(bt, 4 * g + 3), row(ct, 4 * g + 3));
        const float yq = ENDS ? 0.f : quad_sums(p0, p1, p2, p3, q);
        if (ENDS) sum_d += dv;
        else if (live) lane_store(y, oy, from_f<T>(finish(yq, uv, zv)));
        y += 4 * sy;
      }
      if (more <= 0 && count % 4) {
        const int done = count / 4 * 4;
        last(count - done, ru[GROUPS], rd[GROUPS], rz[GROUPS], [&](int j) { return row(bt, done + j); },
             [&](int j) { return row(ct, done + j); });
      }
      fetch_group(more, GROUPS);
    }
    if (!live) return;
  } else {
    if (!live) return;
    auto row = [&](const T* p, int64_t stride) {
      vq v;
#pragma unroll
      for (int i = 0; i < Q; ++i) v[i] = !PAD || q * Q + i < N ? to_f<T>(p[stride + q * Q + i]) : 0.f;
      return v;
    };
    if (it.len)
      last(it.len, ru[GROUPS], rd[GROUPS], rz[GROUPS], [&](int j) { return row(b, j * sb); },
           [&](int j) { return row(c, j * sc); });
  }
  float* to = nullptr;
  if (ENDS) {
    to = k.ws_h + slot;
    sum_d += quad_xor1(sum_d);
    sum_d += quad_xor2(sum_d);
    if (q == 0) k.ws_d[(m * k.n_slots + it.slot) * D + d] = sum_d;
  } else if (a.state_out && it.pos0 + it.len == it.total) {
    to = a.state_out + m * a.state_out_mutant_stride + state;
  }
  if (!to) return;
  if constexpr (PAD) {
#pragma unroll
    for (int i = 0; i < Q; ++i)
      if (q * Q + i < N) to[i] = h[i];
  } else {
    vq hv;
#pragma unroll
    for (int i = 0; i < Q; ++i) hv[i] = h[i];
    *reinterpret_cast<vq_any*>(to) = hv;
  }
}

constexpr int JOIN = 64;                               // one wave a block: a long prompt of 2048 channels has 512 of them

// The chunks' first states from their states from zero, in place: of 256 chunks of 2048 x 16 states 69 MB in 22 us,
// bound by the chains' loads (32768 threads have 16 each in flight).  Where a chunk takes a state out of float's range,
// or an infinite one by decays that may be 0 (0 times infinity is NaN), the state goes through it token by token, with
// the operations of seq_scan_kernel: two parts past float's range may add up to a number.  Rates that make every state
// overflow take 0.7 ms.
template <typename T>
__global__ __launch_bounds__(JOIN) void seq_scan_join_kernel(SeqScanArgs k, DivU32 dn) {
  const mure_seq_scan_args& a = k.a;
  const uint32_t e = blockIdx.x * (unsigned)JOIN + threadIdx.x;
  const int D = a.channels, N = a.states;
  if (e >= (uint32_t)D * (uint32_t)N) return;
  const int64_t m = blockIdx.z, d = divu(dn, e), DN = (int64_t)D * N;
  const float al = a.a.p[m * a.a.mutant_stride + e] * LOG2E, half_al = 0.5f * al;
  for (int i = blockIdx.y; i < k.n_chunked; i += gridDim.y) {
    const SeqChunks ch = k.chunks[i];
    float h = a.state ? a.state[m * a.state_mutant_stride + ch.seq * DN + e] : 0.f;
    float* ws = k.ws_h + (m * k.n_slots + ch.slot0) * DN + e;
    const float* sd = k.ws_d + (m * k.n_slots + ch.slot0) * D + d;
    // the state after chunk j, token by token
    auto walk = [&](int j, float h) {
      const int64_t row = ch.row0 + (int64_t)j * SCAN_CHUNK, n = e - d * N + d / (D / a.groups) * N;
      const T* u = static_cast<const T*>(a.u.p) + m * a.u.mutant_stride + row * a.u.row_stride + d;
      const T* dt = static_cast<const T*>(a.dt.p) + m * a.dt.mutant_stride + row * a.dt.row_stride + d;
      const T* b = static_cast<const T*>(a.b.p) + m * a.b.mutant_stride + row * a.b.row_stride + n;
      const float bias = a.dt_bias.p ? a.dt_bias.p[m * a.dt_bias.mutant_stride + d] : 0.f;
      for (int t0 = 0; t0 < SCAN_CHUNK; t0 += TILE) {
        T ru[TILE], rd[TILE], rb[TILE];
#pragma unroll
        for (int t = 0; t < TILE; ++t) {
          ru[t] = u[(t0 + t) * a.u.row_stride];
          rd[t] = dt[(t0 + t) * a.dt.row_stride];
          rb[t] = b[(t0 + t) * a.b.row_stride];
        }
#pragma unroll
        for (int t = 0; t < TILE; ++t) {
          float dv = to_f<T>(rd[t]) + bias;
          if (a.softplus) dv = softplus(dv);
          const float du = dv * to_f<T>(ru[t]);
          h = fmaf(__builtin_amdgcn_exp2f(dv * al), h, du * to_f<T>(rb[t]));
        }
      }
      return h;
    };
    // AHEAD chunks are loaded at a time, ahead of those being joined.  The last chunk has no state from zero, and none
    // is used.
    constexpr int AHEAD = 8;
    constexpr float LEAST = -62.f;                     // of half: with steps of one sign no token's decay is 0
    float end[AHEAD], s[AHEAD];
    const float* at = ws;
    auto load = [&](int n) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (i < n) end[i] = at[i * DN], s[i] = sd[i * (int64_t)D];
      at += AHEAD * DN;
      sd += AHEAD * (int64_t)D;
    };
    int left = ch.n;
    // n chunks, `ended` of them with ends, and the loads of `more` after them; false: they have to be joined one by one
    auto join = [&](int n, int ended, int more) {
      float e[AHEAD], x[AHEAD], to[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) e[i] = end[i], x[i] = half_al * s[i];
      load(more);
      float last = h;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        to[i] = last;
        if (i < ended) last = carried(x[i], last, e[i]);
      }
      bool plain = isfinite(last) || isnan(h);         // an infinite state or a NaN on the way is one at the end
      if (!plain && isinf(h)) {
        plain = true;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
          if (i < ended) plain = plain && x[i] >= LEAST;
      }
      if (!plain) return false;
      h = last;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (i < n) ws[i * DN] = to[i];
      return true;
    };
    load(min(AHEAD, left - 1));
    for (; left > 0; left -= AHEAD, ws += AHEAD * DN) {
      if (left > 2 * AHEAD ? join(AHEAD, AHEAD, AHEAD) : join(left, left - 1, left - AHEAD - 1)) continue;
      const int j0 = ch.n - left;
      const float* sums = k.ws_d + (m * k.n_slots + ch.slot0 + j0) * D + d;
#pragma unroll 1
      for (int i = 0; i < min(AHEAD, left); ++i) {
        const float end = ws[i * DN], sum = sums[i * (int64_t)D], x = half_al * sum;
        ws[i * DN] = h;
        if (i == left - 1 || isnan(h)) continue;
        const float next = h == 0.f ? end : carried(x, h, end);
        h = isfinite(sum) && (isfinite(h) ? isfinite(next) : x >= LEAST) ? next : walk(j0 + i, h);
      }
    }
  }
}

int64_t seq_scan_blocks(const mure_seq_scan_args& a) {
  return (int64_t)((a.channels / a.groups + 63) / 64) * a.groups * a.n_mutants;
}

template <typename T, int Q, bool PAD, int KIND>
static hipError_t scan_q(SeqScanArgs k, hipStream_t s) {
  const int tiles = (k.a.channels / k.a.groups + 63) / 64;
  const int64_t blocks = seq_scan_blocks(k.a);         // of an item: at most SCAN_GRID (checked by the caller)
  const int most = (int)(SCAN_GRID / blocks);
  for (int left = k.n_items; left > 0; left -= most, k.item0 += most) {
    if (hipError_t e = launch(seq_scan_kernel<T, Q, PAD, KIND>, dim3((unsigned)(blocks * std::min(left, most))), 256, s, k,
                              make_divu32((uint32_t)(tiles * k.a.groups)), make_divu32((uint32_t)k.a.n_mutants),
                              make_divu32((uint32_t)tiles));
        e != hipSuccess)
      return e;
  }
  return hipSuccess;
}

template <typename T, int Q, int KIND>
static hipError_t scan_p(const SeqScanArgs& k, hipStream_t s) {
  // A lane's distance from its rows' first element has 32 bits but in the instances with padding.
  const int64_t most = ((int64_t)UINT32_MAX / (int64_t)sizeof(T) - 64) / 3;
  const bool near = std::max({k.a.u.row_stride, k.a.dt.row_stride, k.a.gate.p ? k.a.gate.row_stride : 0, k.a.out.row_stride}) <= most;
  return k.a.states == 4 * Q && near ? scan_q<T, Q, false, KIND>(k, s) : scan_q<T, Q, true, KIND>(k, s);
}

template <typename T, int KIND>
static hipError_t scan_t(const SeqScanArgs& k, hipStream_t s) {
  const int N = k.a.states;
  if (N <= 4) return scan_p<T, 1, KIND>(k, s);
  if (N <= 8) return scan_p<T, 2, KIND>(k, s);
  if (N <= 16) return scan_p<T, 4, KIND>(k, s);
  if (N <= 32) return scan_p<T, 8, KIND>(k, s);
  return scan_p<T, 16, KIND>(k, s);
}

template <int KIND>
static hipError_t scan_any(const SeqScanArgs& k, hipStream_t s) {
  return k.a.dtype == MURE_F32 ? scan_t<float, KIND>(k, s) : scan_t<bf16_t, KIND>(k, s);
}

hipError_t launch_seq_scan(const SeqScanArgs& k, hipStream_t s) { return k.longest < 4 ? scan_any<STEPS>(k, s) : scan_any<RUNS>(k, s); }

hipError_t launch_seq_scan_ends(const SeqScanArgs& k, hipStream_t s) { return scan_any<ENDS_ONLY>(k, s); }

hipError_t launch_seq_scan_join(const SeqScanArgs& k, hipStream_t s) {
  const int64_t DN = (int64_t)k.a.channels * k.a.states;
  const auto kernel = k.a.dtype == MURE_F32 ? seq_scan_join_kernel<float> : seq_scan_join_kernel<bf16_t>;
  return launch(kernel, dim3((unsigned)((DN + JOIN - 1) / JOIN), (unsigned)std::min(k.n_chunked, 65535), (unsigned)k.a.n_mutants), JOIN,
                s, k, make_divu32((uint32_t)k.a.states));
}

}  // namespace mure
