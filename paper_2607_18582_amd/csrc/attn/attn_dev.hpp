// Device parts of attention: tiles of keys and values in LDS, a wave's 32 rows
// of queries against them.
//
// A wave holds 32 rows (token, head) as columns of the transposed products
//   S^T = K Q^T   [keys x rows],   O^T = V^T P^T   [head_dim x rows]
// in 32x32 matrix instructions: lane l has row l % 32 of the queries, and of
// every 32 keys the 16 numbered 8 (i / 4) + 4 (l / 32) + i % 4.  So a row's
// maximum and sum stay within two lanes, the row's factors are one register
// each, and the weights P^T are the second product's operand as they are: the
// order of keys within an instruction's sum is free, and the values are read
// in the same one.
#pragma once

#include "../seq/seq_dev.hpp"
#include "attn.hpp"

namespace mure {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void;
typedef v4u __attribute__((aligned(2))) v4u_any;  // the GPU's global loads and stores take any address

// What a copy to LDS reads where there is nothing.
__device__ const uint32_t ZEROS[4] = {};

// The matrix instruction of a type: N elements of the summed axis per lane and operand.
template <typename T> struct Mma;
template <> struct Mma<bf16_t> {
  static constexpr int N = 8;
  typedef v8bf frag;
  static __device__ __forceinline__ v16f mma(frag a, frag b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mma<float> {
  static constexpr int N = 1;
  typedef float frag;
  static __device__ __forceinline__ v16f mma(frag a, frag b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
};

// Sizes of a head of up to 32 DB channels of T.
template <typename T, int DB> struct Head {
  static constexpr int BYTES = 32 * DB * (int)sizeof(T);
  static constexpr int ROW = BYTES <= 64 ? 64 : BYTES <= 128 ? 128 : BYTES <= 256 ? 256 : BYTES <= 512 ? 512 : 1024;   // of a tile, in LDS
  static constexpr int PIECES = ROW / 16;
  static constexpr int STEPS = BYTES / 32;     // two 16-byte pieces of a row of keys, one per half wave
};

// The place of a row's 16-byte pieces in LDS is xored with a number of the row's, so that the rows that lanes read
// together lie in different banks: 16-byte reads of one piece of 16 keys, 8-byte reads of 64 bytes of 4 values (of
// 128 bytes of two, in float32).
template <int PIECES> __device__ __forceinline__ int k_twist(int key) {
  return PIECES >= 16 ? key & 15 : PIECES == 8 ? (key >> 1) & 7 : (key >> 2) & 3;
}
template <typename T, int PIECES> __device__ __forceinline__ int v_twist(int key) {
  if (sizeof(T) == 4) return PIECES >= 16 ? ((key >> 2) & 1) << 3 : 0;
  return PIECES >= 16 ? (key & 3) << 2 : PIECES == 8 ? ((key >> 1) & 1) << 2 : 0;
}

// The rows of one sequence's keys (or values) of one head: its cache's first, then the call's own.
template <typename T> struct Rows {
  const T* held;
  const T* own;
  int64_t held_stride, own_stride;
  int past;
  __device__ __forceinline__ const T* at(int j) const { return j < past ? held + j * held_stride : own + (int64_t)(j - past) * own_stride; }
};

// Waits for the wave's own copies to LDS.
__device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// 16 bytes from p + first on of a row of n elements, zeros behind its end.
template <typename T> __device__ __forceinline__ v4u load_piece(const T* p, int first, int n) {
  constexpr int E = 16 / sizeof(T);
  if (first + E <= n) return *reinterpret_cast<const v4u_any*>(p + first);
  union {
    v4u v;
    T e[E];
  } u;
  u.v = v4u{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (first + i < n) u.e[i] = p[first + i];
  return u.v;
}

// Copies KT keys' rows from key t0 on into a tile, zeros from key `end` on and behind n elements: 1024 bytes a wave
// and step.  FAST: rows are whole aligned pieces and go to LDS directly (wait_copies).
template <typename T, int DB, int KT, bool VALUES, bool FAST>
__device__ __forceinline__ void fetch(char* tile, const Rows<T>& rows, int t0, int end, int n, int first, int step, int lane) {
  using H = Head<T, DB>;
  constexpr int COPIES = KT * H::ROW / 1024;
#pragma unroll
  for (int s = 0; s < COPIES; ++s) {
    const int q = first + s * step;
    if (q >= COPIES) break;
    const int byte = q * 1024 + lane * 16, key = byte / H::ROW, slot = byte % H::ROW / 16;
    const int piece = slot ^ (VALUES ? v_twist<T, H::PIECES>(key) : k_twist<H::PIECES>(key)), e = piece * (16 / (int)sizeof(T));
    const bool in = t0 + key < end && e < n;
    if constexpr (FAST) {
      const void* p = in ? static_cast<const void*>(rows.at(t0 + key) + e) : ZEROS;
      __builtin_amdgcn_global_load_lds(p, (lds_void*)(tile + q * 1024), 16, 0, 0);
    } else {
      *reinterpret_cast<v4u*>(tile + byte) = in ? load_piece<T>(rows.at(t0 + key), e, n) : v4u{0, 0, 0, 0};
    }
  }
}

// A row of queries times the scale's sign, as the second operand of S^T: pieces 2 s + (lane / 32) of it.  Scores are
// then scaled by a positive number, which keeps their order and hides a key by -inf.
template <typename T, int DB> using Query = v4u[Head<T, DB>::STEPS];
template <typename T, int DB> __device__ __forceinline__ void load_query(Query<T, DB>& q, const T* p, int n, int half, float scale) {
#pragma unroll
  for (int s = 0; s < Head<T, DB>::STEPS; ++s) {
    const int e = (2 * s + half) * (16 / (int)sizeof(T));
    q[s] = e < n ? load_piece<T>(p, e, n) : v4u{0, 0, 0, 0};
    if (scale < 0.f) q[s] ^= sizeof(T) == 4 ? 0x80000000u : 0x80008000u;
    if (scale == 0.f) {                        // 0, or NaN of what is not finite
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w = q[s][i], hi = (w & 0x7f800000u) == 0x7f800000u ? 0x7fc00000u : 0u;
        q[s][i] = sizeof(T) == 4 ? hi : hi | ((w & 0x7f80u) == 0x7f80u ? 0x7fc0u : 0u);
      }
    }
  }
}

// The factor of the scores, for exponents of 2.
__device__ __forceinline__ float factor(float scale) { return (scale == 0.f ? 1.f : fabsf(scale)) * 1.44269504088896340736f; }

template <typename T> __device__ __forceinline__ v16f mma_piece(v4u a, v4u b, v16f c) {
  if constexpr (sizeof(T) == 2) return Mma<T>::mma(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c);
  else {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = Mma<T>::mma(__uint_as_float(a[i]), __uint_as_float(b[i]), c);
    return c;
  }
}

// S^T of 32 keys of a tile from key k0 on
template <typename T, int DB> __device__ __forceinline__ v16f scores(const char* tile, int k0, int lane, const Query<T, DB>& q) {
  using H = Head<T, DB>;
  const int key = k0 + (lane & 31), twist = k_twist<H::PIECES>(key);
  const char* row = tile + key * H::ROW;
  v16f s = {};
#pragma unroll
  for (int i = 0; i < H::STEPS; ++i) s = mma_piece<T>(*reinterpret_cast<const v4u*>(row + ((2 * i + (lane >> 5)) ^ twist) * 16), q[i], s);
  return s;
}

// The first operand of O^T: channels 32 db + l % 32 of the values of instruction `step` of 32 keys from k0 on.
template <typename T, int DB> __device__ __forceinline__ typename Mma<T>::frag values(const char* tile, int k0, int step, int db, int lane) {
  using H = Head<T, DB>;
  const int half = lane >> 5;
  if constexpr (sizeof(T) == 2) {
    // each read transposes 4 keys x 16 channels among 16 lanes
    v4s r[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int key = k0 + 16 * step + 8 * i + 4 * half + (lane & 15) / 4, c = 32 * db + (lane & 16) + (lane & 3) * 4;
      const char* p = tile + key * H::ROW + (((c >> 3) ^ v_twist<T, H::PIECES>(key)) << 4) + (c & 4) * 2;
      r[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)p);
    }
    return __builtin_bit_cast(v8bf, __builtin_shufflevector(r[0], r[1], 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    const int key = k0 + 8 * (step / 4) + 4 * half + step % 4, c = 32 * db + (lane & 31);
    return *reinterpret_cast<const float*>(tile + key * H::ROW + (((c >> 2) ^ v_twist<T, H::PIECES>(key)) << 4) + (c & 3) * 4);
  }
}

// Bits that say whether some of a fragment's values are infinite or NaN (add them up by |, ask with nonfinite).
template <typename T> __device__ __forceinline__ uint32_t test_values(typename Mma<T>::frag f) {
  if constexpr (sizeof(T) == 4) {
    return (__float_as_uint(f) & 0x7f800000u) + 0x00800000u;    // exponents of ones carry into the sign's place
  } else {
    const v4u w = __builtin_bit_cast(v4u, f);
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) t |= (w[i] & 0x7f807f80u) + 0x00800080u;
    return t;
  }
}
template <typename T> __device__ __forceinline__ bool nonfinite(uint32_t t) { return __any((t & (sizeof(T) == 4 ? 0x80000000u : 0x80008000u)) != 0); }

// A fragment with zeros in the place of what is not finite.
template <typename T> __device__ __forceinline__ typename Mma<T>::frag finite_only(typename Mma<T>::frag f) {
  if constexpr (sizeof(T) == 4) {
    return (__float_as_uint(f) & 0x7f800000u) == 0x7f800000u ? 0.f : f;
  } else {
    v4u w = __builtin_bit_cast(v4u, f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = w[i];
      w[i] = ((x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u) | ((x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu);
    }
    return __builtin_bit_cast(v8bf, w);
  }
}

// Adds the values of channels 32 db ... that are not finite to the sums of the rows that see their keys.
template <typename T, int DB>
__device__ __forceinline__ v16f add_nonfinite(const char* tile, int keys, int db, int lo, int hi, int half, v16f acc) {
  using H = Head<T, DB>;
#pragma unroll 1
  for (int key = max(0, lo); key < min(keys, hi); ++key) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int c = 32 * db + 8 * (i / 4) + 4 * half + i % 4, at = c * (int)sizeof(T);
      const float v = to_f<T>(*reinterpret_cast<const T*>(tile + key * H::ROW + (((at >> 4) ^ v_twist<T, H::PIECES>(key)) << 4) + (at & 15)));
      acc[i] += fabsf(v) < __builtin_inff() ? 0.f : v;
    }
  }
  return acc;
}

// The running softmax of a wave's rows: exponents of 2, the largest so far and the sum of the lane's half of the keys.
template <int DB> struct Running {
  v16f o[DB];
  float m, l;
  __device__ __forceinline__ void start() {
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i] = v16f{};
    m = -__builtin_inff();
    l = 0.f;
  }
};

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

// Takes KB times 32 keys of a tile into a wave's sums.  Rows see keys lo ... hi - 1, counted from the tile's first.
// MASKED: some key is hidden from some row.  c: the scores' factor, log2(e) included.
template <typename T, int DB, int KB, bool MASKED>
__device__ __forceinline__ void take(Running<DB>& run, v16f (&s)[KB], const char* vtile, int lo, int hi, float c, int lane) {
  constexpr float LOWEST = -__builtin_inff();
  const int half = lane >> 5;
  if constexpr (MASKED) {
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = 32 * b + 8 * (i / 4) + 4 * half + i % 4;
        s[b][i] = key >= lo && key < hi ? s[b][i] : LOWEST;
      }
  }
  float m = s[0][0];
#pragma unroll
  for (int b = 0; b < KB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) m = fmaxf(m, s[b][i]);
  m = fmaxf(m, other_half(m)) * c;
  m = fmaxf(run.m, m);
  const float base = m == LOWEST ? 0.f : m;    // nothing above -inf yet: every weight is 0
  const float old = __builtin_amdgcn_exp2f(run.m - base);
  run.m = m;
  float l = 0.f;
#pragma unroll
  for (int b = 0; b < KB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], c, -base));
      l += s[b][i];
    }
  run.l = run.l * old + l;
#pragma unroll
  for (int d = 0; d < DB; ++d) run.o[d] *= old;
  constexpr int N = Mma<T>::N, STEPS = 16 / N;
  typename Mma<T>::frag p[KB][STEPS];
#pragma unroll
  for (int b = 0; b < KB; ++b)
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      if constexpr (N == 1) p[b][st] = s[b][st];
      else {
        v4u w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = f2bf2(s[b][8 * st + 2 * i], s[b][8 * st + 2 * i + 1]);
        p[b][st] = __builtin_bit_cast(v8bf, w);
      }
    }
#pragma unroll
  for (int d = 0; d < DB; ++d) {
    if constexpr (!MASKED) {
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int st = 0; st < STEPS; ++st) run.o[d] = Mma<T>::mma(values<T, DB>(vtile, 32 * b, st, d, lane), p[b][st], run.o[d]);
    } else {
      // A hidden key's weight is 0, which infinity or NaN must not meet: where a value is not finite, the finite ones
      // are summed again without it, and it is added for the rows that see it.
      v16f acc = {};
      uint32_t test = 0;
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
          const auto v = values<T, DB>(vtile, 32 * b, st, d, lane);
          test |= test_values<T>(v);
          acc = Mma<T>::mma(v, p[b][st], acc);
        }
      if (nonfinite<T>(test)) {
        acc = v16f{};
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
          for (int st = 0; st < STEPS; ++st) acc = Mma<T>::mma(finite_only<T>(values<T, DB>(vtile, 32 * b, st, d, lane)), p[b][st], acc);
        acc = add_nonfinite<T, DB>(vtile, 32 * KB, d, lo, hi, half, acc);
      }
      run.o[d] += acc;
    }
  }
}

// Four neighbouring channels c ... of n
template <typename T> __device__ __forceinline__ void store4(T* p, int c, int n, float a, float b, float d, float e) {
  const float v[4] = {a, b, d, e};
  if (c + 4 <= n) {
    if constexpr (sizeof(T) == 2) {
      typedef uint32_t v2u __attribute__((ext_vector_type(2)));
      typedef v2u __attribute__((aligned(2))) any;
      *reinterpret_cast<any*>(p + c) = v2u{f2bf2(a, b), f2bf2(d, e)};
    } else {
      typedef v4f __attribute__((aligned(4))) any;
      *reinterpret_cast<any*>(p + c) = v4f{a, b, d, e};
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (c + i < n) p[c + i] = from_f<T>(v[i]);
}

template <typename T, int DB> __device__ __forceinline__ void store_row(T* p, int n, const v16f (&o)[DB], float f, int half) {
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4) store4<T>(p, 32 * d + 2 * i + 4 * half, n, o[d][i] * f, o[d][i + 1] * f, o[d][i + 2] * f, o[d][i + 3] * f);
}

// The range of keys that a token at position `pos` of a sequence of `total` sees.
__device__ __forceinline__ void sees(const mure_attn_attend_args& a, int pos, int total, int& lo, int& hi) {
  const int64_t w = a.window;
  lo = w && pos >= w ? (int)(pos - w + 1) : 0;
  hi = a.causal ? pos + 1 : w && pos + w < total ? (int)(pos + w) : total;
}

}  // namespace mure
