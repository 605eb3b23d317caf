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
typedef __attribute__((address_space(3))) void lds_void;
typedef v4u __attribute__((aligned(2))) v4u_any;  // the GPU's global loads and stores take any address

// Two floats -> two bfloat16 (lo in bits 0-15), to nearest even, by the compiler's conversion: it keeps the wait state
// between an exponential and the use of its result, which inline assembly does not.
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v2f{lo, hi}, v2bf));
}

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

// What a tile holds, by the reads of it: keys in 16-byte pieces of 16 rows, values in 64 bytes of 4 rows (float32: 128
// bytes of two) for 32x32 products, values in 32 bytes of 8 rows (float32: 64 of four) for 16x16 products.
enum Reads { KEYS, VALUES32, VALUES16 };

// The place of a row's 16-byte pieces in LDS is xored with a number of the row's, so that the rows that lanes read
// together lie in different banks.  PERIOD: rows after which the numbers repeat.
template <typename T, int PIECES, Reads R> struct Twist {
  static constexpr int PERIOD = R == KEYS ? 16 : R == VALUES16 ? sizeof(T) == 4 ? 16 : 8 : sizeof(T) == 4 ? 8 : 4;
  static __device__ __forceinline__ int of(int key) {
    if (R == KEYS) return PIECES >= 16 ? key & 15 : PIECES == 8 ? (key >> 1) & 7 : (key >> 2) & 3;
    if (R == VALUES32) {
      if (sizeof(T) == 4) return PIECES >= 16 ? ((key >> 2) & 1) << 3 : 0;
      return PIECES >= 16 ? (key & 3) << 2 : PIECES == 8 ? ((key >> 1) & 1) << 2 : 0;
    }
    if (sizeof(T) == 4) return PIECES >= 16 ? ((key >> 2) & 3) << 2 : ((key >> 2) & 1) << 2;
    return PIECES >= 16 ? (key & 7) << 1 : PIECES == 8 ? ((key >> 1) & 3) << 1 : ((key >> 2) & 1) << 1;
  }
};

// The rows of one sequence's keys (or values) of one head: its cache's first, then the call's own.
template <typename T> struct Rows {
  const T* held;
  const T* own;
  int64_t held_stride, own_stride;
  int past;
  __device__ __forceinline__ const T* at(int j) const { return j < past ? held + j * held_stride : own + (int64_t)(j - past) * own_stride; }
};

// A number that is the same in all lanes, for the scalar unit (a division leaves it in the vector unit's registers).
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
template <typename T> __device__ __forceinline__ T* uniform(T* p) {
  const uint64_t v = (uint64_t)p;
  return (T*)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}

// Waits for the wave's own copies to LDS but the last N.
template <int N = 0> __device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// 16 bytes from p + first on of a row of n elements, zeros behind its end.
template <typename T> __device__ __forceinline__ v4u load_piece(const T* p, int first, int n) {
  constexpr int E = 16 / sizeof(T);
  if (first + E <= n) return *reinterpret_cast<const v4u_any*>(p + first);
  v4u v = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (first + i < n) {
      if constexpr (sizeof(T) == 4) v[i] = __float_as_uint(p[first + i]);
      else v[i / 2] |= (uint32_t)p[first + i] << (i & 1 ? 16 : 0);
    }
  return v;
}

// The same of a row of whole words, at least one piece long, without a branch: the row's last piece, moved down.
template <typename T> __device__ __forceinline__ v4u load_words(const T* p, int first, int n) {
  constexpr int E = 16 / sizeof(T);
  v4u v = *reinterpret_cast<const v4u_any*>(p + min(first, n - E));
  const int by = (first - (n - E)) * (int)sizeof(T) / 4;       // words
  if (by > 0) {
    if (by & 1) v = v4u{v[1], v[2], v[3], 0};
    if (by & 2) v = v4u{v[2], v[3], 0, 0};
    if (by >= 4) v = v4u{0, 0, 0, 0};
  }
  return v;
}

// 16 bytes a lane from `off` on of a buffer of `bytes` bytes at p (zeros behind it) to `to`, one lane after the other.  As the
// compiler's builtin every later read of LDS would wait for it; this one only wait_copies waits for.  The wait states are
// those between a scalar's write by the vector unit, or m0's, and its use here.  Nothing else in these kernels uses m0, so
// the warning that the compiler need not keep it is moot.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy16(const void* p, int bytes, unsigned off, char* to) {
  const uint64_t at = (uint64_t)p;
  const v4u r = {(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, (uint32_t)bytes, 0x00027000u};
  const uint32_t lds = (uint32_t)(uintptr_t)(lds_void*)to;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(uniform((int)lds)), "v"(off), "s"(r) : "memory", "m0");
}

// Copies of KT keys' rows into a tile by W waves, 1024 bytes a wave and step.
template <typename T, int DB, int KT, int W, Reads R> struct Copy {
  using H = Head<T, DB>;
  using Tw = Twist<T, H::PIECES, R>;
  static constexpr int COPIES = KT * H::ROW / 1024, STEPS = (COPIES + W - 1) / W, EACH = 1024 / H::ROW;      // keys of a copy
  static_assert(COPIES % W == 0 || COPIES < W, "");

  // The place of the lane's piece of copy q: its key in the tile, its first element there.
  static __device__ __forceinline__ void place(int q, int lane, int& key, int& e) {
    const int byte = q * 1024 + lane * 16;
    key = byte / H::ROW;
    e = (byte % H::ROW / 16 ^ Tw::of(key)) * (16 / (int)sizeof(T));
  }

  // Rows of n elements from key t0 on, zeros from key `end` on and behind the row, element by element where need be.
  static __device__ __forceinline__ void slowly(char* tile, const Rows<T>& rows, int t0, int end, int n, int wave, int lane) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int q = wave + s * W;
      if (COPIES % W && q >= COPIES) break;
      int key, e;
      place(q, lane, key, e);
      *reinterpret_cast<v4u*>(tile + q * 1024 + lane * 16) = t0 + key < end && e < n ? load_piece<T>(rows.at(t0 + key), e, n) : v4u{0, 0, 0, 0};
    }
  }

  // Keys from ... to - 1 of the tile whose key 0 is (or would be) at p, straight to LDS (wait_copies) through a buffer that
  // ends with key to - 1: what lies behind it, or behind a row, reads as zeros.  A tile's rows lie within 2^31 bytes.
  static __device__ __forceinline__ void straight(char* tile, const T* p, int64_t stride, int from, int to, int n, int wave, int lane) {
    // scalars, every one of them: a buffer's description in vector registers costs a loop around each copy
    const int pitch = uniform((int)(stride * (int)sizeof(T))), bytes = uniform((to - 1) * pitch + n * (int)sizeof(T));
    char* const base = uniform(const_cast<char*>(reinterpret_cast<const char*>(p)));
    if constexpr (W * EACH % Tw::PERIOD) asm("" : "+v"(lane));     // places stay out of registers between tiles
    int key, e;
    place(wave, lane, key, e);
    unsigned off = (unsigned)(key * pitch) + (e < n ? (unsigned)(e * (int)sizeof(T)) : 0x80000000u);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int q = wave + s * W;
      if (COPIES % W && q >= COPIES) break;
      // the step's own place is in the buffer's base, so that the lanes' offsets are the same in every step
      const int first = s * W * EACH * pitch;
      if (s && W * EACH % Tw::PERIOD) {
        int k;
        place(q, lane, k, e);
        off = (unsigned)(key * pitch) + (e < n ? (unsigned)(e * (int)sizeof(T)) : 0x80000000u);
      }
      if (from <= 0) copy16(base + first, max(0, bytes - first), off, tile + q * 1024);
      else if (key + s * W * EACH >= from) copy16(base + first, max(0, bytes - first), off, tile + q * 1024);
    }
  }

  // `straight` of a whole tile in four steps, with few scalar instructions: the steps' places are the buffer's scalar
  // offsets (which must lie inside the buffer, and do in a whole tile).
  static __device__ __forceinline__ void whole(char* tile, const T* p, int64_t stride, int n, int wave, int lane) {
    const int pitch = uniform((int)(stride * (int)sizeof(T)));
    int key, e;
    place(wave, lane, key, e);
    const unsigned off = (unsigned)(key * pitch) + (e < n ? (unsigned)(e * (int)sizeof(T)) : 0x80000000u);
    const uint64_t at = (uint64_t)uniform(p);
    const v4u r = {(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, (uint32_t)uniform((KT - 1) * pitch + n * (int)sizeof(T)), 0x00027000u};
    const uint32_t lds = (uint32_t)uniform((int)(uint32_t)(uintptr_t)(lds_void*)(tile + wave * 1024));
    const int step = W * EACH * pitch;
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds\n\t"
        "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds\n\t"
        "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %4 offen lds\n\t"
        "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %5 offen lds" ::"s"(lds), "v"(off), "s"(r), "s"(step), "s"(2 * step), "s"(3 * step), "n"(W * 1024)
        : "memory", "m0", "scc");
  }

  // Rows that are whole words but no whole pieces: after the copies, zeros behind the row in its last piece, each by the wave
  // that copied it.
  static __device__ __forceinline__ void trim(char* tile, int n, int wave, int lane) {
    constexpr int E = 16 / (int)sizeof(T);
    static_assert(KT <= 64, "");
    if (n % E == 0) return;
    const int piece = lane * H::PIECES + (n / E ^ Tw::of(lane)), words = n % E * (int)sizeof(T) / 4;
    if (lane >= KT || piece / 64 % W != wave) return;
    uint32_t* to = reinterpret_cast<uint32_t*>(tile + piece * 16);
    if (words < 2) to[1] = 0;
    if (words < 3) to[2] = 0;
    to[3] = 0;
  }

  // A tile at key t0; at least STEPS copies a wave.
  template <int FAST> static __device__ __forceinline__ void run(char* tile, const Rows<T>& rows, int t0, int end, int n, int wave, int lane) {
    if constexpr (FAST) {
      if constexpr (COPIES == 4 * W && W * EACH % Tw::PERIOD == 0) {
        if (t0 >= rows.past && t0 + KT <= end) return whole(tile, rows.own + (int64_t)(t0 - rows.past) * rows.own_stride, rows.own_stride, n, wave, lane);
        if (t0 + KT <= rows.past) return whole(tile, rows.held + (int64_t)t0 * rows.held_stride, rows.held_stride, n, wave, lane);
      }
      const int held = min(rows.past - t0, KT);                // keys of the tile that the cache holds: the others come from the call's own rows
      if (held > 0) straight(tile, rows.held + (int64_t)t0 * rows.held_stride, rows.held_stride, 0, held, n, wave, lane);
      if (held < KT) straight(tile, rows.own + (int64_t)(t0 - rows.past) * rows.own_stride, rows.own_stride, held, min(end - t0, KT), n, wave, lane);
    } else {
      slowly(tile, rows, t0, end, n, wave, lane);
    }
  }
};
#pragma clang diagnostic pop

// A row of queries times the scale's sign, as the second operand of S^T: pieces W s + w of it.  Scores are then scaled by a
// positive number, which keeps their order and hides a key by -inf.
template <typename T, int DB> using Query = v4u[Head<T, DB>::STEPS];
template <typename T, int STEPS, int W> __device__ __forceinline__ void load_query(v4u* q, const T* p, int n, int w, float scale) {
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int e = (W * s + w) * (16 / (int)sizeof(T));
    q[s] = e < n ? load_piece<T>(p, e, n) : v4u{0, 0, 0, 0};
    if (scale < 0.f) q[s] ^= sizeof(T) == 4 ? 0x80000000u : 0x80008000u;
    if (scale == 0.f) {                        // 0, or NaN of what is not finite
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = q[s][i], hi = (x & 0x7f800000u) == 0x7f800000u ? 0x7fc00000u : 0u;
        q[s][i] = sizeof(T) == 4 ? hi : hi | ((x & 0x7f80u) == 0x7f80u ? 0x7fc0u : 0u);
      }
    }
  }
}

// The factor of the scores, for exponents of 2: finite, so that scores of 0 stay 0.
__device__ __forceinline__ float factor(float scale) { return fminf((scale == 0.f ? 1.f : fabsf(scale)) * 1.44269504088896340736f, 3.402823466e38f); }

template <typename T> __device__ __forceinline__ v16f mma_piece(v4u a, v4u b, v16f c) {
  if constexpr (sizeof(T) == 2) return Mma<T>::mma(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c);
  else {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = Mma<T>::mma(__uint_as_float(a[i]), __uint_as_float(b[i]), c);
    return c;
  }
}

// A lane's places in a tile, from which all of its reads are constant steps or bits away.
template <typename T, int DB> struct Reader {
  using H = Head<T, DB>;
  int k, v;
  __device__ __forceinline__ explicit Reader(int lane) {
    const int half = lane >> 5, key = lane & 31;
    k = key * H::ROW + ((half ^ Twist<T, H::PIECES, KEYS>::of(key)) << 4);
    if constexpr (sizeof(T) == 2) {
      const int vk = 4 * half + (lane & 15) / 4, c = (lane & 16) + (lane & 3) * 4;
      v = vk * H::ROW + (((c >> 3) ^ Twist<T, H::PIECES, VALUES32>::of(vk)) << 4) + (c & 4) * 2;
    } else {
      const int vk = 4 * half, c = lane & 31;
      v = vk * H::ROW + (((c >> 2) ^ Twist<T, H::PIECES, VALUES32>::of(vk)) << 4) + (c & 3) * 4;
    }
  }

  // A piece of the lane's key of 32 from key k0 (a multiple of 32) on: twists have a period of at most 32 keys
  __device__ __forceinline__ v4u piece(const char* tile, int k0, int i) const { return *reinterpret_cast<const v4u*>(tile + (k ^ (i << 5)) + k0 * H::ROW); }

  // S^T of 32 keys of a tile
  __device__ __forceinline__ v16f scores(const char* tile, int k0, const Query<T, DB>& q) const {
    // some pieces ahead of their products, and the next ones beside them
    constexpr int G = H::STEPS % 4 == 0 ? 4 : H::STEPS % 3 == 0 ? 3 : 2;
    v16f s = {};
    v4u a[2][G];
#pragma unroll
    for (int i = 0; i < G; ++i) a[0][i] = piece(tile, k0, i);
#pragma unroll
    for (int g = 0; g < H::STEPS; g += G) {
      if (g + G < H::STEPS)
#pragma unroll
        for (int i = 0; i < G; ++i) a[g / G + 1 & 1][i] = piece(tile, k0, g + G + i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < G; ++i) s = mma_piece<T>(a[g / G & 1][i], q[g + i], s);
    }
    return s;
  }

  // The first operand of O^T: channels 32 db + l % 32 of the values of instruction `step` of 32 keys from k0 on.
  __device__ __forceinline__ typename Mma<T>::frag values(const char* tile, int k0, int step, int db) const {
    if constexpr (sizeof(T) == 2) {
      // each read transposes 4 keys x 16 channels among 16 lanes
      v4s r[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        r[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(tile + (v ^ (db << 6)) + (k0 + 16 * step + 8 * i) * H::ROW));
      return __builtin_bit_cast(v8bf, __builtin_shufflevector(r[0], r[1], 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      return *reinterpret_cast<const float*>(tile + (v ^ (db << 7)) + (k0 + 8 * (step / 4) + step % 4) * H::ROW);
    }
  }
};

// Puts zeros in the place of what is infinite or NaN in keys from ... to - 1 of a tile, and says whether there was any.
// A hidden key's weight is 0, which must not meet it; the rows that see the key get it by add_nonfinite, when all is summed.
template <typename T, int DB> __device__ __forceinline__ bool clean(char* tile, int from, int to, int tid, int threads) {
  // exponents of ones carry into the sign's place
  constexpr uint32_t ONES = sizeof(T) == 4 ? 0x7f800000u : 0x7f807f80u, CARRY = sizeof(T) == 4 ? 0x00800000u : 0x00800080u;
  constexpr uint32_t SIGN = sizeof(T) == 4 ? 0x80000000u : 0x80008000u;
  bool found = false;
#pragma unroll 1
  for (int byte = from * Head<T, DB>::ROW + tid * 16; byte < to * Head<T, DB>::ROW; byte += threads * 16) {
    v4u w = *reinterpret_cast<const v4u*>(tile + byte);
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) any |= (w[i] & ONES) + CARRY;
    if (!(any & SIGN)) continue;
    found = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t t = ((w[i] & ONES) + CARRY) & SIGN;
      w[i] &= sizeof(T) == 4 ? (t ? 0u : ~0u) : (t & 0x80000000u ? 0u : 0xffff0000u) | (t & 0x8000u ? 0u : 0xffffu);
    }
    *reinterpret_cast<v4u*>(tile + byte) = w;
  }
  return found;
}

// The weights of 32 keys, as operands of O^T.  In bfloat16 each is rounded once, to half a step of 2^-8 of itself: in two
// halves they would double the second product, half of the matrix instructions.  The sum below a result adds them
// unrounded.  The measured cases' errors against float64 are 0.0020 to 0.0023 of the result's norm so, and 0.0016 from the
// rounding of the results alone.
template <typename T> struct Weights {
  static constexpr int N = 16 / Mma<T>::N;
  typename Mma<T>::frag p[N];
  __device__ __forceinline__ void set(int i, const v16f& s) {
    if constexpr (Mma<T>::N == 1) p[i] = s[i];
    else {
      v4u w;
#pragma unroll
      for (int x = 0; x < 4; ++x) w[x] = pack2(s[8 * i + 2 * x], s[8 * i + 2 * x + 1]);
      p[i] = __builtin_bit_cast(v8bf, w);
    }
  }
};

// Scores of keys that the lane's row does not see: it sees lo ... hi - 1 of the 32.
__device__ __forceinline__ void hide(v16f& s, int lo, int hi, int half) {
  lo -= 4 * half;                              // so that the keys' numbers are constants
  hi -= 4 * half;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int key = 8 * (i / 4) + i % 4;
    s[i] = key >= lo && key < hi ? s[i] : -__builtin_inff();
  }
}

// A lane's number and that of the lane 32 further, in both.
struct Halves {
  float a, b;
  __device__ __forceinline__ explicit Halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
  }
};

// The running softmax of a wave's rows: exponents of 2, their base and the sum of the lane's half of the keys' weights.
template <int DB> struct Running {
  v16f o[DB];
  float m, l;
  static __device__ __forceinline__ int channel(int i, int lane) { return i / 16 * 32 + 8 * (i / 4 % 4) + 4 * (lane >> 5) + i % 4; }
  __device__ __forceinline__ void start() {
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i] = v16f{};
    m = -__builtin_inff();
    l = 0.f;
  }

  // The base for 32 more scores: it stays where it is until a weight would pass 2^8, then, row by row, the largest exponent
  // becomes the base.  True: the row's sums have to be multiplied by `old` (l has been) before such weights are added.
  // c: the scores' factor, log2(e) included.
  __device__ __forceinline__ bool base_for(const v16f& s, float c, float& old) {
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    const Halves both(top);
    top = fmaxf(both.a, both.b) * c;
    const bool grows = top > m + 8.f;
    old = grows ? __builtin_amdgcn_exp2f(m - top) : 1.f;       // 0 of an infinite sum is NaN, which add_nonfinite mends
    m = grows ? top : m;
    l *= old;
    return grows;
  }
  __device__ __forceinline__ void rescale(float old) {
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] *= old;
  }

  // The weights of 32 scores; nothing above -inf yet: every weight is 0.
  __device__ __forceinline__ float weight(float s, float c, float base) { return __builtin_amdgcn_exp2f(fmaf(s, c, -base)); }
  template <typename T> __device__ __forceinline__ Weights<T> weigh(v16f s, float c) {
    const float base = m == -__builtin_inff() ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = weight(s[i], c, base);
      sum += s[i];
    }
    l += sum;
    Weights<T> w;
#pragma unroll
    for (int i = 0; i < Weights<T>::N; ++i) w.set(i, s);
    return w;
  }

  // Adds the values of 32 keys of a tile from key k0 on.
  template <typename T> __device__ __forceinline__ void add(const Reader<T, DB>& read, const char* tile, int k0, const Weights<T>& w) {
    // some fragments ahead of their products, and the next ones beside them
    constexpr int N = Weights<T>::N, G = N < 4 ? N : 4;
    typename Mma<T>::frag v[2][G];
    const auto fill = [&](int g) {
#pragma unroll
      for (int i = 0; i < G; ++i) v[g & 1][i] = read.values(tile, k0, g * G % N + i, g * G / N);
    };
    fill(0);
#pragma unroll
    for (int g = 0; g < DB * N / G; ++g) {
      if (g + 1 < DB * N / G) fill(g + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < G; ++i) o[g * G / N] = Mma<T>::mma(v[g & 1][i], w.p[g * G % N + i], o[g * G / N]);
    }
  }

  // weigh of these scores, the next keys' scores and add of the last ones: after every product a share of the softmax, its
  // operand read some products ahead.
  template <typename T>
  __device__ __forceinline__ void mixed(const v16f& s, float c, Weights<T>& mine, const Reader<T, DB>& read, const char* next, int next_at, const Query<T, DB>& q, v16f& after,
                                        const char* last, int last_at, const Weights<T>& w) {
    static_assert(sizeof(T) == 2, "");
    constexpr int QK = Head<T, DB>::STEPS, PRODUCTS = 2 * QK, AHEAD = 3;
    const float base = m == -__builtin_inff() ? 0.f : m;
    v4u ring[AHEAD + 1];
    const auto fetch = [&](int n) {
      if (n < QK) ring[n % (AHEAD + 1)] = read.piece(next, next_at, n);
      else if (n < PRODUCTS) ring[n % (AHEAD + 1)] = __builtin_bit_cast(v4u, read.values(last, last_at, (n - QK) % 2, (n - QK) / 2));
    };
    v16f p;
    float sum = 0.f;
    v4u packed[2];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) fetch(n);
#pragma unroll
    for (int n = 0; n < PRODUCTS; ++n) {
      fetch(n + AHEAD);
      const v8bf f = __builtin_bit_cast(v8bf, ring[n % (AHEAD + 1)]);
      if (n < QK) after = Mma<T>::mma(f, __builtin_bit_cast(v8bf, q[n]), n ? after : v16f{});
      else o[(n - QK) / 2] = Mma<T>::mma(f, w.p[(n - QK) % 2], o[(n - QK) / 2]);
#pragma unroll
      for (int i = n * 16 / PRODUCTS; i < (n + 1) * 16 / PRODUCTS; ++i) {
        float x = weight(s[i], c, base);
        sum += x;
        asm volatile("" : "+v"(x), "+v"(sum));                 // here, not where the weights are needed
        p[i] = x;
        if (i & 1) {
          uint32_t pair = pack2(p[i - 1], x);
          asm volatile("" : "+v"(pair));
          packed[i / 8][i / 2 % 4] = pair;
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    l += sum;
    mine.p[0] = __builtin_bit_cast(v8bf, packed[0]);
    mine.p[1] = __builtin_bit_cast(v8bf, packed[1]);
  }
};

// 64 bytes of the summed axis of 16 x 16 results, a lane's piece being a quarter of them: one instruction, or in float32 four.
template <typename T> __device__ __forceinline__ v4f mma16_part(v4u a, v4u b, int e, v4f c) {
  if constexpr (sizeof(T) == 2) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
}
template <typename T> __device__ __forceinline__ v4f mma16(v4u a, v4u b, v4f c) {
#pragma unroll
  for (int e = 0; e < (sizeof(T) == 2 ? 1 : 4); ++e) c = mma16_part<T>(a, b, e, c);
  return c;
}

// Four neighbouring channels c ... of n
template <typename T> __device__ __forceinline__ void store4(T* p, int c, int n, float a, float b, float d, float e) {
  const float v[4] = {a, b, d, e};
  if (c + 4 <= n) {
    if constexpr (sizeof(T) == 2) {
      typedef uint32_t v2u __attribute__((ext_vector_type(2)));
      typedef v2u __attribute__((aligned(2))) any;
      *reinterpret_cast<any*>(p + c) = v2u{pack2(a, b), pack2(d, e)};
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

// What is not finite, added to the stored sums of the wave's rows that see it (`row`: the lane has a row whose weights are
// numbers; l: their sum).  Its weight counts for nothing but where it is 0, which makes NaN:
//   - of the keys that some row of the block does not see, below mid_lo and from mid_hi on, whose values clean has taken out
//     (`apart`: it has found any);
//   - of all keys, where a sum is NaN: a weight that is 0 in float32 and not in the formula makes NaN of an infinite value
//     there.  Without such a value the sum stays NaN: finite ones have passed float32.
// A weight is 0 in the formula where the score is -inf: where the key is not finite (any other score that such a key has
// would make the weights NaN), or in all of a row (l = 0).
// The row sees keys lo ... hi - 1 of the tiles of `width` at `first`, `step` further and so on below `to`; N sums a lane, at
// out[channel(i, lane)], four neighbours each.  For all lanes of the wave.
template <int N, typename T, typename O, typename F>
__device__ __forceinline__ void add_nonfinite(bool row, float l, bool apart, O* out, const Rows<T>& keys, const Rows<T>& values, int n, int first, int step, int width, int to, int lo,
                                              int hi, int mid_lo, int mid_hi, int lane, F&& channel) {
  constexpr float INF = __builtin_inff();
  constexpr int EACH = 4;                      // keys whose values are on their way at a time
  // f(first, end) for the tiles' keys from `least` on and below `most`: all, or those outside mid_lo ... mid_hi - 1
  const auto spans = [&](bool all, int least, int most, auto&& f) {
#pragma unroll 1
    for (int t = first; t < most; t += step)
#pragma unroll 1
      for (int side = 0; side < (all ? 1 : 2); ++side) {
        const int from = max(max(t, least), side ? max(mid_lo, mid_hi) : 0), end = min(min(t + width, most), all || side ? most : mid_lo);
        if (from < end && !f(from, end)) return;
      }
  };
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");          // the stores
  bool infinite = false, renewed = false;
#pragma unroll 1
  for (int i = 0; i < N; i += 4) {
    const int c = channel(i, lane);
#pragma unroll 1
    for (int all = 1; all >= 0; --all) {       // sums that are NaN by all keys, then the others by those apart
      if (!row || !(all || apart)) continue;
      float y[4], sum[4] = {};
      bool mine[4], any = false;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        y[x] = c + x < n ? to_f<O>(out[c + x]) : 0.f;
        mine[x] = c + x < n && (y[x] != y[x]) == (bool)all;
        any |= mine[x];
      }
      if (!any) continue;
      spans(all, lo, min(to, hi), [&](int from, int end) {
#pragma unroll 1
        for (int key = from; key < end; key += EACH)
#pragma unroll
          for (int j = 0; j < EACH; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const float v = to_f<T>(values.at(min(key + j, end - 1))[min(c + x, n - 1)]);
              sum[x] += fabsf(v) < INF ? 0.f : v;                      // the last key twice is no other sum
            }
        bool open = false;                     // a sum that a further value may change
#pragma unroll
        for (int x = 0; x < 4; ++x) open |= mine[x] && sum[x] == sum[x];
        return open;
      });
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if (!mine[x] || sum[x] == 0.f) continue;
        if (l == 0.f) sum[x] *= 0.f;
        out[c + x] = from_f<O>(all ? sum[x] : y[x] + sum[x]);
        infinite |= sum[x] == sum[x];
        renewed |= all;
      }
    }
  }
  if (!__any(infinite)) return;
  // 0 times infinity: keys that are not finite
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  spans(__any(renewed), 0, to, [&](int from, int end) {
#pragma unroll 1
    for (int key0 = from; key0 < end; key0 += 64) {
      // exponents of ones carry into the sign's place
      constexpr uint32_t ONES = sizeof(T) == 4 ? 0x7f800000u : 0x7f807f80u, CARRY = sizeof(T) == 4 ? 0x00800000u : 0x00800080u;
      uint32_t any = 0;
      if (key0 + lane < end) {
        const T* p = keys.at(key0 + lane);
#pragma unroll 1
        for (int e = 0; e < n; e += 16 / (int)sizeof(T)) {
          const v4u w = load_piece<T>(p, e, n);
#pragma unroll
          for (int i = 0; i < 4; ++i) any |= (w[i] & ONES) + CARRY;
        }
      }
#pragma unroll 1
      for (uint64_t bad = __ballot((any & (sizeof(T) == 4 ? 0x80000000u : 0x80008000u)) != 0); bad; bad &= bad - 1) {
        const int key = key0 + __builtin_ctzll(bad);
        if (!infinite || key < lo || key >= hi) continue;
#pragma unroll 1
        for (int i = 0; i < N; ++i) {
          const int c = channel(i, lane);
          if (c < n && !(fabsf(to_f<T>(values.at(key)[c])) < INF)) out[c] = from_f<O>(__builtin_nanf(""));
        }
      }
    }
    return true;
  });
}

// The sum v of parts' sums and the next one, x, whose base is log2(f) below: an infinite one stays infinite, however small its
// weights are beside the others'.
__device__ __forceinline__ float join_sum(float x, float f, float v) { return fmaf(x, fabsf(x) == __builtin_inff() ? 1.f : f, v); }

// The range of keys that a token at position `pos` of a sequence of `total` sees.
__device__ __forceinline__ void sees(const mure_attn_attend_args& a, int pos, int total, int& lo, int& hi) {
  const int64_t w = a.window;
  lo = w && pos >= w ? (int)(pos - w + 1) : 0;
  hi = a.causal ? pos + 1 : w && pos + w < total ? (int)(pos + w) : total;
}

}  // namespace mure
