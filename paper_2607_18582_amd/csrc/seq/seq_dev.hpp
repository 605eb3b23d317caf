// Device helpers of the sequence operators: vectors of elements at any
// alignment, activations.
#pragma once

#include <tuple>
#include <utility>

#include "../dev.hpp"
#include "seq.hpp"

namespace mure {

// Enqueues a kernel and returns the launch's own status: hipGetLastError would report what another call of this thread
// has left there.
template <typename... P, typename... A>
hipError_t launch(void (*kernel)(P...), dim3 grid, unsigned block, hipStream_t s, A&&... a) {
  std::tuple<P...> params(std::forward<A>(a)...);
  return std::apply(
      [&](auto&... p) {
        void* at[] = {&p...};
        return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(block), at, 0, s);
      },
      params);
}

// 16 bytes of elements of T at the alignment of T: the GPU's global loads and
// stores take any address (a vector that crosses a cache line costs both).
template <typename T> struct Vec {
  static constexpr int N = 16 / sizeof(T);
  typedef T raw __attribute__((ext_vector_type(N)));
  typedef raw __attribute__((aligned(sizeof(T)))) any;
};

// N elements at p (N = Vec<T>::N: one 16-byte load; N = 1: one element) as floats
template <typename T, int N> __device__ __forceinline__ void load_n(const T* p, float (&v)[N]) {
  if constexpr (N == 1) {
    v[0] = to_f<T>(*p);
  } else {
    const typename Vec<T>::raw r = *reinterpret_cast<const typename Vec<T>::any*>(p);
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = to_f<T>(r[j]);
  }
}

// Results stream past the L2: a large convolution takes 202 us so and 209 with
// plain stores (65536 x 4096 bfloat16).
template <typename T, int N> __device__ __forceinline__ void store_n(T* p, const float (&v)[N]) {
  if constexpr (N == 1) {
    *p = from_f<T>(v[0]);
  } else if constexpr (sizeof(T) == 2) {
    typedef uint32_t words __attribute__((ext_vector_type(N / 2)));
    typedef words __attribute__((aligned(2))) any;
    words r;
#pragma unroll
    for (int j = 0; j < N; j += 2) r[j / 2] = f2bf2(v[j], v[j + 1]);
    __builtin_nontemporal_store(r, reinterpret_cast<any*>(p));
  } else {
    typename Vec<T>::raw r;
#pragma unroll
    for (int j = 0; j < N; ++j) r[j] = v[j];
    __builtin_nontemporal_store(r, reinterpret_cast<typename Vec<T>::any*>(p));
  }
}

// Elements first ... N - 1 of v only.
template <typename T, int N> __device__ __forceinline__ void store_from(T* p, const float (&v)[N], int first) {
  if (first == 0) {
    store_n<T, N>(p, v);
    return;
  }
#pragma unroll
  for (int j = 1; j < N; ++j)
    if (j >= first) p[j] = from_f<T>(v[j]);
}

// sigmoid(z) = 1 / (1 + e^-z) from the hardware exponential and reciprocal,
// each within an ulp; 0 where e^-z is infinite.
__device__ __forceinline__ float seq_sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * z));
}
__device__ __forceinline__ float seq_silu(float z) { return z * seq_sigmoid(z); }

}  // namespace mure
