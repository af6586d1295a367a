// Loads, stores and sums that the operators' kernels share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace evg {

typedef _Float16 half_t;
typedef __bf16 bf16_t;

template <typename T> __device__ __forceinline__ float to_f(T v) { return (float)v; }
// Rounds to the nearest, ties to even.
template <typename T> __device__ __forceinline__ T from_f(float v) { return (T)v; }

// N consecutive elements at any alignment that their type allows: global accesses of 16 bytes need none on gfx950.
template <typename T, int N> struct __attribute__((packed, aligned(sizeof(T)))) Pack { T v[N]; };

template <int N, typename T>
__device__ __forceinline__ void load_n(const T* p, float* v) {
  const Pack<T, N> r = *reinterpret_cast<const Pack<T, N>*>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = to_f(r.v[i]);
}

template <int N, typename T>
__device__ __forceinline__ void store_n(T* p, const float* v) {
  Pack<T, N> r;
#pragma unroll
  for (int i = 0; i < N; ++i) r.v[i] = from_f<T>(v[i]);
  *reinterpret_cast<Pack<T, N>*>(p) = r;
}

// Non-temporal: what is not read again soon should not push out what is.
template <int N, typename T>
__device__ __forceinline__ void load_n_once(const T* p, float* v) {
  typedef uint32_t words __attribute__((ext_vector_type(N * sizeof(T) / 4), aligned(sizeof(T))));
  const words w = __builtin_nontemporal_load(reinterpret_cast<const words*>(p));
  const Pack<T, N> r = __builtin_bit_cast(Pack<T, N>, w);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = to_f(r.v[i]);
}

template <int N, typename T>
__device__ __forceinline__ void store_n_once(T* p, const float* v) {
  typedef uint32_t words __attribute__((ext_vector_type(N * sizeof(T) / 4), aligned(sizeof(T))));
  Pack<T, N> r;
#pragma unroll
  for (int i = 0; i < N; ++i) r.v[i] = from_f<T>(v[i]);
  __builtin_nontemporal_store(__builtin_bit_cast(words, r), reinterpret_cast<words*>(p));
}

// The first n of N elements (n may be <= 0 or >= N); the others are 0.
template <int N, typename T>
__device__ __forceinline__ void load_upto(const T* p, int n, float* v) {
  if (n >= N) {
    load_n<N>(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < n ? to_f(p[i]) : 0.f;
  }
}

template <int N, typename T>
__device__ __forceinline__ void store_upto(T* p, int n, const float* v) {
  if (n >= N) {
    store_n<N>(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = from_f<T>(v[i]);
  }
}

// The first n of N elements as they are; the others are 0.  ONCE: past the caches.
template <int N, bool ONCE = false, typename T>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p, int n) {
  typedef uint32_t words __attribute__((ext_vector_type(N * sizeof(T) / 4), aligned(sizeof(T))));
  if (n >= N) {
    if constexpr (ONCE) return __builtin_bit_cast(Pack<T, N>, __builtin_nontemporal_load(reinterpret_cast<const words*>(p)));
    return *reinterpret_cast<const Pack<T, N>*>(p);
  }
  Pack<T, N> r;
#pragma unroll
  for (int i = 0; i < N; ++i) r.v[i] = i < n ? p[i] : (T)0.f;
  return r;
}

template <int N, bool ONCE = false, typename T>
__device__ __forceinline__ void store_pack(T* p, int n, const Pack<T, N>& r) {
  typedef uint32_t words __attribute__((ext_vector_type(N * sizeof(T) / 4), aligned(sizeof(T))));
  if (n >= N) {
    if constexpr (ONCE) __builtin_nontemporal_store(__builtin_bit_cast(words, r), reinterpret_cast<words*>(p));
    else *reinterpret_cast<Pack<T, N>*>(p) = r;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = r.v[i];
  }
}

// The sum over a wavefront, in every lane; the order is fixed.
template <typename F>
__device__ __forceinline__ F wave_sum(F v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}

// The same of 32-bit values without the LDS permutes, whose latency a row's dependent sums would add up: the lanes of 16 by data-parallel
// moves, then rows of 16 into the next and halves into the last lane, from where it is uniform.
template <int CTRL, int ROWS>
__device__ __forceinline__ float moved(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROWS, 0xf, false));
}
// Over each 2, 4, 8 or 16 lanes, in all of them: each adds the same pairs, so they get the same bits.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
  v += moved<0xB1, 0xf>(v);                               // lanes 1 0 3 2
  if constexpr (LANES >= 4) v += moved<0x4E, 0xf>(v);     // lanes 2 3 0 1
  if constexpr (LANES >= 8) v += moved<0x141, 0xf>(v);    // mirrored within 8
  if constexpr (LANES >= 16) v += moved<0x140, 0xf>(v);   // mirrored within 16
  return v;
}
__device__ __forceinline__ float wave_sum_uniform(float v) {
  v = lanes_sum<16>(v);
  v += moved<0x142, 0xa>(v);   // row 0's into row 1, row 2's into row 3
  v += moved<0x143, 0xc>(v);   // the lower half's into the upper one
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

}  // namespace evg
