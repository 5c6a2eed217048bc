// Elements of the sequence operators: float, bfloat16 or half in memory, float in registers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cnn.h"

namespace cnn {

inline bool type_known(int type) { return type == CNN_F32 || type == CNN_BF16 || type == CNN_F16; }
inline size_t type_bytes(int type) { return type == CNN_F32 ? 4 : 2; }

// N elements that are loaded and stored together (16 bytes at a time where they have that many).
template <class T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Pack {
  T v[N];
};

// Loads and stores past the caches, for packs of whole sixteen bytes.
using Words = uint32_t __attribute__((ext_vector_type(4)));
template <class P>
struct Sixteens {
  static_assert(sizeof(P) % 16 == 0, "packs of whole sixteen bytes");
  Words w[sizeof(P) / 16];
};
template <class P>
__device__ __forceinline__ void put_past_caches(P* at, const P& v) {
  const Sixteens<P> words = __builtin_bit_cast(Sixteens<P>, v);
#pragma unroll
  for (int i = 0; i < (int)(sizeof(P) / 16); ++i) __builtin_nontemporal_store(words.w[i], reinterpret_cast<Words*>(at) + i);
}
template <class P>
__device__ __forceinline__ P got_past_caches(const P* at) {
  Sixteens<P> words;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(P) / 16); ++i) words.w[i] = __builtin_nontemporal_load(reinterpret_cast<const Words*>(at) + i);
  return __builtin_bit_cast(P, words);
}

// N elements at any multiple of their own size: global memory takes loads and stores of up to sixteen bytes there.
template <class T, int N>
struct Loose {
  T v[N];
};

// The first `count` of N elements, zeros behind them; a whole pack is one access.  Nothing looks at them here, so several packs that are got one after
// the other are on their way together (a conversion would wait for each).
template <int N, class T>
__device__ __forceinline__ Loose<T, N> got_loose(const T* at, int count) {
  Loose<T, N> p;
  if (count >= N) {
    p = *reinterpret_cast<const Loose<T, N>*>(at);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) p.v[j] = j < count ? at[j] : (T)0.0f;
  }
  return p;
}
template <int N, class T>
__device__ __forceinline__ void widen(float (&to)[N], const Loose<T, N>& p) {
#pragma unroll
  for (int j = 0; j < N; ++j) to[j] = (float)p.v[j];
}
// Whole packs past the caches.
template <int N, class T>
__device__ __forceinline__ Loose<T, N> got_loose_past_caches(const T* at) {
  static_assert(N * sizeof(T) % 16 == 0, "packs of whole sixteen bytes");
  using Words = uint32_t __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  struct All {
    uint32_t __attribute__((ext_vector_type(4))) w[N * sizeof(T) / 16];
  } all;
#pragma unroll
  for (int i = 0; i < (int)(N * sizeof(T) / 16); ++i) all.w[i] = __builtin_nontemporal_load(reinterpret_cast<const Words*>(at) + i);
  using To = Loose<T, N>;
  return __builtin_bit_cast(To, all);
}
template <int N, class T>
__device__ __forceinline__ void put_loose_past_caches(T* at, const float (&from)[N]) {
  using Words = uint32_t __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  Loose<T, N> p;
#pragma unroll
  for (int j = 0; j < N; ++j) p.v[j] = (T)from[j];
  struct All {
    uint32_t __attribute__((ext_vector_type(4))) w[N * sizeof(T) / 16];
  };
  const All all = __builtin_bit_cast(All, p);
#pragma unroll
  for (int i = 0; i < (int)(N * sizeof(T) / 16); ++i) __builtin_nontemporal_store(all.w[i], reinterpret_cast<Words*>(at) + i);
}
template <int N, class T>
__device__ __forceinline__ Loose<T, N> got_loose(const T* at, int count, bool past_caches) {
  if constexpr (N * sizeof(T) % 16 == 0)
    if (past_caches && count >= N) return got_loose_past_caches<N>(at);
  return got_loose<N>(at, count);
}
// The same as floats, for a pack that is needed at once; and stores.
template <int N, class T>
__device__ __forceinline__ void get_loose(float (&to)[N], const T* at, int count) {
  widen(to, got_loose<N>(at, count));
}
template <int N, class T>
__device__ __forceinline__ void put_loose(T* at, const float (&from)[N], int count) {
  if (count >= N) {
    Loose<T, N> p;
#pragma unroll
    for (int j = 0; j < N; ++j) p.v[j] = (T)from[j];
    *reinterpret_cast<Loose<T, N>*>(at) = p;
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < count) at[j] = (T)from[j];
  }
}

template <int N, class T>
__device__ __forceinline__ void put_loose(T* at, const float (&from)[N], int count, bool past_caches) {
  if constexpr (N * sizeof(T) % 16 == 0)
    if (past_caches && count >= N) return put_loose_past_caches(at, from);
  put_loose(at, from, count);
}

// Packs as they were loaded, sixteen-bit elements two to a register: what is widened before this is not kept in registers for behind it.
template <class P>
__device__ __forceinline__ void forget(P& pack) {
  static_assert(sizeof(P) % 4 == 0, "packs of whole words");
  struct All {
    uint32_t w[sizeof(P) / 4];
  } all = __builtin_bit_cast(All, pack);
#pragma unroll
  for (int i = 0; i < (int)(sizeof(P) / 4); ++i) asm volatile("" : "+v"(all.w[i]));
  pack = __builtin_bit_cast(P, all);
}

// Elements as the floats that they are: a product and sum whose result is stored as a half may else be rounded to that at once, not to a float first, where
// nothing comes between, and a result would depend on the path that it takes (an ulp of one half in 2^14).
template <int N>
__device__ __forceinline__ void as_floats(float (&v)[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j) asm("" : "+v"(v[j]));
}

// Calls fn with a value of the element type that `type` names.
template <class FN>
auto with_type(int type, FN fn) {
  if (type == CNN_F32) return fn(float{});
  if (type == CNN_BF16) return fn(__bf16{});
  return fn(_Float16{});
}

// Workgroups 0 .. n - 1, and perhaps some more, as a grid of two dimensions: one of them holds less than 2^32 threads, or the launch is refused; a workgroup
// has up to 1024.
inline dim3 grid_of(int64_t n) {
  const int64_t x = n < 1 << 21 ? n : 1 << 21;
  return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}
__device__ __forceinline__ int64_t workgroup() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

inline int launch_status() {
  if (hipGetLastError() != hipSuccess) return CNN_EHIP;
  return CNN_OK;
}

}  // namespace cnn
