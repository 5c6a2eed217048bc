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

// Calls fn with a value of the element type that `type` names.
template <class FN>
auto with_type(int type, FN fn) {
  if (type == CNN_F32) return fn(float{});
  if (type == CNN_BF16) return fn(__bf16{});
  return fn(_Float16{});
}

// Workgroups 0 .. n - 1, and perhaps some more, as a grid of two dimensions: one of them holds less than 2^32 threads.
inline dim3 grid_of(int64_t n) {
  const int64_t x = n < 1 << 22 ? n : 1 << 22;
  return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}
__device__ __forceinline__ int64_t workgroup() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

inline int launch_status() {
  if (hipGetLastError() != hipSuccess) return CNN_EHIP;
  return CNN_OK;
}

}  // namespace cnn
