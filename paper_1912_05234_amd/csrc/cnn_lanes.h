// Sums and other reductions over neighbouring lanes of a wave, without LDS: data-parallel moves within sixteen lanes, swaps of rows beyond.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cnn {

constexpr int SWAP_1 = 0xB1, SWAP_2 = 0x4E, HALF_MIRROR = 0x141, MIRROR = 0x140, ROTATE_8 = 0x128;

template <int CTRL>
__device__ __forceinline__ uint32_t lane_moved(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ float lane_moved(float v) {
  return __uint_as_float(lane_moved<CTRL>(__float_as_uint(v)));
}
template <int CTRL>
__device__ __forceinline__ uint64_t lane_moved(uint64_t v) {
  return (uint64_t)lane_moved<CTRL>((uint32_t)(v >> 32)) << 32 | lane_moved<CTRL>((uint32_t)v);
}

// fn(own half's, other half's) of 32 (ROWS = 1: of 16) lanes each, the same in both: op(lower, upper).
template <bool HALVES, class T, class OP>
__device__ __forceinline__ T across_rows(T v, OP op) {
  static_assert(sizeof(T) == 4 || sizeof(T) == 8, "one or two words");
  uint32_t lower[sizeof(T) / 4], upper[sizeof(T) / 4], words[sizeof(T) / 4];
  __builtin_memcpy(words, &v, sizeof(T));
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 4); ++i) {
    const auto r = HALVES ? __builtin_amdgcn_permlane32_swap(words[i], words[i], false, false) : __builtin_amdgcn_permlane16_swap(words[i], words[i], false, false);
    lower[i] = r[0], upper[i] = r[1];
  }
  T a, b;
  __builtin_memcpy(&a, lower, sizeof(T));
  __builtin_memcpy(&b, upper, sizeof(T));
  return op(a, b);
}

// op over LANES neighbouring lanes, for a commutative op; every lane has the same result, bit for bit.
template <int LANES, class T, class OP>
__device__ __forceinline__ T over_lanes(T v, OP op) {
  if constexpr (LANES > 1) v = op(v, lane_moved<SWAP_1>(v));
  if constexpr (LANES > 2) v = op(v, lane_moved<SWAP_2>(v));
  if constexpr (LANES > 4) v = op(v, lane_moved<HALF_MIRROR>(v));
  if constexpr (LANES > 8) v = op(v, lane_moved<MIRROR>(v));
  if constexpr (LANES > 16) v = across_rows<false>(v, op);
  if constexpr (LANES > 32) v = across_rows<true>(v, op);
  return v;
}
// (A product that is summed is rounded first: fused into the addition, each lane would have its own unrounded and the others' rounded.)
template <int LANES>
__device__ __forceinline__ float sum_over(float v) {
  return over_lanes<LANES>(v, [](float a, float b) {
#pragma clang fp contract(off)
    return a + b;
  });
}
template <int LANES>
__device__ __forceinline__ float max_over(float v) {
  return over_lanes<LANES>(v, [](float a, float b) { return fmaxf(a, b); });
}

}  // namespace cnn
