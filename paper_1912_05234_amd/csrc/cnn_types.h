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

// Calls fn with a value of the element type that `type` names.
template <class FN>
auto with_type(int type, FN fn) {
  if (type == CNN_F32) return fn(float{});
  if (type == CNN_BF16) return fn(__bf16{});
  return fn(_Float16{});
}

inline int launch_status() {
  if (hipGetLastError() != hipSuccess) return CNN_EHIP;
  return CNN_OK;
}

}  // namespace cnn
