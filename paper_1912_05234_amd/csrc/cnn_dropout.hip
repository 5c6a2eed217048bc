// Dropout from a counter-based generator.
//
//   y[e] = u(e) >= round(p 2^32) ? x[e] / (1 - p) : 0     (+ residual[e])
//
// u(e) is a 32-bit number that depends on the seed, the offset and e alone, so the backward pass draws the same mask again and
// none is stored.  The generator is Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// 2011): ten rounds of two 32 x 32 -> 64 bit products turn a counter of 128 bits into four words.
//
// Eight elements share a call: its four words are the sixteen HIGH bits of eight numbers.  The sixteen low bits, from a second
// call with the top bit of the counter's second word set, decide only where the high bits equal those of the limit, one element
// in 65536, and only there the call is made.  So p has its 32 bits at the price of sixteen.
//
// Memory bounds it: 67 M bfloat16 elements with a residual (402 MB read and written) take 69 us, 5.8 TB/s; a copy of 1 GiB reaches 5.15.  A thread's
// two blocks of eight elements are loaded before the generator runs.
#include <type_traits>

#include "cnn_common.h"
#include "cnn_types.h"

namespace cnn {
namespace {

constexpr int DROP_THREADS = 256;
constexpr int DROP_BLOCKS = 2;  // of eight elements, per thread

struct DropArgs {
  const void *x, *residual;
  void* y;
  size_t n;
  uint32_t limit_high, limit_low;  // of the number below which an element is dropped
  float scale;
  uint64_t seed, offset;
  const int64_t* step;
};

__device__ __forceinline__ uint4 philox(uint64_t block, uint32_t call, uint64_t offset, uint64_t seed) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32) | call << 31, c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0, c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c1 = (uint32_t)b, c3 = (uint32_t)a;
    k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
  }
  return uint4{c0, c1, c2, c3};
}

__device__ __forceinline__ uint32_t half_of(const uint4& w, int j) {
  const uint32_t word = j < 2 ? w.x : j < 4 ? w.y : j < 6 ? w.z : w.w;
  return j & 1 ? word >> 16 : word & 0xffffu;
}

// The decisions on the eight elements of a block, one bit each.
__device__ __forceinline__ uint32_t kept(const DropArgs& a, uint64_t block, uint64_t offset) {
  const uint4 high = philox(block, 0, offset, a.seed);
  uint32_t keep = 0, open = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t h = half_of(high, j);
    keep |= (uint32_t)(h >= a.limit_high) << j;
    open |= (uint32_t)(h == a.limit_high) << j;
  }
  if (open && a.limit_low) {
    const uint4 low = philox(block, 1, offset, a.seed);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (open >> j & 1 && half_of(low, j) < a.limit_low) keep &= ~(1u << j);
  }
  return keep;
}

template <class T, bool RESIDUAL, bool PAST_CACHES>
__global__ __launch_bounds__(DROP_THREADS) void dropout_kernel(DropArgs a) {
  const T *x = static_cast<const T*>(a.x), *res = static_cast<const T*>(a.residual);
  T* y = static_cast<T*>(a.y);
  const uint64_t offset = a.offset + (a.step ? (uint64_t)*a.step : 0);
  const size_t first = (size_t)workgroup() * (DROP_THREADS * DROP_BLOCKS) + threadIdx.x;
  Pack<T, 8> in[DROP_BLOCKS], add[DROP_BLOCKS];
#pragma unroll
  for (int i = 0; i < DROP_BLOCKS; ++i) {
    const size_t e = (first + (size_t)i * DROP_THREADS) * 8;
    if (e + 8 <= a.n) {
      const auto *from = reinterpret_cast<const Pack<T, 8>*>(x + e), *more = reinterpret_cast<const Pack<T, 8>*>(res + e);
      if constexpr (PAST_CACHES) in[i] = got_past_caches(from);
      else in[i] = *from;
      if constexpr (RESIDUAL && PAST_CACHES) add[i] = got_past_caches(more);
      else if constexpr (RESIDUAL) add[i] = *more;
    }
  }
#pragma unroll
  for (int i = 0; i < DROP_BLOCKS; ++i) {
    const size_t block = first + (size_t)i * DROP_THREADS, e = block * 8;
    if (e >= a.n) return;
    const uint32_t keep = kept(a, block, offset);
    if (e + 8 <= a.n) {
      Pack<T, 8> out;
#pragma unroll
      for (int j = 0; j < 8; ++j) {  // a dropped element is zero whatever it holds
        const float v = keep >> j & 1 ? (float)in[i].v[j] * a.scale : 0.0f;
        out.v[j] = (T)(RESIDUAL ? v + (float)add[i].v[j] : v);
      }
      if constexpr (PAST_CACHES) put_past_caches(reinterpret_cast<Pack<T, 8>*>(y + e), out);
      else *reinterpret_cast<Pack<T, 8>*>(y + e) = out;
    } else {
      for (int j = 0; e + j < a.n; ++j) {
        const float v = keep >> j & 1 ? (float)x[e + j] * a.scale : 0.0f;
        y[e + j] = (T)(RESIDUAL ? v + (float)res[e + j] : v);
      }
    }
  }
}

int dropout(const void* x, const void* residual, void* y, size_t n, int type, double p, uint64_t seed, uint64_t offset,
            const int64_t* step, void* hip_stream) {
  if (!x || !y || n < 1 || n > (size_t)1 << 40 || !type_known(type) || !(p >= 0.0 && p <= 1.0)) return CNN_EINVAL;
  if (!aligned16(x) || !aligned16(y) || (residual && !aligned16(residual)) || (reinterpret_cast<uintptr_t>(step) & 7)) return CNN_EINVAL;
  const uint64_t limit = (uint64_t)__builtin_floor(p * 4294967296.0 + 0.5);
  const DropArgs a{x, residual, y, n, (uint32_t)(limit >> 16), (uint32_t)limit & 0xffffu, p < 1.0 ? (float)(1.0 / (1.0 - p)) : 0.0f,
                   seed, offset, step};
  const size_t groups = (n + DROP_THREADS * DROP_BLOCKS * 8 - 1) / (DROP_THREADS * DROP_BLOCKS * 8);
  const size_t bytes = n * type_bytes(type) * (residual ? 3 : 2);
  // More than the last cache holds goes past it: 400 MB of bfloat16 75 -> 68 us, 320 MB 60 -> 54, 192 MB 36 -> 37.  Not floats, whose lanes
  // take 32 bytes in two halves: 400 MB 70 -> 74 us.
  const bool past_caches = bytes >= (size_t)256 << 20 && type != CNN_F32;
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    const auto launch = [&](auto add, auto past) {
      dropout_kernel<T, decltype(add)::value, decltype(past)::value><<<grid_of((int64_t)groups), DROP_THREADS, 0, (hipStream_t)hip_stream>>>(a);
      return launch_status();
    };
    const std::true_type yes;
    const std::false_type no;
    if constexpr (sizeof(T) == 2)
      if (past_caches) return residual ? launch(yes, yes) : launch(no, yes);
    return residual ? launch(yes, no) : launch(no, no);
  });
}

}  // namespace
}  // namespace cnn

extern "C" {

int cnn_dropout_fwd(const void* x, const void* residual, void* y, size_t n, int type, double p, uint64_t seed, uint64_t offset,
                    const int64_t* step, void* hip_stream) {
  return cnn::dropout(x, residual, y, n, type, p, seed, offset, step, hip_stream);
}

int cnn_dropout_bwd(const void* d_y, void* d_x, size_t n, int type, double p, uint64_t seed, uint64_t offset, const int64_t* step,
                    void* hip_stream) {
  return cnn::dropout(d_y, nullptr, d_x, n, type, p, seed, offset, step, hip_stream);
}

}  // extern "C"
