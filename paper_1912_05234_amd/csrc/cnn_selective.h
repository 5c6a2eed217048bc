// Selective state space scan: N states to every channel d of a sequence, whose decays the data choose.
//
//   D_t = softplus(dt_t + dt_bias) (or dt_t + dt_bias),   h_t = exp(D_t A) h_{t-1} + D_t x_t B_t,   y_t = sum_n C_t h_t + skip x_t
//
// with A[d,n] a parameter and B_t, C_t [n] shared by the channels of a group.  Backward, with q the error that the future leaves in h_t,
//
//   g = q + C d_y,  d_C = sum_d h d_y,  d_B = sum_d g D x,  d_x = D sum_n g B + skip d_y,
//   q' = exp(D A) g,  d_D = x sum_n g B + sum_n A q' h_{t-1},  d_A = sum_t D q' h_{t-1}          (q' is the next q, one token back)
//
// Layout.  A wave takes 64 / S channels of one sequence; S neighbouring lanes share a channel and hold NL of its states each, in
// registers, so sums over states are mostly a lane's own.  The S lanes also share the work on what a channel has once a token: each
// loads, and takes the softplus of, one token of S.  B and C come through LDS, as floats.
//
// What bounds it: the vector unit, an exponential and four or five products for every state and token (the hardware's exponential takes
// as long as four products).  Where channels are too few to fill the chip the sequences are cut into segments: a first pass leaves each
// segment's own end state and the sum of its D, from which the decay of a whole segment is exp(A sum D), a second kernel joins them, and
// the real pass starts every segment from its true state.
//
// Backward a segment is walked twice: forwards, leaving every eighth state in LDS, and backwards, eight tokens at a time, whose
// states and decays are computed again into registers.  The first pass leaves the segment's error of its first state
// beside its end state: sum_t (product of the decays up to t) C_t d_y_t, a running product and no second exponential.
#pragma once

#include <type_traits>

#include "cnn_common.h"
#include "cnn_types.h"

namespace cnn {
namespace selective {

using f4 = float __attribute__((ext_vector_type(4)));

constexpr int U = 8;          // tokens whose inputs are on their way together
constexpr int LONGEST = 64;   // of a segment's tokens, backward: eight checkpoints in LDS

struct Tokens {
  const void* data;
  int64_t batch, token, group;
};

struct Args {
  Tokens x, dt, b, c, d_y;
  const float *a, *skip, *dt_bias;  // [D][N], [D], [D]; the last two nullable
  const int32_t* lengths;
  const float *first, *d_last;  // [B][D][N], nullable
  void *y, *d_x, *d_dt;         // [B][T][D]
  float* last;                  // the final state, or the error of the first; nullable
  float *ends, *errors, *sums;  // of the segments: [segments][B][D][N], the same, [segments][B][D]
  float *partial, *shared;      // backward: [segments][B][D][N + 2], [channel blocks][B][T][G][2][NP]
  int64_t T, length;            // of a segment
  int B, D, N, G, per, blocks, segments, softplus;  // per: channels of a group; blocks: waves that these take
};

__device__ __forceinline__ int64_t length_of(const Args& a, int64_t b) {
  if (!a.lengths) return a.T;
  const int64_t n = a.lengths[b];
  return n < 0 ? 0 : n > a.T ? a.T : n;
}

template <int CTRL>
__device__ __forceinline__ float lane_moved(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
constexpr int SWAP_1 = 0xB1, SWAP_2 = 0x4E, HALF_MIRROR = 0x141, MIRROR = 0x140, ROTATE_8 = 0x128;

// The sum over S neighbouring lanes, in all of them.
template <int S>
__device__ __forceinline__ float shared_sum(float v) {
  if constexpr (S > 1) v += lane_moved<SWAP_1>(v);
  if constexpr (S > 2) v += lane_moved<SWAP_2>(v);
  if constexpr (S > 4) v += lane_moved<HALF_MIRROR>(v);
  if constexpr (S > 8) v += lane_moved<MIRROR>(v);
  return v;
}

// Lane k's value of S neighbouring lanes, in all of them.
template <int S, int K>
__device__ __forceinline__ float from_lane(float v) {
  if constexpr (S == 1) return v;
  else if constexpr (S == 2) return lane_moved<K | K << 2 | (K + 2) << 4 | (K + 2) << 6>(v);
  else if constexpr (S == 4) return lane_moved<K | K << 2 | K << 4 | K << 6>(v);
  else return __shfl(v, (int)(threadIdx.x & ~(S - 1)) + K);
}

// softplus(z) = ln(1 + e^z).  ln(1 + e) for small e by Kahan's formula e ln(w) / (w - 1) with w = 1 + e rounded (Goldberg, "What every
// computer scientist should know about floating-point arithmetic", theorem 4).
__device__ __forceinline__ float softplus_of(float z) {
  const float e = __builtin_amdgcn_exp2f(z * -NEG_LOG2E), w = 1.0f + e;
  const float l = __builtin_amdgcn_logf(w) * 0.69314718055994530942f;
  const float r = w == 1.0f ? e : e * l * __builtin_amdgcn_rcpf(w - 1.0f);
  return z > 20.0f ? z : r;  // (z + e^-z: the same float)
}

// A wave's place: its channel and states, the tokens of its segment.
struct Place {
  int64_t b, t0, t1, end;  // tokens t0 .. t1 - 1, of which those from `end` on are past the sequence
  int segment, group, channel, state, s, block;
  bool mine;  // a channel of the group (else the lane has the last one's parameters, inputs and errors of zero, and stores nothing)
};

template <int NL, int S>
__device__ __forceinline__ Place place_of(const Args& a) {
  constexpr int CHANNELS = 64 / S;
  Place p;
  int64_t w = workgroup();
  p.block = (int)(w % a.blocks), w /= a.blocks;
  p.group = (int)(w % a.G), w /= a.G;
  p.b = w % a.B, p.segment = (int)(w / a.B);
  const int lane = threadIdx.x, in = p.block * CHANNELS + lane / S;
  p.mine = in < a.per;
  p.channel = p.group * a.per + (p.mine ? in : a.per - 1);
  p.s = lane % S, p.state = p.s * NL;
  p.t0 = p.segment * a.length;
  p.t1 = p.t0 + a.length < a.T ? p.t0 + a.length : a.T;
  const int64_t n = length_of(a, p.b);
  p.end = n < p.t0 ? p.t0 : n < p.t1 ? n : p.t1;
  return p;
}

template <int NL>
__device__ __forceinline__ void get_states(float (&h)[NL], const float* from, const Place& p, const Args& a) {
  const float* at = from + (int64_t)p.channel * a.N + p.state;
#pragma unroll
  for (int i = 0; i < NL; i += 4) get_loose<4>(*reinterpret_cast<float(*)[4]>(h + i), at + i, a.N - p.state - i);
}
template <int NL>
__device__ __forceinline__ void put_states(float* to, const float (&h)[NL], const Place& p, const Args& a) {
  float* at = to + (int64_t)p.channel * a.N + p.state;
  if (p.mine)
#pragma unroll
    for (int i = 0; i < NL; i += 4) put_loose<4>(at + i, *reinterpret_cast<const float(*)[4]>(h + i), a.N - p.state - i);
}

// What U tokens have once a channel, each lane its tokens k S + s; zeros past the sequence.
template <class T, int S>
struct Once {
  static constexpr int EACH = U > S ? U / S : 1;
  float v[EACH];
  __device__ __forceinline__ void get(const Tokens& from, const Place& p, int64_t t) {
    const T* at = static_cast<const T*>(from.data) + p.b * from.batch + p.channel;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int64_t k = t + i * S + p.s;
      v[i] = p.mine && (S <= U || p.s < U) && k >= p.t0 && k < p.end ? (float)at[k * from.token] : 0.0f;
    }
  }
  template <int K>
  __device__ __forceinline__ float of() const {  // token K's
    return from_lane<S, K % S>(v[K / S]);
  }
};

// Rows of B and C of U tokens on their way through LDS, as floats; zeros past the sequence and past N.
template <class T, int NP>
struct Row {
  static constexpr int EACH = U * NP >= 64 ? U * NP / 64 : 1;
  T v[EACH];
  __device__ __forceinline__ void get(const Tokens& from, const Place& p, const Args& a, int64_t t) {
    const T* at = static_cast<const T*>(from.data) + p.b * from.batch + p.group * from.group;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int e = i * 64 + (int)threadIdx.x, k = e / NP, n = e % NP;
      const int64_t token = t + k;
      v[i] = (T)0.0f;
      if (k < U && n < a.N && token >= p.t0 && token < p.end) v[i] = at[token * from.token + n];
    }
  }
  __device__ __forceinline__ void put(float* to) const {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int e = i * 64 + (int)threadIdx.x;
      if (e < U * NP) to[e] = (float)v[i];
    }
  }
};

template <int NL>
__device__ __forceinline__ void get_row(float (&to)[NL], const float* from) {  // from LDS, 16 bytes at a time
#pragma unroll
  for (int i = 0; i < NL; i += 4) {
    const f4 q = *reinterpret_cast<const f4*>(from + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) to[i + j] = q[j];
  }
}

// Calls fn with the constants 0 .. COUNT - 1.
template <int COUNT, class FN>
__device__ __forceinline__ void each(FN fn) {
  if constexpr (COUNT > 0) {
    each<COUNT - 1>(fn);
    fn(std::integral_constant<int, COUNT - 1>{});
  }
}

template <int NL>
__device__ __forceinline__ void get_decays(float (&a2)[NL], const Args& a, const Place& p) {
  get_states(a2, a.a, p, a);
#pragma unroll
  for (int i = 0; i < NL; ++i) a2[i] *= -NEG_LOG2E;
}

// D_t and D_t x_t of a lane's own tokens.
template <class T, int S>
__device__ __forceinline__ void get_steps(const Args& a, const Place& p, int64_t t, float bias, const Once<T, S>& x, const Once<T, S>& dt, Once<T, S>& delta,
                                          Once<T, S>& u) {
#pragma unroll
  for (int i = 0; i < Once<T, S>::EACH; ++i) {
    const float z = dt.v[i] + bias;
    delta.v[i] = t + i * S + p.s < p.end ? (a.softplus ? softplus_of(z) : z) : 0.0f;  // past the sequence the state stays
    u.v[i] = delta.v[i] * x.v[i];
  }
}

// ---- forward -------------------------------------------------------------------------------------------------------------
// ENDS: a segment's own end state (from zero) and its sum of D; with ERRORS its first state's error too.  Else y, and the final state where there is
// one segment.
template <class T, int NL, int S, bool ENDS, bool ERRORS>
__global__ __launch_bounds__(64) void selective_tokens_kernel(Args a) {
  constexpr int NP = NL * S;
  __shared__ __align__(16) float rows[2][2][U * NP];
  const Place p = place_of<NL, S>(a);
  float a2[NL], h[NL], q[ERRORS ? NL : 1], run[ERRORS ? NL : 1];
  get_decays(a2, a, p);
  const int64_t states = (int64_t)a.D * a.N;
  const float bias = a.dt_bias ? a.dt_bias[p.channel] : 0.0f, skip = a.skip ? a.skip[p.channel] : 0.0f;
  const float* from = ENDS ? nullptr : a.segments > 1 ? a.ends + ((int64_t)p.segment * a.B + p.b) * states : a.first ? a.first + p.b * states : nullptr;
#pragma unroll
  for (int i = 0; i < NL; ++i) h[i] = 0.0f;
  if (from) get_states(h, from, p, a);
  if constexpr (ERRORS)
#pragma unroll
    for (int i = 0; i < NL; ++i) q[i] = 0.0f, run[i] = 1.0f;
  float sum = 0.0f;
  constexpr bool NEEDS_C = !ENDS || ERRORS;
  Once<T, S> x, dt, d_y, next_x, next_dt, next_d;
  Row<T, NP> b, c;
  next_x.get(a.x, p, p.t0), next_dt.get(a.dt, p, p.t0);
  if constexpr (ERRORS) next_d.get(a.d_y, p, p.t0);
  b.get(a.b, p, a, p.t0);
  if constexpr (NEEDS_C) c.get(a.c, p, a, p.t0);
  const int64_t stop = ENDS ? p.end : p.t1;
  T* y = static_cast<T*>(a.y) + p.b * a.T * a.D + p.channel;
  int turn = 0;
  for (int64_t t = p.t0; t < stop; t += U, turn ^= 1) {
    x = next_x, dt = next_dt;
    if constexpr (ERRORS) d_y = next_d;
    b.put(rows[turn][0]);
    if constexpr (NEEDS_C) c.put(rows[turn][1]);
    __syncthreads();
    next_x.get(a.x, p, t + U), next_dt.get(a.dt, p, t + U);
    if constexpr (ERRORS) next_d.get(a.d_y, p, t + U);
    b.get(a.b, p, a, t + U);
    if constexpr (NEEDS_C) c.get(a.c, p, a, t + U);
    Once<T, S> delta, u, out;
    get_steps(a, p, t, bias, x, dt, delta, u);
    each<U>([&](auto k) {
      constexpr int K = decltype(k)::value;
      const float d = delta.template of<K>(), input = u.template of<K>();
      float B[NL], C[NL], y_t = 0.0f, error = 0.0f;
      get_row(B, rows[turn][0] + K * NP + p.state);
      if constexpr (NEEDS_C) get_row(C, rows[turn][1] + K * NP + p.state);
      if constexpr (ERRORS) error = d_y.template of<K>();
      if constexpr (ENDS) sum += d;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const float decay = __builtin_amdgcn_exp2f(d * a2[i]);
        h[i] = decay * h[i] + input * B[i];
        if constexpr (!ENDS) y_t += C[i] * h[i];
        if constexpr (ERRORS) {
          run[i] *= decay;
          q[i] += run[i] * (C[i] * error);
        }
      }
      if constexpr (!ENDS) {
        y_t = shared_sum<S>(y_t);
        if (p.s == K % S) out.v[K / S] = y_t;
      }
    });
    if constexpr (!ENDS)
#pragma unroll
      for (int i = 0; i < Once<T, S>::EACH; ++i) {
        const int64_t k = t + i * S + p.s;
        if (p.mine && (S <= U || p.s < U) && k < p.t1) y[k * a.D] = (T)(k < p.end ? out.v[i] + skip * x.v[i] : 0.0f);
      }
  }
  if constexpr (ENDS) {
    const int64_t at = (int64_t)p.segment * a.B + p.b;
    put_states(a.ends + at * states, h, p, a);
    if constexpr (ERRORS) put_states(a.errors + at * states, q, p, a);
    if (p.mine && p.s == 0) a.sums[at * a.D + p.channel] = sum;
  } else if (a.last && a.segments == 1) {
    put_states(a.last + p.b * states, h, p, a);
  }
}

// ---- backward --------------------------------------------------------------------------------------------------------------
// One level of a sum over lanes whose values are divided at the same time: of COUNT values the lanes with BIT unset keep the sums of the first half,
// the others of the second.
template <int BIT, int COUNT>
__device__ __forceinline__ void halve(float (&v)[16]) {
  constexpr int HALF = COUNT / 2;
#pragma unroll
  for (int i = 0; i < HALF; ++i) {
    const float x = v[i], y = v[i + HALF];
    if constexpr (BIT == 32) {
      const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
      v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    } else if constexpr (BIT == 16) {
      const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
      v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    } else {
      const bool upper = threadIdx.x & BIT;
      const float keep = upper ? y : x, give = upper ? x : y;
      float got;
      if constexpr (BIT == 8) got = lane_moved<ROTATE_8>(give);
      else if constexpr (BIT == 4) got = __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(give), 0x101f));  // lane ^ 4
      else if constexpr (BIT == 2) got = lane_moved<SWAP_2>(give);
      else got = lane_moved<SWAP_1>(give);
      v[i] = keep + got;
    }
  }
}

template <int BIT>
__device__ __forceinline__ float add_across(float v) {
  if constexpr (BIT == 8) return v + lane_moved<ROTATE_8>(v);
  else if constexpr (BIT == 4) return v + __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(v), 0x101f));
  else if constexpr (BIT == 2) return v + lane_moved<SWAP_2>(v);
  else return v + lane_moved<SWAP_1>(v);
}

// Sums of COUNT values over the channels of a wave (lane bits from S on): v[0 .. left - 1] are those of value first + i, in lanes
// of which those with `writes` have different ones.
template <int S, int COUNT>
struct ChannelSums {
  static constexpr int BITS = S == 1 ? 6 : S == 2 ? 5 : S == 4 ? 4 : S == 8 ? 3 : 2;
  static constexpr int HALVINGS = COUNT == 16 ? (BITS < 4 ? BITS : 4) : (BITS < 3 ? BITS : 3);
  static constexpr int LEFT = COUNT >> HALVINGS;
  static __device__ __forceinline__ void sum(float (&v)[16]) {
    halve<32, COUNT>(v);
    halve<16, COUNT / 2>(v);
    if constexpr (HALVINGS > 2) halve<8, COUNT / 4>(v);
    if constexpr (HALVINGS > 3) halve<4, COUNT / 8>(v);
    if constexpr (HALVINGS == 3 && BITS > 3) v[0] = add_across<4>(v[0]);
    if constexpr (BITS > 4) v[0] = add_across<2>(v[0]);
    if constexpr (BITS > 5) v[0] = add_across<1>(v[0]);
  }
  static __device__ __forceinline__ int first() {
    const int lane = threadIdx.x;
    int at = 0;
    if (lane & 32) at += COUNT / 2;
    if (lane & 16) at += COUNT / 4;
    if (HALVINGS > 2 && lane & 8) at += COUNT / 8;
    if (HALVINGS > 3 && lane & 4) at += COUNT / 16;
    return at;
  }
  static __device__ __forceinline__ bool writes() {  // one of the lanes that have the same
    constexpr int SAME = (1 << (6 - HALVINGS)) - 1;
    return (threadIdx.x & SAME & ~(S - 1)) == 0;
  }
};

template <class T, int NL, int S>
__global__ __launch_bounds__(64) void selective_gradient_kernel(Args a) {
  constexpr int NP = NL * S, EACH = Once<T, S>::EACH;
  using Sums = ChannelSums<S, 2 * NL>;
  __shared__ __align__(16) float rows[2][2][U * NP];
  __shared__ __align__(16) f4 kept[LONGEST / U][NL / 4][64];
  const Place p = place_of<NL, S>(a);
  float a2[NL], h[NL], q[NL], d_a[NL], d_skip = 0.0f, d_bias = 0.0f;
  get_decays(a2, a, p);
  const int64_t states = (int64_t)a.D * a.N, at = (int64_t)p.segment * a.B + p.b;
  const float bias = a.dt_bias ? a.dt_bias[p.channel] : 0.0f, skip = a.skip ? a.skip[p.channel] : 0.0f;
  const float* from = a.segments > 1 ? a.ends + at * states : a.first ? a.first + p.b * states : nullptr;
  const float* error_from = a.segments > 1 ? a.errors + at * states : a.d_last ? a.d_last + p.b * states : nullptr;
#pragma unroll
  for (int i = 0; i < NL; ++i) h[i] = q[i] = d_a[i] = 0.0f;
  if (from) get_states(h, from, p, a);
  if (error_from) get_states(q, error_from, p, a);
  const int chunks = (int)((p.end - p.t0 + U - 1) / U);
  Once<T, S> x, dt, d_y, next_x, next_dt, next_d, delta, u;
  Row<T, NP> b, c;
  int turn = 0;
  // forwards: the state in front of every chunk
  next_x.get(a.x, p, p.t0), next_dt.get(a.dt, p, p.t0), b.get(a.b, p, a, p.t0);
  for (int j = 0; j < chunks; ++j, turn ^= 1) {
    const int64_t t = p.t0 + j * U;
#pragma unroll
    for (int i = 0; i < NL; i += 4) kept[j][i / 4][threadIdx.x] = f4{h[i], h[i + 1], h[i + 2], h[i + 3]};
    if (j == chunks - 1) break;
    x = next_x, dt = next_dt;
    b.put(rows[turn][0]);
    __syncthreads();
    next_x.get(a.x, p, t + U), next_dt.get(a.dt, p, t + U), b.get(a.b, p, a, t + U);
    get_steps(a, p, t, bias, x, dt, delta, u);
    each<U>([&](auto k) {
      constexpr int K = decltype(k)::value;
      const float d = delta.template of<K>(), input = u.template of<K>();
      float B[NL];
      get_row(B, rows[turn][0] + K * NP + p.state);
#pragma unroll
      for (int i = 0; i < NL; ++i) h[i] = __builtin_amdgcn_exp2f(d * a2[i]) * h[i] + input * B[i];
    });
  }
  __syncthreads();
  // backwards; next_x, next_dt and b hold the last chunk
  const int64_t last = p.t0 + (int64_t)(chunks - 1) * U;
  next_d.get(a.d_y, p, last), c.get(a.c, p, a, last);
  T *d_x = static_cast<T*>(a.d_x) + p.b * a.T * a.D + p.channel, *d_dt = static_cast<T*>(a.d_dt) + p.b * a.T * a.D + p.channel;
  const int value = Sums::first(), row = value < NL ? 0 : 1, state = p.state + value - row * NL;
  float* shared = a.shared + ((((int64_t)p.block * a.B + p.b) * a.T) * a.G + p.group) * 2 * NP + row * NP + state;
  for (int j = chunks - 1; j >= 0; --j, turn ^= 1) {
    const int64_t t = p.t0 + j * U;
    x = next_x, dt = next_dt, d_y = next_d;
    b.put(rows[turn][0]), c.put(rows[turn][1]);
    __syncthreads();
    next_x.get(a.x, p, t - U), next_dt.get(a.dt, p, t - U), next_d.get(a.d_y, p, t - U);
    b.get(a.b, p, a, t - U), c.get(a.c, p, a, t - U);
    get_steps(a, p, t, bias, x, dt, delta, u);
    float before[U + 1][NL], decay[U][NL];  // before[k]: the state in front of token k
#pragma unroll
    for (int i = 0; i < NL; i += 4) {
      const f4 v = kept[j][i / 4][threadIdx.x];
#pragma unroll
      for (int l = 0; l < 4; ++l) before[0][i + l] = v[l];
    }
    each<U>([&](auto k) {
      constexpr int K = decltype(k)::value;
      const float d = delta.template of<K>(), input = u.template of<K>();
      float B[NL];
      get_row(B, rows[turn][0] + K * NP + p.state);
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        decay[K][i] = __builtin_amdgcn_exp2f(d * a2[i]);
        before[K + 1][i] = decay[K][i] * before[K][i] + input * B[i];
      }
    });
    Once<T, S> sum_b, sum_a;  // of g B; of A q' h
    each<U>([&](auto k) {
      constexpr int K = U - 1 - decltype(k)::value;
      const float d = delta.template of<K>(), input = u.template of<K>(), error = d_y.template of<K>();
      float B[NL], C[NL], v[16], by_b = 0.0f, by_a = 0.0f;
      get_row(B, rows[turn][0] + K * NP + p.state);
      get_row(C, rows[turn][1] + K * NP + p.state);
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const float g = q[i] + C[i] * error;
        v[i] = g * input;
        v[NL + i] = before[K + 1][i] * error;
        by_b += g * B[i];
        q[i] = decay[K][i] * g;
        const float along = q[i] * before[K][i];
        d_a[i] += d * along;
        by_a += a2[i] * along;
      }
      by_b = shared_sum<S>(by_b), by_a = shared_sum<S>(by_a);
      if (p.s == K % S) sum_b.v[K / S] = by_b, sum_a.v[K / S] = by_a;
      Sums::sum(v);
      if (Sums::writes() && t + K < p.end)
#pragma unroll
        for (int i = 0; i < Sums::LEFT; ++i) shared[(t + K) * a.G * 2 * NP + i] = v[i];
    });
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int64_t k = t + i * S + p.s;
      if ((S > U && p.s >= U) || k >= p.end) continue;
      const float z = dt.v[i] + bias;
      const float d_delta = x.v[i] * sum_b.v[i] + sum_a.v[i] * 0.69314718055994530942f;
      const float d_z = a.softplus ? d_delta * logistic(z) : d_delta;
      d_skip += d_y.v[i] * x.v[i], d_bias += d_z;
      if (!p.mine) continue;
      d_x[k * a.D] = (T)(delta.v[i] * sum_b.v[i] + skip * d_y.v[i]);
      d_dt[k * a.D] = (T)d_z;
    }
  }
  if (p.mine && p.s == 0) {
    for (int64_t k = p.end; k < p.t1; ++k) d_x[k * a.D] = (T)0.0f, d_dt[k * a.D] = (T)0.0f;
  }
  if (a.last && p.segment == 0) put_states(a.last + p.b * states, q, p, a);
  d_skip = shared_sum<S>(d_skip), d_bias = shared_sum<S>(d_bias);
  float* partial = a.partial + (at * a.D + p.channel) * (a.N + 2);
  if (p.mine) {
#pragma unroll
    for (int i = 0; i < NL; ++i)
      if (p.state + i < a.N) partial[p.state + i] = d_a[i];
    if (p.s == 0) partial[a.N] = d_skip, partial[a.N + 1] = d_bias;
  }
}

// ---- launches, one source to an element type ---------------------------------------------------------------------------------
enum Pass { TOKENS, ENDS, ENDS_AND_ERRORS, GRADIENT };

struct Form {  // states to a lane, lanes to a channel
  int states, lanes;
};

void launch_f32(const Args& a, Pass pass, Form f, dim3 grid, hipStream_t st);
void launch_bf16(const Args& a, Pass pass, Form f, dim3 grid, hipStream_t st);
void launch_f16(const Args& a, Pass pass, Form f, dim3 grid, hipStream_t st);

template <class T, int NL, int S>
void launch_form(const Args& a, Pass pass, dim3 grid, hipStream_t st) {
  // Forward any division of the states; backward eight to a lane (four where there are no more).
  if constexpr (NL == 8 || (NL == 4 && S == 1)) {
    if (pass == ENDS_AND_ERRORS) return selective_tokens_kernel<T, NL, S, true, true><<<grid, 64, 0, st>>>(a);
    if (pass == GRADIENT) return selective_gradient_kernel<T, NL, S><<<grid, 64, 0, st>>>(a);
  }
  if (pass == ENDS) selective_tokens_kernel<T, NL, S, true, false><<<grid, 64, 0, st>>>(a);
  else selective_tokens_kernel<T, NL, S, false, false><<<grid, 64, 0, st>>>(a);
}

template <class T>
void launch_type(const Args& a, Pass pass, Form f, dim3 grid, hipStream_t st) {
  const auto at = [&](auto nl, auto s) {
    if (f.states == decltype(nl)::value && f.lanes == decltype(s)::value) launch_form<T, decltype(nl)::value, decltype(s)::value>(a, pass, grid, st);
  };
  using std::integral_constant;
  const integral_constant<int, 1> one;
  const integral_constant<int, 2> two;
  const integral_constant<int, 4> four;
  const integral_constant<int, 8> eight;
  const integral_constant<int, 16> sixteen;
  at(four, one), at(four, two), at(four, four);
  at(eight, one), at(eight, two), at(eight, four), at(eight, eight), at(eight, sixteen);
  at(sixteen, one), at(sixteen, two), at(sixteen, four), at(sixteen, eight);
}

}  // namespace selective
}  // namespace cnn
