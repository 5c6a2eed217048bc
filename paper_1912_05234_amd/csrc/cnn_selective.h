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
//
// Measured: a prompt of 2 x 4096 tokens of 2048 x 16 states, bfloat16, 142 us (71 first pass, 86 second, 9 between them, of which the vector unit
// issues three quarters of the time; without segments, 32 x 256 tokens, 77); the gradients of 100 x 784 tokens of 128 x 16 states, floats, 237 (60 + 9 + 160
// + 7 + 8; memory alone would take 43), of 2 x 2047 x 1024 x 16, fp16, 111.
#pragma once

#include <type_traits>

#include "cnn_common.h"
#include "cnn_lanes.h"
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
  void *d_b, *d_c;              // [B][T][G][N]
  float* last;                  // the final state, or the error of the first; nullable
  float *ends, *errors, *sums;  // of the segments: [segments][B][D][N], the same, [segments][B][D]
  float *partial, *shared;      // backward: [segments][B][D][N + 2]; [workgroups][B][T][G][2][NP] where these are several
  int T, length;                // of a segment
  int B, D, N, G, per, blocks, workgroups, segments, softplus;  // per: channels of a group; blocks: waves that these take; workgroups: backward
};

__device__ __forceinline__ int length_of(const Args& a, int b) {
  if (!a.lengths) return a.T;
  const int n = a.lengths[b];
  return n < 0 ? 0 : n > a.T ? a.T : n;
}

// Lane k's value of S neighbouring lanes, in all of them.
template <int S, int K>
__device__ __forceinline__ float from_lane(float v) {
  if constexpr (S == 1) return v;
  else if constexpr (S == 2) return lane_moved<K | K << 2 | (K + 2) << 4 | (K + 2) << 6>(v);
  else if constexpr (S == 4) return lane_moved<K | K << 2 | K << 4 | K << 6>(v);
  else return __shfl(v, (int)(threadIdx.x & ~(S - 1)) + K);
}

// softplus(z) = ln(1 + e^z) = max(z, 0) + ln(1 + e) with e = exp(-|z|), and its slope 1 / (1 + e^-z).  With w = 1 + e rounded, ln(1 + e) = ln w + (1 + e - w) / w up to
// the square of the last term; what the rounding left out, 1 + e - w, is exact in two subtractions and at most 2^-24, so that its division by
// w (1 to 2, and 1 where e is small) is left out.
__device__ __forceinline__ float softplus_of(float z, float& slope) {
  const float e = __builtin_amdgcn_exp2f(__builtin_fabsf(z) * NEG_LOG2E), w = 1.0f + e, rest = e - (w - 1.0f);
  slope = (z < 0.0f ? e : 1.0f) * __builtin_amdgcn_rcpf(w);
  return fmaxf(z, 0.0f) + __builtin_fmaf(__builtin_amdgcn_logf(w), 0.69314718055994530942f, rest);
}
__device__ __forceinline__ float softplus_of(float z) {
  float slope;
  return softplus_of(z, slope);
}

// A lane's place: its channel and states, the tokens of its wave's segment.
struct Place {
  int b, t0, t1, end;  // tokens t0 .. t1 - 1, of which those from `end` on are past the sequence
  int segment, group, channel, state, s, block;
  bool mine;  // a channel of the group (else the lane has the last one's parameters, inputs and errors of zero, and stores nothing)
};

template <int NL, int S, int WAVES>
__device__ __forceinline__ Place place_of(const Args& a, int blocks) {
  constexpr int CHANNELS = WAVES * 64 / S;
  Place p;
  int64_t w = workgroup();
  p.block = (int)(w % blocks), w /= blocks;
  p.group = (int)(w % a.G), w /= a.G;
  p.b = (int)(w % a.B), p.segment = (int)(w / a.B);
  const int lane = threadIdx.x, in = p.block * CHANNELS + lane / S;  // (of all waves)
  p.mine = in < a.per;
  p.channel = p.group * a.per + (p.mine ? in : a.per - 1);
  p.s = lane % S, p.state = p.s * NL;
  p.t0 = p.segment * a.length;
  p.t1 = a.T - p.t0 < a.length ? a.T : p.t0 + a.length;
  const int n = length_of(a, p.b);
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

// What U tokens have once a channel, each lane its tokens k S + s.
template <int S>
struct Own {
  static constexpr int EACH = U > S ? U / S : 1;
};
template <class T, int S>
struct Once {
  static constexpr int EACH = Own<S>::EACH;
  T v[EACH];
  template <int K>
  __device__ __forceinline__ T of() const {  // token K's
    return from_lane<S, K % S>(v[K / S]);
  }
};

// The loads of a tensor's U tokens of one chunk.  They are not looked at here, so that all of a chunk's are on their way together: no
// lane has a branch of its own, and where a chunk ends past its segment the last token is taken again.  Chunks outside
// the segment are not read.  A chunk's address is the same in all lanes, their offsets from it are below 2^31 bytes.
template <class T, int S>
struct Source {
  const T* base;
  int64_t token;
  uint32_t lane;
  int own;
  __device__ __forceinline__ Source(const Tokens& from, const Place& p)
      : base(static_cast<const T*>(from.data) + p.b * from.batch), token(from.token), own(p.s % U) {
    lane = (uint32_t)p.channel + (uint32_t)own * (uint32_t)token;
  }
  __device__ __forceinline__ void get(Once<T, S>& to, const Place& p, int t) const {
    if (t < p.t0 || t >= p.end) return;
    const T* row = base + t * token;
    if (t + U <= p.end) {
#pragma unroll
      for (int i = 0; i < Own<S>::EACH; ++i) to.v[i] = row[lane + (uint32_t)(i * S) * (uint32_t)token];
    } else {
#pragma unroll
      for (int i = 0; i < Own<S>::EACH; ++i) {
        const int k = i * S + own, last = p.end - 1 - t;
        to.v[i] = row[(uint32_t)p.channel + (uint32_t)(k < last ? k : last) * (uint32_t)token];
      }
    }
  }
};

// Stores of U tokens of one chunk, contiguous rows of D: of the tokens below `stop`.
template <class T, int S>
__device__ __forceinline__ void put_tokens(T* to, const Once<float, S>& from, const Place& p, const Args& a, int t, int stop) {
  if (!p.mine || (S > U && p.s >= U)) return;
  T* row = to + ((int64_t)p.b * a.T + t) * a.D;
  const uint32_t lane = (uint32_t)p.channel + (uint32_t)p.s * (uint32_t)a.D;
  if (t + U <= stop) {
#pragma unroll
    for (int i = 0; i < Own<S>::EACH; ++i) row[lane + (uint32_t)(i * S) * (uint32_t)a.D] = (T)from.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < Own<S>::EACH; ++i)
      if (t + i * S + p.s < stop) row[lane + (uint32_t)(i * S) * (uint32_t)a.D] = (T)from.v[i];
  }
}

// Rows of B and C of U tokens on their way through LDS, as floats; zeros past N.
template <class T, int NP, int THREADS = 64>
struct Row {
  static constexpr int EACH = U * NP >= THREADS ? U * NP / THREADS : 1;
  const T* base;
  int64_t token;
  T v[EACH];
  __device__ __forceinline__ Row(const Tokens& from, const Place& p)
      : base(static_cast<const T*>(from.data) + p.b * from.batch + p.group * from.group), token(from.token) {}
  __device__ __forceinline__ void get(const Place& p, const Args& a, int t) {
    if (t < p.t0 || t >= p.end) return;
    const T* row = base + t * token;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int e = i * THREADS + (int)threadIdx.x, k = e / NP % U, n = e % NP, last = p.end - 1 - t;
      v[i] = row[(uint32_t)(k < last ? k : last) * (uint32_t)token + (uint32_t)(n < a.N ? n : a.N - 1)];
    }
  }
  __device__ __forceinline__ void put(float* to, const Args& a) const {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int e = i * THREADS + (int)threadIdx.x;
      if (e < U * NP) to[e] = e % NP < a.N ? (float)v[i] : 0.0f;
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

// D_t, its slope, D_t x_t and x_t of a lane's own tokens; zeros past the sequence (there the state stays) and for channels that are none.
template <class T, int S>
__device__ __forceinline__ void get_steps(const Args& a, const Place& p, int t, float bias, const Once<T, S>& x, const Once<T, S>& dt, Once<float, S>& slope,
                                          Once<float, S>& delta, Once<float, S>& u, Once<float, S>& input) {
  const bool whole = t + U <= p.end;  // the same in all lanes
#pragma unroll
  for (int i = 0; i < Own<S>::EACH; ++i) {
    const bool there = p.mine && (whole || t + i * S + p.s < p.end);
    const float z = (float)dt.v[i] + bias;
    slope.v[i] = 1.0f;
    delta.v[i] = there ? (a.softplus ? softplus_of(z, slope.v[i]) : z) : 0.0f;
    input.v[i] = there ? (float)x.v[i] : 0.0f;
    u.v[i] = delta.v[i] * input.v[i];
  }
}

template <class T, int S>
__device__ __forceinline__ void get_errors(const Place& p, int t, const Once<T, S>& d_y, Once<float, S>& error) {
#pragma unroll
  for (int i = 0; i < Own<S>::EACH; ++i) error.v[i] = p.mine && t + i * S + p.s < p.end ? (float)d_y.v[i] : 0.0f;
}

// ---- forward -------------------------------------------------------------------------------------------------------------
// ENDS: a segment's own end state (from zero) and its sum of D; with ERRORS its first state's error too.  Else y, and the final state where there is
// one segment.
template <class T, int NL, int S, bool ENDS, bool ERRORS>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(S == 1 ? 2 : S == 16 ? 3 : 4))) void selective_tokens_kernel(Args a) {
  constexpr int NP = NL * S;
  __shared__ __align__(16) float rows[2][2][U * NP];
  const Place p = place_of<NL, S, 1>(a, a.blocks);
  if (p.segment >= a.segments) return;  // (a grid of two dimensions may have more workgroups than are wanted)
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
  const Source<T, S> from_x(a.x, p), from_dt(a.dt, p), from_d(ERRORS ? a.d_y : a.x, p);
  Once<T, S> next_x, next_dt, next_d;
  Row<T, NP> b(a.b, p), c(a.c, p);
  from_x.get(next_x, p, p.t0), from_dt.get(next_dt, p, p.t0);
  if constexpr (ERRORS) from_d.get(next_d, p, p.t0);
  b.get(p, a, p.t0);
  if constexpr (NEEDS_C) c.get(p, a, p.t0);
  int turn = 0, t = p.t0;
  for (; t < p.end; t += U, turn ^= 1) {
    Once<float, S> slope, delta, u, x, d_y, out;
    get_steps(a, p, t, bias, next_x, next_dt, slope, delta, u, x);
    if constexpr (ERRORS) get_errors(p, t, next_d, d_y);
    b.put(rows[turn][0], a);
    if constexpr (NEEDS_C) c.put(rows[turn][1], a);
    __syncthreads();
    from_x.get(next_x, p, t + U), from_dt.get(next_dt, p, t + U);
    if constexpr (ERRORS) from_d.get(next_d, p, t + U);
    b.get(p, a, t + U);
    if constexpr (NEEDS_C) c.get(p, a, t + U);
    float next_B[NL], next_C[NL];  // a token ahead: all of them at once would take too many registers
    get_row(next_B, rows[turn][0] + p.state);
    if constexpr (NEEDS_C) get_row(next_C, rows[turn][1] + p.state);
    each<U>([&](auto k) {
      constexpr int K = decltype(k)::value;
      const float d = delta.template of<K>(), input = u.template of<K>();
      float B[NL], C[NL], y_t = 0.0f, error = 0.0f;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        B[i] = next_B[i];
        if constexpr (NEEDS_C) C[i] = next_C[i];
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (K + 1 < U) {
        get_row(next_B, rows[turn][0] + (K + 1) * NP + p.state);
        if constexpr (NEEDS_C) get_row(next_C, rows[turn][1] + (K + 1) * NP + p.state);
      }
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
        y_t = sum_over<S>(y_t);
        if (p.s == K % S) out.v[K / S] = y_t;
      }
    });
    if constexpr (!ENDS) {
#pragma unroll
      for (int i = 0; i < Own<S>::EACH; ++i) out.v[i] = t + i * S + p.s < p.end ? out.v[i] + skip * x.v[i] : 0.0f;
      put_tokens(static_cast<T*>(a.y), out, p, a, t, p.t1);
    }
  }
  if constexpr (!ENDS) {  // rows past the sequence
    Once<float, S> zero;
#pragma unroll
    for (int i = 0; i < Own<S>::EACH; ++i) zero.v[i] = 0.0f;
    for (; t < p.t1; t += U) put_tokens(static_cast<T*>(a.y), zero, p, a, t, p.t1);
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
    const int lane = threadIdx.x;  // (its low six bits)
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

// WAVES waves to a workgroup, of neighbouring channels: they share the rows of B and C, and their sums over channels meet in LDS.
template <class T, int NL, int S, int WAVES>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(NL == 4 && S > 2 ? 3 : 2))) void selective_gradient_kernel(Args a) {
  constexpr int NP = NL * S, EACH = Own<S>::EACH, THREADS = 64 * WAVES;
  using Sums = ChannelSums<S, 2 * NL>;
  __shared__ __align__(16) float rows[2][2][U * NP];
  __shared__ __align__(16) f4 kept[WAVES][LONGEST / U][NL / 4][64];
  __shared__ float sums[2][WAVES][U * 2 * NP];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const Place p = place_of<NL, S, WAVES>(a, a.workgroups);
  if (p.segment >= a.segments) return;  // (the whole workgroup, as above)
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
  const int chunks = (p.end - p.t0 + U - 1) / U;
  const Source<T, S> from_x(a.x, p), from_dt(a.dt, p), from_d(a.d_y, p);
  Once<T, S> next_x, next_dt, next_d;
  Once<float, S> slope, delta, u, x, d_y;
  Row<T, NP, THREADS> b(a.b, p), c(a.c, p);
  int turn = 0;
  // forwards: the state in front of every chunk
  from_x.get(next_x, p, p.t0), from_dt.get(next_dt, p, p.t0), b.get(p, a, p.t0);
  for (int j = 0; j < chunks; ++j, turn ^= 1) {
    const int t = p.t0 + j * U;
#pragma unroll
    for (int i = 0; i < NL; i += 4) kept[wave][j][i / 4][lane] = f4{h[i], h[i + 1], h[i + 2], h[i + 3]};
    if (j == chunks - 1) break;
    get_steps(a, p, t, bias, next_x, next_dt, slope, delta, u, x);
    b.put(rows[turn][0], a);
    __syncthreads();
    from_x.get(next_x, p, t + U), from_dt.get(next_dt, p, t + U), b.get(p, a, t + U);
    float next_B[NL];
    get_row(next_B, rows[turn][0] + p.state);
    each<U>([&](auto k) {
      constexpr int K = decltype(k)::value;
      const float d = delta.template of<K>(), input = u.template of<K>();
      float B[NL];
#pragma unroll
      for (int i = 0; i < NL; ++i) B[i] = next_B[i];
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (K + 1 < U) get_row(next_B, rows[turn][0] + (K + 1) * NP + p.state);
#pragma unroll
      for (int i = 0; i < NL; ++i) h[i] = __builtin_amdgcn_exp2f(d * a2[i]) * h[i] + input * B[i];
    });
  }
  __syncthreads();
  // backwards; next_x, next_dt and b hold the last chunk
  const int last = p.t0 + (chunks - 1) * U;
  from_d.get(next_d, p, last), c.get(p, a, last);
  const int value = Sums::first(), sum_at = (value < NL ? 0 : NP - NL) + p.state + value;
  // The sums of the chunk from token t on, which every wave has left in sums[from]: one after the other, U tokens of 2 NP values to the workgroup.
  const auto put_sums = [&](int t, int from) {
    for (int e = threadIdx.x; e < U * 2 * NP; e += THREADS) {
      const int k = e / (2 * NP), which = e / NP % 2, n = e % NP;
      if (t + k >= p.end) break;
      float s = sums[from][0][e];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) s += sums[from][w][e];
      const int64_t row = ((int64_t)p.b * a.T + t + k) * a.G + p.group;
      if (a.workgroups > 1) a.shared[((int64_t)p.block * a.B * a.T * a.G + row) * 2 * NP + e % (2 * NP)] = s;
      else if (n < a.N) static_cast<T*>(which ? a.d_c : a.d_b)[row * a.N + n] = (T)s;
    }
  };
  for (int j = chunks - 1; j >= 0; --j, turn ^= 1) {
    const int t = p.t0 + j * U;
    get_steps(a, p, t, bias, next_x, next_dt, slope, delta, u, x);
    get_errors(p, t, next_d, d_y);
    b.put(rows[turn][0], a), c.put(rows[turn][1], a);
    __syncthreads();
    if (j < chunks - 1) put_sums(t + U, turn ^ 1);
    from_x.get(next_x, p, t - U), from_dt.get(next_dt, p, t - U), from_d.get(next_d, p, t - U);
    b.get(p, a, t - U), c.get(p, a, t - U);
    float before[U + 1][NL], decay[U][NL];  // before[k]: the state in front of token k
#pragma unroll
    for (int i = 0; i < NL; i += 4) {
      const f4 v = kept[wave][j][i / 4][lane];
#pragma unroll
      for (int l = 0; l < 4; ++l) before[0][i + l] = v[l];
    }
    float next_B[NL], next_C[NL];
    get_row(next_B, rows[turn][0] + p.state);
    each<U>([&](auto k) {
      constexpr int K = decltype(k)::value;
      const float d = delta.template of<K>(), input = u.template of<K>();
      float B[NL];
#pragma unroll
      for (int i = 0; i < NL; ++i) B[i] = next_B[i];
      __builtin_amdgcn_sched_barrier(0);
      get_row(next_B, rows[turn][0] + (K + 1 < U ? K + 1 : K) * NP + p.state);
      if constexpr (K + 1 == U) get_row(next_C, rows[turn][1] + K * NP + p.state);
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        decay[K][i] = __builtin_amdgcn_exp2f(d * a2[i]);
        before[K + 1][i] = decay[K][i] * before[K][i] + input * B[i];
      }
    });
    Once<float, S> sum_b, sum_a;  // of g B; of A q' h
    float over_channels[U][Sums::LEFT];
    each<U>([&](auto k) {
      constexpr int K = U - 1 - decltype(k)::value;
      const float d = delta.template of<K>(), input = u.template of<K>(), error = d_y.template of<K>();
      float B[NL], C[NL], v[16], by_b = 0.0f, by_a = 0.0f;
#pragma unroll
      for (int i = 0; i < NL; ++i) B[i] = next_B[i], C[i] = next_C[i];
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (K > 0) {
        get_row(next_B, rows[turn][0] + (K - 1) * NP + p.state);
        get_row(next_C, rows[turn][1] + (K - 1) * NP + p.state);
      }
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
      by_b = sum_over<S>(by_b), by_a = sum_over<S>(by_a);
      if (p.s == K % S) sum_b.v[K / S] = by_b, sum_a.v[K / S] = by_a;
      Sums::sum(v);
#pragma unroll
      for (int i = 0; i < Sums::LEFT; ++i) over_channels[K][i] = v[i];
    });
    if (Sums::writes())
#pragma unroll
      for (int k = 0; k < U; ++k)
#pragma unroll
        for (int i = 0; i < Sums::LEFT; ++i) sums[turn][wave][k * 2 * NP + sum_at + i] = over_channels[k][i];
    Once<float, S> to_x, to_dt;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const float d_delta = x.v[i] * sum_b.v[i] + sum_a.v[i] * 0.69314718055994530942f;
      to_x.v[i] = delta.v[i] * sum_b.v[i] + skip * d_y.v[i], to_dt.v[i] = d_delta * slope.v[i];
      const bool there = (S <= U || p.s < U) && t + i * S + p.s < p.end;
      d_skip += there ? d_y.v[i] * x.v[i] : 0.0f, d_bias += there ? to_dt.v[i] : 0.0f;
    }
    put_tokens(static_cast<T*>(a.d_x), to_x, p, a, t, p.end);
    put_tokens(static_cast<T*>(a.d_dt), to_dt, p, a, t, p.end);
  }
  __syncthreads();
  if (chunks > 0) put_sums(p.t0, turn ^ 1);
  if (a.workgroups == 1)  // (else the kernel that adds up the workgroups' sums clears what is past the sequence)
    for (int64_t e = threadIdx.x; e < (int64_t)(p.t1 - p.end) * a.N; e += THREADS) {
      const int64_t to = (((int64_t)p.b * a.T + p.end + e / a.N) * a.G + p.group) * a.N + e % a.N;
      static_cast<T*>(a.d_b)[to] = (T)0.0f, static_cast<T*>(a.d_c)[to] = (T)0.0f;
    }
  if (p.mine && p.s == 0) {
    for (int k = p.end; k < p.t1; ++k) {
      const int64_t to = ((int64_t)p.b * a.T + k) * a.D + p.channel;
      static_cast<T*>(a.d_x)[to] = (T)0.0f, static_cast<T*>(a.d_dt)[to] = (T)0.0f;
    }
  }
  if (a.last && p.segment == 0) put_states(a.last + p.b * states, q, p, a);
  d_skip = sum_over<S>(d_skip), d_bias = sum_over<S>(d_bias);
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

// Of a workgroup of the backward pass, by the states that a channel's lanes hold.  Checkpoints, sums and rows take 35 to 42 KB of LDS up to 16 states, 28 up to
// 32; beyond, with one wave, 24 and 48 KB, of which a compute unit holds six and three.  More waves there are not measured: they would have fewer
// workgroups' sums of d_b and d_c to add (4 x 1000 tokens of 256 x 16 states take 48 us, of 32 88, of 64 213, of 128 593).
constexpr int waves_of(int states) { return states <= 16 ? 4 : states <= 32 ? 2 : 1; }

struct Form {  // states to a lane, lanes to a channel
  int states, lanes;
};

void launch_f32(const Args& a, Pass pass, Form f, dim3 grid, hipStream_t st);
void launch_bf16(const Args& a, Pass pass, Form f, dim3 grid, hipStream_t st);
void launch_f16(const Args& a, Pass pass, Form f, dim3 grid, hipStream_t st);

template <class T, int NL, int S>
void launch_form(const Args& a, Pass pass, dim3 grid, hipStream_t st) {
  // Backward a lane has four states, whose U tokens, with their decays, are 64 registers (eight, with 128, spill: 100 x 784 tokens of 128 x 16 states took
  // 410 us that way and 259 this way; here 10 registers spill, 14 to 22 where a channel has one lane or eight); eight only where a channel has more than 16 lanes
  // hold.  Forward eight,
  // which share a token's work on its channel among more states (a prompt of 2 x 4096 tokens of 2048 x 16 states: 147 us, and 150 with four),
  // or four where there are no more or more waves are wanted.
  if constexpr (NL == 4 || S == 16) {
    if (pass == ENDS_AND_ERRORS) return selective_tokens_kernel<T, NL, S, true, true><<<grid, 64, 0, st>>>(a);
    constexpr int WAVES = waves_of(NL * S);
    if (pass == GRADIENT) return selective_gradient_kernel<T, NL, S, WAVES><<<grid, 64 * WAVES, 0, st>>>(a);
  }
  if constexpr (NL == 8 || S < 8) {
    if (pass == ENDS) selective_tokens_kernel<T, NL, S, true, false><<<grid, 64, 0, st>>>(a);
    if (pass == TOKENS) selective_tokens_kernel<T, NL, S, false, false><<<grid, 64, 0, st>>>(a);
  }
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
  at(four, one), at(four, two), at(four, four), at(four, eight), at(four, sixteen);
  at(eight, two), at(eight, four), at(eight, eight), at(eight, sixteen);
}

}  // namespace selective
}  // namespace cnn
