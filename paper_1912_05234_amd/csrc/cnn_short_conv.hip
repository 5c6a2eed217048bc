// Causal convolution of a few taps along every channel of a sequence, with silu or without, its gradient, and its form for single tokens.
//
//   p[t] = bias + sum_k w[k] x[t - K + 1 + k],   y = silu(p) or p           (x before the sequence: a state of K - 1 inputs, or zeros)
//   d_p = d_y silu'(p),   d_x[t] = sum_k w[k] d_p[t + K - 1 - k],   d_w[k] = sum_t d_p[t] x[t - K + 1 + k],   d_b = sum_t d_p[t]
//
// Memory bounds it: x (and d_y) read once, y (d_x) written once.  A thread holds a pack of channels, its weights and the last K - 1
// inputs in registers and walks over a chunk of tokens, the next few of them on their way together; only a chunk's first K - 1 inputs are
// read twice (from the caches).  Backward it recomputes p, keeps the last K - 1 errors d_p beside the inputs, and a chunk goes K - 1
// tokens past its end for them.  The weights' gradients are summed in registers over a chunk, over a workgroup's chunks in LDS, and
// over workgroups by a second kernel, in an order that the shape alone fixes.  100 sequences of up to 784 tokens of 128 floats (60 MB) take 14.8 us forward;
// 4 x 4093 x 2048 bfloat16 backward (201 MB) 66: two waves to a SIMD, as many as the launch has (159 registers, floats 168, would leave three), wait for half of
// their time, and the 31 us in which the vector unit issues are only partly those in which memory moves its 39.
#include <utility>

#include "cnn_common.h"
#include "cnn_fold.h"
#include "cnn_types.h"

namespace cnn {
namespace short_conv {
namespace {

constexpr int THREADS = 256, MOST_TAPS = 8, MOST_CHANNELS = 1 << 20;

struct Tokens {
  const void* data;
  int64_t batch, token;
};

struct Args {
  Tokens x, d_y;
  const float *weight, *bias;  // [D][K]; nullable
  const int32_t* lengths;
  const void *first, *d_last;  // [B][K - 1][D]; nullable
  void *out, *last;            // y or d_x [B][T][D]; the final state, or the error of the first, nullable
  float* partial;              // backward: [row blocks][D][K + 1]
  int64_t T, chunk, chunks, rows, D;  // rows: chunks of all sequences
  int lanes, channel_blocks, silu;
};

__device__ __forceinline__ int64_t length_of(const Args& a, int64_t b) {
  if (!a.lengths) return a.T;
  const int64_t n = a.lengths[b];
  return n < 0 ? 0 : n > a.T ? a.T : n;
}

// The thread's part: channels c .. c + V - 1 (`count` of them there), tokens t0 .. t1 - 1 of sequence b; count <= 0: none.
struct Part {
  int64_t b, c, t0, t1, n, row;
  int count;
};

template <int V>
__device__ __forceinline__ Part part_of(const Args& a) {
  Part p;
  const int lane = (int)threadIdx.x % a.lanes, beside = (int)threadIdx.x / a.lanes;
  const int64_t group = workgroup() / a.channel_blocks, block = workgroup() % a.channel_blocks;
  p.c = (block * a.lanes + lane) * V;
  p.row = group * (THREADS / a.lanes) + beside;
  const int64_t left = a.D - p.c;
  p.count = p.row >= a.rows ? 0 : left < V ? (int)left : V;
  p.b = p.row / a.chunks;
  p.t0 = p.row % a.chunks * a.chunk;
  p.t1 = p.t0 + a.chunk < a.T ? p.t0 + a.chunk : a.T;
  p.n = p.count > 0 ? length_of(a, p.b) : 0;
  return p;
}

template <int K, int V>
__device__ __forceinline__ void get_weights(const Args& a, const Part& p, float (&w)[K][V], float (&bias)[V]) {
  const Loose<float, K * V> all = got_loose<K * V>(a.weight + p.c * K, p.count * K);
  Loose<float, V> b{};
  if (a.bias) b = got_loose<V>(a.bias + p.c, p.count);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    bias[j] = b.v[j];
#pragma unroll
    for (int k = 0; k < K; ++k) w[k][j] = all.v[j * K + k];
  }
}

// Input at position t < n, which may lie in the state before the sequence.
template <class T, int K, int V>
__device__ __forceinline__ Loose<T, V> got_input(const Args& a, const Part& p, int64_t t) {
  if (t >= 0) return got_loose<V>(static_cast<const T*>(a.x.data) + p.b * a.x.batch + t * a.x.token + p.c, p.count);
  if (a.first) return got_loose<V>(static_cast<const T*>(a.first) + (p.b * (K - 1) + t + K - 1) * a.D + p.c, p.count);
  return got_loose<V>(static_cast<const T*>(nullptr), 0);
}

// AHEAD tokens from t on: their loads together, without a branch for each where the whole chunk is inside the sequence.
template <class T, int V, int AHEAD>
__device__ __forceinline__ void get_tokens(Loose<T, V> (&to)[AHEAD], const T* at, int64_t token, int64_t t, int64_t end, int count) {
  const T* row = at + t * token;
  if (t + AHEAD <= end && count >= V) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) to[i] = *reinterpret_cast<const Loose<T, V>*>(row + i * token);
  } else {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (t + i < end) to[i] = got_loose<V>(row + i * token, count);
  }
}

template <class T, int K, int V>
__global__ __launch_bounds__(THREADS) void conv_tokens_kernel(Args a) {
  constexpr int AHEAD = 4;
  const Part p = part_of<V>(a);
  if (p.count <= 0) return;
  float w[K][V], bias[V], seen[AHEAD + K - 1][V];
  get_weights(a, p, w, bias);
#pragma unroll
  for (int i = 0; i < K - 1; ++i) {
    const int64_t t = p.t0 - (K - 1) + i;
    if (t < p.n) widen(seen[i], got_input<T, K, V>(a, p, t));
  }
  const T* x = static_cast<const T*>(a.x.data) + p.b * a.x.batch + p.c;
  Loose<T, V> next[AHEAD];
  get_tokens(next, x, a.x.token, p.t0, p.n, p.count);
  T* y = static_cast<T*>(a.out) + p.b * a.T * a.D + p.c;
  // INSIDE: all AHEAD tokens are the sequence's and the chunk's, and the pack is whole.
  const auto walk = [&](int64_t t, auto inside) {
    constexpr bool INSIDE = decltype(inside)::value;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) widen(seen[K - 1 + i], next[i]);
    if (t + AHEAD < p.t1) get_tokens(next, x, a.x.token, t + AHEAD, p.n, p.count);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (!INSIDE && t + i >= p.t1) break;
      float out[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float s = bias[j];
#pragma unroll
        for (int k = 0; k < K; ++k) s += w[k][j] * seen[i + k][j];
        out[j] = s;
      }
      if (a.silu)
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] *= logistic(out[j]);
      if (!INSIDE && t + i >= p.n)
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = 0.0f;
      put_loose(y + (t + i) * a.D, out, INSIDE ? V : p.count);
    }
#pragma unroll
    for (int i = 0; i < K - 1; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) seen[i][j] = seen[AHEAD + i][j];
  };
  const int64_t within = p.n < p.t1 ? p.n : p.t1;
  for (int64_t t = p.t0; t < p.t1; t += AHEAD) {
    if (t + AHEAD <= within && p.count >= V) walk(t, std::true_type{});
    else walk(t, std::false_type{});
  }
  if (a.last && p.t0 == 0)
#pragma unroll
    for (int i = 0; i < K - 1; ++i) {
      float v[V];
      widen(v, got_input<T, K, V>(a, p, p.n - (K - 1) + i));
      put_loose(static_cast<T*>(a.last) + (p.b * (K - 1) + i) * a.D + p.c, v, p.count);
    }
}

template <class T, int K, int V>
__global__ __launch_bounds__(THREADS) void conv_tokens_backward_kernel(Args a) {
  constexpr int AHEAD = 8;
  __shared__ float sums[THREADS * V];
  const Part p = part_of<V>(a);
  if (workgroup() / a.channel_blocks * (THREADS / a.lanes) >= a.rows) return;  // (the whole workgroup: a grid of two dimensions may have more than are wanted)
  float d_w[K][V], d_b[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    d_b[j] = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) d_w[k][j] = 0.0f;
  }
  if (p.count > 0) {
    float w[K][V], bias[V], seen[AHEAD + K - 1][V], error[AHEAD + K - 1][V];
    get_weights(a, p, w, bias);
#pragma unroll
    for (int i = 0; i < K - 1; ++i) {
      const int64_t t = p.t0 - (K - 1) + i;
      if (t < p.n) widen(seen[i], got_input<T, K, V>(a, p, t));
#pragma unroll
      for (int j = 0; j < V; ++j) error[i][j] = 0.0f;
    }
    const T* d_y = static_cast<const T*>(a.d_y.data) + p.b * a.d_y.batch + p.c;
    T* d_x = static_cast<T*>(a.out) + p.b * a.T * a.D + p.c;
    const int64_t end = p.t1 + K - 1;  // token s completes the error of input s - K + 1
    const T* x = static_cast<const T*>(a.x.data) + p.b * a.x.batch + p.c;
    Loose<T, V> next_x[AHEAD], next_d[AHEAD];
    get_tokens(next_x, x, a.x.token, p.t0, p.n, p.count), get_tokens(next_d, d_y, a.d_y.token, p.t0, p.n, p.count);
    // INSIDE: all AHEAD tokens are the sequence's and the chunk's, the errors that they complete the chunk's, and the pack is whole.
    const auto walk = [&](int64_t t, auto inside) {
      constexpr bool INSIDE = decltype(inside)::value;
      float d[AHEAD][V];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) widen(seen[K - 1 + i], next_x[i]), widen(d[i], next_d[i]);
      if (t + AHEAD < end) {
        get_tokens(next_x, x, a.x.token, t + AHEAD, p.n, p.count), get_tokens(next_d, d_y, a.d_y.token, t + AHEAD, p.n, p.count);
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int64_t s = t + i, u = s - (K - 1);
        if (!INSIDE && s >= end) break;
        float e[V];
#pragma unroll
        for (int j = 0; j < V; ++j) e[j] = d[i][j];
        if (a.silu)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            float pre = bias[j];
#pragma unroll
            for (int k = 0; k < K; ++k) pre += w[k][j] * seen[i + k][j];
            const float sigmoid = logistic(pre);
            e[j] *= sigmoid * (1.0f + pre * (1.0f - sigmoid));
          }
        if (!INSIDE && s >= p.n)
#pragma unroll
          for (int j = 0; j < V; ++j) e[j] = 0.0f;
        if (INSIDE || (s < p.n && s < p.t1))
#pragma unroll
          for (int j = 0; j < V; ++j) {
            d_b[j] += e[j];
#pragma unroll
            for (int k = 0; k < K; ++k) d_w[k][j] += e[j] * seen[i + k][j];
          }
#pragma unroll
        for (int j = 0; j < V; ++j) error[K - 1 + i][j] = e[j];
        if (!INSIDE && u < p.t0 && !(p.t0 == 0 && a.last)) continue;  // an earlier chunk's, or one that nobody asked for
        float out[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          float sum = 0.0f;
#pragma unroll
          for (int k = 0; k < K; ++k) sum += w[K - 1 - k][j] * error[i + k][j];
          out[j] = sum;
        }
        if constexpr (std::is_same<T, _Float16>::value) as_floats(out);
        if constexpr (INSIDE) {
          put_loose(d_x + u * a.D, out, V);
          continue;
        }
        const int64_t kept = u - (p.n - (K - 1));  // its place in the final state
        if (a.d_last && kept >= 0 && kept < K - 1) {
          float more[V];
          get_loose(more, static_cast<const T*>(a.d_last) + (p.b * (K - 1) + kept) * a.D + p.c, p.count);
#pragma unroll
          for (int j = 0; j < V; ++j) out[j] += more[j];
        }
        if (u >= 0) {
          if (u >= p.n)
#pragma unroll
            for (int j = 0; j < V; ++j) out[j] = 0.0f;
          put_loose(d_x + u * a.D, out, p.count);
        } else {
          put_loose(static_cast<T*>(a.last) + (p.b * (K - 1) + u + K - 1) * a.D + p.c, out, p.count);
        }
      }
#pragma unroll
      for (int i = 0; i < K - 1; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) seen[i][j] = seen[AHEAD + i][j], error[i][j] = error[AHEAD + i][j];
    };
    const int64_t within = p.n < p.t1 ? p.n : p.t1;
    for (int64_t t = p.t0; t < end; t += AHEAD) {
      if (t + AHEAD <= within && t - (K - 1) >= p.t0 && p.count >= V) walk(t, std::true_type{});
      else walk(t, std::false_type{});
    }
  }
  // [lanes][V] for each chunk beside the others, one tap after the other
  float* partial = a.partial + workgroup() / a.channel_blocks * a.D * (K + 1);
#pragma unroll
  for (int k = 0; k <= K; ++k) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; ++j) sums[threadIdx.x * V + j] = k < K ? d_w[k < K ? k : 0][j] : d_b[j];
    __syncthreads();
    for (int i = threadIdx.x; i < a.lanes * V; i += THREADS) {
      const int64_t c = workgroup() % a.channel_blocks * a.lanes * V + i;
      float s = 0.0f;
      for (int r = i; r < THREADS * V; r += a.lanes * V) s += sums[r];
      if (c < a.D) partial[c * (K + 1) + k] = s;
    }
  }
}

struct PutGradients {
  float *d_weight, *d_bias;
  int taps;
  __device__ void operator()(int64_t i, float sum) const {
    const int64_t c = i / (taps + 1);
    const int k = (int)(i % (taps + 1));
    if (k < taps) d_weight[c * taps + k] = sum;
    else if (d_bias) d_bias[c] = sum;
  }
};

// ---- one token ---------------------------------------------------------------------------------------------------------
struct OneArgs {
  const void* x;
  int64_t batch, pool, total, packs, D;  // total: packs of all rows
  const float *weight, *bias;
  void *state, *y;  // [pool][K - 1][D]
  const int32_t* slots;
  int silu;
};

// A thread moves a pack of a row's state on by one input.  Latency bounds it: the slot, then the state; the weights come meanwhile.
constexpr int ONE_PACK = 4;
template <class T, int K, int V>
__global__ __launch_bounds__(THREADS) void conv_one_token_kernel(OneArgs a) {
  const int64_t i = workgroup() * THREADS + threadIdx.x;
  if (i >= a.total) return;
  const int64_t b = i / a.packs, c = i % a.packs * V, left = a.D - c;
  const int count = left < V ? (int)left : V;
  const int64_t slot = a.slots ? a.slots[b] : b;
  const Loose<float, K * V> w = got_loose<K * V>(a.weight + c * K, count * K);
  const Loose<T, V> x = got_loose<V>(static_cast<const T*>(a.x) + b * a.batch + c, count);
  Loose<float, V> bias{};
  if (a.bias) bias = got_loose<V>(a.bias + c, count);
  T* y = static_cast<T*>(a.y) + b * a.D + c;
  float out[V];
#pragma unroll
  for (int j = 0; j < V; ++j) out[j] = 0.0f;
  if (slot >= 0 && slot < a.pool) {
    T* state = static_cast<T*>(a.state) + slot * (K - 1) * a.D + c;
    Loose<T, V> raw[K];
#pragma unroll
    for (int k = 0; k < K - 1; ++k) raw[k] = got_loose<V>(state + k * a.D, count);
    raw[K - 1] = x;
    float seen[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) widen(seen[k], raw[k]);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float s = bias.v[j];
#pragma unroll
      for (int k = 0; k < K; ++k) s += w.v[j * K + k] * seen[k][j];
      out[j] = a.silu ? s * logistic(s) : s;
    }
#pragma unroll
    for (int k = 0; k < K - 1; ++k) put_loose(state + k * a.D, seen[k + 1], count);
  }
  put_loose(y, out, count);
}

// ---- plans ---------------------------------------------------------------------------------------------------------------
bool shape_ok(const cnn_causal_conv_shape* s) {
  return s && s->B >= 1 && s->T >= 1 && s->D >= 1 && s->D <= MOST_CHANNELS && s->K >= 2 && s->K <= MOST_TAPS && type_known(s->type) &&
         (int64_t)s->B * s->T < (int64_t)1 << 31;
}

bool tokens_ok(const cnn_tokens* t, int type) {
  return t && t->data && reinterpret_cast<uintptr_t>(t->data) % type_bytes(type) == 0 && t->batch >= 0 && t->token >= 0;
}

bool all_aligned(std::initializer_list<const void*> all) {
  for (const void* p : all)
    if (!aligned16(p)) return false;
  return true;
}

struct Plan {
  int lanes, channel_blocks;
  int64_t chunk, chunks, rows, groups;
  size_t bytes;
};

// Lanes along the channels: as many as leave at most an eighth of them idle, else the number that leaves fewest.  Chunks: as long as enough threads
// remain, which each want a few tokens on their way: forward 262144; backward, where a chunk goes K - 1 tokens further and leaves a row of
// partial sums, 65536 (4 x 4093 x 2048 bfloat16 69 us, with 131072 76, with 262144 79).
Plan plan_of(const cnn_causal_conv_shape& s, int pack, bool backward) {
  Plan p{};
  const int64_t packs = (s.D + pack - 1) / pack;
  const auto taken = [&](int lanes) { return (packs + lanes - 1) / lanes * lanes; };
  p.lanes = THREADS;
  for (int lanes = THREADS / 2; lanes >= 8 && taken(p.lanes) * 7 > packs * 8; lanes /= 2)
    if (taken(lanes) < taken(p.lanes)) p.lanes = lanes;
  p.channel_blocks = (int)((packs + p.lanes - 1) / p.lanes);
  const int64_t want = backward ? 65536 : 262144, all = (int64_t)s.B * s.T * packs;
  p.chunk = backward ? 16 : 8;
  while (p.chunk < 128 && all / (p.chunk * 2) >= want) p.chunk *= 2;
  p.chunks = (s.T + p.chunk - 1) / p.chunk;
  p.rows = p.chunks * s.B;
  p.groups = (p.rows + THREADS / p.lanes - 1) / (THREADS / p.lanes);
  p.bytes = backward ? (size_t)p.groups * s.D * (s.K + 1) * 4 : 0;
  return p;
}

Args args_of(const cnn_causal_conv_shape& s, const Plan& p, const cnn_tokens* x, const float* weight, const float* bias, const int32_t* lengths,
             const void* first) {
  Args a{};
  a.x = {x->data, x->batch, x->token};
  a.weight = weight, a.bias = bias, a.lengths = lengths, a.first = first;
  a.T = s.T, a.chunk = p.chunk, a.chunks = p.chunks, a.rows = p.rows, a.D = s.D;
  a.lanes = p.lanes, a.channel_blocks = p.channel_blocks, a.silu = s.silu != 0;
  return a;
}

// Calls fn with the number of taps as a constant.
template <class FN>
void with_taps(int taps, FN fn) {
  const auto at = [&](auto k) {
    if (decltype(k)::value == taps) fn(k);
  };
  at(std::integral_constant<int, 2>{}), at(std::integral_constant<int, 3>{}), at(std::integral_constant<int, 4>{}), at(std::integral_constant<int, 5>{});
  at(std::integral_constant<int, 6>{}), at(std::integral_constant<int, 7>{}), at(std::integral_constant<int, 8>{});
}

// Two channels to a lane and eight tokens ahead backward: 4 x 4093 x 2048 bfloat16 69 us, 4 x 4093 x 2048 floats 92, 2 x 645 x 112 13.4; four
// channels and four tokens 68, 96 and 19, two and four 86, 89 and 13.3.
constexpr int BACK_PACK = 2;
int pack_of(int type) { return type == CNN_F32 ? 4 : 8; }

}  // namespace
}  // namespace short_conv
}  // namespace cnn

extern "C" {

int cnn_causal_conv_fwd(const cnn_causal_conv_shape* s, const cnn_tokens* x, const float* weight, const float* bias, const int32_t* lengths,
                        const void* initial_state, void* y, void* final_state, void* hip_stream) {
  using namespace cnn;
  using namespace cnn::short_conv;
  if (!shape_ok(s) || !tokens_ok(x, s->type) || !weight || !y || !all_aligned({weight, bias, lengths, initial_state, y, final_state})) return CNN_EINVAL;
  const Plan p = plan_of(*s, pack_of(s->type), false);
  Args a = args_of(*s, p, x, weight, bias, lengths, initial_state);
  a.out = y, a.last = final_state;
  return with_type(s->type, [&](auto t) {
    using T = decltype(t);
    with_taps(s->K, [&](auto k) {
      conv_tokens_kernel<T, decltype(k)::value, sizeof(T) == 4 ? 4 : 8><<<grid_of(p.groups * p.channel_blocks), THREADS, 0, (hipStream_t)hip_stream>>>(a);
    });
    return launch_status();
  });
}

size_t cnn_causal_conv_bwd_workspace_bytes(const cnn_causal_conv_shape* s) {
  return cnn::short_conv::shape_ok(s) ? cnn::short_conv::plan_of(*s, cnn::short_conv::BACK_PACK, true).bytes : 0;
}

int cnn_causal_conv_bwd(const cnn_causal_conv_shape* s, const cnn_tokens* x, const cnn_tokens* d_y, const float* weight, const float* bias,
                        const int32_t* lengths, const void* initial_state, const void* d_final_state, void* d_x, float* d_weight, float* d_bias,
                        void* d_initial_state, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace cnn;
  using namespace cnn::short_conv;
  if (!shape_ok(s) || !tokens_ok(x, s->type) || !tokens_ok(d_y, s->type) || !weight || !d_x || !d_weight || !workspace) return CNN_EINVAL;
  if (!all_aligned({weight, bias, lengths, initial_state, d_final_state, d_x, d_weight, d_bias, d_initial_state, workspace})) return CNN_EINVAL;
  const Plan p = plan_of(*s, BACK_PACK, true);
  if (workspace_bytes < p.bytes) return CNN_EWORKSPACE;
  Args a = args_of(*s, p, x, weight, bias, lengths, initial_state);
  a.d_y = {d_y->data, d_y->batch, d_y->token};
  a.d_last = d_final_state, a.out = d_x, a.last = d_initial_state, a.partial = static_cast<float*>(workspace);
  hipStream_t st = (hipStream_t)hip_stream;
  return with_type(s->type, [&](auto t) {
    using T = decltype(t);
    with_taps(s->K, [&](auto k) {
      conv_tokens_backward_kernel<T, decltype(k)::value, BACK_PACK><<<grid_of(p.groups * p.channel_blocks), THREADS, 0, st>>>(a);
    });
    if (launch_status() != CNN_OK) return CNN_EHIP;
    return fold(a.partial, p.groups, (int64_t)s->D * (s->K + 1), PutGradients{d_weight, d_bias, s->K}, st);
  });
}

int cnn_causal_conv_step(const cnn_causal_conv_shape* s, const cnn_tokens* x, const float* weight, const float* bias, void* state, int64_t pool,
                         const int32_t* slots, void* y, void* hip_stream) {
  using namespace cnn;
  using namespace cnn::short_conv;
  if (!shape_ok(s) || s->T != 1 || !tokens_ok(x, s->type) || !weight || !state || !y || !all_aligned({weight, bias, state, slots, y})) return CNN_EINVAL;
  if (pool < 1 || pool > 1 << 30 || (!slots && pool < s->B)) return CNN_EINVAL;
  const int64_t packs = (s->D + ONE_PACK - 1) / ONE_PACK, total = packs * s->B;
  const OneArgs a{x->data, x->batch, pool, total, packs, s->D, weight, bias, state, y, slots, s->silu != 0};
  return with_type(s->type, [&](auto t) {
    using T = decltype(t);
    with_taps(s->K, [&](auto k) {
      conv_one_token_kernel<T, decltype(k)::value, ONE_PACK><<<grid_of((total + THREADS - 1) / THREADS), THREADS, 0, (hipStream_t)hip_stream>>>(a);
    });
    return launch_status();
  });
}

}  // extern "C"
