// Entry points of the selective scan, its form for single tokens, and the kernels around those of cnn_selective.h.
#include "cnn_selective.h"

#include "cnn_fold.h"

namespace cnn {
namespace selective {
namespace {

constexpr int MOST_STATES = 128, MOST_CHANNELS = 1 << 20;
constexpr int64_t MOST_STRIDE = 1 << 26;  // from token to token: a chunk's lie within 2^31 bytes
constexpr float LOG2E = 1.44269504088896340736f;

// ---- states between segments ---------------------------------------------------------------------------------------------
// ends[j] holds what segment j leaves of a state of zero, errors[j] what reaches its first token's state from its own tokens; afterwards the state
// that segment j starts from, and (backwards, by the second half of the grid) the error that it gets from the next.  A chain along the segments, whose loads are a batch
// ahead of it.
constexpr int JOIN_THREADS = 256, JOIN_AHEAD = 8;
template <bool ERRORS>
__device__ __forceinline__ void join_segments(const Args& a, int64_t i) {
  const int64_t states = (int64_t)a.D * a.N, b = i / states, dn = i % states;
  const float a2 = a.a[dn] * LOG2E;
  const int64_t each = a.B * states, every = (int64_t)a.B * a.D;
  float* all = (ERRORS ? a.errors : a.ends) + i;
  const float* sums = a.sums + b * a.D + dn / a.N;
  const auto place = [&](int j) { return ERRORS ? a.segments - 1 - j : j; };
  float own[JOIN_AHEAD], by[JOIN_AHEAD], next_own[JOIN_AHEAD], next_by[JOIN_AHEAD];
  const auto get = [&](int j0) {
#pragma unroll
    for (int k = 0; k < JOIN_AHEAD; ++k)
      if (j0 + k < a.segments) next_own[k] = all[place(j0 + k) * each], next_by[k] = sums[place(j0 + k) * every];
  };
  const float* first = ERRORS ? a.d_last : a.first;
  float run = first ? first[i] : 0.0f;
  get(0);
  for (int j0 = 0; j0 < a.segments; j0 += JOIN_AHEAD) {
#pragma unroll
    for (int k = 0; k < JOIN_AHEAD; ++k) own[k] = next_own[k], by[k] = next_by[k];
    get(j0 + JOIN_AHEAD);
#pragma unroll
    for (int k = 0; k < JOIN_AHEAD; ++k)
      if (j0 + k < a.segments) {
        all[place(j0 + k) * each] = run;
        run = run * __builtin_amdgcn_exp2f(by[k] * a2) + own[k];
      }
  }
  if (!ERRORS && a.last) a.last[i] = run;
}

__global__ __launch_bounds__(JOIN_THREADS) void selective_join_kernel(Args a, bool backward) {
  const int64_t all = a.B * ((int64_t)a.D * a.N), i = workgroup() * JOIN_THREADS + threadIdx.x, groups = (all + JOIN_THREADS - 1) / JOIN_THREADS;
  if (backward) a.last = nullptr;  // (there the error of the first state)
  if (i < groups * JOIN_THREADS) {
    if (i < all) join_segments<false>(a, i);
  } else if (backward) {
    if (i - groups * JOIN_THREADS < all) join_segments<true>(a, i - groups * JOIN_THREADS);
  }
}

// ---- d_b and d_c: sums over the workgroups of a group's channels -------------------------------------------------------------------
struct SharedArgs {
  const float* shared;  // [blocks][rows][2][NP]
  const int32_t* lengths;
  void *d_b, *d_c;  // [rows][N]
  int64_t rows, T;  // rows: B * T * G
  int G, N, NP, blocks;
};

// PARTS threads share a pack of four sums, each taking every PARTS-th workgroup's.
template <class T, int PARTS>
__global__ __launch_bounds__(256) void selective_shared_kernel(SharedArgs a) {
  __shared__ f4 sums[PARTS > 1 ? 256 : 1];
  constexpr int WIDE = 256 / PARTS;
  const int packs = 2 * a.NP / 4, part = threadIdx.x / WIDE;
  const int64_t i = workgroup() * WIDE + threadIdx.x % WIDE, row = i / packs;
  f4 sum{0.0f, 0.0f, 0.0f, 0.0f};
  if (row < a.rows && (!a.lengths || row / a.G % a.T < a.lengths[row / a.G / a.T])) {
    const f4* from = reinterpret_cast<const f4*>(a.shared) + i;
#pragma unroll 8
    for (int k = part; k < a.blocks; k += PARTS) sum += from[k * a.rows * packs];
  }
  if constexpr (PARTS > 1) {
    sums[threadIdx.x] = sum;
    __syncthreads();
    if (part) return;
#pragma unroll
    for (int k = 1; k < PARTS; ++k) sum += sums[k * WIDE + threadIdx.x];
  }
  if (row >= a.rows) return;
  const int at = (int)(i % packs) * 4, n = at % a.NP;
  const float v[4] = {sum[0], sum[1], sum[2], sum[3]};
  put_loose<4>(static_cast<T*>(at < a.NP ? a.d_b : a.d_c) + row * a.N + n, v, a.N - n);
}

struct PutParameters {
  float *d_a, *d_skip, *d_dt_bias;
  int N;
  __device__ void operator()(int64_t i, float sum) const {
    const int64_t d = i / (N + 2);
    const int n = (int)(i % (N + 2));
    if (n < N) d_a[d * N + n] = sum;
    else if (n == N && d_skip) d_skip[d] = sum;
    else if (n > N && d_dt_bias) d_dt_bias[d] = sum;
  }
};

// ---- one token -------------------------------------------------------------------------------------------------------------
struct OneArgs {
  Tokens x, dt, b, c;
  const float *a, *skip, *dt_bias;
  float* state;  // [pool][D][N]
  const int32_t* slots;
  void* y;  // [B][D]
  int64_t pool;
  int B, D, N, per, lanes, softplus;
};

// Four states to a lane, so many lanes to a channel; neighbouring lanes' states are neighbours in memory, which bounds it.  A lane takes AHEAD
// channels, whose loads are on their way together.  (256 rows of 2048 x 16 states, 70 MB, 16.8 us.)
constexpr int ONE_THREADS = 256;
template <class T, int AHEAD>
__global__ __launch_bounds__(ONE_THREADS) void selective_one_token_kernel(OneArgs a) {
  const int lane = (int)threadIdx.x % a.lanes, n = lane * 4, channels = ONE_THREADS / a.lanes, blocks = (a.D + AHEAD * channels - 1) / (AHEAD * channels);
  const int64_t b = workgroup() / blocks;
  const int first = (int)(workgroup() % blocks) * AHEAD * channels + (int)threadIdx.x / a.lanes, count = a.N - n;
  if (b >= a.B) return;
  const int64_t slot = a.slots ? a.slots[b] : b;
  const bool there = slot >= 0 && slot < a.pool;  // (else no sequence here)
  Loose<float, 4> h[AHEAD], decays[AHEAD];
  Loose<T, 4> B[AHEAD], C[AHEAD];
  T x[AHEAD], dt[AHEAD];
  float bias[AHEAD], skip[AHEAD];
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) {
    const int channel = first + k * channels;
    if (!there || channel >= a.D) continue;  // (a channel's lanes together)
    const int group = channel / a.per;
    h[k] = got_loose<4>(a.state + (slot * a.D + channel) * a.N + n, count);
    decays[k] = got_loose<4>(a.a + (int64_t)channel * a.N + n, count);
    B[k] = got_loose<4>(static_cast<const T*>(a.b.data) + b * a.b.batch + group * a.b.group + n, count);
    C[k] = got_loose<4>(static_cast<const T*>(a.c.data) + b * a.c.batch + group * a.c.group + n, count);
    x[k] = static_cast<const T*>(a.x.data)[b * a.x.batch + channel], dt[k] = static_cast<const T*>(a.dt.data)[b * a.dt.batch + channel];
    bias[k] = a.dt_bias ? a.dt_bias[channel] : 0.0f, skip[k] = a.skip ? a.skip[channel] : 0.0f;
  }
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) {
    const int channel = first + k * channels;
    if (channel >= a.D) return;
    float sum = 0.0f;
    if (there) {
      const float z = (float)dt[k] + bias[k], delta = a.softplus ? softplus_of(z) : z, u = delta * (float)x[k];
      float state[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        state[j] = __builtin_amdgcn_exp2f(delta * (decays[k].v[j] * LOG2E)) * h[k].v[j] + u * (float)B[k].v[j];
        sum += (float)C[k].v[j] * state[j];
      }
      put_loose(a.state + (slot * a.D + channel) * a.N + n, state, count);
      for (int d = 1; d < a.lanes; d *= 2) sum += __shfl_xor(sum, d);
      sum += skip[k] * (float)x[k];
    }
    if (lane == 0) static_cast<T*>(a.y)[b * a.D + channel] = (T)sum;
  }
}

// ---- plans -----------------------------------------------------------------------------------------------------------------
bool shape_ok(const cnn_selective_scan_shape* s) {
  return s && s->B >= 1 && s->T >= 1 && s->D >= 1 && s->D <= MOST_CHANNELS && s->N >= 1 && s->N <= MOST_STATES && s->G >= 1 && s->D % s->G == 0 &&
         type_known(s->type) && (int64_t)s->B * s->D <= 1 << 24 && (int64_t)s->B * s->T <= INT32_MAX - 64;
}

bool tokens_ok(const cnn_tokens* t, int type) {
  return t && t->data && reinterpret_cast<uintptr_t>(t->data) % type_bytes(type) == 0 && t->batch >= 0 && t->token >= 0 && t->token <= MOST_STRIDE;
}
bool heads_ok(const cnn_heads* h, int type) {
  return h && h->data && reinterpret_cast<uintptr_t>(h->data) % type_bytes(type) == 0 && h->batch >= 0 && h->token >= 0 && h->token <= MOST_STRIDE && h->head >= 0;
}

bool all_aligned(std::initializer_list<const void*> all) {
  for (const void* p : all)
    if (!aligned16(p)) return false;
  return true;
}

struct Plan {
  Form form;
  int blocks, workgroups, segments;
  int64_t length;
  size_t ends, errors, sums, partial, shared, bytes;  // offsets in the workspace
};

size_t rounded(size_t b) { return (b + 255) & ~(size_t)255; }

// About how long a pass takes, in a SIMD's cycles: `alone` a token for a wave that has a SIMD to itself, `shared` for each of several.  (Measured forward,
// 4096 tokens by one wave to a SIMD: four states to a lane 315, eight 475; 2 x 4096 x 2048 x 16 states by eight waves to a SIMD: 190 and 360.)
double pass_cost(int64_t waves, int64_t length, double alone, double shared) {
  const double load = (double)((waves + 1023) / 1024);
  return (double)length * (load * shared > alone ? load * shared : alone) + 3000.0;
}

Plan plan_of(const cnn_selective_scan_shape& s, bool backward) {
  Plan p{};
  const int64_t per = s.D / s.G;
  const auto blocks = [&](int lanes) { return (per * lanes + 63) / 64; };
  double best = 0.0;
  for (const int states : {8, 4})
    for (const int lanes : {1, 2, 4, 8, 16}) {
      // the fewest lanes that hold a channel's states, of those that have a kernel
      if (states * lanes < s.N || (lanes > 1 && states * lanes / 2 >= s.N)) continue;
      if (backward ? states == 8 && (lanes < 16 || s.N <= 64) : states == 8 ? lanes < 2 : lanes > 4) continue;
      const int64_t waves = (int64_t)s.B * s.G * blocks(lanes);
      const double alone = 180.0 + 40.0 * states, shared = 20.0 + 38.0 * states;
      for (int64_t length = 16; ; length *= 2) {
        if (backward && length > LONGEST) break;
        if (length > s.T) length = (s.T + U - 1) / U * U;
        const int64_t segments = (s.T + length - 1) / length;
        double cost = pass_cost(waves * segments, length, alone * (backward ? 2.9 : 1.0), shared * (backward ? 4.2 : 1.0));
        if (segments > 1)  // the first pass, two more launches, the chain along the segments and its bytes
          cost += pass_cost(waves * segments, length, alone * (backward ? 1.1 : 0.75), shared * (backward ? 1.4 : 0.75)) + 13000.0 +
                  2500.0 * (double)((segments + 7) / 8) + (double)s.B * s.D * s.N * segments * (backward ? 0.012 : 0.006);
        if (best == 0.0 || cost < best) best = cost, p.form = {states, lanes}, p.length = length, p.segments = (int)segments;
        if (length >= s.T) break;
      }
    }
  p.blocks = (int)blocks(p.form.lanes);
  const int waves = waves_of(p.form.states * p.form.lanes);
  p.workgroups = (p.blocks + waves - 1) / waves;
  const size_t states = rounded((size_t)p.segments * s.B * s.D * s.N * 4);
  p.ends = 0;
  if (p.segments > 1) {
    p.errors = states, p.sums = p.errors + (backward ? states : 0);
    p.bytes = p.sums + rounded((size_t)p.segments * s.B * s.D * 4);
  }
  if (backward) {
    p.partial = p.bytes, p.shared = p.partial + rounded((size_t)p.segments * s.B * s.D * (s.N + 2) * 4);
    p.bytes = p.shared + (p.workgroups > 1 ? (size_t)p.workgroups * s.B * s.T * s.G * 2 * p.form.states * p.form.lanes * 4 : 0);
  }
  return p;
}

Tokens tokens_of(const cnn_tokens* t) { return {t->data, t->batch, t->token, 0}; }
Tokens tokens_of(const cnn_heads* h) { return {h->data, h->batch, h->token, h->head}; }

Args args_of(const cnn_selective_scan_shape& s, const Plan& p, void* workspace) {
  Args a{};
  char* ws = static_cast<char*>(workspace);
  a.ends = reinterpret_cast<float*>(ws + p.ends), a.errors = reinterpret_cast<float*>(ws + p.errors), a.sums = reinterpret_cast<float*>(ws + p.sums);
  a.partial = reinterpret_cast<float*>(ws + p.partial), a.shared = reinterpret_cast<float*>(ws + p.shared);
  a.T = s.T, a.length = (int)p.length, a.B = s.B, a.D = s.D, a.N = s.N, a.G = s.G, a.per = s.D / s.G, a.blocks = p.blocks, a.workgroups = p.workgroups, a.segments = p.segments;
  a.softplus = s.softplus != 0;
  return a;
}

int run(const Args& a, const Plan& p, int type, bool backward, hipStream_t st) {
  const auto launch = type == CNN_F32 ? launch_f32 : type == CNN_BF16 ? launch_bf16 : launch_f16;
  const dim3 grid = grid_of((int64_t)p.blocks * a.G * a.B * p.segments);
  if (p.segments > 1) {
    launch(a, backward ? ENDS_AND_ERRORS : ENDS, p.form, grid, st);
    if (launch_status() != CNN_OK) return CNN_EHIP;
    const int64_t groups = ((int64_t)a.B * a.D * a.N + JOIN_THREADS - 1) / JOIN_THREADS;
    selective_join_kernel<<<grid_of(backward ? 2 * groups : groups), JOIN_THREADS, 0, st>>>(a, backward);
    if (launch_status() != CNN_OK) return CNN_EHIP;
  }
  launch(a, backward ? GRADIENT : TOKENS, p.form, backward ? grid_of((int64_t)p.workgroups * a.G * a.B * p.segments) : grid, st);
  return launch_status();
}

}  // namespace
}  // namespace selective
}  // namespace cnn

extern "C" {

size_t cnn_selective_scan_fwd_workspace_bytes(const cnn_selective_scan_shape* s) {
  return cnn::selective::shape_ok(s) ? cnn::selective::plan_of(*s, false).bytes : 0;
}

size_t cnn_selective_scan_bwd_workspace_bytes(const cnn_selective_scan_shape* s) {
  return cnn::selective::shape_ok(s) ? cnn::selective::plan_of(*s, true).bytes : 0;
}

int cnn_selective_scan_fwd(const cnn_selective_scan_shape* s, const cnn_tokens* x, const cnn_tokens* dt, const float* a_, const cnn_heads* b, const cnn_heads* c,
                           const float* skip, const float* dt_bias, const int32_t* lengths, const float* initial_state, void* y, float* final_state,
                           void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace cnn;
  using namespace cnn::selective;
  if (!shape_ok(s) || !tokens_ok(x, s->type) || !tokens_ok(dt, s->type) || !heads_ok(b, s->type) || !heads_ok(c, s->type) || !a_ || !y) return CNN_EINVAL;
  if (!all_aligned({a_, skip, dt_bias, lengths, initial_state, y, final_state, workspace})) return CNN_EINVAL;
  const Plan p = plan_of(*s, false);
  if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return CNN_EWORKSPACE;
  Args a = args_of(*s, p, workspace);
  a.x = tokens_of(x), a.dt = tokens_of(dt), a.b = tokens_of(b), a.c = tokens_of(c);
  a.a = a_, a.skip = skip, a.dt_bias = dt_bias, a.lengths = lengths, a.first = initial_state, a.y = y, a.last = final_state;
  return run(a, p, s->type, false, (hipStream_t)hip_stream);
}

int cnn_selective_scan_bwd(const cnn_selective_scan_shape* s, const cnn_tokens* x, const cnn_tokens* dt, const float* a_, const cnn_heads* b, const cnn_heads* c,
                           const cnn_tokens* d_y, const float* skip, const float* dt_bias, const int32_t* lengths, const float* initial_state,
                           const float* d_final_state, void* d_x, void* d_dt, float* d_a, void* d_b, void* d_c, float* d_skip, float* d_dt_bias,
                           float* d_initial_state, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace cnn;
  using namespace cnn::selective;
  if (!shape_ok(s) || !tokens_ok(x, s->type) || !tokens_ok(dt, s->type) || !heads_ok(b, s->type) || !heads_ok(c, s->type) || !tokens_ok(d_y, s->type)) return CNN_EINVAL;
  if (!a_ || !d_x || !d_dt || !d_a || !d_b || !d_c || !workspace) return CNN_EINVAL;
  if (!all_aligned({a_, skip, dt_bias, lengths, initial_state, d_final_state, d_x, d_dt, d_a, d_b, d_c, d_skip, d_dt_bias, d_initial_state, workspace})) return CNN_EINVAL;
  const Plan p = plan_of(*s, true);
  if (workspace_bytes < p.bytes) return CNN_EWORKSPACE;
  Args a = args_of(*s, p, workspace);
  a.x = tokens_of(x), a.dt = tokens_of(dt), a.b = tokens_of(b), a.c = tokens_of(c), a.d_y = tokens_of(d_y);
  a.a = a_, a.skip = skip, a.dt_bias = dt_bias, a.lengths = lengths, a.first = initial_state, a.d_last = d_final_state;
  a.d_x = d_x, a.d_dt = d_dt, a.d_b = d_b, a.d_c = d_c, a.last = d_initial_state;
  hipStream_t st = (hipStream_t)hip_stream;
  const int rc = run(a, p, s->type, true, st);
  if (rc != CNN_OK) return rc;
  const SharedArgs g{a.shared, lengths, d_b, d_c, (int64_t)s->B * s->T * s->G, s->T, s->G, s->N, p.form.states * p.form.lanes, p.workgroups};
  const int64_t packs = g.rows * (2 * g.NP / 4);
  const int status = p.workgroups == 1 ? CNN_OK : with_type(s->type, [&](auto t) {
    using T = decltype(t);
    // (Two tokens of 31 sequences of 2496 channels, 39 workgroups to a sum.)
    if (g.blocks > 8) selective_shared_kernel<T, 8><<<grid_of((packs + 31) / 32), 256, 0, st>>>(g);
    else selective_shared_kernel<T, 1><<<grid_of((packs + 255) / 256), 256, 0, st>>>(g);
    return launch_status();
  });
  if (status != CNN_OK) return status;
  return fold(a.partial, (int64_t)p.segments * s->B, (int64_t)s->D * (s->N + 2), PutParameters{d_a, d_skip, d_dt_bias, s->N}, st);
}

int cnn_selective_scan_step(const cnn_selective_scan_shape* s, const cnn_tokens* x, const cnn_tokens* dt, const float* a_, const cnn_heads* b, const cnn_heads* c,
                            const float* skip, const float* dt_bias, float* state, int64_t pool, const int32_t* slots, void* y, void* hip_stream) {
  using namespace cnn;
  using namespace cnn::selective;
  if (!shape_ok(s) || s->T != 1 || !tokens_ok(x, s->type) || !tokens_ok(dt, s->type) || !heads_ok(b, s->type) || !heads_ok(c, s->type)) return CNN_EINVAL;
  if (!a_ || !state || !y || !all_aligned({a_, skip, dt_bias, state, slots, y})) return CNN_EINVAL;
  if (pool < 1 || pool > 1 << 30 || (!slots && pool < s->B)) return CNN_EINVAL;
  int lanes = 1;
  while (lanes * 4 < s->N) lanes *= 2;
  const OneArgs a{tokens_of(x), tokens_of(dt), tokens_of(b), tokens_of(c), a_, skip, dt_bias, state, slots, y, pool, s->B, s->D, s->N, s->D / s->G, lanes, s->softplus != 0};
  const int channels = ONE_THREADS / lanes;
  const auto grid = [&](int ahead) { return grid_of((int64_t)s->B * ((s->D + ahead * channels - 1) / (ahead * channels))); };
  return with_type(s->type, [&](auto t) {
    using T = decltype(t);
    if ((int64_t)s->B * s->D / channels < 2048) selective_one_token_kernel<T, 1><<<grid(1), ONE_THREADS, 0, (hipStream_t)hip_stream>>>(a);
    else selective_one_token_kernel<T, 2><<<grid(2), ONE_THREADS, 0, (hipStream_t)hip_stream>>>(a);
    return launch_status();
  });
}

}  // extern "C"
