// Norms around a block: RMS norm of groups of `width` elements, after a scaled addition or in front of a gate.
//
//   n = v / sqrt(mean(v^2) + eps)
//   ADD    v = residual + scale x,  r = v,  y = n w
//   GATE   v = x,                   y = residual + scale n w silu(gate)
//
// Backward, with d the error of n, rstd = 1 / sqrt(mean(v^2) + eps):  d_v = rstd (d - n mean(d n)).  Both means come from one pass
// over the row (sum v^2 and sum d v), so nothing but the inputs of the forward pass is kept for it.
//
// Memory bounds it: every element is read and written once.  A team of lanes holds a group in registers between the sums and the
// results, sixteen elements to a lane at most (packs of sixteen bytes, or of four elements where one of the tensors holds floats); teams are as
// narrow as the group allows, a workgroup takes the groups of several rows side by side and goes on to further rows with its
// weights in registers.  The weight's gradient is summed over a workgroup's rows in registers, over its teams in LDS, and over the workgroups by a second
// kernel, in an order that the shape alone fixes.  16381 rows of 2048 bfloat16 with a stream of floats, backward (537 MB), take 90 us: 85 at 6.3 TB/s and
// 4.5 for the second kernel (a copy of 1 GiB reaches 5.2); 78400 rows of 2 x 64 floats behind a gate, backward (201 MB), 44; 64 rows of 64 floats
// 5.5, the call.
//
// Groups of more than 8192 elements, whose sixteen waves leave 128 registers to a lane, spill: backward 20 to 105 of them (4000 rows of 12000 floats behind a gate 543
// us of 185 at a copy's rate, 4000 of 16384 bfloat16 with a stream of floats 356 of 202), forward 6 to 17 behind a gate with a stream of floats (116 of 111).
#pragma once

#include "cnn_common.h"
#include "cnn_lanes.h"
#include "cnn_types.h"

namespace cnn {
namespace norm {

enum Mode { ADD, GATE };

struct Rows {
  const void* data;
  int64_t row;  // elements from one to the next
};

struct Args {
  Rows x, residual, gate;  // residual and gate nullable; backward: x is what was normalised
  Rows d_y, d_r;           // backward; d_r nullable
  const float* weight;
  void *y, *r;             // ADD: r nullable; backward: d_x (ADD: nullable) and d_residual (ADD) or d_gate (GATE: nullable)
  float* partial;          // backward: [row blocks][groups * width]
  int64_t rows, row_blocks;
  int groups, width;
  int at_once, beside, group_blocks;  // groups of a workgroup; rows side by side in it; workgroups for all groups of a row
  float scale, eps, by_width;
  bool past_caches;
};

template <class T, class R>
struct Types {
  using X = T;
  using S = R;
  static constexpr int PACK = sizeof(T) == 2 && sizeof(R) == 2 ? 8 : 4;
};

// Sums of COUNT values over a team; every lane of it has them afterwards.
template <int LANES, int COUNT>
struct TeamSum {
  static constexpr int WAVES = LANES > 64 ? LANES / 64 : 1;
  float buffer[LANES > 64 ? 2 : 1][LANES > 64 ? WAVES : 1][COUNT];
  __device__ __forceinline__ void sum(float (&v)[COUNT], int turn) {
#pragma unroll
    for (int c = 0; c < COUNT; ++c) v[c] = sum_over<(LANES < 64 ? LANES : 64)>(v[c]);
    if constexpr (LANES > 64) {
      // (turns use the two buffers by turns: whoever writes one again has passed the barrier of the turn between)
      float(&b)[WAVES][COUNT] = buffer[turn & 1];
      if (threadIdx.x % 64 == 0)
#pragma unroll
        for (int c = 0; c < COUNT; ++c) b[threadIdx.x / 64][c] = v[c];
      __syncthreads();
#pragma unroll
      for (int c = 0; c < COUNT; ++c) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += b[w][c];
        v[c] = s;
      }
    }
  }
};

__device__ __forceinline__ float silu_of(float z, float& sigmoid) {
  sigmoid = logistic(z);
  return z * sigmoid;
}

// 1 / sqrt(mean + eps): the hardware's estimate and one step of Newton's method, which leaves it within an ulp or so.
__device__ __forceinline__ float inverse_root(float v) {
  const float e = __builtin_amdgcn_rsqf(v), h = 0.5f * v * e;
  const float refined = e + e * __builtin_fmaf(-h, e, 0.5f);
  return e < 1e18f && e > 1e-18f ? refined : e;  // (no infinities out of the step)
}

// A lane's pack of a group: `count` elements from `at` on, of which the first `skip` are another lane's too.  The last pack of a group of no whole number of
// packs ends with it and overlaps the one before, so that it is one access like the others: sums leave the shared elements to that one, results
// are written twice, the same.  (Element by element, rows of 541 bfloat16 took 153 us where this takes 69.)
struct Slot {
  int at, count, skip;
};
template <int V>
__device__ __forceinline__ Slot slot_of(int at, int width) {
  if (at >= width) return {0, 0, 0};
  if (at + V <= width) return {at, V, 0};
  if (width < V) return {at, width, 0};
  return {width - V, V, at - (width - V)};
}

constexpr int threads_of(int lanes) { return lanes > 256 ? lanes : 256; }

template <class TY, Mode MODE, int LANES, int PACKS>
__global__ __launch_bounds__(threads_of(LANES)) void norm_forward_kernel(Args a) {
  using T = typename TY::X;
  using R = typename TY::S;
  constexpr int V = TY::PACK, TEAMS = threads_of(LANES) / LANES;
  __shared__ TeamSum<LANES, 1> shared;
  const int lane = threadIdx.x % LANES, team = TEAMS > 1 ? threadIdx.x / LANES : 0;
  const int64_t rb = workgroup() / a.group_blocks;
  const int group = (int)(workgroup() % a.group_blocks) * a.at_once + team % a.at_once, beside = team / a.at_once;
  if (rb >= a.row_blocks) return;                                       // (the whole workgroup)
  const bool works = beside < a.beside && group < a.groups;
  if (TEAMS > 1 && !works) return;  // (teams of more than a wave are alone in their workgroup, which has a group)
  const int first = group * a.width;
  Slot slot[PACKS];
  float w[PACKS][V];
#pragma unroll
  for (int p = 0; p < PACKS; ++p) {
    slot[p] = slot_of<V>((p * LANES + lane) * V, a.width);
    get_loose(w[p], a.weight + first + slot[p].at, slot[p].count);
  }
  int turn = 0;
  for (int64_t n = rb * a.beside + beside; n < a.rows; n += a.row_blocks * a.beside, ++turn) {
    float v[PACKS][V], z[PACKS][V], res[PACKS][V];
    const T* x = static_cast<const T*>(a.x.data) + n * a.x.row + first;
    const R* residual = static_cast<const R*>(a.residual.data) + n * a.residual.row + first;
    const T* gate = static_cast<const T*>(a.gate.data) + n * a.gate.row + first;
    Loose<T, V> raw_x[PACKS], raw_gate[PACKS];
    Loose<R, V> raw_residual[PACKS];
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      raw_x[p] = got_loose<V>(x + slot[p].at, slot[p].count, a.past_caches);
      if (a.residual.data) raw_residual[p] = got_loose<V>(residual + slot[p].at, slot[p].count, a.past_caches);
      if (MODE == GATE && a.gate.data) raw_gate[p] = got_loose<V>(gate + slot[p].at, slot[p].count, a.past_caches);
    }
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      widen(v[p], raw_x[p]);
      if (a.residual.data) widen(res[p], raw_residual[p]);
      if (MODE == GATE && a.gate.data) widen(z[p], raw_gate[p]);
    }
    float sum[1] = {0.0f};
#pragma unroll
    for (int p = 0; p < PACKS; ++p)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (MODE == ADD && a.residual.data) v[p][j] = res[p][j] + a.scale * v[p][j];
        sum[0] += j < slot[p].skip ? 0.0f : v[p][j] * v[p][j];
      }
    shared.sum(sum, turn);
    const float rstd = inverse_root(sum[0] * a.by_width + a.eps);
    const int64_t to = n * a.groups * a.width + first;
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      if (MODE == ADD && a.r) put_loose(static_cast<R*>(a.r) + to + slot[p].at, v[p], slot[p].count, a.past_caches);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float y = v[p][j] * rstd * w[p][j], sigmoid;
        if constexpr (MODE == GATE) {
          if (a.gate.data) y *= silu_of(z[p][j], sigmoid);
          y = a.residual.data ? res[p][j] + a.scale * y : a.scale * y;
        }
        v[p][j] = y;
      }
      if constexpr (MODE == ADD) put_loose(static_cast<T*>(a.y) + to + slot[p].at, v[p], slot[p].count, a.past_caches);
      else put_loose(static_cast<R*>(a.y) + to + slot[p].at, v[p], slot[p].count, a.past_caches);
    }
  }
}

template <class TY, Mode MODE, int LANES, int PACKS>
__global__ __launch_bounds__(threads_of(LANES)) void norm_backward_kernel(Args a) {
  using T = typename TY::X;
  using R = typename TY::S;
  constexpr int V = TY::PACK, TEAMS = threads_of(LANES) / LANES;
  using X = typename std::conditional<MODE == ADD, R, T>::type;  // of what was normalised
  using D = typename std::conditional<MODE == ADD, T, R>::type;  // of y
  // Sixteen waves share the registers of a compute unit's four SIMDs: there weights and gates are taken again where they are used, and elements kept as they
  // were loaded.
  constexpr bool KEEPS = LANES < 1024;
  __shared__ TeamSum<LANES, 2> shared;
  __shared__ float sums[TEAMS > 1 ? TEAMS * LANES * PACKS * V : 1];
  const int lane = threadIdx.x % LANES, team = TEAMS > 1 ? threadIdx.x / LANES : 0;
  const int64_t rb = workgroup() / a.group_blocks;
  const int group0 = (int)(workgroup() % a.group_blocks) * a.at_once, group = group0 + team % a.at_once, beside = team / a.at_once;
  if (rb >= a.row_blocks) return;  // (the whole workgroup)
  const bool works = beside < a.beside && group < a.groups;
  const int first = works ? group * a.width : 0;
  Slot slot[PACKS];
  float w[PACKS][V], dw[PACKS][V];
#pragma unroll
  for (int p = 0; p < PACKS; ++p) {
    slot[p] = slot_of<V>((p * LANES + lane) * V, a.width);
    if constexpr (KEEPS) get_loose(w[p], a.weight + first + slot[p].at, slot[p].count);
#pragma unroll
    for (int j = 0; j < V; ++j) dw[p][j] = 0.0f;
  }
  int turn = 0;
  for (int64_t n = works ? rb * a.beside + beside : a.rows; n < a.rows; n += a.row_blocks * a.beside, ++turn) {
    float v[PACKS][V], d[PACKS][V], z[PACKS][V];  // z: the gate, or the error of r
    const X* x = static_cast<const X*>(a.x.data) + n * a.x.row + first;
    const D* d_y = static_cast<const D*>(a.d_y.data) + n * a.d_y.row + first;
    const R* d_r = static_cast<const R*>(a.d_r.data) + n * a.d_r.row + first;
    const T* gate = static_cast<const T*>(a.gate.data) + n * a.gate.row + first;
    Loose<X, V> raw_x[PACKS];
    Loose<D, V> raw_d[PACKS];
    Loose<typename std::conditional<MODE == ADD, R, T>::type, V> raw_z[PACKS] = {};
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      raw_x[p] = got_loose<V>(x + slot[p].at, slot[p].count, a.past_caches);
      raw_d[p] = got_loose<V>(d_y + slot[p].at, slot[p].count, a.past_caches);
      if constexpr (MODE == ADD) {
        if (a.d_r.data) raw_z[p] = got_loose<V>(d_r + slot[p].at, slot[p].count, a.past_caches);
      } else {
        if (a.gate.data) raw_z[p] = got_loose<V>(gate + slot[p].at, slot[p].count, a.past_caches);
      }
    }
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      widen(v[p], raw_x[p]), widen(d[p], raw_d[p]);
      if (MODE == ADD ? a.d_r.data : a.gate.data) widen(z[p], raw_z[p]);
    }
    float sum[2] = {0.0f, 0.0f}, sigmoid[PACKS][V];
    const auto factor = [&](int p, int j) { return MODE == ADD ? 1.0f : a.gate.data ? a.scale * (z[p][j] * sigmoid[p][j]) : a.scale; };
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      if constexpr (!KEEPS) get_loose(w[p], a.weight + first + slot[p].at, slot[p].count);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (MODE == GATE && a.gate.data) sigmoid[p][j] = logistic(z[p][j]);
        sum[0] += j < slot[p].skip ? 0.0f : v[p][j] * v[p][j];
        sum[1] += j < slot[p].skip ? 0.0f : d[p][j] * w[p][j] * factor(p, j) * v[p][j];
      }
    }
    shared.sum(sum, turn);
    const float rstd = inverse_root(sum[0] * a.by_width + a.eps), mean = sum[1] * a.by_width * rstd;
    // A group of one element is 1 or -1 but for eps: d - n (d n) = d (1 - n^2) = d eps rstd^2, of which the difference would leave nothing.
    const bool alone = a.width == 1;
    const float left = a.eps * rstd * rstd;
    const int64_t to = n * a.groups * a.width + first;
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      float d_gate[V];
      if constexpr (!KEEPS) {
        get_loose(w[p], a.weight + first + slot[p].at, slot[p].count);
        forget(raw_x[p]), forget(raw_d[p]), forget(raw_z[p]);
        widen(v[p], raw_x[p]), widen(d[p], raw_d[p]);
        if (MODE == ADD ? a.d_r.data : a.gate.data) widen(z[p], raw_z[p]);
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (MODE == GATE && a.gate.data) sigmoid[p][j] = logistic(z[p][j]);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float hat = v[p][j] * rstd, error = d[p][j], by = factor(p, j);
        dw[p][j] += error * hat * by;
        const float d_n = error * w[p][j] * by;
        v[p][j] = rstd * (alone ? d_n * left : d_n - hat * mean);
        if (MODE == ADD && a.d_r.data) v[p][j] += z[p][j];
        if (MODE == GATE && a.gate.data) {
          const float s = sigmoid[p][j];
          d_gate[j] = a.scale * error * hat * w[p][j] * s * (1.0f + z[p][j] * (1.0f - s));
        }
      }
      if constexpr (MODE == ADD) {
        put_loose(static_cast<R*>(a.r) + to + slot[p].at, v[p], slot[p].count, a.past_caches);
        if (a.y) {
#pragma unroll
          for (int j = 0; j < V; ++j) v[p][j] *= a.scale;
          put_loose(static_cast<T*>(a.y) + to + slot[p].at, v[p], slot[p].count, a.past_caches);
        }
      } else {
        put_loose(static_cast<T*>(a.y) + to + slot[p].at, v[p], slot[p].count, a.past_caches);
        if (a.gate.data) put_loose(static_cast<T*>(a.r) + to + slot[p].at, d_gate, slot[p].count, a.past_caches);
      }
    }
  }
  float* partial = a.partial + rb * a.groups * a.width;
  if constexpr (TEAMS == 1) {
#pragma unroll
    for (int p = 0; p < PACKS; ++p)
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j >= slot[p].skip && j < slot[p].count) partial[first + slot[p].at + j] = dw[p][j];
  } else {
    constexpr int WIDE = LANES * PACKS * V;
#pragma unroll
    for (int p = 0; p < PACKS; ++p)
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j >= slot[p].skip && j < slot[p].count) sums[team * WIDE + slot[p].at + j] = dw[p][j];
    __syncthreads();
    const int here = a.groups - group0 < a.at_once ? a.groups - group0 : a.at_once;
    for (int c = threadIdx.x; c < here * a.width; c += TEAMS * LANES) {
      const int g = c / a.width, j = c % a.width;
      float s = 0.0f;
      for (int b = 0; b < a.beside; ++b) s += sums[(b * a.at_once + g) * WIDE + j];
      partial[group0 * a.width + c] = s;
    }
  }
}

// How a shape is cut; `pack` elements to a load.
struct Cut {
  int lanes, packs;
};
inline Cut cut_of(int width, int pack) {
  const int packs = (width + pack - 1) / pack, most = 16 / pack;  // of a lane
  for (int lanes = 1; lanes <= 32; lanes *= 2)
    if (packs <= lanes) return {lanes, 1};
  for (int lanes : {64, 256, 1024})
    for (int p = 1; p <= most; p *= 2)
      if (packs <= lanes * p) return {lanes, p};
  return {0, 0};
}
inline int pack_of(int type, int stream_type) { return type != CNN_F32 && stream_type != CNN_F32 ? 8 : 4; }

void launch_f32(const Args& a, int stream_type, Mode mode, bool backward, Cut cut, unsigned grid, hipStream_t st);
void launch_bf16(const Args& a, int stream_type, Mode mode, bool backward, Cut cut, unsigned grid, hipStream_t st);
void launch_f16(const Args& a, int stream_type, Mode mode, bool backward, Cut cut, unsigned grid, hipStream_t st);

template <class TY, Mode MODE, int LANES, int PACKS>
void launch_cut(const Args& a, bool backward, unsigned grid, hipStream_t st) {
  if (backward) norm_backward_kernel<TY, MODE, LANES, PACKS><<<grid, threads_of(LANES), 0, st>>>(a);
  else norm_forward_kernel<TY, MODE, LANES, PACKS><<<grid, threads_of(LANES), 0, st>>>(a);
}

template <class TY, Mode MODE>
void launch_mode(const Args& a, bool backward, Cut c, unsigned grid, hipStream_t st) {
  if (c.lanes == 1) return launch_cut<TY, MODE, 1, 1>(a, backward, grid, st);
  if (c.lanes == 2) return launch_cut<TY, MODE, 2, 1>(a, backward, grid, st);
  if (c.lanes == 4) return launch_cut<TY, MODE, 4, 1>(a, backward, grid, st);
  if (c.lanes == 8) return launch_cut<TY, MODE, 8, 1>(a, backward, grid, st);
  if (c.lanes == 16) return launch_cut<TY, MODE, 16, 1>(a, backward, grid, st);
  if (c.lanes == 32) return launch_cut<TY, MODE, 32, 1>(a, backward, grid, st);
  const auto with_lanes = [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    if constexpr (TY::PACK == 8 || L == 64)  // (four packs of four come before one more lane)
      if (c.packs == 1) return launch_cut<TY, MODE, L, 1>(a, backward, grid, st);
    if (c.packs == 2) return launch_cut<TY, MODE, L, 2>(a, backward, grid, st);
    if constexpr (TY::PACK == 4) launch_cut<TY, MODE, L, 4>(a, backward, grid, st);
  };
  if (c.lanes == 64) with_lanes(std::integral_constant<int, 64>{});
  else if (c.lanes == 256) with_lanes(std::integral_constant<int, 256>{});
  else with_lanes(std::integral_constant<int, 1024>{});
}

template <class T>
void launch_type(const Args& a, int stream_type, Mode mode, bool backward, Cut c, unsigned grid, hipStream_t st) {
  const auto with = [&](auto types) {
    using TY = decltype(types);
    if (mode == ADD) launch_mode<TY, ADD>(a, backward, c, grid, st);
    else launch_mode<TY, GATE>(a, backward, c, grid, st);
  };
  if constexpr (sizeof(T) == 4) with(Types<T, T>{});
  else if (stream_type == CNN_F32) with(Types<T, float>{});
  else with(Types<T, T>{});
}

}  // namespace norm
}  // namespace cnn
