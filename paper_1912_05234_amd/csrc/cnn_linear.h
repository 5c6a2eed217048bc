// Linear attention with a decay for each head, over whole sequences.
//
//   S_t = a S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t
//
// taken in chunks of C tokens, t counted from the chunk's start and S the state before it:
//
//   O = scale ( a^{t+1} Q S + (a^{t-s} [s <= t] Q K^T) V ),   S' = a^C S + sum_s k_s (a^{C-1-s} v_s)^T
//
// so that almost everything is a matrix product, and every power of a has an exponent that is not negative.
//
// The gradients are the same operator with other roles (d_q: q' = d_o, k' = v, v' = k; d_k: q' = v, k' = d_o, v' = q; d_v: q' = k,
// k' = q, v' = d_o, the last two with time reversed), so one kernel serves all four.  Below, q, k, v are a role's, DK is the
// width of its q and k, DV that of its v and out.
//
// A workgroup takes a block of DV columns of one sequence and head, and walks the chunks of its segment of the time axis; the
// state stays in the accumulators of the matrix instructions, fp32, each wave holding 16 NW columns.  Where there are too few
// heads to fill the GPU the time axis is cut into segments: a first pass finds what each segment adds to the state, a scan over
// the segments turns that into the state that each starts from, and the second pass runs them side by side.
//
// Operands are bfloat16 pieces (x = h + m + l, eight bits each): a bfloat16 is one piece, a half two, a float three, and products
// of two pieces are left out where they are below the last bit kept (2^-16 of the result for halves, 2^-24 for floats).
// What the kernel computes itself is not rounded to the input's type: state and scores are cut into two pieces (three for floats),
// a^{C-1-s} v_s into three, so that the state is exact to fp32 sums for every type.
#pragma once

#include "cnn_common.h"
#include "cnn_types.h"

namespace cnn {
namespace linear {

using bf8 = __bf16 __attribute__((ext_vector_type(8)));
using bf2 = __bf16 __attribute__((ext_vector_type(2)));
using f4 = float __attribute__((ext_vector_type(4)));
using f2 = float __attribute__((ext_vector_type(2)));
using s4 = short __attribute__((ext_vector_type(4)));

struct Operand {  // [batch][token][head][width], strides in elements, the last one is 1
  const void* data;
  int64_t batch, token, head;
  int share;  // query heads that use one head of it
};

struct Role {
  Operand q, k, v;
  void* out;  // [batch][token][head][DV], contiguous; float where `wide`, else of the element type
  const float* first;  // state before the sequence, nullable: element (i, j) of unit u at u * DK * DV + i * first_i + j * first_j
  float* last;         // state after it, nullable, [unit][DK][DV]
  float* carry;        // [unit][segment][DK][DV]
  int first_i, first_j;
  int DK, DV, blocks;  // blocks of columns
  float scale, first_by, last_by;
  int reversed;  // the last token of a sequence comes first; the first state then already stands at the first token
  int wide, packed;  // packed: rows are made of whole packs of eight elements at addresses that are multiples of 16 bytes
};

constexpr int ROLES = 3;
struct Args {
  Role role[ROLES];
  const float* decay;      // [heads]
  const int32_t* lengths;  // [batch], nullable
  int64_t units, T, segment_length;  // units: sequences times heads
  int heads, segments;
};

template <class T>
constexpr int PIECES = sizeof(T) == 4 ? 3 : 2;
template <>
inline constexpr int PIECES<__bf16> = 1;
constexpr int at_least_two(int n) { return n < 2 ? 2 : n; }

__device__ __forceinline__ f4 mfma(bf8 a, bf8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// c += a b from the pieces' products down to the last piece of the longer operand, small ones first.
template <int NA, int NB>
__device__ __forceinline__ f4 product(const bf8 (&a)[NA], const bf8 (&b)[NB], f4 c) {
  constexpr int LAST = (NA > NB ? NA : NB) - 1;
#pragma unroll
  for (int s = LAST; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < NA; ++i)
      if (s - i >= 0 && s - i < NB) c = mfma(a[i], b[s - i], c);
  return c;
}

// Pieces of eight floats, each rounded to nearest.
template <int N>
__device__ __forceinline__ void cut(const float (&x)[8], bf8 (&piece)[N]) {
  float rest[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) rest[j] = x[j];
#pragma unroll
  for (int p = 0; p < N; ++p) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const bf2 h = __builtin_convertvector(f2{rest[j], rest[j + 1]}, bf2);
      piece[p][j] = h[0], piece[p][j + 1] = h[1];
      if (p + 1 < N) rest[j] -= (float)h[0], rest[j + 1] -= (float)h[1];
    }
  }
}

// Four rows of one column of a row-major tile in LDS: lane (g, r) gives the address of elements 4 (r % 4) .. + 3 (of the sixteen
// columns wanted) of row 4 g + r / 4 and receives rows 4 g .. 4 g + 3 of column r.
__device__ __forceinline__ s4 read_transposed(const __bf16* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)(p));
}
__device__ __forceinline__ bf8 joined(s4 a, s4 b) {
  using s8 = short __attribute__((ext_vector_type(8)));
  return __builtin_bit_cast(bf8, s8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
}

// Shape of a kernel: DKP columns of q and k (DK padded with zeros), chunks of 16 CT tokens, WAVES waves of 16 NW columns each.
template <class T, int DKP, int CT, int WAVES, int NW>
struct Shape {
  static constexpr int C = 16 * CT, DVC = WAVES * 16 * NW, THREADS = 64 * WAVES;
  static constexpr int NP = PIECES<T>, MP = at_least_two(NP);  // pieces of the inputs, and of state and scores
  // rows of q and k are read sixteen bytes to a lane, of v and k also four rows to a lane: the padding spreads them over the banks
  static constexpr int QS = DKP + 8, VS = DVC + 16;
  static constexpr int K = 0, V = K + NP * C * QS, Q = V + NP * C * VS, P = Q + NP * C * QS;  // offsets of the tiles in LDS
  static constexpr int TILES = CT * (CT + 1) / 2;  // of the scores, on and below the diagonal
  static constexpr int ALL = P + TILES * MP * 256;
};

// Units of eight elements of a tile that a thread brings from memory to LDS.
template <class T, int ROWS, int WIDTH, int THREADS>
struct Stage {
  static constexpr int UNITS = ROWS * WIDTH / 8, EACH = (UNITS + THREADS - 1) / THREADS;
  Pack<T, 8> u[EACH];

  // rows t0 .. of a sequence of n tokens; zeros past it and past `width`
  __device__ __forceinline__ void load(const T* base, int64_t stride, int64_t t0, int64_t n, int width, bool reversed, bool packed) {
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int i = e * THREADS + threadIdx.x, c = i % (WIDTH / 8) * 8;
      const int64_t t = t0 + i / (WIDTH / 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) u[e].v[j] = (T)0.0f;
      if (i >= UNITS || t >= n || c >= width) continue;
      const T* row = base + (reversed ? n - 1 - t : t) * stride + c;
      if (packed) {
        u[e] = *reinterpret_cast<const Pack<T, 8>*>(row);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (c + j < width) u[e].v[j] = row[j];
      }
    }
  }

  template <int STRIDE>
  __device__ __forceinline__ void store(__bf16* tile) const {  // NP planes of [ROWS][STRIDE]
    constexpr int NP = PIECES<T>;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int i = e * THREADS + threadIdx.x, at = i / (WIDTH / 8) * STRIDE + i % (WIDTH / 8) * 8;
      if (i >= UNITS) continue;
      bf8 piece[NP];
      if constexpr (NP == 1) {
        piece[0] = __builtin_bit_cast(bf8, u[e]);
      } else {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)u[e].v[j];
        cut<NP>(x, piece);
      }
#pragma unroll
      for (int p = 0; p < NP; ++p) *reinterpret_cast<bf8*>(tile + p * ROWS * STRIDE + at) = piece[p];
    }
  }
};

// log2 of a decay, finite also for a = 0 (a^0 = 1 and a^n = 0 then come out right), to fp32 also next to 1.
__device__ __forceinline__ float log2_decay(float a) {
  const double l = log2((double)a);
  return l > -1.0e4 ? (float)l : -1.0e4f;
}
__device__ __forceinline__ float power(float log2a, int e) { return __builtin_amdgcn_exp2f(log2a * (float)e); }

template <class T, int DKP, int CT, int WAVES, int NW, bool STATE_ONLY>
__global__ __launch_bounds__(64 * WAVES) void scan_kernel(Args args) {
  using S = Shape<T, DKP, CT, WAVES, NW>;
  constexpr int C = S::C, THREADS = S::THREADS, NP = S::NP, MP = S::MP, KS = CT / 2, M = DKP / 16;
  __shared__ __align__(16) __bf16 tile[STATE_ONLY ? S::Q : S::ALL];
  const Role& R = args.role[blockIdx.y];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;

  const int64_t job = blockIdx.x / R.blocks, unit = job / args.segments;
  const int segment = (int)(job % args.segments), block = (int)(blockIdx.x % R.blocks);
  if (unit >= args.units) return;  // (a role of fewer column blocks has fewer workgroups)
  const int64_t batch = unit / args.heads;
  const int head = (int)(unit % args.heads), dv0 = block * S::DVC;
  const int64_t n = args.lengths ? (args.lengths[batch] < 0 ? 0 : args.lengths[batch] < args.T ? args.lengths[batch] : args.T) : args.T;
  const int64_t begin = segment * args.segment_length, end = begin + args.segment_length < args.T ? begin + args.segment_length : args.T;
  const int DK = R.DK, DV = R.DV, width = DV - dv0 < S::DVC ? DV - dv0 : S::DVC;
  const bool reversed = R.reversed, packed = R.packed;
  const auto base = [&](const Operand& o) { return static_cast<const T*>(o.data) + batch * o.batch + head / o.share * o.head; };
  const T *q = base(R.q), *k = base(R.k), *v = base(R.v) + dv0;
  const float log2a = log2_decay(args.decay[head]);

  // S: tile m of sixteen rows, register i: row 32 (m / 2) + 8 g + 4 (m % 2) + i, so that a pair of tiles is the second operand of a
  // product over 32 rows as it is; column 16 (NW wave + w) + r
  const auto row_of = [&](int m, int i) { return 32 * (m >> 1) + 8 * g + 4 * (m & 1) + i; };
  const auto column_of = [&](int w) { return 16 * (NW * wave + w) + r; };
  f4 state[M][NW];
  const bool whole = args.segments == 1;
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int w = 0; w < NW; ++w)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = row_of(m, i), col = dv0 + column_of(w);
        float x = 0.0f;
        if (!STATE_ONLY && row < DK && col < DV) {
          if (!whole) x = R.carry[((unit * args.segments + segment) * DK + row) * DV + col];
          else if (R.first) x = R.first[unit * DK * DV + (int64_t)row * R.first_i + (int64_t)col * R.first_j] * R.first_by;
        }
        state[m][w][i] = x;
      }
  int shift = reversed && begin == 0 ? 0 : 1;  // powers of a between the state before the chunk and the chunk's first token

  Stage<T, C, DKP, THREADS> q_in, k_in;
  Stage<T, C, S::DVC, THREADS> v_in;
  const auto load = [&](int64_t t0) {
    if (!STATE_ONLY) q_in.load(q, R.q.token, t0, n, DK, reversed, packed);
    k_in.load(k, R.k.token, t0, n, DK, reversed, packed);
    v_in.load(v, R.v.token, t0, n, width, reversed, packed);
  };
  const int64_t busy = end < n ? end : n;  // where the sequence, or the segment, ends
  if (begin < busy) load(begin);
  for (int64_t t0 = begin; t0 < busy; t0 += C) {
    const int count = busy - t0 < C ? (int)(busy - t0) : C;
    if (!STATE_ONLY) q_in.template store<S::QS>(tile + S::Q);
    k_in.template store<S::QS>(tile + S::K);
    v_in.template store<S::VS>(tile + S::V);
    __syncthreads();
    if (t0 + C < busy) load(t0 + C);

    f4 acc[CT][NW];
    if constexpr (!STATE_ONLY) {
      // scores, transposed: columns t, rows s; four consecutive s to a lane are half an operand of the product with V
      for (int i = wave; i < S::TILES; i += WAVES) {
        const int tt = i < 1 ? 0 : i < 3 ? 1 : i < 6 ? 2 : 3, st = i - tt * (tt + 1) / 2;
        f4 p{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < DKP / 32; ++s) {
          bf8 a[NP], b[NP];
#pragma unroll
          for (int z = 0; z < NP; ++z) {
            a[z] = *reinterpret_cast<const bf8*>(tile + S::K + (z * C + 16 * st + r) * S::QS + 32 * s + 8 * g);
            b[z] = *reinterpret_cast<const bf8*>(tile + S::Q + (z * C + 16 * tt + r) * S::QS + 32 * s + 8 * g);
          }
          p = product(a, b, p);
        }
        const int e = 16 * (tt - st) + r - 4 * g;  // t - s of register 0
        float rest[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) rest[j] = e >= j ? p[j] * power(log2a, e - j) : 0.0f;
#pragma unroll
        for (int z = 0; z < MP; ++z) {
          const bf2 h0 = __builtin_convertvector(f2{rest[0], rest[1]}, bf2), h1 = __builtin_convertvector(f2{rest[2], rest[3]}, bf2);
          *reinterpret_cast<bf2*>(tile + S::P + ((i * MP + z) * 64 + lane) * 4) = h0;
          *reinterpret_cast<bf2*>(tile + S::P + ((i * MP + z) * 64 + lane) * 4 + 2) = h1;
          rest[0] -= (float)h0[0], rest[1] -= (float)h0[1], rest[2] -= (float)h1[0], rest[3] -= (float)h1[1];
        }
      }
      // Q S
#pragma unroll
      for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int w = 0; w < NW; ++w) acc[t][w] = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < M / 2; ++s) {
        bf8 b[NW][MP];
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const f4 lo = state[2 * s][w], hi = state[2 * s + 1][w];
          const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
          cut<MP>(x, b[w]);
        }
#pragma unroll
        for (int t = 0; t < CT; ++t) {
          bf8 a[NP];
#pragma unroll
          for (int z = 0; z < NP; ++z) a[z] = *reinterpret_cast<const bf8*>(tile + S::Q + (z * C + 16 * t + r) * S::QS + 32 * s + 8 * g);
#pragma unroll
          for (int w = 0; w < NW; ++w) acc[t][w] = product(a, b[w], acc[t][w]);
        }
      }
#pragma unroll
      for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float by = power(log2a, 16 * t + 4 * g + i + shift);
#pragma unroll
          for (int w = 0; w < NW; ++w) acc[t][w][i] *= by;
        }
      __syncthreads();  // the scores are there
    }

    // the state: decayed, and the chunk's products added
    const float by = power(log2a, count + shift - 1);
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int i = 0; i < 4; ++i) state[m][w][i] *= by;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      bf8 b[NW][3];
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        bf8 raw[NP];
#pragma unroll
        for (int z = 0; z < NP; ++z) {
          const __bf16* p = tile + S::V + (z * C + 32 * s + 4 * g + (r >> 2)) * S::VS + 16 * (NW * wave + w) + 4 * (r & 3);
          raw[z] = joined(read_transposed(p), read_transposed(p + 16 * S::VS));
        }
        if constexpr (!STATE_ONLY) {
          // scores times V; the tile above the diagonal is zero
#pragma unroll
          for (int t = 2 * s; t < CT; ++t) {
            bf8 a[MP];
#pragma unroll
            for (int z = 0; z < MP; ++z) {
              const int i = t * (t + 1) / 2 + 2 * s;
              const s4 lo = *reinterpret_cast<const s4*>(tile + S::P + ((i * MP + z) * 64 + lane) * 4);
              s4 hi{0, 0, 0, 0};
              if (2 * s + 1 <= t) hi = *reinterpret_cast<const s4*>(tile + S::P + (((i + 1) * MP + z) * 64 + lane) * 4);
              a[z] = joined(lo, hi);
            }
            acc[t][w] = product(a, raw, acc[t][w]);
          }
        }
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = 0.0f;
#pragma unroll
          for (int z = NP - 1; z >= 0; --z) x[j] += (float)raw[z][j];
          const int e = count - 1 - (32 * s + 16 * (j >> 2) + 4 * g + (j & 3));  // tokens that follow in the chunk
          x[j] = e >= 0 ? x[j] * power(log2a, e) : 0.0f;
        }
        cut<3>(x, b[w]);
      }
#pragma unroll
      for (int m = 0; m < M; ++m) {
        bf8 a[NP];
#pragma unroll
        for (int z = 0; z < NP; ++z) {
          const __bf16* p = tile + S::K + (z * C + 32 * s + 4 * g + (r >> 2)) * S::QS + 32 * (m >> 1) + 8 * (r & 3) + 4 * (m & 1);
          a[z] = joined(read_transposed(p), read_transposed(p + 16 * S::QS));
        }
#pragma unroll
        for (int w = 0; w < NW; ++w) state[m][w] = product(a, b[w], state[m][w]);
      }
    }
    if constexpr (!STATE_ONLY) {
#pragma unroll
      for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = 16 * t + 4 * g + i;
          if (at >= count) continue;
          const int64_t token = reversed ? n - 1 - (t0 + at) : t0 + at;
          const int64_t row = ((batch * args.T + token) * args.heads + head) * DV;
#pragma unroll
          for (int w = 0; w < NW; ++w) {
            const int col = column_of(w);
            if (col >= width) continue;
            const float x = acc[t][w][i] * R.scale;
            if (R.wide) static_cast<float*>(R.out)[row + dv0 + col] = x;
            else static_cast<T*>(R.out)[row + dv0 + col] = (T)x;
          }
        }
    }
    shift = 1;
    __syncthreads();  // the tiles may be overwritten
  }

  if constexpr (!STATE_ONLY) {  // rows past the sequence are zero
    const int64_t from = begin > n ? begin : n;
    for (int64_t i = threadIdx.x; i < (end - from) * width; i += THREADS) {
      const int64_t at = ((batch * args.T + from + i / width) * args.heads + head) * DV + dv0 + i % width;
      if (R.wide) static_cast<float*>(R.out)[at] = 0.0f;
      else static_cast<T*>(R.out)[at] = (T)0.0f;
    }
  }
  if (STATE_ONLY || (whole && R.last)) {
    // a reversed sequence's state stands at its first token; one decay more and the scale make it the error of the state before it
    const float by = STATE_ONLY || n == 0 ? 1.0f : R.last_by * (reversed ? args.decay[head] : 1.0f);
    float* to = STATE_ONLY ? R.carry + (unit * args.segments + segment) * DK * DV : R.last + unit * DK * DV;
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = row_of(m, i), col = dv0 + column_of(w);
          if (row >= DK || col >= DV) continue;
          float x = state[m][w][i] * by;
          if (!STATE_ONLY && n == 0) x = R.first ? R.first[unit * DK * DV + (int64_t)row * R.first_i + (int64_t)col * R.first_j] : 0.0f;
          to[(int64_t)row * DV + col] = x;
        }
  }
}

// ---- launches, one translation unit to each element type ---------------------------------------------------------------
constexpr int padded(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : d <= 128 ? 128 : 256; }
// Columns of a workgroup: all of a narrow role's, else 128, or 64 where the state has 256 rows, so that it takes 64 registers.
constexpr int block_columns(int DK, int DV) { return DV <= 32 ? 32 : DV <= 64 || DK > 128 ? 64 : 128; }

template <class T, int DKP, int WAVES, int NW>
int launch_scan(const Args& a, int roles, bool state_only, hipStream_t st) {
  constexpr int CT = sizeof(T) == 2 && PIECES<T> == 1 ? 4 : 2;  // chunks of 64 tokens of one piece, of 32 of more
  int blocks = 1;
  for (int r = 0; r < roles; ++r) blocks = a.role[r].blocks > blocks ? a.role[r].blocks : blocks;
  const dim3 grid((unsigned)(a.units * a.segments * blocks), (unsigned)roles);
  if (state_only) scan_kernel<T, DKP, CT, WAVES, NW, true><<<grid, 64 * WAVES, 0, st>>>(a);
  else scan_kernel<T, DKP, CT, WAVES, NW, false><<<grid, 64 * WAVES, 0, st>>>(a);
  return launch_status();
}

template <class T, int DKP>
int launch_scan(const Args& a, int roles, int columns, bool state_only, hipStream_t st) {
  if (columns == 32) return launch_scan<T, DKP, 2, 1>(a, roles, state_only, st);
  if constexpr (DKP < 256)
    if (columns == 128) return launch_scan<T, DKP, 4, 2>(a, roles, state_only, st);
  return launch_scan<T, DKP, 4, 1>(a, roles, state_only, st);
}

// One pass of all roles; those of one shape in one launch.
template <class T>
int run_scan(const Args& all, int roles, bool state_only, hipStream_t st) {
  for (int r = 0; r < roles;) {
    Args a = all;
    const int dk = padded(all.role[r].DK), columns = block_columns(all.role[r].DK, all.role[r].DV);
    int same = 0;
    for (; r + same < roles; ++same) {
      const Role& o = all.role[r + same];
      if (padded(o.DK) != dk || block_columns(o.DK, o.DV) != columns) break;
      a.role[same] = o;
    }
    const int rc = dk == 32    ? launch_scan<T, 32>(a, same, columns, state_only, st)
                   : dk == 64  ? launch_scan<T, 64>(a, same, columns, state_only, st)
                   : dk == 128 ? launch_scan<T, 128>(a, same, columns, state_only, st)
                               : launch_scan<T, 256>(a, same, columns, state_only, st);
    if (rc != CNN_OK) return rc;
    r += same;
  }
  return CNN_OK;
}

int run_scan_f32(const Args& a, int roles, bool state_only, hipStream_t st);
int run_scan_bf16(const Args& a, int roles, bool state_only, hipStream_t st);
int run_scan_f16(const Args& a, int roles, bool state_only, hipStream_t st);

}  // namespace linear
}  // namespace cnn
