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
// A workgroup takes a block of DV columns (32 to 128, a wave to 32) of one sequence and head, and walks the chunks of its segment of the time axis; the
// state stays in the accumulators of the matrix instructions, fp32, each wave holding 32 columns.  Where there are too few
// heads to fill the GPU the time axis is cut into segments: a first pass finds what each segment adds to the state, a scan over
// the segments turns that into the state that each starts from, and the second pass runs them side by side.
//
// Operands are bfloat16 pieces (x = h + m + l, eight bits each): a bfloat16 is one piece, a half two, a float three, and products
// of two pieces are left out where they are below the last bit kept (2^-16 of the result for halves, 2^-24 for floats).
// What the kernel computes itself is not rounded to the input's type: state and scores are cut into two pieces (2^-17 of each is
// lost, of results that are rounded to 2^-9 or 2^-12), three for floats; a^{C-1-s} v_s into three, so that the state is exact to fp32
// sums for every type, or two in the second pass over segments, whose own state is no result.
//
// Measured (MI355X; in brackets the bytes that have to be moved at a copy's 5.15 TB/s): 8192 tokens of 2 x 16 heads of 128 (bf16) 118 us
// (53): 32 for the first pass, 14 for the scan over 16 segments, 72 for the second pass, in which a SIMD's two waves issue vector
// instructions, most of them cutting and decaying the state, 60 % of the time and its matrix unit is busy 35 %.  100 x 2 heads of 784 tokens,
// 32 wide (fp32): 33 us forward on uneven lengths (10), 72 us backward (27), bound by the cutting of floats, some 840 vector instructions
// for 32 tokens and a role, with what stands around the loop.  3 x 12 heads of 2047 tokens, 64 and 96 wide (fp16), backward: 105 us (10),
// of six dependent launches.
#pragma once

#include <type_traits>

#include "cnn_common.h"
#include "cnn_types.h"

namespace cnn {
namespace linear {

using bf8 = __bf16 __attribute__((ext_vector_type(8)));
using bf2 = __bf16 __attribute__((ext_vector_type(2)));
using f4 = float __attribute__((ext_vector_type(4)));
using f2 = float __attribute__((ext_vector_type(2)));
using s4 = short __attribute__((ext_vector_type(4)));
using bf4 = __bf16 __attribute__((ext_vector_type(4)));

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
  float* carry;        // [unit][segment], states in the order of the kernel's registers
  const float* flipped;  // instead: those of a role whose states are this one's transposed
  int first_i, first_j;
  int DK, DV, DKP, columns, blocks;  // DK padded, columns of a workgroup, workgroups to a state
  int flipped_rows;                  // DKP of that role
  int64_t flipped_floats;            // of one of its states
  float scale;    // of out
  float inside;   // of what the tokens add to the state: the scale where the state before the sequence already holds it
  float last_by;  // of the state after it: the scale where neither the tokens nor the state before them hold it
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

// Tokens of a sequence, and of one of its segments: these end where the sequence does, the first of them may be short or empty.
__device__ __forceinline__ int64_t length_of(const Args& a, int64_t batch) {
  if (!a.lengths) return a.T;
  const int64_t n = a.lengths[batch];
  return n < 0 ? 0 : n < a.T ? n : a.T;
}
__device__ __forceinline__ int64_t segment_end(const Args& a, int64_t n, int segment) {
  const int64_t e = n - (a.segments - 1 - segment) * a.segment_length;
  return e > 0 ? e : 0;
}
__device__ __forceinline__ int64_t segment_begin(const Args& a, int64_t n, int segment) { return segment_end(a, n, segment - 1); }

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

// Shape of a kernel: DKP columns of q and k (DK padded with zeros), WAVES waves of 32 columns of v (NW tiles of 16), chunks of 32
// tokens: products over the tokens of a chunk are one step of the matrix instruction, and the scores are three of its tiles, which
// every wave computes for itself.
constexpr int C = 32, NW = 2;
template <class T, int DKP, int WAVES>
struct Shape {
  static constexpr int DVC = WAVES * 16 * NW, THREADS = 64 * WAVES;
  static constexpr int NP = PIECES<T>, MP = at_least_two(NP);  // pieces of the inputs, and of state and scores
  // rows of q and k are read sixteen bytes to a lane, of v and k also four rows to a lane: the padding spreads them over the banks
  static constexpr int QS = DKP + 8, VS = DVC + 16;
  // A single wave of narrow rows takes q from memory in the order of its operands: without it in LDS eight waves of floats fit a
  // compute unit, not six.
  static constexpr bool Q_DIRECT = WAVES == 1 && DKP == 32;
  // Columns of v belong to one wave each.  Floats come from memory in the order of its operands; elements of 16 bits pass through LDS,
  // whose reads turn the tile, and are cut after that: the uncut number is wanted too.
  static constexpr bool V_DIRECT = sizeof(T) == 4;
  static constexpr int K = 0, V = K + NP * C * QS, Q = V + (V_DIRECT ? 0 : C * VS), ALL = Q + (Q_DIRECT ? 0 : NP * C * QS);  // offsets of the tiles in LDS
  // two sets of tiles, and one barrier a chunk, where eight waves of a compute unit have room for them
  static constexpr int SETS = 2 * ALL * 2 <= 20 * 1024 * WAVES ? 2 : 1;
};

// Units of eight elements of a tile that a thread brings from memory to LDS: one column of units, every STEP-th row.
//
// Rows that are no tokens (before `pad`, in a sequence's first chunk) and columns past the width repeat others, so that the loads
// need no branches; what they add to a result is zero because k's are zeros in LDS: clear() and blank() see to that.
template <class T, int ROWS, int WIDTH, int THREADS>
struct Stage {
  static constexpr int COLUMNS = WIDTH / 8, STEP = THREADS / COLUMNS, EACH = (ROWS + STEP - 1) / STEP;
  // Threads past STEP whole rows bring in the next row's units a second time; rows past the last are left out.
  static constexpr bool PAST = ROWS % STEP != 0 || THREADS % COLUMNS != 0;
  Pack<T, 8> u[EACH];
  uint32_t at[EACH];  // PACKED: bytes from the chunk's lowest address, which is row 0's, or in reversed order the last row's
  int width, stride;  // in elements

  __device__ __forceinline__ int column() const { return threadIdx.x % COLUMNS * 8; }
  __device__ __forceinline__ int row(int e) const {
    const int r = threadIdx.x / COLUMNS + e * STEP;
    return PAST && r >= ROWS ? ROWS - 1 : r;
  }
  __device__ __forceinline__ int place(int row, int pad, bool reversed) const {
    row = row > pad ? row : pad;
    return reversed ? ROWS - 1 - row : row;
  }
  __device__ __forceinline__ void set(int columns, int64_t token_stride, int pad, bool reversed) {
    width = columns, stride = (int)token_stride;
    const int c = column() < width ? column() : 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e)  // (rows of a chunk are less than 2^31 bytes apart)
      at[e] = __umul24(place(row(e), pad, reversed), (uint32_t)stride * (uint32_t)sizeof(T)) + c * (uint32_t)sizeof(T);
  }
  __device__ __forceinline__ void load(const T* low) {
#pragma unroll
    for (int e = 0; e < EACH; ++e) u[e] = *reinterpret_cast<const Pack<T, 8>*>(reinterpret_cast<const char*>(low) + at[e]);
  }
  // the same element by element, for any width, stride and alignment
  __device__ __forceinline__ void load_any(const T* low, int64_t token_stride, int columns, int pad, bool reversed) {
    const int c = column();
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const T* from = low + place(row(e), pad, reversed) * token_stride;
#pragma unroll
      for (int j = 0; j < 8; ++j) u[e].v[j] = c + j < columns ? from[c + j] : (T)0.0f;
    }
  }

  // Rows before `pad` as zeros.
  __device__ __forceinline__ void clear(int pad) {
#pragma unroll
    for (int e = 0; e < EACH; ++e)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if ((int)threadIdx.x / COLUMNS + e * STEP < pad) u[e].v[j] = (T)0.0f;
  }

  // planes of [ROWS][STRIDE], one to a piece, or one of uncut elements of 16 bits; `all`: columns past the width too
  template <int STRIDE, bool UNCUT = false>
  __device__ __forceinline__ void store(__bf16* tile, bool all) const {
    constexpr int NP = UNCUT ? 1 : PIECES<T>;
    if (!all && column() >= width) return;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int r = threadIdx.x / COLUMNS + e * STEP;
      if (PAST && r >= ROWS) continue;
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
      for (int p = 0; p < NP; ++p) *reinterpret_cast<bf8*>(tile + (p * ROWS + r) * STRIDE + column()) = piece[p];
    }
  }
  // columns past the width as zeros, once
  template <int STRIDE>
  __device__ __forceinline__ void blank(__bf16* tile) const {
    if (column() < width) return;
    for (int r = threadIdx.x / COLUMNS; r < PIECES<T> * ROWS; r += STEP) *reinterpret_cast<bf8*>(tile + r * STRIDE + column()) = bf8{};
  }
};

__host__ __device__ constexpr int padded(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : d <= 96 ? 96 : d <= 128 ? 128 : 256; }
// Columns of a workgroup, 32 to a wave, as few as the number of workgroups allows.  (One wave brings in the rows of at most 64
// columns of q and k by itself, two of 128.)
__host__ __device__ constexpr int block_columns(int DK, int DV) {
  if (DV <= 32 && DK <= 64) return 32;
  if (DV <= 64 && DK <= 128) return 64;
  return DK <= 128 && (DV + 95) / 96 == (DV + 127) / 128 ? 96 : 128;
}
// Floats of a state as the kernel holds it.
__host__ __device__ inline int64_t carry_floats(const Role& r) { return (int64_t)r.DKP * r.blocks * r.columns; }

// Rows of q of a single wave, as operands of its products: row 16 t + lane % 16, columns 32 s + 8 (lane / 16) .. + 7.
template <class T, int DKP>
struct Direct {
  static constexpr int ST = DKP / 32;
  Pack<T, 8> u[2][ST];
  uint32_t at[2];
  int column;  // as far as it is one; a column past the width meets zeros of k

  __device__ __forceinline__ int place(int t, int pad, bool reversed) const {
    int row = 16 * t + (threadIdx.x & 15);
    row = row > pad ? row : pad;
    return reversed ? C - 1 - row : row;
  }
  __device__ __forceinline__ void set(int width, int64_t token_stride, int pad, bool reversed) {
    column = threadIdx.x / 16 % 4 * 8 < width ? threadIdx.x / 16 % 4 * 8 : 0;
#pragma unroll
    for (int t = 0; t < 2; ++t) at[t] = __umul24(place(t, pad, reversed), (uint32_t)token_stride * (uint32_t)sizeof(T)) + column * (uint32_t)sizeof(T);
  }
  __device__ __forceinline__ void load(const T* low) {
    static_assert(ST == 1, "columns of one step");
#pragma unroll
    for (int t = 0; t < 2; ++t) u[t][0] = *reinterpret_cast<const Pack<T, 8>*>(reinterpret_cast<const char*>(low) + at[t]);
  }
  __device__ __forceinline__ void load_any(const T* low, int64_t token_stride, int width, int pad, bool reversed) {
    const int c = threadIdx.x / 16 % 4 * 8;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const T* from = low + place(t, pad, reversed) * token_stride;
#pragma unroll
      for (int j = 0; j < 8; ++j) u[t][0].v[j] = c + j < width ? from[c + j] : (T)0.0f;
    }
  }
  template <int NP>
  __device__ __forceinline__ void pieces(bf8 (&out)[2][NP]) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if constexpr (NP == 1) {
        out[t][0] = __builtin_bit_cast(bf8, u[t][0]);
      } else {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)u[t][0].v[j];
        cut<NP>(x, out[t]);
      }
    }
  }
};

// Columns of v of one wave as operands: eight tokens, 16 (j / 4) + 4 (lane / 16) + j % 4, of column lane % 16 of each of its tiles.
template <class T>
struct Columns {
  T u[NW][8];
  uint32_t at[NW];  // bytes from the row that its place in the wave does not change

  __device__ __forceinline__ int column(int w) const { return (threadIdx.x >> 6) * 16 * NW + 16 * w + (threadIdx.x & 15); }
  __device__ __forceinline__ static int group() { return threadIdx.x >> 4 & 3; }
  __device__ __forceinline__ void set(int width, int64_t token_stride, bool reversed) {
    const uint32_t row = __umul24(reversed ? 12 - 4 * group() : 4 * group(), (uint32_t)token_stride * (uint32_t)sizeof(T));
#pragma unroll
    for (int w = 0; w < NW; ++w) at[w] = row + (column(w) < width ? column(w) : 0) * (uint32_t)sizeof(T);
  }
  __device__ __forceinline__ void load(const T* low, int64_t token_stride, bool reversed) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int place = 16 * (j >> 2) + (j & 3);
      const char* row = reinterpret_cast<const char*>(low + (reversed ? 19 - place : place) * token_stride);
#pragma unroll
      for (int w = 0; w < NW; ++w) u[w][j] = *reinterpret_cast<const T*>(row + at[w]);
    }
  }
  __device__ __forceinline__ void load_any(const T* low, int64_t token_stride, int width, int pad, bool reversed) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      int row = 16 * (j >> 2) + 4 * group() + (j & 3);
      row = row > pad ? row : pad;
      const T* from = low + (reversed ? C - 1 - row : row) * token_stride;
#pragma unroll
      for (int w = 0; w < NW; ++w) u[w][j] = column(w) < width ? from[column(w)] : (T)0.0f;
    }
  }
};

// log2 of a decay, finite also for a = 0 (a^0 = 1 and a^n = 0 then come out right), to fp32 also next to 1; NaN for a NaN, which so shows.
__device__ __forceinline__ float log2_decay(float a) {
  const double l = log2((double)a);
  return l < -1.0e4 ? -1.0e4f : (float)l;
}
__device__ __forceinline__ float power(float log2a, int e) { return __builtin_amdgcn_exp2f(log2a * (float)e); }

// Keeps operands read from LDS for a later step from taking registers now.
__device__ __forceinline__ void in_steps() { __builtin_amdgcn_sched_barrier(0); }
// A number that the compiler takes for a new one, so that nothing computed from it is held through the loop before.
__device__ __forceinline__ int anew(int x) {
  asm volatile("" : "+s"(x));
  return x;
}

using Bytes = __attribute__((address_space(1))) char;  // memory of the GPU
// Waits for the loads from memory that are under way.  The compiler's own waits in a loop allow for what may be pending on any way to
// them: without this one before the loop the products with the state waited in every chunk for the next chunk's rows, and without the
// one before rows are stored to LDS, which some lanes skip, the next loads waited for all stores to memory.
__device__ __forceinline__ void loads_done() { __builtin_amdgcn_s_waitcnt(0x0f70); }  // (vmcnt 0, the other counters at their most)

// Where a state's register i of tile m of a wave's lane stands.  A pair of tiles is an operand of a product over 32 rows as it is.
__device__ __forceinline__ int state_row(int m, int lane, int i) { return 32 * (m >> 1) + 8 * (lane >> 4) + 4 * (m & 1) + i; }
__device__ __forceinline__ int state_column(int tile, int lane) { return 16 * tile + (lane & 15); }  // tile: of sixteen columns
// The other way: index of an element in a state of `tiles` tiles of rows to a tile of columns.
__device__ __forceinline__ uint32_t state_index(int row, int column, int tiles) {
  const int m = 2 * (row >> 5) + (row >> 2 & 1), lane = 16 * (row >> 3 & 3) + (column & 15);
  return (uint32_t)((((column >> 4) * tiles + m) * 64 + lane) * 4 + (row & 3));
}

// Waves to a SIMD, which bound the registers of a kernel.  (Three would spill: the pixel sequences' gradients took 105 us, not 71.)
// Two make floats of 96 and 128 columns of q and k spill 3 to 21 registers where two or three waves share v, and 185 where rows of 128 are
// not made of packs: 8 x 8 heads of 1024 tokens, 128 x 64, forward 74 us (20), of 126 x 62 116 us.  Not changed, not compared with one.
constexpr int waves_wanted(int DKP) { return DKP <= 128 ? 2 : 1; }

// STATE_ONLY: the first pass.  EXACT: the state is a result, not only what the segment's own tokens see.
template <class T, int DKP, int WAVES, bool PACKED, bool STATE_ONLY, bool EXACT>
__global__ __launch_bounds__(64 * WAVES, waves_wanted(DKP)) void scan_kernel(Args args) {
  using S = Shape<T, DKP, WAVES>;
  constexpr int THREADS = S::THREADS, NP = S::NP, MP = S::MP, WP = EXACT ? 3 : MP, M = DKP / 16;
  constexpr int SET = STATE_ONLY ? S::Q : S::ALL;
  __shared__ __align__(16) __bf16 tiles[S::SETS * SET];
  const Role& R = args.role[blockIdx.y];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;

  const int64_t job = blockIdx.x / R.blocks, unit = job / args.segments;
  const int segment = (int)(job % args.segments), block = (int)(blockIdx.x % R.blocks);
  if (unit >= args.units) return;  // (a role of fewer column blocks has fewer workgroups)
  const int64_t batch = unit / args.heads;
  const int head = (int)(unit % args.heads), dv0 = block * S::DVC;
  const int64_t n = length_of(args, batch), end = segment_end(args, n, segment), begin = segment_begin(args, n, segment);
  const int DK = R.DK, DV = R.DV, width = DV - dv0 < S::DVC ? DV - dv0 : S::DVC;
  const bool reversed = R.reversed;

  // Chunks end where the segment does; the first one may begin before it, with `pad` rows that are no tokens.
  int pad = (int)((C - (end - begin) % C) % C);
  std::conditional_t<S::Q_DIRECT, Direct<T, 32>, Stage<T, C, DKP, THREADS>> q_in;
  Stage<T, C, DKP, THREADS> k_in;
  std::conditional_t<S::V_DIRECT, Columns<T>, Stage<T, C, S::DVC, THREADS>> v_in;
  bf8 direct[2][NP];  // q's operands of the present chunk, where they do not pass through LDS
  const int64_t low = reversed ? n - (begin - pad) - C : begin - pad, advance = reversed ? -C : C;  // in tokens
  const auto base = [&](const Operand& o) __attribute__((always_inline)) { return static_cast<const T*>(o.data) + batch * o.batch + head / o.share * o.head + low * o.token; };
  const T *q = base(R.q), *k = base(R.k), *v = base(R.v) + dv0;
  const int64_t q_step = advance * R.q.token, k_step = advance * R.k.token, v_step = advance * R.v.token;
  const auto load_v = [&](int pad, bool first) __attribute__((always_inline)) {
    if constexpr (S::V_DIRECT) {
      if (PACKED && !first) v_in.load(v, R.v.token, reversed);
      else v_in.load_any(v, R.v.token, width, pad, reversed);
    } else {
      if (PACKED) v_in.load(v);
      else v_in.load_any(v, R.v.token, width, pad, reversed);
    }
    v += v_step;
  };
  const auto load = [&](int pad) __attribute__((always_inline)) {
    if constexpr (PACKED) {
      k_in.load(k);
      if (!STATE_ONLY) q_in.load(q);
    } else {
      k_in.load_any(k, R.k.token, DK, pad, reversed);
      if (!STATE_ONLY) q_in.load_any(q, R.q.token, DK, pad, reversed);
    }
    q += q_step, k += k_step;
    if constexpr (!S::V_DIRECT) load_v(pad, false);
  };
  const auto store = [&](__bf16* tile) __attribute__((always_inline)) {
    k_in.template store<S::QS>(tile + S::K, !PACKED);
    if constexpr (!S::V_DIRECT) v_in.template store<S::VS, true>(tile + S::V, true);
    if constexpr (STATE_ONLY) return;
    else if constexpr (S::Q_DIRECT) q_in.pieces(direct);
    else q_in.template store<S::QS>(tile + S::Q, true);
  };
  const auto set = [&](int pad) __attribute__((always_inline)) {
    k_in.set(DK, R.k.token, pad, reversed);
    if constexpr (!S::V_DIRECT) v_in.set(width, R.v.token, pad, reversed);
    if (!STATE_ONLY) q_in.set(DK, R.q.token, pad, reversed);
  };
  set(pad);
  if constexpr (S::V_DIRECT) v_in.set(width, R.v.token, reversed);
  if (begin < end) {
    load(pad);
    if constexpr (S::V_DIRECT) load_v(pad, true);
  }
  if (pad) set(0);
  if (PACKED && DK < DKP)
    for (int i = 0; i < S::SETS; ++i) k_in.template blank<S::QS>(tiles + i * SET + S::K);

  f4 state[M][NW];
  const bool whole = args.segments == 1;
  const int64_t carry_size = (int64_t)DKP * R.blocks * S::DVC;  // [tile of columns][tile of rows][lane][4]
  f4* carry = reinterpret_cast<f4*>(R.carry + (unit * args.segments + segment) * carry_size) + (block * WAVES + wave) * NW * M * 64 + lane;
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int w = 0; w < NW; ++w) state[m][w] = f4{0.0f, 0.0f, 0.0f, 0.0f};
  // Rows 32 m + 8 g + j, j < 8, of a column are registers j % 4 of its tiles 2 m + j / 4.
  const int rows = DK - 8 * g;  // of the state from 8 g on
  if (!STATE_ONLY && !whole && R.flipped) {
    // their columns are rows here: an element's place in their registers, taken apart into what depends on the lane and what does not
    const int tiles = R.flipped_rows / 16;
    const float* from = R.flipped + (unit * args.segments + segment) * R.flipped_floats;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const int column = dv0 + state_column(NW * wave + w, lane);
      if (column >= R.flipped_rows) continue;
      const float* p = from + state_index(column, 8 * g, tiles);
#pragma unroll
      for (int m = 0; m < M / 2; ++m) {
        if (PACKED && 32 * m >= rows) continue;  // (their columns past the width hold something)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (PACKED || 32 * m + j < rows) state[2 * m + (j >> 2)][w][j & 3] = p[4 * j + m * 512 * tiles];
      }
    }
  } else if (!STATE_ONLY && !whole) {
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int w = 0; w < NW; ++w) state[m][w] = carry[(w * M + m) * 64];
  } else if (!STATE_ONLY && R.first) {
    const float* from = R.first + unit * DK * DV;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const int column = state_column(NW * wave + w, lane);
      if (column >= width) continue;
      const float* p = from + 8 * g * R.first_i + (dv0 + column) * R.first_j;
#pragma unroll
      for (int m = 0; m < M / 2; ++m) {
        if (PACKED && 32 * m >= rows) continue;  // whole packs of rows
        if (PACKED && R.first_i == 1) {
          state[2 * m][w] = *reinterpret_cast<const f4*>(p + 32 * m);
          state[2 * m + 1][w] = *reinterpret_cast<const f4*>(p + 32 * m + 4);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (PACKED || 32 * m + j < rows) state[2 * m + (j >> 2)][w][j & 3] = p[(32 * m + j) * R.first_i];
        }
      }
    }
  }
  int shift = reversed && begin == 0 ? 0 : 1;  // powers of a between the state before the chunk and the chunk's first token

  const float log2a = log2_decay(args.decay[head]);
  // weights of the scores, by t - s = 16 (t's tile - s's tile) + r - 4 g - i, and of the tokens in the state at the chunk's end
  float on_diagonal[4], below[4], follow[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = r - 4 * g - i;
    on_diagonal[i] = power(log2a, e > 0 ? e : 0);
    below[i] = power(log2a, 16 + e);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) follow[j] = power(log2a, C - 1 - 16 * (j >> 2) - (j & 3) - 4 * g);
  if (const float inside = R.inside; inside != 1.0f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) on_diagonal[i] *= inside, below[i] *= inside;
#pragma unroll
    for (int j = 0; j < 8; ++j) follow[j] *= inside;
  }

  // out: rows of a chunk are tokens, columns 4 g + i of a tile of sixteen
  const bool wide = R.wide;
  const int out_column = 16 * NW * wave + 4 * g, out_size = wide ? 4 : (int)sizeof(T);
  const int64_t out_stride = (int64_t)args.heads * DV * out_size, out_step = advance * out_stride;  // in bytes
  Bytes* out = (Bytes*)R.out + (((batch * args.T + low) * args.heads + head) * DV + dv0) * out_size;
  uint32_t out_at[2];  // PACKED: rows of a chunk are less than 2^31 bytes apart
#pragma unroll
  for (int t = 0; t < 2; ++t) out_at[t] = (uint32_t)((reversed ? C - 1 - 16 * t - r : 16 * t + r) * (int)out_stride + out_column * out_size);
  const float scale = R.scale;

  __bf16* tile = tiles;
  loads_done();
  if (begin < end) {
    if (pad) k_in.clear(pad);  // what is no token adds nothing
    store(tile);
    __syncthreads();
  }
  for (int64_t t0 = begin - pad; t0 < end; t0 += C) {
    const bool more = t0 + C < end;
    if (more) load(0);

    f4 acc[2][NW];  // of the result, transposed: rows are columns 4 g + i of out, column r is token r
    bf8 score[2][MP];
    if constexpr (!STATE_ONLY) {
      // Q S, and the scores, transposed: columns t, rows s, so that a pair of tiles is an operand of the product with V
      f4 p00{0.0f, 0.0f, 0.0f, 0.0f}, p01 = p00, p11 = p00;  // [s][t]
#pragma unroll
      for (int w = 0; w < NW; ++w) acc[0][w] = acc[1][w] = p00;
#pragma unroll
      for (int s = 0; s < M / 2; ++s) {
        bf8 row[2][NP], query[2][NP];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int z = 0; z < NP; ++z) {
            if constexpr (S::Q_DIRECT) query[t][z] = direct[t][z];
            else query[t][z] = *reinterpret_cast<const bf8*>(tile + S::Q + (z * C + 16 * t + r) * S::QS + 32 * s + 8 * g);
            row[t][z] = *reinterpret_cast<const bf8*>(tile + S::K + (z * C + 16 * t + r) * S::QS + 32 * s + 8 * g);
          }
        p00 = product(row[0], query[0], p00);
        p01 = product(row[0], query[1], p01);
        p11 = product(row[1], query[1], p11);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const f4 lo = state[2 * s][w], hi = state[2 * s + 1][w];
          const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
          bf8 a[MP];
          cut<MP>(x, a);
          acc[0][w] = product(a, query[0], acc[0][w]);
          acc[1][w] = product(a, query[1], acc[1][w]);
        }
        if (NP > 1 || (s & 1)) in_steps();
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int e = 16 * t + r - pad + shift;
        const float by = power(log2a, e > 0 ? e : 0);
#pragma unroll
        for (int w = 0; w < NW; ++w) acc[t][w] *= by;
        float x[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool on = r >= 4 * g + j;
          x[j] = t ? p01[j] * below[j] : on ? p00[j] * on_diagonal[j] : 0.0f;
          x[4 + j] = t && on ? p11[j] * on_diagonal[j] : 0.0f;
        }
        cut<MP>(x, score[t]);
      }
    }

    // the scores' product with V; the state: decayed, and the chunk's products added
    // (the first pass leaves the state as it is and weights each token by what is left of its segment: fewer products)
    const float by = power(log2a, STATE_ONLY ? (int)(end - t0 - C) : C - pad + shift - 1);
    bf8 weighted[NW][WP];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      bf8 raw[NP];
      float x[8];
      if constexpr (S::V_DIRECT) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)v_in.u[w][j];
        cut<NP>(x, raw);
      } else {
        const __bf16* p = tile + S::V + (4 * g + (r >> 2)) * S::VS + 16 * (NW * wave + w) + 4 * (r & 3);
        raw[0] = joined(read_transposed(p), read_transposed(p + 16 * S::VS));
        const auto uncut = __builtin_bit_cast(Pack<T, 8>, raw[0]);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)uncut.v[j];
        if constexpr (NP > 1) cut<NP>(x, raw);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] *= STATE_ONLY ? follow[j] * by : follow[j];
      cut<WP>(x, weighted[w]);
      if constexpr (!STATE_ONLY) {
        acc[0][w] = product(raw, score[0], acc[0][w]);
        acc[1][w] = product(raw, score[1], acc[1][w]);
      }
    }
    if constexpr (S::V_DIRECT)
      if (more) load_v(0, false);
#pragma unroll
    for (int m = 0; m < M; ++m) {
      bf8 a[NP];
#pragma unroll
      for (int z = 0; z < NP; ++z) {
        const __bf16* p = tile + S::K + (z * C + 4 * g + (r >> 2)) * S::QS + 32 * (m >> 1) + 8 * (r & 3) + 4 * (m & 1);
        a[z] = joined(read_transposed(p), read_transposed(p + 16 * S::QS));
      }
#pragma unroll
      for (int w = 0; w < NW; ++w) state[m][w] = product(a, weighted[w], STATE_ONLY ? state[m][w] : state[m][w] * by);
      if ((m & 3) == 3 || (NP > 1 && (m & 1))) in_steps();
    }

    __bf16* const next = S::SETS == 1 || tile != tiles ? tiles : tiles + SET;
    if constexpr (S::SETS == 1) __syncthreads();  // the tiles may be overwritten
    loads_done();
    if (more) store(next);
    if constexpr (!STATE_ONLY) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (16 * t + r < pad) continue;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const f4 y = acc[t][w] * scale;
          if constexpr (PACKED) {  // whole packs, so width is a multiple of eight
            if (out_column + 16 * w >= width) continue;
            using Four = std::conditional_t<sizeof(T) == 4, f4, f2>;
            const Four narrow = __builtin_bit_cast(Four, Pack<T, 4>{{(T)y[0], (T)y[1], (T)y[2], (T)y[3]}});
            if (wide) *(__attribute__((address_space(1))) f4*)(out + out_at[t] + 64 * w) = y;
            else *(__attribute__((address_space(1))) Four*)(out + out_at[t] + 16 * w * (int)sizeof(T)) = narrow;
          } else {
            Bytes* const to = out + (reversed ? C - 1 - 16 * t - r : 16 * t + r) * out_stride + (out_column + 16 * w) * out_size;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (out_column + 16 * w + i >= width) continue;
              if (wide) ((__attribute__((address_space(1))) float*)to)[i] = y[i];
              else ((__attribute__((address_space(1))) T*)to)[i] = (T)y[i];
            }
          }
        }
      }
      out += out_step;
    }
    shift = 1, pad = 0, tile = next;
    __syncthreads();
  }

  if constexpr (!STATE_ONLY) {  // rows past the sequence are zero; the segments share them out
    const int64_t past = args.T - n, first = n + past * segment / args.segments, last = n + past * (segment + 1) / args.segments;
    constexpr int LANES = S::DVC / 4, ROWS = THREADS / LANES;
    const int column = threadIdx.x % LANES * 4;
    for (int64_t t = first + threadIdx.x / LANES; t < last; t += ROWS) {
      const int64_t at = ((batch * args.T + t) * args.heads + head) * DV + dv0 + column;
      if (PACKED && column < width) {
        if (wide) *reinterpret_cast<f4*>(static_cast<float*>(R.out) + at) = f4{0.0f, 0.0f, 0.0f, 0.0f};
        else *reinterpret_cast<Pack<T, 4>*>(static_cast<T*>(R.out) + at) = Pack<T, 4>{};
      }
      if (!PACKED)
        for (int i = 0; i < 4; ++i) {
          if (column + i >= width) continue;
          if (wide) static_cast<float*>(R.out)[at + i] = 0.0f;
          else static_cast<T*>(R.out)[at + i] = (T)0.0f;
        }
    }
  }
  if constexpr (STATE_ONLY) {
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int w = 0; w < NW; ++w) carry[(w * M + m) * 64] = state[m][w];
  } else if (whole && R.last) {
    float* to = R.last + unit * DK * DV + dv0;
    if (n == 0) {  // as it was given
      const float* from = R.first ? R.first + unit * DK * DV : nullptr;
      for (int i = threadIdx.x; i < DK * width; i += THREADS) {
        const int row = i / width, column = i % width;
        to[row * DV + column] = from ? from[row * R.first_i + (dv0 + column) * R.first_j] : 0.0f;
      }
      return;
    }
    // a reversed sequence's state stands at its first token; one decay more and the scale make it the error of the state before it
    const float by = R.last_by * (reversed ? args.decay[head] : 1.0f);
    const int left = anew(DK) - 8 * g, stride = anew(DV);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const int column = state_column(NW * wave + w, lane);
      if (column >= width) continue;
      float* p = to + 8 * g * stride + column;
#pragma unroll
      for (int m = 0; m < M / 2; ++m) {
        if (PACKED && 32 * m >= left) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (PACKED || 32 * m + j < left) p[(32 * m + j) * stride] = state[2 * m + (j >> 2)][w][j & 3] * by;
        in_steps();
      }
    }
  }
}

// ---- launches, one translation unit to each element type ---------------------------------------------------------------
template <class T, int DKP, int WAVES>
int launch_scan(const Args& a, int roles, bool state_only, hipStream_t st) {
  int blocks = 1;
  for (int r = 0; r < roles; ++r) blocks = a.role[r].blocks > blocks ? a.role[r].blocks : blocks;
  const dim3 grid((unsigned)(a.units * a.segments * blocks), (unsigned)roles);
  const auto launch = [&](auto packed, auto only, auto exact) {
    scan_kernel<T, DKP, WAVES, decltype(packed)::value, decltype(only)::value, decltype(exact)::value><<<grid, 64 * WAVES, 0, st>>>(a);
  };
  const std::true_type yes;
  const std::false_type no;
  const std::bool_constant<PIECES<T> == 3> floats;  // (their pieces are three either way)
  const auto any_exact = [&](auto packed) {
    if (state_only) launch(packed, yes, yes);
    else if (a.segments == 1) launch(packed, no, yes);
    else launch(packed, no, floats);
  };
  if (a.role[0].packed) any_exact(yes);
  else any_exact(no);
  return launch_status();
}

template <class T, int DKP>
int launch_scan(const Args& a, int roles, int columns, bool state_only, hipStream_t st) {
  if constexpr (DKP <= 64)
    if (columns == 32) return launch_scan<T, DKP, 1>(a, roles, state_only, st);
  if constexpr (DKP <= 128)
    if (columns == 64) return launch_scan<T, DKP, 2>(a, roles, state_only, st);
  if constexpr (DKP <= 128)
    if (columns == 96) return launch_scan<T, DKP, 3>(a, roles, state_only, st);
  return launch_scan<T, DKP, 4>(a, roles, state_only, st);
}

// One pass of all roles; those of one shape in one launch.
template <class T>
int run_scan(const Args& all, int roles, bool state_only, hipStream_t st) {
  for (int r = 0; r < roles;) {
    Args a = all;
    const int dk = all.role[r].DKP, columns = all.role[r].columns;
    int same = 0;
    for (; r + same < roles && all.role[r + same].DKP == dk && all.role[r + same].columns == columns; ++same) a.role[same] = all.role[r + same];
    const int rc = dk == 32    ? launch_scan<T, 32>(a, same, columns, state_only, st)
                   : dk == 64  ? launch_scan<T, 64>(a, same, columns, state_only, st)
                   : dk == 96  ? launch_scan<T, 96>(a, same, columns, state_only, st)
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
