// Embedding lookup and its gradient.
//
//   out[n] = scale table[token[n]],   d_table[r] = scale sum_{n : token[n] = r} d_out[n]
//
// A token outside [0, V) is padding: its output row is zero and its error goes nowhere.
//
// The gradient sorts the positions by token (a stable radix sort of eight bits a pass, padding left out in the first), cuts the
// sorted list into tiles of equal length and lets one workgroup sum each tile's rows in order: a row whose tokens all lie in one
// tile is finished there, the others leave partial sums that a second kernel adds tile by tile.  So every sum has a fixed order,
// in fp32, whatever the distribution of the tokens: a token that a third of all positions hold costs what any other row costs.
// (Adding into the table with atomics would be shorter, but its results change from run to run and bfloat16 has none.)
//
// Bounds: the lookup is memory (131071 rows of 2 KB: 55 us).  The gradient of 65521 words over 32003 rows of 1000 (bfloat16, 196 MB that
// have to be moved, 38 us at a copy's rate) takes 70 to 74 us: the sums 28 (4.7 TB/s), the sort 27 (of four dependent kernels, with the table
// cleared on the side), the join 7.  Of 78400 pixels over 256 rows of 64 floats: 28 us, all of it round trips of four dependent kernels.
#include <type_traits>

#include "cnn_common.h"
#include "cnn_types.h"

namespace cnn {
namespace {

constexpr int EMBED_THREADS = 256;

struct EmbedArgs {
  const void *table, *tokens;
  void* out;
  int64_t N, V;
  int cols;       // of VN elements, per row
  int lanes_log;  // lanes that share a row
  float scale;
};

template <class I>
__device__ __forceinline__ int64_t token_at(const void* tokens, int64_t n) {
  return (int64_t) static_cast<const I*>(tokens)[n];
}

// Lanes in groups that each take ROWS rows at once, so that as many loads are in flight.
template <class T, int VN, class I, int ROWS, bool PAST_CACHES>
__global__ __launch_bounds__(EMBED_THREADS) void embed_fwd_kernel(EmbedArgs a) {
  using P = Pack<T, VN>;
  const P* table = static_cast<const P*>(a.table);
  P* out = static_cast<P*>(a.out);
  const int lanes = 1 << a.lanes_log, groups = EMBED_THREADS >> a.lanes_log;
  const int64_t row0 = workgroup() * (groups * ROWS) + (threadIdx.x >> a.lanes_log);
  int64_t token[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int64_t n = row0 + r * groups;
    token[r] = n < a.N ? token_at<I>(a.tokens, n) : -1;
  }
  for (int c = threadIdx.x & (lanes - 1); c < a.cols; c += lanes) {
    P v[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
      if ((uint64_t)token[r] < (uint64_t)a.V) v[r] = table[token[r] * a.cols + c];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int64_t n = row0 + r * groups;
      if (n >= a.N) continue;
      P w;
#pragma unroll
      for (int j = 0; j < VN; ++j) w.v[j] = (T)((uint64_t)token[r] < (uint64_t)a.V ? (float)v[r].v[j] * a.scale : 0.0f);
      if constexpr (PAST_CACHES) put_past_caches(out + n * a.cols + c, w);
      else out[n * a.cols + c] = w;
    }
  }
}

// ---- the gradient ------------------------------------------------------------------------------------------------------
struct Entry {  // of the sorted list
  uint32_t token, position;
};

constexpr int RADIX = 256;
constexpr int SORT_THREADS = 256, SORT_WAVES = SORT_THREADS / 64;
constexpr int SORT_EACH = 4;        // positions that a lane holds at once, so that their loads are under way together (8: 74.7 us for the 70.2 of the text above, inputs in turn)
constexpr int SORT_CHUNK = SORT_THREADS * SORT_EACH;  // positions to a workgroup, at least
constexpr int SORT_GROUPS = 256;    // workgroups of a pass, at most: each adds up the counts of those before it
constexpr int SMALL_THREADS = 1024, SMALL_WAVES = SMALL_THREADS / 64, SMALL_EACH = 4;
constexpr int SMALL = SMALL_THREADS * SMALL_EACH;  // positions that one workgroup sorts in LDS

// Rows of the table that no token names are zero: the sorting kernels, which use little of the memory's rate, clear the table on
// the side, a share in each.
struct Fill {
  uint4* at;
  int64_t begin, end;  // in units of 16 bytes
  int tail;            // in the last share: units of 2 bytes past the end
};

__device__ __forceinline__ void fill(const Fill& f, int64_t group, int64_t groups, int threads) {
  for (int64_t i = f.begin + group * threads + threadIdx.x; i < f.end; i += groups * threads) f.at[i] = uint4{0, 0, 0, 0};
  if (group == 0 && (int)threadIdx.x < f.tail) reinterpret_cast<uint16_t*>(f.at + f.end)[threadIdx.x] = 0;
}

struct SortArgs {
  const void* tokens;   // first pass
  const Entry* from;    // later passes
  Entry* to;
  uint32_t* counts;     // [workgroup][RADIX]
  uint32_t* total;      // entries that are no padding
  int64_t N, V;
  int chunk, groups, shift;
  Fill clear;
};

// Entry i of a pass: false for padding and past the end.
template <class I, bool FIRST>
__device__ __forceinline__ bool entry_at(const SortArgs& a, int64_t i, int64_t end, Entry& e) {
  if (i >= end) return false;
  if (!FIRST) {
    e = a.from[i];
    return true;
  }
  const int64_t t = token_at<I>(a.tokens, i);
  e = Entry{(uint32_t)t, (uint32_t)i};
  return (uint64_t)t < (uint64_t)a.V;
}

// Entries begin + 64 r + lane of a wave, r = 0 .. SORT_EACH - 1.
template <class I, bool FIRST>
__device__ __forceinline__ void entries_at(const SortArgs& a, int64_t begin, int64_t end, Entry (&e)[SORT_EACH], bool (&any)[SORT_EACH]) {
#pragma unroll
  for (int r = 0; r < SORT_EACH; ++r) {
    e[r] = Entry{0, 0};
    any[r] = entry_at<I, FIRST>(a, begin + 64 * r + (threadIdx.x & 63), end, e[r]);
  }
}

template <class I, bool FIRST>
__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(SortArgs a) {
  if ((int)blockIdx.x >= a.groups) return fill(a.clear, blockIdx.x - a.groups, gridDim.x - a.groups, SORT_THREADS);
  __shared__ uint32_t count[SORT_WAVES][RADIX];
  const int wave = threadIdx.x >> 6;
  for (int w = 0; w < SORT_WAVES; ++w) count[w][threadIdx.x] = 0;
  __syncthreads();
  const int64_t all = FIRST ? a.N : (int64_t)*a.total, part = a.chunk / SORT_WAVES;
  const int64_t begin = (int64_t)blockIdx.x * a.chunk + wave * part, end = begin + part < all ? begin + part : all;
  for (int64_t i = begin; i < end; i += 64 * SORT_EACH) {
    Entry e[SORT_EACH];
    bool any[SORT_EACH];
    entries_at<I, FIRST>(a, i, end, e, any);
#pragma unroll
    for (int r = 0; r < SORT_EACH; ++r)
      if (any[r]) atomicAdd(&count[wave][e[r].token >> a.shift & (RADIX - 1)], 1u);
  }
  __syncthreads();
  uint32_t sum = 0;
  for (int w = 0; w < SORT_WAVES; ++w) sum += count[w][threadIdx.x];
  a.counts[(int64_t)blockIdx.x * RADIX + threadIdx.x] = sum;
}

// Lanes of the wave that hold the same digit as this one, among those that hold any.
__device__ __forceinline__ uint64_t peers(uint32_t digit, bool any) {
  uint64_t same = __ballot(any);
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const uint64_t set = __ballot(digit >> b & 1);
    same &= digit >> b & 1 ? set : ~set;
  }
  return same;
}

// What the lanes of a wave read from LDS before this is read before what they write after it, and the other way round.
__device__ __forceinline__ void wave_in_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Sum of `v` over the lower lanes of a workgroup of WAVES waves, all of which call it.  `sums` is LDS of WAVES words.
template <int WAVES>
__device__ __forceinline__ uint32_t exclusive_sum(uint32_t v, uint32_t* sums) {
  const int lane = threadIdx.x & 63;
  uint32_t s = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = __shfl_up(s, d);
    if (lane >= d) s += o;
  }
  if (lane == 63) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) before += sums[w];
  return before + s - v;
}

// The pass itself: each wave takes a quarter of the chunk, in order, and keeps its own next place for each digit.
template <class I, bool FIRST>
__global__ __launch_bounds__(SORT_THREADS) void sort_scatter_kernel(SortArgs a) {
  if ((int)blockIdx.x >= a.groups) return fill(a.clear, blockIdx.x - a.groups, gridDim.x - a.groups, SORT_THREADS);
  __shared__ uint32_t place[SORT_WAVES][RADIX], sums[SORT_WAVES];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, digit = threadIdx.x;
  const int64_t all = FIRST ? a.N : (int64_t)*a.total;
  const int64_t part = a.chunk / SORT_WAVES;  // a multiple of 64 SORT_EACH
  const int64_t begin = (int64_t)blockIdx.x * a.chunk + wave * part;
  const int64_t end = begin + part < all ? begin + part : all;
  Entry e[SORT_EACH];
  bool any[SORT_EACH];
  entries_at<I, FIRST>(a, begin, end, e, any);
  // entries of this thread's digit in earlier workgroups, and in all
  uint32_t before = 0, total = 0;
#pragma unroll 16
  for (int g = 0; g < a.groups; ++g) {
    const uint32_t c = a.counts[(int64_t)g * RADIX + digit];
    before += g < (int)blockIdx.x ? c : 0;
    total += c;
  }
  for (int w = 0; w < SORT_WAVES; ++w) place[w][digit] = 0;
  const uint32_t base = before + exclusive_sum<SORT_WAVES>(total, sums);  // (its barrier also follows the clearing)
  if (FIRST && blockIdx.x == 0 && threadIdx.x == RADIX - 1) *a.total = base - before + total;
  for (int64_t i = begin; i < end; i += 64 * SORT_EACH) {
    if (part > 64 * SORT_EACH) entries_at<I, FIRST>(a, i, end, e, any);
#pragma unroll
    for (int r = 0; r < SORT_EACH; ++r)
      if (any[r]) atomicAdd(&place[wave][e[r].token >> a.shift & (RADIX - 1)], 1u);
  }
  __syncthreads();
  uint32_t next = base;
  for (int w = 0; w < SORT_WAVES; ++w) {
    const uint32_t c = place[w][digit];
    place[w][digit] = next;
    next += c;
  }
  __syncthreads();
  for (int64_t i = begin; i < end; i += 64 * SORT_EACH) {  // (every lane of the wave makes every step)
    if (part > 64 * SORT_EACH) entries_at<I, FIRST>(a, i, end, e, any);
#pragma unroll
    for (int r = 0; r < SORT_EACH; ++r) {
      const uint32_t d = e[r].token >> a.shift & (RADIX - 1);
      const uint64_t same = peers(d, any[r]);
      const int rank = __popcll(same & ((1ull << lane) - 1));
      const uint32_t at = any[r] ? place[wave][d] : 0;
      wave_in_order();
      if (any[r]) {
        if (rank == 0) place[wave][d] = at + (uint32_t)__popcll(same);
        a.to[at + rank] = e[r];
      }
      wave_in_order();
    }
  }
}

// All passes for up to SMALL positions, by one workgroup in LDS; the others clear the table.
template <class I>
__global__ __launch_bounds__(SMALL_THREADS) void sort_small_kernel(SortArgs a, int passes) {
  if (blockIdx.x) return fill(a.clear, blockIdx.x - 1, gridDim.x - 1, SMALL_THREADS);
  __shared__ Entry list[SMALL];
  __shared__ uint32_t place[SMALL_WAVES][RADIX], sums[SMALL_WAVES], entries;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int64_t all = a.N;
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = 8 * pass;
    Entry e[SMALL_EACH];
    bool any[SMALL_EACH];
#pragma unroll
    for (int r = 0; r < SMALL_EACH; ++r) {
      const int i = (wave * SMALL_EACH + r) * 64 + lane;
      e[r] = Entry{0, 0};
      if (pass == 0) {
        any[r] = entry_at<I, true>(a, i, all, e[r]);
      } else {
        any[r] = i < all;
        if (any[r]) e[r] = list[i];
      }
    }
    for (int i = threadIdx.x; i < SMALL_WAVES * RADIX; i += SMALL_THREADS) (&place[0][0])[i] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < SMALL_EACH; ++r)
      if (any[r]) atomicAdd(&place[wave][e[r].token >> shift & (RADIX - 1)], 1u);
    __syncthreads();
    uint32_t total = 0;
    if (threadIdx.x < RADIX)
      for (int w = 0; w < SMALL_WAVES; ++w) total += place[w][threadIdx.x];
    uint32_t next = exclusive_sum<SMALL_WAVES>(total, sums);
    if (threadIdx.x < RADIX)
      for (int w = 0; w < SMALL_WAVES; ++w) {
        const uint32_t c = place[w][threadIdx.x];
        place[w][threadIdx.x] = next;
        next += c;
      }
    if (threadIdx.x == RADIX - 1) entries = next;
    __syncthreads();
    all = entries;
#pragma unroll
    for (int r = 0; r < SMALL_EACH; ++r) {
      const uint32_t d = e[r].token >> shift & (RADIX - 1);
      const uint64_t same = peers(d, any[r]);
      const int rank = __popcll(same & ((1ull << lane) - 1));
      const uint32_t at = any[r] ? place[wave][d] : 0;
      wave_in_order();
      if (any[r]) {
        if (rank == 0) place[wave][d] = at + (uint32_t)__popcll(same);
        list[at + rank] = e[r];
      }
      wave_in_order();
    }
    __syncthreads();
  }
  for (int64_t i = threadIdx.x; i < all; i += SMALL_THREADS) a.to[i] = list[i];
  if (threadIdx.x == 0) *a.total = (uint32_t)all;
}

struct SumArgs {
  const void* d_out;
  void* d_table;
  const Entry* sorted;
  const uint32_t* total;
  float* partial;  // [tile][2][D]: of the run that enters a tile, of the one that leaves it
  int cols;        // of VN elements, per row
  int lanes_log, stretch, tile;  // entries of a walker, of a workgroup
  float scale;
};

template <int VN>
struct Sum {
  float v[VN];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int j = 0; j < VN; ++j) v[j] = 0.0f;
  }
  template <class T>
  __device__ __forceinline__ void add(const Pack<T, VN>& p) {
#pragma unroll
    for (int j = 0; j < VN; ++j) v[j] += (float)p.v[j];
  }
  template <class T>
  __device__ __forceinline__ void store(T* row, int c, float scale) const {
    Pack<T, VN> p;
#pragma unroll
    for (int j = 0; j < VN; ++j) p.v[j] = (T)(v[j] * scale);
    reinterpret_cast<Pack<T, VN>*>(row)[c] = p;
  }
};

// A walker of 1 << lanes_log lanes takes a stretch of the sorted list and 1 << lanes_log packs of the columns; a workgroup's walkers
// take the stretches of one tile and add up, through LDS, the parts of rows that lie in more than one of them.
constexpr int AHEAD = 8;
template <class T, int VN>
__global__ __launch_bounds__(EMBED_THREADS) void embed_sum_kernel(SumArgs a) {
  using P = Pack<T, VN>;
  __shared__ float parts[2][EMBED_THREADS * VN];  // of the run that enters a stretch, of the one that leaves it
  __shared__ bool through[EMBED_THREADS];         // by stretch: it is part of a run that goes on on both sides
  const P* d_out = static_cast<const P*>(a.d_out);
  T* d_table = static_cast<T*>(a.d_table);
  const int64_t total = *a.total, width = (int64_t)a.cols * VN;
  const int walkers = EMBED_THREADS >> a.lanes_log, walker = threadIdx.x >> a.lanes_log, lane = threadIdx.x & ((1 << a.lanes_log) - 1);
  const int c = (blockIdx.y << a.lanes_log) + lane;
  const int64_t begin = (int64_t)blockIdx.x * a.tile + (int64_t)walker * a.stretch;
  const int64_t end = begin + a.stretch < total ? begin + a.stretch : total;
  const bool busy = begin < end && c < a.cols;
  uint32_t token = busy ? a.sorted[begin].token : 0;
  const bool entered = busy && begin > 0 && a.sorted[begin - 1].token == token;
  bool inside = !entered;  // the present run began in this stretch
  Sum<VN> sum;
  sum.clear();
  const auto keep = [&](int which) {
#pragma unroll
    for (int j = 0; j < VN; ++j) parts[which][j * EMBED_THREADS + threadIdx.x] = sum.v[j];
  };
  if (busy)
    for (int64_t i = begin; i < end; i += AHEAD) {
      Entry e[AHEAD];
      P row[AHEAD];
#pragma unroll
      for (int r = 0; r < AHEAD; ++r)
        if (i + r < end) e[r] = a.sorted[i + r];
#pragma unroll
      for (int r = 0; r < AHEAD; ++r)
        if (i + r < end) row[r] = d_out[(int64_t)e[r].position * a.cols + c];
#pragma unroll
      for (int r = 0; r < AHEAD; ++r) {
        if (i + r >= end) break;
        if (e[r].token != token) {
          if (inside) sum.store(d_table + token * width, c, a.scale);
          else keep(0);
          sum.clear();
          token = e[r].token, inside = true;
        }
        sum.add(row[r]);
      }
    }
  const bool leaves = busy && end < total && a.sorted[end].token == token;
  if (busy && inside && !leaves) sum.store(d_table + token * width, c, a.scale);
  else if (busy) keep(inside);
  if (lane == 0) through[walker] = busy && !inside && leaves;  // (the first column of a block is never past the width)
  __syncthreads();
  // The run that leaves this stretch: the parts that entered the next ones, up to the stretch or the tile where it ends.
  const auto follow = [&](int which) {
#pragma unroll
    for (int j = 0; j < VN; ++j) sum.v[j] = parts[which][j * EMBED_THREADS + threadIdx.x];
    int w = walker;
    bool on = which == 1 || through[w];
    while (on && ++w < walkers) {
#pragma unroll
      for (int j = 0; j < VN; ++j) sum.v[j] += parts[0][j * EMBED_THREADS + (w << a.lanes_log) + lane];
      on = through[w];
    }
    return on;  // it leaves the tile
  };
  if (busy && inside && leaves) {
    if (follow(1)) sum.store(a.partial + (2 * (int64_t)blockIdx.x + 1) * width, c, 1.0f);
    else sum.store(d_table + token * width, c, a.scale);
  }
  if (walker == 0 && entered) {
    follow(0);
    sum.store(a.partial + 2 * (int64_t)blockIdx.x * width, c, 1.0f);
  }
}

// Rows whose tokens lie in more than one tile: the part that left the tile where they began, then the parts that entered the
// following ones, added in an order that depends on their number alone.  Each walker takes a row of few parts; for a row of many
// the whole workgroup shares the parts out.
constexpr int JOIN_THREADS = 1024, JOIN_TILES = 16, JOIN_FEW = 8;
template <class T, int VN>
__global__ __launch_bounds__(JOIN_THREADS) void embed_join_kernel(SumArgs a) {
  __shared__ uint32_t begun[JOIN_TILES][2];  // by tile: parts of the row that begins in it and leaves it (0: none), its token
  __shared__ float lds[JOIN_THREADS * VN];
  const int64_t total = *a.total;
  const int lanes = 1 << a.lanes_log, groups = JOIN_THREADS >> a.lanes_log;
  const int lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> a.lanes_log;
  const int64_t width = (int64_t)a.cols * VN, first = (int64_t)blockIdx.x * JOIN_TILES;
  if (threadIdx.x < JOIN_TILES) {
    const int64_t tile = first + threadIdx.x, begin = tile * a.tile, end = begin + a.tile;
    uint32_t parts = 0, token = 0;
    if (end < total) {
      uint32_t at[JOIN_FEW];  // tokens at the starts of the following tiles
#pragma unroll
      for (int j = 0; j < JOIN_FEW; ++j) {
        const int64_t i = end + (int64_t)j * a.tile;
        at[j] = i < total ? a.sorted[i].token : ~0u;
      }
      token = at[0];
      const bool leaves = a.sorted[end - 1].token == token;
      const bool entered = begin > 0 && a.sorted[begin - 1].token == token;
      if (leaves && !entered) {
        parts = 1;
#pragma unroll
        for (int j = 0; j < JOIN_FEW; ++j)
          if (parts == (uint32_t)j + 1 && at[j] == token) ++parts;
      }
    }
    begun[threadIdx.x][0] = parts, begun[threadIdx.x][1] = token;
  }
  __syncthreads();
  T* d_table = static_cast<T*>(a.d_table);
  const int c = (blockIdx.y << a.lanes_log) + lane;
  const auto part = [&](int64_t tile, int64_t p) {
    return reinterpret_cast<const Pack<float, VN>*>(a.partial + (2 * (tile + p) + (p == 0)) * width)[c];
  };
  for (int k = group; k < JOIN_TILES; k += groups) {
    const int parts = begun[k][0];
    if (parts == 0 || parts > JOIN_FEW || c >= a.cols) continue;
    Sum<VN> sum;
    sum.clear();
#pragma unroll
    for (int p = 0; p < JOIN_FEW; ++p)
      if (p < parts) sum.add(part(first + k, p));
    sum.store(d_table + begun[k][1] * width, c, a.scale);
  }
  for (int k = 0; k < JOIN_TILES; ++k) {
    if (begun[k][0] <= JOIN_FEW) continue;  // (the same for the whole workgroup)
    // tiles that begin with the row's token: every wave looks at 64 places at a time
    int64_t low = first + k + JOIN_FEW, high = (total + a.tile - 1) / a.tile;  // the last one known, one past the last
    while (high - low > 1) {
      const int64_t step = (high - low + 63) / 64, at = low + step * ((threadIdx.x & 63) + 1);
      low += step * __popcll(__ballot(at < high && a.sorted[at * a.tile].token == begun[k][1]));
      high = low + step < high ? low + step : high;
    }
    const int64_t parts = low - (first + k) + 1;
    Sum<VN> sum;
    sum.clear();
    if (c < a.cols) {
#pragma unroll 8
      for (int64_t p = group; p < parts; p += groups) sum.add(part(first + k, p));
    }
#pragma unroll
    for (int j = 0; j < VN; ++j) lds[(group * VN + j) * lanes + lane] = sum.v[j];
    __syncthreads();
    const int used = parts < groups ? (int)parts : groups;  // walkers that had a part
    for (int i = threadIdx.x; i < VN * lanes; i += JOIN_THREADS) {
      float s = 0.0f;
#pragma unroll 8
      for (int g = 0; g < used; ++g) s += lds[g * VN * lanes + i];
      lds[i] = s;
    }
    __syncthreads();
    if (group == 0 && c < a.cols) {
#pragma unroll
      for (int j = 0; j < VN; ++j) sum.v[j] = lds[j * lanes + lane];
      sum.store(d_table + begun[k][1] * width, c, a.scale);
    }
    __syncthreads();
  }
}

// Elements to a pack: as many of 16 bytes as divide a row.
int pack_of(int D, int type) {
  int n = (int)(16 / type_bytes(type));
  while (D % n) n >>= 1;
  return n;
}

int lanes_log_for(int cols, int most) {
  int l = 0;
  while (l < most && 1 << l < cols) ++l;
  return l;
}

struct EmbedPlan {
  int64_t groups, chunk, tiles, stretch, tile, columns;
  int pack, lanes_log, passes;
  bool small;
  size_t list, list_bytes, counts, partial, bytes;  // offsets and sizes in the workspace; the number of entries is at its start
};

constexpr int64_t SUM_WAVES = 4096;  // of the summing kernel where the list is long: sixteen to a compute unit

EmbedPlan embed_plan(int64_t N, int64_t V, int D, int type) {
  EmbedPlan p{};
  p.small = N <= SMALL;
  p.chunk = SORT_CHUNK;
  while ((N + p.chunk - 1) / p.chunk > SORT_GROUPS) p.chunk *= 2;
  p.groups = (N + p.chunk - 1) / p.chunk;
  p.passes = 1;
  while (p.passes < 4 && V > (int64_t)1 << 8 * p.passes) ++p.passes;
  p.pack = pack_of(D, type);
  const int cols = D / p.pack;
  p.lanes_log = lanes_log_for(cols, 6);
  p.columns = (cols + (1 << p.lanes_log) - 1) >> p.lanes_log;
  // short stretches keep many loads in flight, long ones leave few partial sums
  p.stretch = 16;
  while (p.stretch < 512 && (N / p.stretch * p.columns << p.lanes_log) / 64 > SUM_WAVES) p.stretch *= 2;
  p.tile = p.stretch * (EMBED_THREADS >> p.lanes_log);
  p.tiles = (N + p.tile - 1) / p.tile;
  const auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
  p.list = 256;
  p.list_bytes = up((size_t)N * sizeof(Entry));
  p.counts = p.list + p.list_bytes * (p.small ? 1 : 2);
  p.partial = p.counts + (p.small ? 0 : up((size_t)p.groups * RADIX * 4));
  p.bytes = p.partial + up((size_t)p.tiles * 2 * D * 4);
  return p;
}

bool embed_sizes_fit(int64_t N, int64_t V, int D, int type) {
  return N >= 1 && N < (int64_t)1 << 31 && V >= 1 && V < (int64_t)1 << 31 && D >= 1 && D <= 1 << 16 && type_known(type);
}

template <class I>
int sort_tokens(const EmbedPlan& p, SortArgs a, char* ws, size_t table_bytes, hipStream_t st) {
  Entry* first = reinterpret_cast<Entry*>(ws + p.list);
  const int64_t units = (int64_t)(table_bytes / 16);
  const int tail = (int)(table_bytes % 16 / 2);
  const auto fill_groups = [](int64_t n, int threads) {  // sixteen stores to a thread, one workgroup at least for the tail
    const int64_t g = (n + threads * 16 - 1) / (threads * 16);
    return (unsigned)(g > 2048 ? 2048 : g < 1 ? 1 : g);
  };
  if (p.small) {
    a.to = first;
    a.clear.end = units, a.clear.tail = tail;
    sort_small_kernel<I><<<1 + fill_groups(units, SMALL_THREADS), SMALL_THREADS, 0, st>>>(a, p.passes);
    return launch_status();
  }
  Entry* list[2] = {first, reinterpret_cast<Entry*>(ws + p.list + p.list_bytes)};
  const int shares = 2 * p.passes;
  int share = 0;
  const auto next_share = [&] {
    a.clear.begin = units * share / shares, a.clear.end = units * (share + 1) / shares;
    ++share;
    a.clear.tail = share == shares ? tail : 0;
    return (unsigned)p.groups + fill_groups(a.clear.end - a.clear.begin, SORT_THREADS);
  };
  for (int pass = 0; pass < p.passes; ++pass) {
    a.shift = 8 * pass;
    const int to = (p.passes - 1 - pass) & 1;  // the last pass writes list[0]
    a.from = list[to ^ 1], a.to = list[to];
    unsigned grid = next_share();
    if (pass == 0) sort_count_kernel<I, true><<<grid, SORT_THREADS, 0, st>>>(a);
    else sort_count_kernel<I, false><<<grid, SORT_THREADS, 0, st>>>(a);
    grid = next_share();
    if (pass == 0) sort_scatter_kernel<I, true><<<grid, SORT_THREADS, 0, st>>>(a);
    else sort_scatter_kernel<I, false><<<grid, SORT_THREADS, 0, st>>>(a);
  }
  return launch_status();
}

template <class T, int VN>
int sum_rows(const EmbedPlan& p, const SumArgs& a, hipStream_t st) {
  embed_sum_kernel<T, VN><<<dim3((unsigned)p.tiles, (unsigned)p.columns), EMBED_THREADS, 0, st>>>(a);
  if (p.tiles > 1)
    embed_join_kernel<T, VN><<<dim3((unsigned)((p.tiles + JOIN_TILES - 1) / JOIN_TILES), (unsigned)p.columns), JOIN_THREADS, 0, st>>>(a);
  return launch_status();
}

template <class T, int VN>
int lookup(const EmbedArgs& a, bool wide, bool past_caches, hipStream_t st) {
  constexpr int ROWS = 4;
  const int64_t per = (int64_t)(EMBED_THREADS >> a.lanes_log) * ROWS;
  const dim3 grid = grid_of((a.N + per - 1) / per);
  const auto launch = [&](auto past) {
    constexpr bool PAST = decltype(past)::value;
    if (wide) embed_fwd_kernel<T, VN, int64_t, ROWS, PAST><<<grid, EMBED_THREADS, 0, st>>>(a);
    else embed_fwd_kernel<T, VN, int32_t, ROWS, PAST><<<grid, EMBED_THREADS, 0, st>>>(a);
  };
  if constexpr (VN * sizeof(T) == 16)
    if (past_caches) {
      launch(std::true_type{});
      return launch_status();
    }
  launch(std::false_type{});
  return launch_status();
}

// Calls fn<T, VN> for the pack size of a row.
template <class FN>
int with_pack(int type, int pack, FN fn) {
  return with_type(type, [&](auto t) -> int {
    using T = decltype(t);
    if constexpr (sizeof(T) == 2)
      if (pack == 8) return fn(t, std::integral_constant<int, 8>{});
    if (pack == 4) return fn(t, std::integral_constant<int, 4>{});
    if (pack == 2) return fn(t, std::integral_constant<int, 2>{});
    return fn(t, std::integral_constant<int, 1>{});
  });
}

}  // namespace
}  // namespace cnn

extern "C" {

int cnn_embedding_fwd(const void* table, const void* tokens, void* out, int64_t N, int64_t V, int D, int type, int wide_tokens,
                      float scale, void* hip_stream) {
  using namespace cnn;
  if (!table || !tokens || !out || !embed_sizes_fit(N, V, D, type)) return CNN_EINVAL;
  if (!aligned16(table) || !aligned16(tokens) || !aligned16(out)) return CNN_EINVAL;
  const int pack = pack_of(D, type);
  // A long output is not kept in the caches, which then hold the table: rows of 2 KB of 50021, 256 MB of output 80 -> 53 us, 128 MB 37 -> 28;
  // with a reader behind it 171 -> 156 and 79 -> 80, 64 MB 35.5 -> 36.5.  Rows that end inside a line of 128 bytes lose by it
  // (79338 of 604 floats 34 -> 43 us).
  const size_t row = (size_t)D * type_bytes(type);
  const bool past_caches = row % 128 == 0 && (reinterpret_cast<uintptr_t>(out) & 127) == 0 && (size_t)N * row >= (size_t)96 << 20;
  const EmbedArgs a{table, tokens, out, N, V, D / pack, lanes_log_for(D / pack, 8), scale};
  return with_pack(type, pack, [&](auto t, auto n) { return lookup<decltype(t), decltype(n)::value>(a, wide_tokens != 0, past_caches, (hipStream_t)hip_stream); });
}

size_t cnn_embedding_bwd_workspace_bytes(int64_t N, int64_t V, int D, int type) {
  return cnn::embed_sizes_fit(N, V, D, type) ? cnn::embed_plan(N, V, D, type).bytes : 0;
}

int cnn_embedding_bwd(const void* d_out, const void* tokens, void* d_table, int64_t N, int64_t V, int D, int type, int wide_tokens,
                      float scale, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace cnn;
  if (!d_out || !tokens || !d_table || !workspace || !embed_sizes_fit(N, V, D, type)) return CNN_EINVAL;
  if (!aligned16(d_out) || !aligned16(tokens) || !aligned16(d_table) || !aligned16(workspace)) return CNN_EINVAL;
  const EmbedPlan p = embed_plan(N, V, D, type);
  if (workspace_bytes < p.bytes) return CNN_EWORKSPACE;
  char* ws = static_cast<char*>(workspace);
  hipStream_t st = (hipStream_t)hip_stream;
  SortArgs s{};
  s.tokens = tokens;
  s.total = reinterpret_cast<uint32_t*>(ws);
  s.counts = reinterpret_cast<uint32_t*>(ws + p.counts);
  s.N = N, s.V = V, s.chunk = (int)p.chunk, s.groups = (int)p.groups;
  s.clear.at = static_cast<uint4*>(d_table);
  const size_t table_bytes = (size_t)V * D * type_bytes(type);
  const int rc = wide_tokens ? sort_tokens<int64_t>(p, s, ws, table_bytes, st) : sort_tokens<int32_t>(p, s, ws, table_bytes, st);
  if (rc != CNN_OK) return rc;
  const SumArgs a{d_out, d_table, reinterpret_cast<Entry*>(ws + p.list), s.total, reinterpret_cast<float*>(ws + p.partial), D / p.pack,
                  p.lanes_log, (int)p.stretch, (int)p.tile, scale};
  return with_pack(type, p.pack, [&](auto t, auto n) { return sum_rows<decltype(t), decltype(n)::value>(p, a, st); });
}

}  // extern "C"
