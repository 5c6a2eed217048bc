// Log probabilities of given tokens, entropy and the most probable tokens of rows of logits, and the logits' gradient.
//
//   z = scale l,  m = max z,  ln p_v = z_v - m - ln sum exp(z - m),  H = - sum p ln p
//   d_l_v = scale ( sum_j g_j [v = token_j] - p_v sum_j g_j - d_H p_v (ln p_v + H) )
//
// Memory bounds both: a pass reads the logits once.  A workgroup holds its part of a row in registers, at most 64 elements to a lane (of floats 32),
// so the maximum, the two sums (of e = exp(z - m) and of e (z - m), from which the entropy comes without cancellation: both of its
// terms have one sign) and the choice of the largest elements all work on them.  Rows longer than 65536 (16384 floats; 32768 where rows are few) are cut into
// parts, more of them where rows are few, which a second kernel joins.
//
// The k largest: the k-th largest of the maxima of 64 (128) groups of lanes is a lower bound that few elements reach (24 are expected
// for k = 20 of 64 groups); those go into a list in LDS, and each finds its place by counting the larger ones.  Keys are unique,
// the value's bits in order above the complement of the index, so equal values keep the order of their tokens.  Where the list
// overflows (rows of equal logits) the workgroup takes the largest key k times instead.
//
// Measured: 8191 rows of 32003 bfloat16 150 us forward (524 MB; the vector unit's share, an exponential and some six operations an element, is
// 60 of them), 187 with five top tokens, 181 backward (1.05 GB, 5.8 TB/s, past the caches); 64 rows of 50021 with twenty top tokens 14.7: one workgroup to a
// row, a chain of loads, sums and barriers; 78400 rows of 256 19 (8 at a copy's rate) and 21.  Forward no load is on its way while a row's exponentials are
// computed: memory's time and the vector unit's nearly add up.
#include "cnn_common.h"
#include "cnn_lanes.h"
#include "cnn_types.h"

namespace cnn {
namespace logp {
namespace {

constexpr int MOST_GIVEN = 256, MOST_TOP = 64;
constexpr int64_t MOST_VOCAB = 1 << 24;
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

struct Sums {  // of e and of e (z - m) in powers of two, relative to the maximum m of the logits
  float m, s, t;
};

struct Args {
  const void* logits;
  int64_t row, rows, vocab, part_length;
  const void* tokens;
  float *log_probs, *entropy, *stats, *top_log_probs;
  int32_t* top_tokens;
  Sums* sums;      // [rows][parts]
  uint64_t* keys;  // [rows][parts][top]
  int parts, given, top, wide;
  float scale;
};

__device__ __forceinline__ float minus_infinity() { return -__builtin_inff(); }

// e d for e = 2^d, which is 0 for d = -inf.  (A NaN of d is in e.)
__device__ __forceinline__ float weighted(float e, float d) { return e * fmaxf(d, -1e30f); }

// scale (l - base) from half the difference and twice the scale: rounded as the difference is, but a number where that passes the largest one.
__device__ __forceinline__ float scaled_apart(float l, float base, float scale) { return __builtin_fmaf(l, 0.5f, -0.5f * base) * (2.0f * scale); }

// The sums of a wave's pieces, one to a lane, relative to the largest maximum; c = scale log2(e).  Pieces without a possible token have
// m = -inf, s = t = 0.
__device__ __forceinline__ Sums joined(const Sums& a, float c) {
  const float m = max_over<64>(a.m), ref = m == minus_infinity() ? 0.0f : m;
  const float d = scaled_apart(a.m, ref, c), e = __builtin_amdgcn_exp2f(d);
  return {m, sum_over<64>(a.s * e), sum_over<64>(e * (a.t + weighted(a.s, d)))};
}
// Pieces one after the other.
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b, float c) {
  const float m = fmaxf(a.m, b.m), ref = m == minus_infinity() ? 0.0f : m;
  const float da = scaled_apart(a.m, ref, c), db = scaled_apart(b.m, ref, c);
  const float ea = __builtin_amdgcn_exp2f(da), eb = __builtin_amdgcn_exp2f(db);
  return {m, a.s * ea + b.s * eb, ea * (a.t + weighted(a.s, da)) + eb * (b.t + weighted(b.s, db))};
}

__device__ __forceinline__ uint64_t key_of(float x, int64_t index) {
  const uint32_t bits = __float_as_uint(x + 0.0f);  // (-0 is 0)
  uint32_t order = bits ^ ((uint32_t)((int32_t)bits >> 31) | 0x80000000u);
  if (x != x) order = 0xfffffffeu;  // above infinity, and no key is all ones
  return (uint64_t)order << 32 | (uint32_t)~(uint32_t)index;
}
__device__ __forceinline__ float value_of(uint64_t key) {
  const uint32_t order = (uint32_t)(key >> 32);
  return order == 0xfffffffeu ? __builtin_nanf("") : __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order);
}
__device__ __forceinline__ int64_t index_of(uint64_t key) { return (int64_t)(uint32_t)~(uint32_t)key; }

__device__ __forceinline__ int64_t token_of(const void* tokens, int wide, int64_t i) {
  return wide ? static_cast<const int64_t*>(tokens)[i] : (int64_t) static_cast<const int32_t*>(tokens)[i];
}

// A given token's logit; `known` says whether it is one.
struct Given {
  float logit;
  bool known;
};
template <class T>
__device__ __forceinline__ Given got_given(const Args& a, const T* logits, int64_t n, int j) {
  Given g{0.0f, false};
  if (j >= a.given) return g;
  const int64_t token = token_of(a.tokens, a.wide, n * a.given + j);
  g.known = token >= 0 && token < a.vocab;
  if (g.known) g.logit = (float)logits[token];
  return g;
}

// The row's results from its sums; its lanes share the given tokens, of which each has asked for its first one's logit beforehand.
template <int THREADS, class T>
__device__ __forceinline__ float finish_row(const Args& a, const T* logits, int64_t n, const Sums& r, const Given& first) {
  const int lane = threadIdx.x % THREADS;
  const bool none = r.m == minus_infinity() && r.s == 0.0f;  // (a NaN would be in s)
  const float log_sum = none ? 0.0f : logf(r.s), base = none ? 0.0f : r.m;
  if (lane == 0) {
    // (a row with an infinite or NaN logit has s = NaN)
    const float h = none ? 0.0f : log_sum - r.t * LN2 / r.s;
    if (a.entropy) a.entropy[n] = h;
    if (a.stats) a.stats[n * 3] = r.m, a.stats[n * 3 + 1] = log_sum, a.stats[n * 3 + 2] = h;
  }
  for (int j = lane; j < a.given; j += THREADS) {
    const Given g = j == lane ? first : got_given(a, logits, n, j);
    a.log_probs[n * a.given + j] = g.known ? scaled_apart(g.logit, base, a.scale) - log_sum : 0.0f;
  }
  return log_sum;
}

// Rank `rank` of a row's top tokens.
__device__ __forceinline__ void put_top(const Args& a, int64_t n, int rank, uint64_t key, const Sums& r, float log_sum) {
  const float base = r.m == minus_infinity() ? 0.0f : r.m;
  a.top_tokens[n * a.top + rank] = (int32_t)index_of(key);
  a.top_log_probs[n * a.top + rank] = scaled_apart(value_of(key), base, a.scale) - log_sum;
}

template <int LANES>
__device__ __forceinline__ uint64_t largest_over(uint64_t v) {
  return over_lanes<LANES>(v, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
}

// Waits for the lanes that share a row.  (A wave's own accesses to LDS are in order.)
template <int THREADS>
__device__ __forceinline__ void row_sync() {
  if constexpr (THREADS > 64) {
    __syncthreads();
  } else {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

template <int THREADS>
struct TopShared {
  static constexpr int LIST = THREADS > 64 ? 1024 : THREADS * 8;
  uint64_t list[LIST];
  uint64_t waves[2][THREADS > 64 ? THREADS / 64 : 1];
  int count;
};

// Calls put(rank, key) for the `top` largest of the keys that each(fn) hands out, every thread its own, key 0 where there are fewer; likely(fn) hands out
// some of them, the `top` largest among these.  All of a row's lanes call it; keys are unique and not 0.
template <int THREADS, class LIKELY, class EACH, class PUT>
__device__ void top_keys(TopShared<THREADS>& sh, int top, LIKELY likely, EACH each, PUT put) {
  const int lane = threadIdx.x % THREADS;
  if (lane == 0) sh.count = 0;
  row_sync<THREADS>();
  likely([&](uint64_t key) {
    const int at = atomicAdd(&sh.count, 1);  // (their order in the list does not matter)
    if (at < TopShared<THREADS>::LIST) sh.list[at] = key;
  });
  row_sync<THREADS>();
  const int count = sh.count;
  if (count <= TopShared<THREADS>::LIST) {
    for (int i = lane; i < count; i += THREADS) {
      const uint64_t key = sh.list[i];
      int rank = 0;
      for (int j = 0; j < count; ++j) rank += sh.list[j] > key;
      if (rank < top) put(rank, key);
    }
    for (int i = count + lane; i < top; i += THREADS) put(i, (uint64_t)0);
    return;
  }
  uint64_t last = ~(uint64_t)0;
  for (int r = 0; r < top; ++r) {
    uint64_t best = 0;
    each([&](uint64_t key) {
      if (key < last && key > best) best = key;
    });
    best = largest_over<(THREADS < 64 ? THREADS : 64)>(best);
    if constexpr (THREADS > 64) {
      if (lane % 64 == 0) sh.waves[r & 1][lane / 64] = best;
      row_sync<THREADS>();
#pragma unroll
      for (int w = 0; w < THREADS / 64; ++w) best = sh.waves[r & 1][w] > best ? sh.waves[r & 1][w] : best;
    }
    if (lane == 0) put(r, best);
    last = best;
  }
}

// A lower bound of the k-th largest of LANES * PER values, PER to a lane, the same in these lanes: the sixteen high bits of its key, found bit
// by bit.  NaN, to which nothing compares as smaller, where that is -inf or there are fewer than k.
template <int LANES, int PER>
__device__ __forceinline__ float kth_largest(const float (&v)[PER], int k) {
  uint32_t key[PER], found = 0;
#pragma unroll
  for (int p = 0; p < PER; ++p) key[p] = (uint32_t)(key_of(v[p], 0) >> 32);
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t now = found | 1u << bit;
    int reach = 0;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      uint64_t lanes = __ballot(key[p] >= now);
      if constexpr (LANES < 64) lanes = lanes >> (threadIdx.x & 63 & ~(LANES - 1)) & ((1ull << (LANES & 63)) - 1);
      reach += __popcll(lanes);
    }
    if (reach >= k) found = now;
  }
  return __uint_as_float(found & 0x80000000u ? found ^ 0x80000000u : ~found);
}

// One part of a row to THREADS lanes; where these are a wave or less, a workgroup has several rows.
template <class T, int THREADS, int EACH, bool TOP>
__global__ __launch_bounds__(THREADS > 256 ? THREADS : 256) __attribute__((amdgpu_waves_per_eu(EACH * sizeof(T) > 64 ? 4 : 8))) void logp_part_kernel(Args a) {
  constexpr int V = sizeof(T) == 2 ? 8 : 4, PACKS = EACH / V, LANES = THREADS < 64 ? THREADS : 64, WAVES = THREADS / LANES, ROWS = THREADS > 64 ? 1 : 256 / THREADS;
  __shared__ Sums sums[WAVES];
  const int lane = threadIdx.x % THREADS, beside = ROWS > 1 ? threadIdx.x / THREADS : 0;
  const int64_t unit = workgroup() * ROWS + beside, n = unit / a.parts, begin = unit % a.parts * a.part_length;
  if (n >= a.rows) return;  // (all lanes of a row)
  const int64_t left = a.vocab - begin;
  const int length = (int)(left < a.part_length ? left : a.part_length);  // (every part has an element)
  const T* logits = static_cast<const T*>(a.logits) + n * a.row;
  const T* part = logits + begin;
  const auto at = [&](int p) { return (p * THREADS + lane) * V; };
  Loose<T, V> raw[PACKS];
#pragma unroll
  for (int p = 0; p < PACKS; ++p) {
    raw[p] = got_loose<V>(part + at(p), length - at(p));
    if (length - at(p) < V)
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j >= length - at(p)) raw[p].v[j] = (T)minus_infinity();
  }
  const Given given = a.parts == 1 ? got_given(a, logits, n, lane) : Given{0.0f, false};
  float mine = minus_infinity();
#pragma unroll
  for (int p = 0; p < PACKS; ++p) {
    float x[V];
    widen(x, raw[p]);
#pragma unroll
    for (int j = 0; j < V; ++j) mine = fmaxf(mine, x[j]);
  }
  Sums r{max_over<LANES>(mine), 0.0f, 0.0f};
  // Exponents d = x c - ref', one operation: ref' is ref c rounded, and what the rounding left out, ref c = ref' + rest, is the same for all of them.
  // The largest exponent is rest, at most half a step of ref c: 2^-9 here, but 128 and more past 2^31, where exp2(rest) is no number.  Farther out (a large
  // scale, or a wave whose logits are all masked by a large number) the difference comes first, exact where the exponential is not 0
  // (and past the largest number only where it is): an operation more.
  const float c = a.scale * LOG2E, ref = r.m == minus_infinity() ? 0.0f : r.m, ref_c = ref * c;
  const bool far = !(__builtin_fabsf(ref_c) < 0x1p16f);
  const float rest = far ? 0.0f : __builtin_fmaf(ref, c, -ref_c);
#pragma unroll
  for (int p = 0; p < PACKS; ++p) {
    float x[V];
    __builtin_amdgcn_sched_barrier(0);  // (all packs' exponentials side by side take too many registers)
    forget(raw[p]);
    widen(x, raw[p]);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float d = far ? (x[j] - ref) * c : __builtin_fmaf(x[j], c, -ref_c), e = __builtin_amdgcn_exp2f(d);
      r.s += e, r.t += weighted(e, d);
    }
  }
  const float by = __builtin_amdgcn_exp2f(-rest);
  r.t = by * (r.t - rest * r.s), r.s *= by;
  r.s = sum_over<LANES>(r.s), r.t = sum_over<LANES>(r.t);
  if constexpr (WAVES > 1) {
    if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = r;
    __syncthreads();
    const int w = threadIdx.x % 64;
    r = joined(w < WAVES ? sums[w] : Sums{minus_infinity(), 0.0f, 0.0f}, c);
  }
  float log_sum = 0.0f;
  if (a.parts == 1) log_sum = finish_row<THREADS>(a, logits, n, r, given);
  else if (lane == 0) a.sums[unit] = r;
  if constexpr (!TOP) return;
  __shared__ float groups[128];
  __shared__ TopShared<THREADS> shared[ROWS];
  float least;  // no fewer than `top` elements reach it
  if constexpr (WAVES == 1) {
    const float one[1] = {mine};
    least = kth_largest<LANES>(one, a.top);
  } else {
    constexpr int GROUP = THREADS / 128;  // lanes
    mine = max_over<GROUP>(mine);
    if (lane % GROUP == 0) groups[lane / GROUP] = mine;
    __syncthreads();
    const float two[2] = {groups[lane % 64], groups[lane % 64 + 64]};
    least = kth_largest<64>(two, a.top);
  }
  // The few that reach it are read again, from the caches; so are all of them where the list overflows.
  const auto likely = [&](auto fn) {
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      float x[V];
      forget(raw[p]);
      widen(x, raw[p]);
      uint32_t reach = 0;
#pragma unroll
      for (int j = 0; j < V; ++j) reach |= (uint32_t)!(x[j] < least) << j;
      for (; reach; reach &= reach - 1) {
        const int i = at(p) + __builtin_ctz(reach);
        if (i < length) fn(key_of((float)part[i], begin + i));
      }
    }
  };
  const auto each = [&](auto fn) {
#pragma unroll 4
    for (int i = lane; i < length; i += THREADS) fn(key_of((float)part[i], begin + i));
  };
  top_keys<THREADS>(shared[beside], a.top, likely, each, [&](int rank, uint64_t key) {
    if (a.parts > 1) a.keys[unit * a.top + rank] = key;
    else put_top(a, n, rank, key, r, log_sum);
  });
}

// The parts of a row joined.
constexpr int JOIN_THREADS = 256, JOIN_KEYS = 2;
template <class T>
__global__ __launch_bounds__(JOIN_THREADS) void logp_join_kernel(Args a) {
  __shared__ Sums sums[JOIN_THREADS / 64];
  __shared__ TopShared<JOIN_THREADS> sh;
  const int64_t n = workgroup();
  if (n >= a.rows) return;
  const T* logits = static_cast<const T*>(a.logits) + n * a.row;
  const Given given = got_given(a, logits, n, threadIdx.x);
  const uint64_t* keys = a.keys + n * a.parts * a.top;
  const int count = a.parts * a.top;
  uint64_t own[JOIN_KEYS], least = 0;  // the first keys of this lane; the largest of the parts' last ones, which `top` keys reach
#pragma unroll
  for (int k = 0; k < JOIN_KEYS; ++k) {
    const int i = k * JOIN_THREADS + (int)threadIdx.x;
    own[k] = i < count ? keys[i] : 0;
  }
  const float c = a.scale * LOG2E;
  Sums r{minus_infinity(), 0.0f, 0.0f};
  for (int p = threadIdx.x; p < a.parts; p += JOIN_THREADS) r = join(r, a.sums[n * a.parts + p], c);
  r = joined(r, c);
  const auto each = [&](auto fn) {
#pragma unroll
    for (int k = 0; k < JOIN_KEYS; ++k)
      if (own[k]) fn(own[k], k * JOIN_THREADS + (int)threadIdx.x);
    for (int i = JOIN_KEYS * JOIN_THREADS + (int)threadIdx.x; i < count; i += JOIN_THREADS)
      if (keys[i]) fn(keys[i], i);
  };
  if (a.top) {
    each([&](uint64_t key, int i) {
      if (i % a.top == a.top - 1 && key > least) least = key;
    });
    least = largest_over<64>(least);
  }
  if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = r, sh.waves[0][threadIdx.x / 64] = least;
  __syncthreads();
  r = sums[0];
#pragma unroll
  for (int w = 1; w < JOIN_THREADS / 64; ++w) r = join(r, sums[w], c);
#pragma unroll
  for (int w = 0; w < JOIN_THREADS / 64; ++w) least = sh.waves[0][w] > least ? sh.waves[0][w] : least;
  const float log_sum = finish_row<JOIN_THREADS>(a, logits, n, r, given);
  if (!a.top) return;
  __syncthreads();  // (top_keys writes sh.waves again)
  const auto all = [&](auto fn) { each([&](uint64_t key, int) { fn(key); }); };
  const auto likely = [&](auto fn) {
    each([&](uint64_t key, int) {
      if (key >= least) fn(key);
    });
  };
  top_keys<JOIN_THREADS>(sh, a.top, likely, all, [&](int rank, uint64_t key) { put_top(a, n, rank, key, r, log_sum); });
}

// ---- backward ----------------------------------------------------------------------------------------------------------
struct BackArgs {
  const void* logits;
  int64_t row, rows, vocab;
  const void* tokens;
  const float *stats, *d_log_probs, *d_entropy;
  void* d_logits;
  int tiles, given, wide;
  float scale;
};

// One tile of a row: THREADS lanes with PACKS packs each, all on their way at once; of a wave's lanes or fewer, a workgroup has several rows (of
// fewer, each given one token).
template <class T, int THREADS, int PACKS, bool PAST_CACHES>
__global__ __launch_bounds__(THREADS > 64 ? THREADS : 256) void logp_backward_kernel(BackArgs a) {
  constexpr int V = sizeof(T) == 2 ? 8 : 4, TILE = THREADS * PACKS * V, ROWS = THREADS > 64 ? 1 : 256 / THREADS;
  constexpr bool MANY = THREADS >= 64;
  __shared__ int64_t all_tokens[MANY ? ROWS : 1][MANY ? MOST_GIVEN : 1];
  __shared__ float all_errors[MANY ? ROWS : 1][MANY ? MOST_GIVEN : 1];
  const int lane = threadIdx.x % THREADS, beside = ROWS > 1 ? threadIdx.x / THREADS : 0;
  int64_t* tokens = all_tokens[MANY ? beside : 0];
  float* errors = all_errors[MANY ? beside : 0];
  const int64_t unit = workgroup() * ROWS + beside, n = unit / a.tiles;
  const int begin = (int)(unit % a.tiles) * TILE, left = (int)a.vocab - begin;
  if (n >= a.rows) return;
  const T* logits = static_cast<const T*>(a.logits) + n * a.row;
  T* d_logits = static_cast<T*>(a.d_logits) + n * a.vocab;
  const bool whole = left >= TILE;  // the same in all lanes: no branch for each pack
  Loose<T, V> raw[PACKS];
  const auto at = [&](int p) { return (p * THREADS + lane) * V; };
  if (whole) {
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
      if constexpr (PAST_CACHES) raw[p] = got_loose_past_caches<V>(logits + begin + at(p));
      else raw[p] = *reinterpret_cast<const Loose<T, V>*>(logits + begin + at(p));
    }
  } else {
#pragma unroll
    for (int p = 0; p < PACKS; ++p) raw[p] = got_loose<V>(logits + begin + at(p), left - at(p));
  }
  const float m = a.stats[n * 3], log_sum = a.stats[n * 3 + 1], h = a.stats[n * 3 + 2];
  const float d_h = a.d_entropy ? a.d_entropy[n] : 0.0f;
  const bool none = m == minus_infinity() && log_sum == 0.0f;
  const float base = none ? 0.0f : m;
  float total = 0.0f;  // of the given tokens' errors; the same in every wave
  int64_t token = -1;  // the only one
  float error = 0.0f;
  if (!MANY || a.given == 1) {
    token = token_of(a.tokens, a.wide, n);
    if (token >= 0 && token < a.vocab && !none) total = error = a.d_log_probs[n];
    else token = -1;
  } else {
    for (int j = lane % 64; j < a.given; j += 64) {
      const int64_t t = token_of(a.tokens, a.wide, n * a.given + j);
      const bool known = t >= 0 && t < a.vocab && !none;
      const float g = known ? a.d_log_probs[n * a.given + j] : 0.0f;
      total += g;
      if (lane < 64) tokens[j] = known ? t : -1, errors[j] = g;
    }
    total = sum_over<64>(total);
  }
  const float by = a.scale, c = by * LOG2E, log2_sum = log_sum * LOG2E;
  const auto gradient = [&](float l, float g) {
    const float z = scaled_apart(l, base, c) - log2_sum, p = __builtin_amdgcn_exp2f(z);
    float d = g - p * total;
    if (a.d_entropy) d -= d_h * weighted(p, z * LN2 + h);
    return none ? 0.0f : by * d;
  };
  const int only = (int)token - begin;  // (below 0, or behind the tile, where it is not here)
#pragma unroll
  for (int p = 0; p < PACKS; ++p) {
    float x[V];
    widen(x, raw[p]);
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = gradient(x[j], at(p) + j == only ? error : 0.0f);
    if (!whole) put_loose(d_logits + begin + at(p), x, left - at(p));
    else if constexpr (PAST_CACHES) put_loose_past_caches(d_logits + begin + at(p), x);
    else put_loose(d_logits + begin + at(p), x, V);
  }
  if (!MANY || a.given == 1) return;
  // the row's stores are done before a given token's element is written again
  if constexpr (ROWS > 1) __threadfence_block(), __builtin_amdgcn_wave_barrier();
  else __syncthreads();
  for (int j = lane; j < a.given; j += THREADS) {
    const int64_t t = tokens[j];
    if (t < begin || t >= begin + TILE) continue;
    bool before = false;
    float g = 0.0f;
    for (int i = 0; i < a.given; ++i) {
      if (tokens[i] != t) continue;
      before |= i < j;
      g += errors[i];
    }
    if (!before) d_logits[t] = (T)gradient((float)logits[t], g);
  }
}

// ---- plans ---------------------------------------------------------------------------------------------------------------
bool shape_ok(const cnn_log_probs_shape* s) {
  return s && s->rows >= 1 && s->rows < (int64_t)1 << 31 && s->vocab >= 1 && s->vocab <= MOST_VOCAB && s->given >= 1 && s->given <= MOST_GIVEN && s->top >= 0 &&
         s->top <= MOST_TOP && s->top <= s->vocab && type_known(s->type) && s->scale > 0.0f && s->scale <= 1e30f;
}

bool rows_ok(const cnn_rows* r, int type) {
  return r && r->data && reinterpret_cast<uintptr_t>(r->data) % type_bytes(type) == 0 && r->row >= 0;
}

// The small inputs are read one by one and need only be aligned to their element: slices of a batch serve.
bool element_aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
size_t token_bytes(const cnn_log_probs_shape* s) { return s->wide_tokens ? 8 : 4; }

struct Plan {
  int threads, each, parts;
  int64_t part_length;
  size_t keys, bytes;
};

// One part where a workgroup holds the row.  Else the second kernel is needed anyway, and parts are as short as a thousand workgroups ask.
Plan plan_of(const cnn_log_probs_shape& s) {
  Plan p{};
  constexpr struct { int threads, each; } FORMS[] = {{16, 8}, {32, 8}, {64, 8}, {64, 16}, {64, 32}, {256, 16}, {256, 32}, {1024, 16}, {1024, 32}, {1024, 64}};
  const int most_each = s.type != CNN_F32 ? 64 : s.rows <= 256 ? 32 : 16;
  const int64_t longest = 1024 * most_each;
  int64_t want = s.vocab;
  if (want > longest) {
    want = s.rows * s.vocab / 1024;
    want = want < 4096 ? 4096 : want > longest ? longest : want;
  }
  for (const auto& f : FORMS) {
    if (f.each > most_each) continue;
    p.threads = f.threads, p.each = f.each;
    if (want <= (int64_t)f.threads * f.each) break;
  }
  const int64_t most = (int64_t)p.threads * p.each;
  p.parts = (int)((s.vocab + most - 1) / most);
  p.part_length = ((s.vocab + p.parts - 1) / p.parts + 7) / 8 * 8;
  p.parts = (int)((s.vocab + p.part_length - 1) / p.part_length);
  if (p.parts > 1) {
    p.keys = ((size_t)s.rows * p.parts * sizeof(Sums) + 255) & ~(size_t)255;
    p.bytes = p.keys + (size_t)s.rows * p.parts * s.top * 8;
  }
  return p;
}

template <class T, bool TOP>
void launch_part(const Args& a, const Plan& p, hipStream_t st) {
  const auto with = [&](auto threads, auto each) {
    constexpr int THREADS = decltype(threads)::value, ROWS = THREADS > 64 ? 1 : 256 / THREADS;
    if (p.threads != THREADS || p.each != decltype(each)::value) return;
    logp_part_kernel<T, THREADS, decltype(each)::value, TOP><<<grid_of((a.rows * a.parts + ROWS - 1) / ROWS), THREADS * ROWS, 0, st>>>(a);
  };
  using std::integral_constant;
  const integral_constant<int, 8> e8;
  const integral_constant<int, 16> e16, lanes16;
  const integral_constant<int, 32> e32, lanes32;
  const integral_constant<int, 64> lanes64;
  const integral_constant<int, 256> lanes256;
  const integral_constant<int, 1024> lanes1024;
  with(lanes16, e8), with(lanes32, e8), with(lanes64, e8), with(lanes64, e16), with(lanes64, e32);
  with(lanes256, e16), with(lanes256, e32), with(lanes1024, e16), with(lanes1024, e32);
  if constexpr (sizeof(T) == 2) with(lanes1024, integral_constant<int, 64>{});
}

template <class T, int THREADS, int PACKS, bool PAST_CACHES>
void launch_backward(BackArgs a, hipStream_t st) {
  constexpr int64_t TILE = THREADS * PACKS * (sizeof(T) == 2 ? 8 : 4);
  a.tiles = (int)((a.vocab + TILE - 1) / TILE);
  constexpr int ROWS = THREADS > 64 ? 1 : 256 / THREADS;
  logp_backward_kernel<T, THREADS, PACKS, PAST_CACHES><<<grid_of((a.rows * a.tiles + ROWS - 1) / ROWS), THREADS * ROWS, 0, st>>>(a);
}

}  // namespace
}  // namespace logp
}  // namespace cnn

extern "C" {

size_t cnn_log_probs_fwd_workspace_bytes(const cnn_log_probs_shape* s) { return cnn::logp::shape_ok(s) ? cnn::logp::plan_of(*s).bytes : 0; }

int cnn_log_probs_fwd(const cnn_log_probs_shape* s, const cnn_rows* logits, const void* tokens, float* log_probs, float* entropy, float* stats,
                      float* top_log_probs, int32_t* top_tokens, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace cnn;
  using namespace cnn::logp;
  if (!shape_ok(s) || !rows_ok(logits, s->type) || !tokens || !log_probs || (s->top && (!top_log_probs || !top_tokens))) return CNN_EINVAL;
  if (!element_aligned(tokens, token_bytes(s))) return CNN_EINVAL;
  for (const void* p : {(const void*)log_probs, (const void*)entropy, (const void*)stats, (const void*)top_log_probs,
                        (const void*)top_tokens, (const void*)workspace})
    if (!aligned16(p)) return CNN_EINVAL;
  const Plan p = plan_of(*s);
  if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return CNN_EWORKSPACE;
  char* ws = static_cast<char*>(workspace);
  const Args a{logits->data, logits->row, s->rows, s->vocab, p.part_length, tokens, log_probs, entropy, stats, top_log_probs, top_tokens,
               reinterpret_cast<Sums*>(ws), reinterpret_cast<uint64_t*>(ws + p.keys), p.parts, s->given, s->top, s->wide_tokens != 0, s->scale};
  hipStream_t st = (hipStream_t)hip_stream;
  return with_type(s->type, [&](auto t) {
    using T = decltype(t);
    if (a.top) launch_part<T, true>(a, p, st);
    else launch_part<T, false>(a, p, st);
    if (launch_status() != CNN_OK) return CNN_EHIP;
    if (p.parts == 1) return CNN_OK;
    logp_join_kernel<T><<<grid_of(a.rows), JOIN_THREADS, 0, st>>>(a);
    return launch_status();
  });
}

int cnn_log_probs_bwd(const cnn_log_probs_shape* s, const cnn_rows* logits, const void* tokens, const float* stats, const float* d_log_probs,
                      const float* d_entropy, void* d_logits, void* hip_stream) {
  using namespace cnn;
  using namespace cnn::logp;
  if (!shape_ok(s) || !rows_ok(logits, s->type) || !tokens || !stats || !d_log_probs || !d_logits) return CNN_EINVAL;
  if (!element_aligned(tokens, token_bytes(s)) || !element_aligned(stats, 4) || !element_aligned(d_log_probs, 4) || !element_aligned(d_entropy, 4)) return CNN_EINVAL;
  if (!aligned16(d_logits)) return CNN_EINVAL;
  const BackArgs a{logits->data, logits->row, s->rows, s->vocab, tokens, stats, d_log_probs, d_entropy, d_logits, 1, s->given, s->wide_tokens != 0, s->scale};
  hipStream_t st = (hipStream_t)hip_stream;
  return with_type(s->type, [&](auto t) {
    using T = decltype(t);
    constexpr int PACK = sizeof(T) == 2 ? 8 : 4;
    if (s->vocab <= 16 * PACK && s->given == 1) launch_backward<T, 16, 1, false>(a, st);
    else if (s->vocab <= 32 * PACK && s->given == 1) launch_backward<T, 32, 1, false>(a, st);
    else if (s->vocab <= 64 * PACK) launch_backward<T, 64, 1, false>(a, st);
    else if (s->vocab <= 256 * PACK) launch_backward<T, 256, 1, false>(a, st);
    // What does not fit the last cache (256 MiB) goes past it: 8191 x 32003 bfloat16 258 -> 181 us, 4096 x 32003 floats 208 -> 170.  Smaller results may be
    // read from it by what comes next (1000 x 32003, 128 MB, would take 25 in place of 28 us here).
    else if (a.rows * a.vocab * (int64_t)sizeof(T) * 2 >= (int64_t)256 << 20) launch_backward<T, 256, 16 / PACK, true>(a, st);
    else launch_backward<T, 256, 16 / PACK, false>(a, st);
    return launch_status();
  });
}

}  // extern "C"
