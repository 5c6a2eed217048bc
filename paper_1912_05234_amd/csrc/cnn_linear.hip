// Entry points of linear attention, its form for single tokens, and the kernels around the scan of cnn_linear.h.
#include "cnn_linear.h"

namespace cnn {
namespace linear {
namespace {

// ---- states of the segments --------------------------------------------------------------------------------------------
// carry[unit][j] holds what segment j adds to a state; afterwards the state that segment j starts from.  One pass over the states, each
// thread four elements of all segments, eight of them on their way at once: 16 segments of 32 states of 128 x 128, 67 MB, take 14 us.
constexpr int CARRY_THREADS = 256;
__global__ __launch_bounds__(CARRY_THREADS) void carry_kernel(Args args) {
  const Role& R = args.role[blockIdx.y];
  const int64_t size = carry_floats(R) / 4, groups = (size + CARRY_THREADS - 1) / CARRY_THREADS;
  const int64_t unit = blockIdx.x / groups, at = blockIdx.x % groups * CARRY_THREADS + threadIdx.x;
  if (unit >= args.units || at >= size) return;
  const int64_t n = length_of(args, unit / args.heads);
  const float a = args.decay[unit % args.heads];
  // [tile of columns][tile of rows][lane]
  const int tiles = R.DKP / 16, lane = (int)(at & 63), row = state_row((int)((at >> 6) % tiles), lane, 0);
  const int column = state_column((int)((at >> 6) / tiles), lane);
  f4 raw{0.0f, 0.0f, 0.0f, 0.0f};
  if (R.first && column < R.DV)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (row + i < R.DK) raw[i] = R.first[unit * R.DK * R.DV + (row + i) * R.first_i + column * R.first_j];
  f4 run = raw;
  f4* carry = reinterpret_cast<f4*>(R.carry) + unit * args.segments * size + at;
  const double log2a = log2((double)a);
  const auto power_of = [&](int64_t e) { return e > 0 ? (float)exp2(log2a * (double)e) : 1.0f; };
  const float full = power_of(args.segment_length);
  constexpr int AHEAD = 8;
  for (int j0 = 0; j0 < args.segments; j0 += AHEAD) {
    f4 added[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (j0 + i < args.segments) added[i] = carry[(j0 + i) * size];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int j = j0 + i;
      if (j >= args.segments) break;
      carry[j * size] = run;
      const int64_t begin = segment_begin(args, n, j), count = segment_end(args, n, j) - begin;
      if (count == 0) continue;
      const float by = begin == 0 ? power_of(R.reversed ? count - 1 : count) : full;
      run = run * by + added[i];
    }
  }
  if (R.last && column < R.DV) {
    if (n > 0) run *= R.last_by * (R.reversed ? a : 1.0f);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (row + i < R.DK) R.last[(unit * R.DK + row + i) * R.DV + column] = run[i];
  }
}

// ---- gradients of shared heads -----------------------------------------------------------------------------------------
// out[row][h][d] = sum over the query heads of h of part[row][head][d], part in fp32; for d_k and d_v.  (6141 rows of 12 heads of 64 and
// of 96 onto 4: 47 MB read, 9 us.)
struct ShareArgs {
  const float* part[2];
  void* out[2];
  int64_t rows;  // times key heads
  int width[2], share;
};

template <class T, int VN>
__global__ __launch_bounds__(256) void share_kernel(ShareArgs a) {
  using P = Pack<float, VN>;
  const int width = a.width[blockIdx.y] / VN, share = a.share;
  const P* part = reinterpret_cast<const P*>(a.part[blockIdx.y]);
  Pack<T, VN>* out = static_cast<Pack<T, VN>*>(a.out[blockIdx.y]);
  const int64_t total = a.rows * width;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = total < (int64_t)1 << 32 ? (uint32_t)i / (uint32_t)width : i / width;
    const P* p = part + row * share * width + (i - row * width);
    P sum = p[0];
    for (int h = 1; h < share; ++h) {
      const P q = p[(int64_t)h * width];
#pragma unroll
      for (int j = 0; j < VN; ++j) sum.v[j] += q.v[j];
    }
    Pack<T, VN> r;
#pragma unroll
    for (int j = 0; j < VN; ++j) r.v[j] = (T)sum.v[j];
    out[i] = r;
  }
}

// ---- one token ---------------------------------------------------------------------------------------------------------
struct StepArgs {
  Operand q, k, v;
  const float* decay;
  float* state;          // [pool][heads][DK][DV]
  const int32_t* slots;  // [batch], nullable: row b uses state b
  void* out;             // [batch][heads][DV]
  int64_t pool;
  int heads, DK, DV, blocks;
  float scale;
};

constexpr int STEP_THREADS = 256, STEP_COLUMNS = 32;

// A workgroup takes 32 columns of one state: the whole of DK, so that nothing has to be joined outside it.  Every thread
// updates VN columns of one row in so many, and keeps their products with q; these are added over the rows at the end.
// Memory bounds it: 256 rows of 16 states of 128 x 128 (537 MB read and written) take 96 us, after other work 102, 5.6 to 5.3 TB/s.
template <class T, int VN, bool PAST_CACHES>
__global__ __launch_bounds__(STEP_THREADS) void step_kernel(StepArgs a) {
  constexpr int LANES = STEP_COLUMNS / VN, ROWS = STEP_THREADS / LANES, AHEAD = 4;
  using P = Pack<float, VN>;
  __shared__ float sums[STEP_THREADS / 64][STEP_COLUMNS];
  const int64_t job = blockIdx.x / a.blocks, batch = job / a.heads;
  const int head = (int)(job % a.heads), lane = threadIdx.x % LANES, row0 = threadIdx.x / LANES;
  const int col = (int)(blockIdx.x % a.blocks) * STEP_COLUMNS + lane * VN;
  const int64_t slot = a.slots ? a.slots[batch] : batch;
  T* out = static_cast<T*>(a.out) + job * a.DV;
  const bool mine = col < a.DV;
  if (slot < 0 || slot >= a.pool) {  // no sequence here
    if (threadIdx.x < LANES && mine)
#pragma unroll
      for (int j = 0; j < VN; ++j) out[col + j] = (T)0.0f;
    return;
  }
  const auto base = [&](const Operand& o) { return static_cast<const T*>(o.data) + batch * o.batch + head / o.share * o.head; };
  const T *q = base(a.q), *k = base(a.k), *v = base(a.v);
  float* state = a.state + (slot * a.heads + head) * a.DK * a.DV;
  const float decay = a.decay[head];
  float value[VN], sum[VN];
#pragma unroll
  for (int j = 0; j < VN; ++j) value[j] = mine ? (float)v[col + j] : 0.0f, sum[j] = 0.0f;
  for (int i = row0; i < a.DK; i += ROWS * AHEAD) {
    P s[AHEAD];
    float key[AHEAD], query[AHEAD];
#pragma unroll
    for (int r = 0; r < AHEAD; ++r) {
      const int row = i + r * ROWS;
      if (row >= a.DK || !mine) continue;
      if constexpr (PAST_CACHES) s[r] = got_past_caches(reinterpret_cast<const P*>(state + (int64_t)row * a.DV + col));
      else s[r] = *reinterpret_cast<const P*>(state + (int64_t)row * a.DV + col);
      key[r] = (float)k[row], query[r] = (float)q[row];
    }
#pragma unroll
    for (int r = 0; r < AHEAD; ++r) {
      const int row = i + r * ROWS;
      if (row >= a.DK || !mine) continue;
#pragma unroll
      for (int j = 0; j < VN; ++j) {
        s[r].v[j] = s[r].v[j] * decay + key[r] * value[j];
        sum[j] += query[r] * s[r].v[j];
      }
      if constexpr (PAST_CACHES) put_past_caches(reinterpret_cast<P*>(state + (int64_t)row * a.DV + col), s[r]);
      else *reinterpret_cast<P*>(state + (int64_t)row * a.DV + col) = s[r];
    }
  }
#pragma unroll
  for (int j = 0; j < VN; ++j) {
#pragma unroll
    for (int d = LANES; d < 64; d *= 2) sum[j] += __shfl_xor(sum[j], d);
    if (threadIdx.x % 64 < LANES) sums[threadIdx.x / 64][lane * VN + j] = sum[j];
  }
  __syncthreads();
  if (threadIdx.x < STEP_COLUMNS) {
    const int c = (int)(blockIdx.x % a.blocks) * STEP_COLUMNS + threadIdx.x;
    float s = 0.0f;
    for (int w = 0; w < STEP_THREADS / 64; ++w) s += sums[w][threadIdx.x];
    if (c < a.DV) out[c] = (T)(s * a.scale);
  }
}

// ---- arguments and plans ---------------------------------------------------------------------------------------------------
bool shape_ok(const cnn_linear_shape* s) {
  return s && s->B >= 1 && s->T >= 1 && s->H >= 1 && s->Hk >= 1 && s->H % s->Hk == 0 && s->Dk >= 1 && s->Dk <= 256 && s->Dv >= 1 &&
         s->Dv <= 256 && type_known(s->type) && (int64_t)s->B * s->H <= 1 << 20;
}

bool heads_ok(const cnn_heads* h, int type) {
  return h && h->data && reinterpret_cast<uintptr_t>(h->data) % type_bytes(type) == 0 && h->batch >= 0 && h->token >= 0 && h->head >= 0;
}

// Rows made of whole packs at aligned addresses, whatever token, head and sequence.
bool packed_ok(const cnn_heads* h, int width, int type) {
  const int64_t unit = 16 / (int64_t)type_bytes(type);
  return aligned16(h->data) && width % 8 == 0 && h->batch % unit == 0 && h->token % unit == 0 && h->head % unit == 0 &&
         h->token * (int64_t)type_bytes(type) < 1 << 24;  // (the kernel multiplies by it in 24 bits)
}

// Results whose rows of one chunk lie less than 2^31 bytes apart.
bool near_ok(const cnn_linear_shape* s) { return (int64_t)s->H * (s->Dk > s->Dv ? s->Dk : s->Dv) < 1 << 23; }

Operand operand_of(const cnn_heads* h, int share) { return {h->data, h->batch, h->token, h->head, share}; }

struct Form {  // of a role's kernel
  int DKP, columns, blocks;
  int64_t floats() const { return (int64_t)DKP * columns * blocks; }
};

struct Plan {
  int segments;
  int64_t length;
  Form form[2];        // of the role d_v, and of forward; of the other two roles
  size_t state_bytes;  // of one role's states, all segments
  size_t wide_k, wide_v, bytes;
};

size_t rounded(size_t b) { return (b + 255) & ~(size_t)255; }

// How long the passes take that cut the time axis into segments of `length` tokens, in chunks of one wave of 128 x 32 that a SIMD
// works through (about 2 us).  Waves of a SIMD share it, and one alone leaves it waiting a third of the time (those of 256 columns are
// alone: their registers fill it); a wave's states, brought in and written, cost it as much as a chunk and a half.
double cost_of(const cnn_linear_shape& s, const Plan& p, int roles, int64_t length) {
  constexpr int64_t CUS = 256;
  const int64_t segments = (s.T + length - 1) / length, units = (int64_t)s.B * s.H;
  const auto pass = [&](const Form& f, int same) {
    const int64_t to_cu = (units * segments * f.blocks * same + CUS - 1) / CUS, to_simd = (to_cu * (f.columns / (16 * NW)) + 3) / 4;
    return (f.DKP > 128 ? 1.5 * (double)to_simd : to_simd > 1 ? (double)to_simd : 1.5) * ((double)(length / C) + 1.5) * (f.DKP + 64) / 192.0;
  };
  const bool joint = p.form[0].DKP == p.form[1].DKP && p.form[0].columns == p.form[1].columns;  // in one launch
  const double all = roles == 1 ? pass(p.form[0], 1) : joint ? pass(p.form[0], 3) : pass(p.form[1], 2) + pass(p.form[0], 1);
  if (segments == 1) return all;
  const double states = roles == 1 ? pass(p.form[0], 1) : joint ? pass(p.form[0], 2) : pass(p.form[1], 1) + pass(p.form[0], 1);
  const double moved = 8.0 * (double)(units * segments) * (double)(p.form[0].floats() + (roles == 1 ? 0 : p.form[1].floats()));  // between them
  return all + 0.45 * states + 2.5 + moved * 1.0e-7;  // (10 MB take as long as a chunk)
}

Plan plan_of(const cnn_linear_shape& s, int roles) {
  Plan p{};
  const int64_t units = (int64_t)s.B * s.H;
  // No segments whose state, written and read twice, is more to move than its tokens, both counted without the columns that pad them.
  // (So widths far from the padded ones may have more: Dk = 158, Dv = 6 holds states of 256 x 128, seventeen times the tokens' bytes.)
  const int64_t least = 16 * (int64_t)s.Dk * s.Dv / (2 * (s.Dk + s.Dv) * (int64_t)type_bytes(s.type));
  const int64_t most = s.T / (least > 2 * C ? least : 2 * C);
  double best = 0.0;
  // Each role in its own form, or all in one that holds them, which is one launch for two: 2 x 11 tokens of 12 heads of 80 x 128 (fp16)
  // take 7 us so and 15 us the other way.
  for (int joint = 0; joint < (roles == 1 ? 1 : 2); ++joint) {
    Plan now{};
    for (int f = 0; f < 2; ++f) {
      const int dk = f ? s.Dv : s.Dk, dv = f ? s.Dk : s.Dv;
      Form& form = now.form[f];
      form.DKP = padded(dk), form.columns = block_columns(dk, dv);
      if (joint) {
        const int other = block_columns(dv, dk);
        form.DKP = padded(dk > dv ? dk : dv);
        form.columns = form.columns > other ? form.columns : other;
      }
      form.blocks = (dv + form.columns - 1) / form.columns;
    }
    for (int64_t n = 1; n == 1 || (n <= most && n <= 256); ++n) {
      now.length = ((s.T + n - 1) / n + C - 1) / C * C;
      const double cost = cost_of(s, now, roles, now.length);
      if (best == 0.0 || cost < best) best = cost, p = now;
    }
  }
  p.segments = (int)((s.T + p.length - 1) / p.length);
  const int64_t floats = roles == 1 || p.form[0].floats() > p.form[1].floats() ? p.form[0].floats() : p.form[1].floats();
  p.state_bytes = p.segments > 1 ? rounded((size_t)units * p.segments * floats * 4) : 0;
  p.bytes = p.state_bytes * (roles > 1 ? 2 : 1);  // (d_k's states are d_v's transposed)
  if (roles > 1 && s.H != s.Hk) {
    p.wide_k = p.bytes;
    p.wide_v = p.wide_k + rounded((size_t)units * s.T * s.Dk * 4);
    p.bytes = p.wide_v + rounded((size_t)units * s.T * s.Dv * 4);
  }
  return p;
}

Args args_of(const cnn_linear_shape& s, const Plan& p, const float* decay, const int32_t* lengths) {
  Args a{};
  a.decay = decay, a.lengths = lengths;
  a.units = (int64_t)s.B * s.H, a.T = s.T, a.segment_length = p.length;
  a.heads = s.H, a.segments = p.segments;
  return a;
}

void set_form(Role& r, const Form& f) { r.DKP = f.DKP, r.columns = f.columns, r.blocks = f.blocks; }

int run(Args& a, int type, int roles, hipStream_t st) {
  const auto scan = type == CNN_F32 ? run_scan_f32 : type == CNN_BF16 ? run_scan_bf16 : run_scan_f16;
  if (a.segments > 1) {
    Args own = a;  // the roles that have states of their own
    int count = 0;
    int64_t groups = 0;
    for (int r = 0; r < roles; ++r) {
      if (a.role[r].flipped) continue;
      own.role[count++] = a.role[r];
      const int64_t g = (carry_floats(a.role[r]) / 4 + CARRY_THREADS - 1) / CARRY_THREADS;
      groups = g > groups ? g : groups;
    }
    const int rc = scan(own, count, true, st);
    if (rc != CNN_OK) return rc;
    carry_kernel<<<dim3((unsigned)(a.units * groups), (unsigned)count), CARRY_THREADS, 0, st>>>(own);
    if (launch_status() != CNN_OK) return CNN_EHIP;
  }
  return scan(a, roles, false, st);
}

}  // namespace
}  // namespace linear
}  // namespace cnn

extern "C" {

size_t cnn_linear_attention_fwd_workspace_bytes(const cnn_linear_shape* s) { return cnn::linear::shape_ok(s) ? cnn::linear::plan_of(*s, 1).bytes : 0; }

size_t cnn_linear_attention_bwd_workspace_bytes(const cnn_linear_shape* s) { return cnn::linear::shape_ok(s) ? cnn::linear::plan_of(*s, 3).bytes : 0; }

int cnn_linear_attention_fwd(const cnn_linear_shape* s, const cnn_heads* q, const cnn_heads* k, const cnn_heads* v, const float* decay,
                             float scale, const int32_t* lengths, const float* initial_state, void* o, float* final_state, void* workspace,
                             size_t workspace_bytes, void* hip_stream) {
  using namespace cnn;
  using namespace cnn::linear;
  if (!shape_ok(s) || !heads_ok(q, s->type) || !heads_ok(k, s->type) || !heads_ok(v, s->type) || !decay || !o) return CNN_EINVAL;
  for (const void* p : {(const void*)decay, (const void*)lengths, (const void*)initial_state, (const void*)o, (const void*)final_state, (const void*)workspace})
    if (!aligned16(p)) return CNN_EINVAL;
  const Plan p = plan_of(*s, 1);
  if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return CNN_EWORKSPACE;
  Args a = args_of(*s, p, decay, lengths);
  const int share = s->H / s->Hk;
  Role& r = a.role[0];
  r.q = operand_of(q, 1), r.k = operand_of(k, share), r.v = operand_of(v, share);
  r.out = o, r.first = initial_state, r.last = final_state, r.carry = static_cast<float*>(workspace);
  r.first_i = s->Dv, r.first_j = 1, r.DK = s->Dk, r.DV = s->Dv;
  set_form(r, p.form[0]);
  r.scale = scale, r.inside = r.last_by = 1.0f;
  r.packed = near_ok(s) && packed_ok(q, s->Dk, s->type) && packed_ok(k, s->Dk, s->type) && packed_ok(v, s->Dv, s->type);
  return run(a, s->type, 1, (hipStream_t)hip_stream);
}

int cnn_linear_attention_bwd(const cnn_linear_shape* s, const cnn_heads* q, const cnn_heads* k, const cnn_heads* v, const float* decay,
                             const cnn_heads* d_o, float scale, const int32_t* lengths, const float* initial_state, const float* d_final_state,
                             void* d_q, void* d_k, void* d_v, float* d_initial_state, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace cnn;
  using namespace cnn::linear;
  if (!shape_ok(s) || !heads_ok(q, s->type) || !heads_ok(k, s->type) || !heads_ok(v, s->type) || !heads_ok(d_o, s->type)) return CNN_EINVAL;
  if (!decay || !d_q || !d_k || !d_v) return CNN_EINVAL;
  for (const void* p : {(const void*)decay, (const void*)lengths, (const void*)initial_state, (const void*)d_final_state, (const void*)d_q, (const void*)d_k,
                        (const void*)d_v, (const void*)d_initial_state, (const void*)workspace})
    if (!aligned16(p)) return CNN_EINVAL;
  const float size = __builtin_fabsf(scale);
  if ((d_final_state || d_initial_state) && !(size >= 0x1p-100f && size <= 0x1p100f)) return CNN_EINVAL;
  const Plan p = plan_of(*s, 3);
  if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return CNN_EWORKSPACE;
  Args a = args_of(*s, p, decay, lengths);
  char* ws = static_cast<char*>(workspace);
  const int share = s->H / s->Hk;
  const Operand Q = operand_of(q, 1), K = operand_of(k, share), V = operand_of(v, share), D = operand_of(d_o, 1);
  const bool shared = share > 1;
  const bool packed = near_ok(s) && packed_ok(q, s->Dk, s->type) && packed_ok(k, s->Dk, s->type) && packed_ok(v, s->Dv, s->type) && packed_ok(d_o, s->Dv, s->type);
  for (int i = 0; i < 3; ++i) {
    Role& r = a.role[i];
    r.carry = reinterpret_cast<float*>(ws + (i ? p.state_bytes : 0));
    r.scale = scale, r.inside = 1.0f, r.last_by = scale, r.packed = packed;
    r.reversed = i > 0, r.wide = i > 0 && shared;
    r.DK = i < 2 ? s->Dv : s->Dk, r.DV = i < 2 ? s->Dk : s->Dv;
    set_form(r, p.form[i < 2]);
    r.first = i == 0 ? initial_state : d_final_state;
    r.first_i = i < 2 ? 1 : s->Dv, r.first_j = i < 2 ? s->Dv : 1;  // the first two hold the state transposed
    // An error of the state over the scale may be past the range of numbers, and a scale alone next to its end: the first is taken as it
    // is, and where there is none the scale comes last.
    if (i > 0 && d_final_state) r.scale = r.last_by = 1.0f, r.inside = scale;
  }
  a.role[0].q = D, a.role[0].k = V, a.role[0].v = K, a.role[0].out = d_q;
  a.role[1].q = V, a.role[1].k = D, a.role[1].v = Q, a.role[1].out = shared ? ws + p.wide_k : d_k;
  a.role[2].q = K, a.role[2].k = Q, a.role[2].v = D, a.role[2].out = shared ? ws + p.wide_v : d_v;
  a.role[2].last = d_initial_state;
  if (p.segments > 1) a.role[1].flipped = a.role[2].carry, a.role[1].flipped_rows = p.form[0].DKP, a.role[1].flipped_floats = p.form[0].floats();
  hipStream_t st = (hipStream_t)hip_stream;
  const int rc = run(a, s->type, 3, st);
  if (rc != CNN_OK || !shared) return rc;
  return with_type(s->type, [&](auto t) {
    using T = decltype(t);
    const ShareArgs g{{reinterpret_cast<const float*>(ws + p.wide_k), reinterpret_cast<const float*>(ws + p.wide_v)}, {d_k, d_v},
                      (int64_t)s->B * s->T * s->Hk, {s->Dk, s->Dv}, share};
    const bool fours = s->Dk % 4 == 0 && s->Dv % 4 == 0;
    const int64_t groups = (g.rows * (s->Dk > s->Dv ? s->Dk : s->Dv) / (fours ? 4 : 1) + 255) / 256;
    const dim3 grid((unsigned)(groups < 4096 ? groups : 4096), 2);
    if (fours) share_kernel<T, 4><<<grid, 256, 0, st>>>(g);
    else share_kernel<T, 1><<<grid, 256, 0, st>>>(g);
    return launch_status();
  });
}

int cnn_linear_attention_step(const cnn_linear_shape* s, const cnn_heads* q, const cnn_heads* k, const cnn_heads* v, const float* decay,
                              float scale, float* state, int64_t pool, const int32_t* slots, void* o, void* hip_stream) {
  using namespace cnn;
  using namespace cnn::linear;
  if (!shape_ok(s) || s->T != 1 || !heads_ok(q, s->type) || !heads_ok(k, s->type) || !heads_ok(v, s->type) || !decay || !state || !o) return CNN_EINVAL;
  if (pool < 1 || pool > 1 << 30 || (!slots && pool < s->B)) return CNN_EINVAL;
  for (const void* p : {(const void*)decay, (const void*)state, (const void*)slots, (const void*)o})
    if (!aligned16(p)) return CNN_EINVAL;
  const int share = s->H / s->Hk, blocks = (s->Dv + STEP_COLUMNS - 1) / STEP_COLUMNS;
  const StepArgs a{operand_of(q, 1), operand_of(k, share), operand_of(v, share), decay, state, slots, o, pool, s->H, s->Dk, s->Dv, blocks, scale};
  const unsigned grid = (unsigned)((int64_t)s->B * s->H * blocks);
  // States that do not fit the last cache (256 MiB) go past it.  Again and again, and after other work that filled it: 252 MB of them 78 and
  // 114 us, past the caches 91 and 97; 268 MB 96 and 118, 96 and 102; 302 MB 113 and 130, 108 and 113; 403 MB 160 and 167, 143 and 149;
  // and 134 MB 44 and 67, 50 and 56.  (What a server's other layers leave of smaller states is not known here.)
  const bool past_caches = (int64_t)s->B * s->H * s->Dk * s->Dv * 4 >= (int64_t)256 << 20;
  return with_type(s->type, [&](auto t) {
    using T = decltype(t);
    if (past_caches && s->Dv % 4 == 0) step_kernel<T, 4, true><<<grid, STEP_THREADS, 0, (hipStream_t)hip_stream>>>(a);
    else if (s->Dv % 4 == 0) step_kernel<T, 4, false><<<grid, STEP_THREADS, 0, (hipStream_t)hip_stream>>>(a);
    else step_kernel<T, 1, false><<<grid, STEP_THREADS, 0, (hipStream_t)hip_stream>>>(a);
    return launch_status();
  });
}

}  // extern "C"
