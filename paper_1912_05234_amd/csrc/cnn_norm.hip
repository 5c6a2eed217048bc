// Entry points of the norms around a block, and the sum of their weight's gradient over workgroups.
#include "cnn_norm.h"

#include "cnn_fold.h"

namespace cnn {
namespace norm {
namespace {

constexpr int MOST_WIDTH = 16384, MOST_COLUMNS = 1 << 20;

struct PutWeight {
  float* d_weight;
  __device__ void operator()(int64_t c, float sum) const { d_weight[c] = sum; }
};

// (The hardware's root takes a number below 2^-126 for 0: a smaller eps would make rows of zeros NaN.)
bool shape_ok(const cnn_norm_shape* s) {
  return s && s->rows >= 1 && s->rows < (int64_t)1 << 31 && s->groups >= 1 && s->width >= 1 && s->width <= MOST_WIDTH &&
         (int64_t)s->groups * s->width <= MOST_COLUMNS && type_known(s->type) && (s->stream_type == s->type || s->stream_type == CNN_F32) &&
         s->eps >= 0x1p-126f && s->eps <= 1e30f && __builtin_fabsf(s->scale) <= 1e30f;
}

bool rows_ok(const cnn_rows* r, int type) {
  return r && r->data && reinterpret_cast<uintptr_t>(r->data) % type_bytes(type) == 0 && r->row >= 0;
}
bool rows_ok_or_null(const cnn_rows* r, int type) { return !r || rows_ok(r, type); }

Rows rows_of(const cnn_rows* r) { return r ? Rows{r->data, r->row} : Rows{nullptr, 0}; }

struct Plan {
  Cut cut;
  int at_once, beside, group_blocks;
  int64_t row_blocks;
  size_t bytes;  // of the partial gradients
};

// Workgroups: enough to fill the chip several times over and no more, as each keeps its weights for all its rows.  Backward each
// leaves a row of partial sums.
Plan plan_of(const cnn_norm_shape& s, bool backward) {
  Plan p{};
  p.cut = cut_of(s.width, pack_of(s.type, s.stream_type));
  const int teams = threads_of(p.cut.lanes) / p.cut.lanes;
  p.at_once = s.groups < teams ? s.groups : teams;
  p.beside = teams / p.at_once;
  p.group_blocks = (s.groups + p.at_once - 1) / p.at_once;
  const int64_t all = (s.rows + p.beside - 1) / p.beside;
  int64_t most = (backward ? 1024 : 2048) * 256 / threads_of(p.cut.lanes) / p.group_blocks;
  if (most < 1 || (backward && all <= 4)) most = 1;  // (a few rows after each other take less than a second kernel)
  p.row_blocks = all < most ? all : most;
  p.bytes = backward && p.row_blocks > 1 ? (size_t)p.row_blocks * s.groups * s.width * 4 : 0;
  return p;
}

Args args_of(const cnn_norm_shape& s, const Plan& p, const float* weight) {
  Args a{};
  a.weight = weight;
  a.rows = s.rows, a.row_blocks = p.row_blocks, a.groups = s.groups, a.width = s.width;
  a.at_once = p.at_once, a.beside = p.beside, a.group_blocks = p.group_blocks;
  a.scale = s.scale, a.eps = s.eps, a.by_width = 1.0f / (float)s.width;
  return a;
}

int run(Args& a, const cnn_norm_shape& s, const Plan& p, Mode mode, bool backward, float* d_weight, hipStream_t st) {
  const int64_t e = (int64_t)type_bytes(s.type), stream = (int64_t)type_bytes(s.stream_type);
  const int64_t each = mode == ADD ? (backward ? e + stream + (a.d_r.data ? stream : 0) + (a.y ? e : 0) + stream : 2 * e + (a.residual.data ? stream : 0) + (a.r ? stream : 0))
                                   : (backward ? stream + 2 * e : e + stream + (a.residual.data ? stream : 0)) + (a.gate.data ? (backward ? 2 * e : e) : 0);
  // What does not fit the last cache (256 MiB) goes past it, if rows are whole packs at aligned distances: 16381 rows of 2048, bfloat16 with a stream of
  // floats, forward 76 -> 63 us, backward 106 -> 92; 60000 rows of 541 153 -> 178; 200 MB of floats 38 -> 39.
  const int pack = pack_of(s.type, s.stream_type);
  bool even = s.width % pack == 0;
  for (const Rows* r : {&a.x, &a.residual, &a.gate, &a.d_y, &a.d_r}) even = even && r->row % pack == 0;
  a.past_caches = even && s.rows * s.groups * s.width * each >= (int64_t)256 << 20;
  const unsigned grid = (unsigned)(p.row_blocks * p.group_blocks);
  (s.type == CNN_F32 ? launch_f32 : s.type == CNN_BF16 ? launch_bf16 : launch_f16)(a, s.stream_type, mode, backward, p.cut, grid, st);
  if (launch_status() != CNN_OK) return CNN_EHIP;
  if (!p.bytes) return CNN_OK;
  return fold(a.partial, p.row_blocks, (int64_t)s.groups * s.width, PutWeight{d_weight}, st);
}

bool all_aligned(std::initializer_list<const void*> all) {
  for (const void* p : all)
    if (!aligned16(p)) return false;
  return true;
}

}  // namespace
}  // namespace norm
}  // namespace cnn

extern "C" {

size_t cnn_norm_bwd_workspace_bytes(const cnn_norm_shape* s) { return cnn::norm::shape_ok(s) ? cnn::norm::plan_of(*s, true).bytes : 0; }

int cnn_add_norm_fwd(const cnn_norm_shape* s, const cnn_rows* x, const cnn_rows* residual, const float* weight, void* y, void* r, void* hip_stream) {
  using namespace cnn;
  using namespace cnn::norm;
  if (!shape_ok(s) || !rows_ok(x, s->type) || !rows_ok_or_null(residual, s->stream_type) || !weight || !y || !all_aligned({weight, y, r})) return CNN_EINVAL;
  if (!residual && (r || s->scale != 1.0f || s->stream_type != s->type)) return CNN_EINVAL;
  const Plan p = plan_of(*s, false);
  Args a = args_of(*s, p, weight);
  a.x = rows_of(x), a.residual = rows_of(residual), a.y = y, a.r = r;
  return run(a, *s, p, ADD, false, nullptr, (hipStream_t)hip_stream);
}

int cnn_add_norm_bwd(const cnn_norm_shape* s, const cnn_rows* d_y, const cnn_rows* r, const cnn_rows* d_r, const float* weight, void* d_x,
                     void* d_residual, float* d_weight, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace cnn;
  using namespace cnn::norm;
  if (!shape_ok(s) || !rows_ok(d_y, s->type) || !rows_ok(r, s->stream_type) || !rows_ok_or_null(d_r, s->stream_type)) return CNN_EINVAL;
  if (!weight || !d_residual || !d_weight || !all_aligned({weight, d_x, d_residual, d_weight, workspace})) return CNN_EINVAL;
  const Plan p = plan_of(*s, true);
  if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return CNN_EWORKSPACE;
  Args a = args_of(*s, p, weight);
  a.x = rows_of(r), a.d_y = rows_of(d_y), a.d_r = rows_of(d_r), a.y = d_x, a.r = d_residual;
  a.partial = p.bytes ? static_cast<float*>(workspace) : d_weight;
  return run(a, *s, p, ADD, true, d_weight, (hipStream_t)hip_stream);
}

int cnn_norm_gate_fwd(const cnn_norm_shape* s, const cnn_rows* x, const cnn_rows* gate, const cnn_rows* residual, const float* weight, void* y,
                      void* hip_stream) {
  using namespace cnn;
  using namespace cnn::norm;
  if (!shape_ok(s) || !rows_ok(x, s->type) || !rows_ok_or_null(gate, s->type) || !rows_ok_or_null(residual, s->stream_type)) return CNN_EINVAL;
  if (!weight || !y || !all_aligned({weight, y})) return CNN_EINVAL;
  const Plan p = plan_of(*s, false);
  Args a = args_of(*s, p, weight);
  a.x = rows_of(x), a.gate = rows_of(gate), a.residual = rows_of(residual), a.y = y;
  return run(a, *s, p, GATE, false, nullptr, (hipStream_t)hip_stream);
}

int cnn_norm_gate_bwd(const cnn_norm_shape* s, const cnn_rows* d_y, const cnn_rows* x, const cnn_rows* gate, const float* weight, void* d_x,
                      void* d_gate, float* d_weight, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace cnn;
  using namespace cnn::norm;
  if (!shape_ok(s) || !rows_ok(d_y, s->stream_type) || !rows_ok(x, s->type) || !rows_ok_or_null(gate, s->type)) return CNN_EINVAL;
  if (!weight || !d_x || !d_weight || (gate != nullptr) != (d_gate != nullptr)) return CNN_EINVAL;
  if (!all_aligned({weight, d_x, d_gate, d_weight, workspace})) return CNN_EINVAL;
  const Plan p = plan_of(*s, true);
  if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return CNN_EWORKSPACE;
  Args a = args_of(*s, p, weight);
  a.x = rows_of(x), a.d_y = rows_of(d_y), a.gate = rows_of(gate), a.y = d_x, a.r = d_gate;
  a.partial = p.bytes ? static_cast<float*>(workspace) : d_weight;
  return run(a, *s, p, GATE, true, d_weight, (hipStream_t)hip_stream);
}

}  // extern "C"
