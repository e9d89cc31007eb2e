// Entry points on scaled 8-bit floats, norms, and tokens dealt to experts: host-side checks and dispatch.  Everything is checked
// before anything is launched.
#include "checks.h"
#include "f8.h"

#include <math.h>
#include <string.h>

#include <initializer_list>

using namespace gs;

namespace {

constexpr int64_t kMost = int64_t(1) << 40;       // elements of a pattern

int64_t product(const int64_t* v, int n) {
  int64_t p = 1;
  for (int i = 0; i < n; ++i) p *= v[i];
  return p;
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// A pattern as matrices of rows: the last access dimension, in as many as the others have.
struct Matrices {
  int64_t mats, rows, cols;
  int64_t count() const { return mats * rows; }
};
int64_t values_bytes(const Matrices& m) { return m.count() * f8_blocks(m.cols) * kF8Block; }
int64_t scales_bytes(const Matrices& m, int block_rows) { return m.mats * ceil_div(m.rows, block_rows) * f8_scale_pitch(m.cols) * 4; }

// `need_data` as for check_ap.
int check_f8(const gs_f8* m, bool need_data, Matrices* of) {
  if (!m) return GS_ERR_NULL;
  if (m->rank < 0 || m->rank > GS_MAX_RANK || m->n_access < 0 || m->n_access > m->rank) return GS_ERR_RANK;
  if (m->reserved != 0 || (m->block_rows != 1 && m->block_rows != kF8Block)) return GS_ERR_UNSUPPORTED;
  int64_t n = 1;
  for (int i = 0; i < m->rank; ++i) {
    if (m->shape[i] < 0) return GS_ERR_SHAPE;
    if (m->shape[i] > 0 && n > kMost / m->shape[i]) return GS_ERR_UNSUPPORTED;
    n *= m->shape[i];
  }
  // each part by itself too: where one has no elements, the others may be of any size
  int64_t part[3] = {1, 1, 1};
  for (int i = 0; i < m->rank; ++i) {
    int64_t* side = &part[i >= m->n_access ? 2 : i == m->n_access - 1 ? 1 : 0];
    if (m->shape[i] > 0 && *side > kMost / m->shape[i]) return GS_ERR_UNSUPPORTED;
    *side *= m->shape[i];
  }
  *of = Matrices{part[0], part[1], part[2]};
  if (of->cols > 0 && of->rows > 0 && of->mats > kMost / round_up(of->rows, kF8Block)) return GS_ERR_UNSUPPORTED;
  if (of->cols > 0 && of->mats * of->rows > kMost / round_up(of->cols, 4 * kF8Block)) return GS_ERR_UNSUPPORTED;
  if (need_data && n > 0) {
    if (!m->values || !m->scales) return GS_ERR_NULL;
    if (!aligned16(m->values) || !aligned16(m->scales)) return GS_ERR_UNSUPPORTED;
  }
  return GS_OK;
}

template <typename A, typename B>
bool same_pattern_shape(const A* a, const B* b) {
  if (a->rank != b->rank) return false;
  for (int i = 0; i < a->rank; ++i)
    if (a->shape[i] != b->shape[i]) return false;
  return true;
}

// Does any of the results share bytes with any of the inputs, or with another result?  Each may be NULL.
bool shares(std::initializer_list<const gs_ap*> results, std::initializer_list<const gs_ap*> inputs) {
  for (auto r = results.begin(); r != results.end(); ++r) {
    if (!*r) continue;
    for (const gs_ap* in : inputs)
      if (in && overlaps(*r, in)) return true;
    for (auto other = results.begin(); other != r; ++other)
      if (*other && overlaps(*r, *other)) return true;
  }
  return false;
}

// An array of a pattern held in F8, as bytes.
gs_ap bytes_of(void* data, int64_t bytes) {
  gs_ap a;
  memset(&a, 0, sizeof(a));
  a.data = data;
  a.dtype = GS_I8;
  a.rank = 1;
  a.shape[0] = bytes;
  return a;
}

bool is_float(int dtype) { return dtype == GS_BF16 || dtype == GS_F32; }

int convert_args(const gs_ap* plain, const gs_f8* m, F8ConvertArgs* a) {
  int st = check_ap(plain, true);
  if (st) return st;
  Matrices of;
  st = check_f8(m, true, &of);
  if (st) return st;
  if (plain->rank != m->rank || plain->n_access != m->n_access) return GS_ERR_RANK;
  if (!same_pattern_shape(plain, m)) return GS_ERR_SHAPE;
  if (!is_float(plain->dtype)) return GS_ERR_DTYPE;
  *a = F8ConvertArgs{plain->data, m->values, static_cast<float*>(m->scales), plain->dtype, m->block_rows, of.mats, of.rows, of.cols};
  return GS_OK;
}

int norm_args(const gs_ap* x, const gs_ap* residual, const gs_ap* weight, float eps, const gs_ap* sum, NormArgs* a) {
  int st = check_ap(x, true);
  if (st) return st;
  if (!is_float(x->dtype)) return GS_ERR_DTYPE;
  memset(a, 0, sizeof(*a));
  for (const gs_ap* o : {residual, sum}) {
    if (!o) continue;
    st = check_ap(o, true);
    if (st) return st;
    if (o->rank != x->rank || o->n_access != x->n_access) return GS_ERR_RANK;
    if (!same_pattern_shape(o, x)) return GS_ERR_SHAPE;
    if (o->dtype != x->dtype) return GS_ERR_DTYPE;
  }
  if (weight) {
    st = check_ap(weight, true);
    if (st) return st;
    const int nc = x->rank - x->n_access;
    if (weight->rank != nc || weight->n_access != 0) return GS_ERR_RANK;
    for (int i = 0; i < nc; ++i)
      if (weight->shape[i] != x->shape[x->n_access + i]) return GS_ERR_SHAPE;
    if (!is_float(weight->dtype)) return GS_ERR_DTYPE;
    a->weight = weight->data;
    a->w_dtype = weight->dtype;
  }
  if (!(eps >= 0.0f) || !isfinite(eps)) return GS_ERR_UNSUPPORTED;
  a->x = x->data;
  a->residual = residual ? residual->data : nullptr;
  a->sum = sum ? sum->data : nullptr;
  a->dtype = x->dtype;
  a->eps = eps;
  a->rows = product(x->shape, x->n_access);
  a->cols = product(x->shape + x->n_access, x->rank - x->n_access);
  return GS_OK;
}

// Blocks of 128 rows have to be those of all rows together.
bool blocks_in_line(const gs_f8* m, const Matrices& of) { return m->block_rows == 1 || of.mats <= 1 || of.rows % kF8Block == 0; }

int operand_args(const gs_f8* a0, const gs_f8* a1, bool need_data, Matrices* x, Matrices* w, F8DotArgs* a) {
  int st = check_f8(a0, need_data, x);
  if (st) return st;
  st = check_f8(a1, need_data, w);
  if (st) return st;
  const int nc = a0->rank - a0->n_access;
  if (nc != a1->rank - a1->n_access) return GS_ERR_SHAPE;
  for (int d = 0; d < nc; ++d)
    if (a0->shape[a0->n_access + d] != a1->shape[a1->n_access + d]) return GS_ERR_SHAPE;
  memset(a, 0, sizeof(*a));
  a->x = static_cast<const uint8_t*>(a0->values);
  a->xs = static_cast<const float*>(a0->scales);
  a->w = static_cast<const uint8_t*>(a1->values);
  a->ws = static_cast<const float*>(a1->scales);
  a->x_rows = a0->block_rows;
  a->w_rows = a1->block_rows;
  a->K = f8_blocks(x->cols) * kF8Block;
  a->pitch = f8_scale_pitch(x->cols);
  return GS_OK;
}

// One matrix for all rows.
int dot_args(const gs_f8* a0, const gs_f8* a1, bool need_data, F8DotArgs* a) {
  Matrices x, w;
  const int st = operand_args(a0, a1, need_data, &x, &w, a);
  if (st) return st;
  if (!blocks_in_line(a0, x) || !blocks_in_line(a1, w)) return GS_ERR_UNSUPPORTED;
  a->M = a->x_count = x.count();
  a->N = w.count();
  return GS_OK;
}

// A matrix ((E, N), (K)) of which every expert has N rows.
int expert_args(const gs_f8* a0, int64_t rows, const gs_f8* a1, bool need_data, F8DotArgs* a) {
  Matrices x, w;
  const int st = operand_args(a0, a1, need_data, &x, &w, a);
  if (st) return st;
  if (a1->n_access != 2) return GS_ERR_RANK;
  if (!blocks_in_line(a0, x)) return GS_ERR_UNSUPPORTED;
  if (rows > (int64_t(1) << 30) || x.count() > (int64_t(1) << 31) - 1 || w.mats > (int64_t(1) << 30)) return GS_ERR_UNSUPPORTED;
  a->M = rows;
  a->N = w.rows;
  a->experts = w.mats;
  a->x_count = x.count();
  if (a->x_count == 0) a->K = 0;        // (every row is one that x does not have)
  return GS_OK;
}

int check_result(const gs_ap* out, int act) {
  const int st = check_ap(out, true);
  if (st) return st;
  if (act != GS_ACT_NONE && act != GS_ACT_RELU) return GS_ERR_UNSUPPORTED;
  if (out->n_access != out->rank) return GS_ERR_RANK;
  return is_float(out->dtype) ? GS_OK : GS_ERR_DTYPE;
}

int run_dot(F8DotArgs& a, gs_ap* out, int act, void* workspace, size_t workspace_bytes, void* stream) {
  if (a.offsets && a.experts == 0) return GS_OK;      // (every row is nobody's)
  a.out = out->data;
  a.out_dtype = out->dtype;
  a.relu = act == GS_ACT_RELU;
  const F8DotPlan plan = plan_f8_dot(a.M, a.N, a.K, a.experts);
  if (plan.part_bytes && (!workspace || !aligned16(workspace) || workspace_bytes < plan.part_bytes)) return GS_ERR_WORKSPACE;
  return launch_status(launch_f8_dot(a, plan, workspace, static_cast<hipStream_t>(stream)));
}

// One i32 each of `rank` dimensions, all of them access dimensions.
int check_indices(const gs_ap* a, int rank) {
  const int st = check_ap(a, true);
  if (st) return st;
  if (a->rank != rank || a->n_access != rank) return GS_ERR_RANK;
  return a->dtype == GS_I32 ? GS_OK : GS_ERR_DTYPE;
}

// Tokens (T, cols) and rows (M, cols), both with one access dimension; places (T, choices), weights alike.
int rows_args(const gs_ap* flat, const gs_ap* rows, const gs_ap* places, const gs_ap* weights, ExpertRowsArgs* a) {
  int st = check_ap(flat, true);
  if (st) return st;
  st = check_ap(rows, true);
  if (st) return st;
  st = check_indices(places, 2);
  if (st) return st;
  if (flat->n_access != 1 || rows->n_access != 1 || flat->rank != rows->rank) return GS_ERR_RANK;
  for (int i = 1; i < flat->rank; ++i)
    if (flat->shape[i] != rows->shape[i]) return GS_ERR_SHAPE;
  if (flat->shape[0] != places->shape[0]) return GS_ERR_SHAPE;
  if (weights) {
    st = check_ap(weights, true);
    if (st) return st;
    if (weights->rank != 2 || weights->n_access != 2) return GS_ERR_RANK;
    if (weights->dtype != GS_F32) return GS_ERR_DTYPE;
    if (!same_pattern_shape(weights, places)) return GS_ERR_SHAPE;
  }
  memset(a, 0, sizeof(*a));
  a->places = static_cast<const int32_t*>(places->data);
  a->weights = weights ? static_cast<const float*>(weights->data) : nullptr;
  a->tokens = places->shape[0];
  a->choices = places->shape[1];
  a->cols = product(flat->shape + 1, flat->rank - 1);
  a->count = rows->shape[0];
  return GS_OK;
}

}  // namespace

extern "C" {

int glenside_f8_sizes(const gs_f8* m, size_t* values, size_t* scales) {
  Matrices of;
  const int st = check_f8(m, false, &of);
  if (st) return st;
  if (!values || !scales) return GS_ERR_NULL;
  *values = size_t(values_bytes(of));
  *scales = size_t(scales_bytes(of, m->block_rows));
  return GS_OK;
}

int glenside_f8_quantize(const gs_ap* in, gs_f8* out, void* stream) {
  F8ConvertArgs a;
  const int st = convert_args(in, out, &a);
  return st ? st : launch_status(launch_f8_quantize(a, static_cast<hipStream_t>(stream)));
}

int glenside_f8_dequantize(const gs_f8* in, gs_ap* out, void* stream) {
  F8ConvertArgs a;
  const int st = convert_args(out, in, &a);
  return st ? st : launch_status(launch_f8_dequantize(a, static_cast<hipStream_t>(stream)));
}

int glenside_norm(const gs_ap* x, const gs_ap* residual, const gs_ap* weight, float eps, gs_ap* sum, gs_ap* out, void* stream) {
  NormArgs a;
  int st = norm_args(x, residual, weight, eps, sum, &a);
  if (st) return st;
  st = check_ap(out, true);
  if (st) return st;
  if (out->rank != x->rank || out->n_access != x->n_access) return GS_ERR_RANK;
  if (!same_pattern_shape(out, x)) return GS_ERR_SHAPE;
  if (!is_float(out->dtype)) return GS_ERR_DTYPE;
  if (shares({sum, out}, {x, residual, weight})) return GS_ERR_UNSUPPORTED;
  a.out = out->data;
  a.out_dtype = out->dtype;
  return launch_status(launch_norm(a, static_cast<hipStream_t>(stream)));
}

int glenside_f8_norm(const gs_ap* x, const gs_ap* residual, const gs_ap* weight, float eps, gs_ap* sum, gs_f8* out, void* stream) {
  NormArgs a;
  int st = norm_args(x, residual, weight, eps, sum, &a);
  if (st) return st;
  Matrices of;
  st = check_f8(out, true, &of);
  if (st) return st;
  if (out->rank != x->rank || out->n_access != x->n_access) return GS_ERR_RANK;
  if (!same_pattern_shape(out, x)) return GS_ERR_SHAPE;
  if (out->block_rows != 1) return GS_ERR_UNSUPPORTED;
  const gs_ap values = bytes_of(out->values, values_bytes(of)), scales = bytes_of(out->scales, scales_bytes(of, 1));
  if (shares({sum, &values, &scales}, {x, residual, weight})) return GS_ERR_UNSUPPORTED;
  a.out = out->values;
  a.scales = static_cast<float*>(out->scales);
  a.out_dtype = GS_F8;
  return launch_status(launch_norm(a, static_cast<hipStream_t>(stream)));
}

int glenside_f8_dot(const gs_f8* a0, const gs_f8* a1, gs_ap* out, int act, void* workspace, size_t workspace_bytes, void* stream) {
  F8DotArgs a;
  int st = dot_args(a0, a1, true, &a);
  if (st) return st;
  st = check_result(out, act);
  if (st) return st;
  if (out->rank != a0->n_access + a1->n_access) return GS_ERR_RANK;
  for (int d = 0; d < a0->n_access; ++d)
    if (out->shape[d] != a0->shape[d]) return GS_ERR_SHAPE;
  for (int d = 0; d < a1->n_access; ++d)
    if (out->shape[a0->n_access + d] != a1->shape[d]) return GS_ERR_SHAPE;
  return run_dot(a, out, act, workspace, workspace_bytes, stream);
}

size_t glenside_f8_dot_workspace(const gs_f8* a0, const gs_f8* a1) {
  F8DotArgs a;
  return dot_args(a0, a1, false, &a) ? 0 : plan_f8_dot(a.M, a.N, a.K, 0).part_bytes;
}

int glenside_f8_expert_dot(const gs_f8* a0, const gs_ap* tokens, const gs_ap* offsets, const gs_f8* a1, gs_ap* out, int act, void* workspace,
                           size_t workspace_bytes, void* stream) {
  int st = check_result(out, act);
  if (st) return st;
  if (out->rank != 2) return GS_ERR_RANK;
  F8DotArgs a;
  st = expert_args(a0, out->shape[0], a1, true, &a);
  if (st) return st;
  if (out->shape[1] != a.N) return GS_ERR_SHAPE;
  st = check_indices(offsets, 1);
  if (st) return st;
  if (offsets->shape[0] != a.experts + 1) return GS_ERR_SHAPE;
  a.offsets = static_cast<const int32_t*>(offsets->data);
  if (tokens) {
    st = check_indices(tokens, 1);
    if (st) return st;
    if (tokens->shape[0] != a.M) return GS_ERR_SHAPE;
    a.tokens = static_cast<const int32_t*>(tokens->data);
  } else if (a.x_count != a.M) {
    return GS_ERR_SHAPE;
  }
  return run_dot(a, out, act, workspace, workspace_bytes, stream);
}

size_t glenside_f8_expert_dot_workspace(const gs_f8* a0, int64_t rows, const gs_f8* a1) {
  F8DotArgs a;
  return rows < 0 || expert_args(a0, rows, a1, false, &a) || a.experts == 0 ? 0 : plan_f8_dot(a.M, a.N, a.K, a.experts).part_bytes;
}

size_t glenside_expert_sort_workspace(int64_t choices, int64_t n_experts) {
  if (choices < 0 || n_experts < 0 || n_experts > 4096 || choices > (int64_t(1) << 30)) return 0;
  return expert_sort_workspace(choices, n_experts);
}

int glenside_expert_sort(const gs_ap* experts, gs_ap* offsets, gs_ap* tokens, gs_ap* places, void* workspace, size_t workspace_bytes, void* stream) {
  int st = check_indices(experts, 2);
  if (st) return st;
  st = check_indices(offsets, 1);
  if (st) return st;
  st = check_indices(tokens, 1);
  if (st) return st;
  st = check_indices(places, 2);
  if (st) return st;
  ExpertSortArgs a;
  memset(&a, 0, sizeof(a));
  a.choices = experts->shape[1];
  a.n = experts->shape[0] * a.choices;
  a.n_experts = offsets->shape[0] - 1;
  if (a.n_experts < 0 || tokens->shape[0] != a.n || !same_pattern_shape(places, experts)) return GS_ERR_SHAPE;
  if (a.n > (int64_t(1) << 30) || a.choices > (int64_t(1) << 30) || a.n_experts > 4096) return GS_ERR_UNSUPPORTED;
  const size_t need = expert_sort_workspace(a.n, a.n_experts);
  if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return GS_ERR_WORKSPACE;
  if (shares({offsets, tokens, places}, {experts})) return GS_ERR_UNSUPPORTED;
  a.experts = static_cast<const int32_t*>(experts->data);
  a.offsets = static_cast<int32_t*>(offsets->data);
  a.tokens = static_cast<int32_t*>(tokens->data);
  a.places = static_cast<int32_t*>(places->data);
  a.counts = static_cast<int32_t*>(workspace);
  return launch_status(launch_expert_sort(a, static_cast<hipStream_t>(stream)));
}

int glenside_expert_split(const gs_ap* x, const gs_ap* places, gs_ap* rows, void* stream) {
  ExpertRowsArgs a;
  const int st = rows_args(x, rows, places, nullptr, &a);
  if (st) return st;
  if (x->dtype != rows->dtype) return GS_ERR_DTYPE;
  if (shares({rows}, {x, places})) return GS_ERR_UNSUPPORTED;
  a.flat = x->data;
  a.rows_out = rows->data;
  a.dtype = x->dtype;
  return launch_status(launch_expert_split(a, static_cast<hipStream_t>(stream)));
}

int glenside_expert_join(const gs_ap* rows, const gs_ap* places, const gs_ap* weights, gs_ap* out, void* stream) {
  ExpertRowsArgs a;
  const int st = rows_args(out, rows, places, weights, &a);
  if (st) return st;
  if (!is_float(rows->dtype) || !is_float(out->dtype)) return GS_ERR_DTYPE;
  if (shares({out}, {rows, places, weights})) return GS_ERR_UNSUPPORTED;
  a.flat_out = out->data;
  a.rows = rows->data;
  a.dtype = rows->dtype;
  a.out_dtype = out->dtype;
  return launch_status(launch_expert_join(a, static_cast<hipStream_t>(stream)));
}

int glenside_expert_join_grad(const gs_ap* grad, const gs_ap* rows, const gs_ap* places, const gs_ap* weights, gs_ap* grad_rows, gs_ap* grad_weights,
                              void* stream) {
  ExpertRowsArgs a;
  int st = rows_args(grad, rows, places, weights, &a);
  if (st) return st;
  st = check_ap(grad_rows, true);
  if (st) return st;
  if (grad_rows->rank != rows->rank || grad_rows->n_access != 1) return GS_ERR_RANK;
  if (!same_pattern_shape(grad_rows, rows)) return GS_ERR_SHAPE;
  if (!is_float(grad->dtype) || rows->dtype != grad->dtype || grad_rows->dtype != grad->dtype) return GS_ERR_DTYPE;
  if (grad_weights) {
    st = check_ap(grad_weights, true);
    if (st) return st;
    if (grad_weights->rank != 2 || grad_weights->n_access != 2) return GS_ERR_RANK;
    if (grad_weights->dtype != GS_F32) return GS_ERR_DTYPE;
    if (!same_pattern_shape(grad_weights, places)) return GS_ERR_SHAPE;
    a.grad_weights = static_cast<float*>(grad_weights->data);
  }
  if (shares({grad_rows, grad_weights}, {grad, rows, places, weights})) return GS_ERR_UNSUPPORTED;
  a.flat = grad->data;
  a.rows = rows->data;
  a.rows_out = grad_rows->data;
  a.dtype = grad->dtype;
  return launch_status(launch_expert_join_grad(a, static_cast<hipStream_t>(stream)));
}

// For tests, not part of the interface: how a product of these sizes (K in numbers; experts 0: one matrix) is done, F8DotWay and workgroups that share a
// sum.  Host only.
int gs_test_f8_dot_plan(int64_t M, int64_t N, int64_t K, int64_t experts, int plan[2]) {
  const F8DotPlan p = plan_f8_dot(M, N, f8_blocks(K) * kF8Block, experts);
  plan[0] = p.way;
  plan[1] = p.splits;
  return GS_OK;
}

}  // extern "C"
