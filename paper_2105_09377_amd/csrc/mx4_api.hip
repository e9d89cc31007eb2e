// Entry points on microscaled 4-bit floats: host-side checks and dispatch.  Everything is checked before anything is
// launched.
#include "checks.h"
#include "mx4.h"

#include <limits.h>
#include <math.h>
#include <string.h>

using namespace gs;

namespace {

constexpr int64_t kMost = int64_t(1) << 40;       // elements of a pattern

int64_t product(const int64_t* v, int n) {
  int64_t p = 1;
  for (int i = 0; i < n; ++i) p *= v[i];
  return p;
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Rows and numbers per row of an MX4 pattern; `need_data` as for check_ap.
int check_mx4(const gs_mx4* m, bool need_data, int64_t* rows, int64_t* cols) {
  if (!m) return GS_ERR_NULL;
  if (m->rank < 0 || m->rank > GS_MAX_RANK || m->n_access < 0 || m->n_access > m->rank) return GS_ERR_RANK;
  int64_t n = 1;
  for (int i = 0; i < m->rank; ++i) {
    if (m->shape[i] < 0) return GS_ERR_SHAPE;
    if (m->shape[i] > 0 && n > kMost / m->shape[i]) return GS_ERR_UNSUPPORTED;
    n *= m->shape[i];
  }
  // each side by itself too: where one has no elements, the other may be of any size
  *rows = *cols = 1;
  for (int i = 0; i < m->rank; ++i) {
    int64_t* side = i < m->n_access ? rows : cols;
    if (m->shape[i] > 0 && *side > kMost / m->shape[i]) return GS_ERR_UNSUPPORTED;
    *side *= m->shape[i];
  }
  if (*cols > 0 && *rows > kMost / round_up(*cols, 256)) return GS_ERR_UNSUPPORTED;
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

int convert_args(const gs_ap* plain, const gs_mx4* m, Mx4ConvertArgs* a) {
  int st = check_ap(plain, true);
  if (st) return st;
  int64_t rows, cols;
  st = check_mx4(m, true, &rows, &cols);
  if (st) return st;
  if (plain->rank != m->rank || plain->n_access != m->n_access) return GS_ERR_RANK;
  if (!same_pattern_shape(plain, m)) return GS_ERR_SHAPE;
  if (plain->dtype != GS_BF16 && plain->dtype != GS_F32) return GS_ERR_DTYPE;
  *a = Mx4ConvertArgs{plain->data, m->values, m->scales, plain->dtype, rows, cols};
  return GS_OK;
}

// Checks that do not need data pointers are made where `need_data` is false too (workspace queries).
int check_cache(const gs_mx4_cache* c, bool need_data) {
  if (!c) return GS_ERR_NULL;
  if (c->reserved != 0) return GS_ERR_UNSUPPORTED;
  if (c->n_pages < 0 || c->heads < 1) return GS_ERR_SHAPE;
  if (c->page_size < 16 || c->page_size > 4096 || c->page_size % 16) return GS_ERR_UNSUPPORTED;
  const int d = c->head_dim;
  if (d != 64 && d != 96 && d != 128 && d != 192 && d != 256) return GS_ERR_UNSUPPORTED;
  if (c->heads > (1 << 16) || c->n_pages > kMost / c->heads / c->page_size / (2 * d)) return GS_ERR_UNSUPPORTED;
  if (need_data && c->n_pages > 0) {
    if (!c->data) return GS_ERR_NULL;
    if (!aligned16(c->data)) return GS_ERR_UNSUPPORTED;
  }
  return GS_OK;
}

Mx4CacheShape cache_shape(const gs_mx4_cache* c) {
  Mx4CacheShape s;
  s.data = static_cast<uint8_t*>(c->data);
  s.n_pages = c->n_pages;
  s.page = c->page_size;
  s.heads = c->heads;
  s.dim = c->head_dim;
  s.by_page = FastDiv::make(uint32_t(c->page_size));
  return s;
}

// The table of `batch` sequences; positions stay below 2^30.
int check_table(const gs_ap* table, const gs_mx4_cache* c, int64_t batch, bool need_data) {
  int st = check_ap(table, need_data);
  if (st) return st;
  if (table->rank != 2 || table->n_access != 1) return GS_ERR_RANK;
  if (table->dtype != GS_I32) return GS_ERR_DTYPE;
  if (table->shape[0] != batch) return GS_ERR_SHAPE;
  if (table->shape[1] > (int64_t(1) << 30) / c->page_size) return GS_ERR_UNSUPPORTED;
  return GS_OK;
}
int check_per_sequence(const gs_ap* a, int64_t batch) {
  int st = check_ap(a, true);
  if (st) return st;
  if (a->rank != 1 || a->n_access != 1) return GS_ERR_RANK;
  if (a->dtype != GS_I32) return GS_ERR_DTYPE;
  return a->shape[0] == batch ? GS_OK : GS_ERR_SHAPE;
}

int token_args(const gs_mx4_cache* c, const gs_ap* table, const gs_ap* first, const gs_ap* counts, const gs_ap* k, const gs_ap* v,
               Mx4TokenArgs* a) {
  int st = check_cache(c, true);
  if (st) return st;
  st = check_ap(k, true);
  if (st) return st;
  st = check_ap(v, true);
  if (st) return st;
  if (k->rank != 4 || k->n_access != 3 || v->rank != 4 || v->n_access != 3) return GS_ERR_RANK;
  if (k->dtype != v->dtype || (k->dtype != GS_BF16 && k->dtype != GS_F32)) return GS_ERR_DTYPE;
  if (!same_pattern_shape(k, v) || k->shape[2] != c->heads || k->shape[3] != c->head_dim) return GS_ERR_SHAPE;
  const int64_t batch = k->shape[0];
  st = check_table(table, c, batch, true);
  if (st) return st;
  st = check_per_sequence(first, batch);
  if (st) return st;
  if (counts) {
    st = check_per_sequence(counts, batch);
    if (st) return st;
  }
  memset(a, 0, sizeof(*a));
  a->cache = cache_shape(c);
  a->table = static_cast<const int32_t*>(table->data);
  a->first = static_cast<const int32_t*>(first->data);
  a->counts = counts ? static_cast<const int32_t*>(counts->data) : nullptr;
  a->k = k->data;
  a->v = v->data;
  a->dtype = k->dtype;
  a->batch = batch;
  a->width = table->shape[1];
  a->tokens = k->shape[1];
  return GS_OK;
}

// Shapes of an attention; pointers are looked at by the caller.
int attend_args(const gs_ap* q, const gs_mx4_cache* c, const gs_ap* table, int64_t window, int64_t sinks, bool need_data, Mx4AttendArgs* a) {
  int st = check_cache(c, need_data);
  if (st) return st;
  st = check_ap(q, need_data);
  if (st) return st;
  if (q->rank != 4 || q->n_access != 3) return GS_ERR_RANK;
  if (q->dtype != GS_BF16) return GS_ERR_DTYPE;
  if (q->shape[3] != c->head_dim || q->shape[2] % c->heads) return GS_ERR_SHAPE;
  st = check_table(table, c, q->shape[0], need_data);
  if (st) return st;
  if (window < 0 || sinks < 0) return GS_ERR_SHAPE;
  const int64_t group = q->shape[2] / c->heads;
  if (q->shape[1] > (1 << 30) || group > (1 << 16) || q->shape[1] * group > (1 << 30)) return GS_ERR_UNSUPPORTED;
  memset(a, 0, sizeof(*a));
  a->cache = cache_shape(c);
  a->table = static_cast<const int32_t*>(table->data);
  a->q = q->data;
  a->batch = q->shape[0];
  a->width = c->n_pages > 0 ? table->shape[1] : 0;     // (without pages no sequence has a token, and nothing of the cache is read)
  a->queries = int32_t(q->shape[1]);
  a->group = int32_t(group);
  const int64_t most = a->width * c->page_size;     // a window of everything is none
  a->window = window < most ? window : 0;
  a->sinks = sinks < most ? sinks : most;
  return GS_OK;
}

int check_dot(int rank0, int access0, const int64_t* shape0, const gs_mx4* a1, const gs_ap* out, int act) {
  if (act != GS_ACT_NONE && act != GS_ACT_RELU) return GS_ERR_UNSUPPORTED;
  const int nc = rank0 - access0;
  if (nc != a1->rank - a1->n_access) return GS_ERR_SHAPE;
  for (int d = 0; d < nc; ++d)
    if (shape0[access0 + d] != a1->shape[a1->n_access + d]) return GS_ERR_SHAPE;
  if (out->rank != access0 + a1->n_access || out->n_access != out->rank) return GS_ERR_RANK;
  for (int d = 0; d < access0; ++d)
    if (out->shape[d] != shape0[d]) return GS_ERR_SHAPE;
  for (int d = 0; d < a1->n_access; ++d)
    if (out->shape[access0 + d] != a1->shape[d]) return GS_ERR_SHAPE;
  if (out->dtype != GS_F32 && out->dtype != GS_BF16) return GS_ERR_DTYPE;
  return GS_OK;
}

int run_dot(Mx4DotArgs a, const gs_mx4* a1, gs_ap* out, int act, void* workspace, size_t workspace_bytes, void* stream) {
  a.w = a1->values;
  a.ws = static_cast<const uint8_t*>(a1->scales);
  a.out = out->data;
  a.out_dtype = out->dtype;
  a.relu = act == GS_ACT_RELU;
  const Mx4DotPlan plan = plan_mx4_dot(!a.xs, a.M, a.N, a.K);
  const size_t need = plan.workspace();
  if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return GS_ERR_WORKSPACE;
  return launch_status(launch_mx4_dot(a, plan, workspace, static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

int glenside_mx4_sizes(const gs_mx4* m, size_t* values_bytes, size_t* scales_bytes) {
  int64_t rows, cols;
  const int st = check_mx4(m, false, &rows, &cols);
  if (st) return st;
  if (!values_bytes || !scales_bytes) return GS_ERR_NULL;
  *values_bytes = size_t(rows * mx4_blocks(cols) * 16);
  *scales_bytes = size_t(rows * mx4_scale_pitch(cols));
  return GS_OK;
}

int glenside_mx4_quantize(const gs_ap* in, gs_mx4* out, void* stream) {
  Mx4ConvertArgs a;
  const int st = convert_args(in, out, &a);
  return st ? st : launch_status(launch_mx4_quantize(a, static_cast<hipStream_t>(stream)));
}

int glenside_mx4_dequantize(const gs_mx4* in, gs_ap* out, void* stream) {
  Mx4ConvertArgs a;
  const int st = convert_args(out, in, &a);
  return st ? st : launch_status(launch_mx4_dequantize(a, static_cast<hipStream_t>(stream)));
}

int glenside_mx4_dot(const gs_mx4* a0, const gs_mx4* a1, gs_ap* out, int act, void* workspace, size_t workspace_bytes, void* stream) {
  Mx4DotArgs a;
  memset(&a, 0, sizeof(a));
  int st = check_mx4(a0, true, &a.M, &a.K);
  if (st) return st;
  st = check_mx4(a1, true, &a.N, &a.K);
  if (st) return st;
  st = check_ap(out, true);
  if (st) return st;
  st = check_dot(a0->rank, a0->n_access, a0->shape, a1, out, act);
  if (st) return st;
  a.x = a0->values;
  // (without numbers there may be no scales; the kernels then read none)
  a.xs = a0->scales ? static_cast<const uint8_t*>(a0->scales) : reinterpret_cast<const uint8_t*>(16);
  return run_dot(a, a1, out, act, workspace, workspace_bytes, stream);
}

size_t glenside_mx4_dot_workspace(const gs_mx4* a0, const gs_mx4* a1) {
  int64_t M, N, K, K1;
  if (check_mx4(a0, false, &M, &K) || check_mx4(a1, false, &N, &K1) || K != K1) return 0;
  return plan_mx4_dot(false, M, N, K).workspace();
}

int glenside_mx4_weight_dot(const gs_ap* a0, const gs_mx4* a1, gs_ap* out, int act, void* workspace, size_t workspace_bytes, void* stream) {
  Mx4DotArgs a;
  memset(&a, 0, sizeof(a));
  int st = check_ap(a0, true);
  if (st) return st;
  st = check_mx4(a1, true, &a.N, &a.K);
  if (st) return st;
  st = check_ap(out, true);
  if (st) return st;
  if (a0->dtype != GS_BF16) return GS_ERR_DTYPE;
  st = check_dot(a0->rank, a0->n_access, a0->shape, a1, out, act);
  if (st) return st;
  a.M = product(a0->shape, a0->n_access);
  a.x = a0->data;
  return run_dot(a, a1, out, act, workspace, workspace_bytes, stream);
}

size_t glenside_mx4_weight_dot_workspace(const gs_ap* a0, const gs_mx4* a1) {
  int64_t N, K;
  if (check_ap(a0, false) || check_mx4(a1, false, &N, &K)) return 0;
  if (product(a0->shape + a0->n_access, a0->rank - a0->n_access) != K) return 0;
  return plan_mx4_dot(true, product(a0->shape, a0->n_access), N, K).workspace();
}

size_t glenside_mx4_cache_bytes(const gs_mx4_cache* cache) {
  if (check_cache(cache, false)) return 0;
  const Mx4CacheShape s = cache_shape(cache);
  return size_t(s.n_pages * s.heads * s.block_bytes());
}

int glenside_mx4_cache_append(const gs_mx4_cache* cache, const gs_ap* table, const gs_ap* first, const gs_ap* counts, const gs_ap* k,
                              const gs_ap* v, void* stream) {
  Mx4TokenArgs a;
  const int st = token_args(cache, table, first, counts, k, v, &a);
  return st ? st : launch_status(launch_mx4_append(a, static_cast<hipStream_t>(stream)));
}

int glenside_mx4_cache_read(const gs_mx4_cache* cache, const gs_ap* table, const gs_ap* first, gs_ap* k, gs_ap* v, void* stream) {
  Mx4TokenArgs a;
  const int st = token_args(cache, table, first, nullptr, k, v, &a);
  return st ? st : launch_status(launch_mx4_read(a, static_cast<hipStream_t>(stream)));
}

int glenside_mx4_attend(const gs_ap* q, const gs_mx4_cache* cache, const gs_ap* table, const gs_ap* lengths, float scale, int64_t window,
                        int64_t sinks, gs_ap* out, void* workspace, size_t workspace_bytes, void* stream) {
  Mx4AttendArgs a;
  int st = attend_args(q, cache, table, window, sinks, true, &a);
  if (st) return st;
  st = check_per_sequence(lengths, a.batch);
  if (st) return st;
  st = check_ap(out, true);
  if (st) return st;
  if (out->rank != q->rank || out->n_access != q->n_access) return GS_ERR_RANK;
  if (!same_pattern_shape(out, q)) return GS_ERR_SHAPE;
  if (out->dtype != GS_BF16 && out->dtype != GS_F32) return GS_ERR_DTYPE;
  if (!isfinite(scale * 1.44269504088896340736f)) return GS_ERR_UNSUPPORTED;     // (the unit that scores are computed in)
  a.lengths = static_cast<const int32_t*>(lengths->data);
  a.out = out->data;
  a.out_dtype = out->dtype;
  a.scale = scale;
  const size_t need = mx4_attend_workspace(a);
  if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return GS_ERR_WORKSPACE;
  a.partial = static_cast<float*>(workspace);
  return launch_status(launch_mx4_attend(a, static_cast<hipStream_t>(stream)));
}

size_t glenside_mx4_attend_workspace(const gs_ap* q, const gs_mx4_cache* cache, const gs_ap* table) {
  Mx4AttendArgs a;
  if (attend_args(q, cache, table, 0, 0, false, &a)) return 0;
  return mx4_attend_workspace(a);
}

// For tests, not part of the interface: how a product (Mx4DotWay, workgroups that share a sum) and an attention (Mx4AttendPlan) of
// these sizes are done.  Host only.
int gs_test_mx4_dot_plan(int x_is_bf16, int64_t M, int64_t N, int64_t K, int plan[2]) {
  const Mx4DotPlan p = plan_mx4_dot(x_is_bf16 != 0, M, N, K);
  plan[0] = p.way;
  plan[1] = p.splits;
  return GS_OK;
}
int gs_test_mx4_attend_plan(const gs_ap* q, const gs_mx4_cache* cache, const gs_ap* table, int64_t window, int64_t sinks, int plan[5]) {
  Mx4AttendArgs a;
  const int st = attend_args(q, cache, table, window, sinks, false, &a);
  if (st) return st;
  const Mx4AttendPlan p = mx4_attend_plan(a);
  plan[0] = p.rows;
  plan[1] = p.waves;
  plan[2] = p.parts;
  plan[3] = p.slots;
  plan[4] = p.joined_alone;
  return GS_OK;
}

}  // extern "C"
