// Entry points of grouped products and adapters: arguments, and which kernels a call takes.
#include <initializer_list>

#include "group.cuh"

namespace {
using namespace grp;

constexpr long long kMaxRows = 1ll << 30;
constexpr int kMaxWidth = 1 << 20;

dc_status check_sizes(long long rows, int c_in, int c_out, dc_dtype dtype) {
  if (rows < 0 || c_in < 1 || c_out < 1 || (dtype != DC_F32 && dtype != DC_BF16)) return DC_ERR_INVALID_ARG;
  if (rows > kMaxRows || c_in > kMaxWidth || c_out > kMaxWidth) return DC_ERR_UNSUPPORTED;
  return DC_OK;
}
dc_status check_adapters(const dc_adapters *a) {
  if (!a || a->count < 1 || a->rank < 1) return DC_ERR_INVALID_ARG;
  if (a->count > kMaxRuns || a->rank > kMaxRank) return DC_ERR_UNSUPPORTED;
  return DC_OK;
}
bool aligned(std::initializer_list<const void *> all) {
  for (const void *p : all)
    if (!dc_aligned16(p)) return false;
  return true;
}
dc_status status(cudaError_t e) { return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? DC_OK : DC_ERR_CUDA; }

size_t saved_bytes(long long rows, int rank, dc_dtype dtype) { return (size_t)rows * (size_t)rank_pad(rank) * (dtype == DC_BF16 ? 4 : 6); }

// A workspace's parts, one behind the other: `base` NULL where only their bytes are wanted.  bf16 rows that do not begin on 16 bytes are copied to rows
// that do, fp32 ones are cut into terms: the tensor core's kernels read by TMA.  (A copy takes a tenth of the time that reading value by value cost.)
struct Parts {
  uint8_t *base;
  dc_dtype dtype;
  size_t bytes = sizeof(DcWsHeader);
  Copy copies[kMaxCopies];
  int count = 0;
  Parts(void *workspace, dc_dtype type) : base((uint8_t *)workspace), dtype(type) {}
  void *add(size_t n) {
    uint8_t *at = base ? base + bytes : nullptr;
    bytes += dc_round_up(n, 256);
    return at;
  }
  bool apart(int cols) const { return dtype == DC_F32 || cols % 8 != 0; }
  // whole lines of 128 bytes, which is what a load takes of a row
  int pitch(int cols) const { return apart(cols) ? (int)dc_round_up((size_t)cols, 64) : cols; }
  void *room(long long rows, int cols) { return add((size_t)rows * (size_t)pitch(cols) * (dtype == DC_BF16 ? 2 : 6)); }
  void reserve(long long rows, int cols) {
    if (apart(cols)) room(rows, cols);
  }
  const void *rows_of(const void *x, long long rows, int cols) {
    if (!x || rows == 0 || !apart(cols)) return x;
    void *to = room(rows, cols);
    copies[count++] = {x, to, rows, cols, pitch(cols)};
    return to;
  }
  cudaError_t copy(cudaStream_t st) { return copies_tc(copies, count, dtype, st); }
};
// Whether fp32 rows go by FMAs, straight from the caller's arrays: by terms x and all matrices are copied first, 10 bytes a number and a launch.
bool direct(const RowsJob &j) {
  if (j.dtype != DC_F32) return false;
  double us = 0.0;
  rows_tc(j, false, nullptr, nullptr, nullptr, &us);
  const double numbers = j.w ? (double)j.rows * j.k + (double)j.runs.weights * j.n * j.k : 0.0;
  return rows_few_us(j) < us + 3.0 + 3.0 + numbers * 10 / 4.5e6;
}
// A grouped product's sizes: forward, or of the rows' gradients.
RowsJob group_job(long long rows, int c_in, int c_out, const int *offsets, int groups, const void *w, bool backward, dc_dtype dtype) {
  RowsJob j = {};
  j.rows = (int)rows;
  j.k = backward ? c_out : c_in;
  j.n = backward ? c_in : c_out;
  j.w = j.raw_w = w;
  j.w_across = backward;
  j.runs = {offsets, nullptr, groups, (int)rows, groups, 0};
  j.dtype = dtype;
  return j;
}

}  // namespace

extern "C" dc_status dc_group_workspace_bytes(long long rows, int groups, int c_in, int c_out, dc_dtype dtype, size_t *bytes) {
  const dc_status s = check_sizes(rows, c_in, c_out, dtype);
  if (s != DC_OK) return s;
  if (!bytes || groups < 1) return DC_ERR_INVALID_ARG;
  if (groups > kMaxRuns) return DC_ERR_UNSUPPORTED;
  Parts need(nullptr, dtype);
  need.reserve(rows, c_in);
  need.reserve(rows, c_out);
  need.reserve((long long)groups * c_out, c_in);
  *bytes = need.bytes;
  return DC_OK;
}

extern "C" dc_status dc_group_forward(const void *x, long long rows, int c_in, const int *offsets, int groups, const void *w, int c_out,
                                      const float *bias, dc_act act, void *y, dc_dtype dtype, void *workspace, size_t workspace_bytes,
                                      dc_stream stream) {
  size_t need;
  const dc_status s = dc_group_workspace_bytes(rows, groups, c_in, c_out, dtype, &need);
  if (s != DC_OK) return s;
  if (act != DC_ACT_IDENTITY && act != DC_ACT_RELU6) return DC_ERR_INVALID_ARG;
  if (!offsets || !w || (rows && (!x || !y))) return DC_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < need) return DC_ERR_WORKSPACE;
  if (!aligned({x, w, bias, y, workspace}) || (reinterpret_cast<uintptr_t>(offsets) & 3u)) return DC_ERR_ALIGNMENT;
  if (rows == 0) return DC_OK;
  Parts parts(workspace, dtype);
  RowsJob j = group_job(rows, c_in, c_out, offsets, groups, w, false, dtype);
  j.x = j.raw_x = x;
  j.x_pitch = j.w_pitch = parts.pitch(c_in);
  j.bias = bias;
  j.bias_each = 1;
  j.act = (int)act;
  j.y = y;
  if (direct(j)) return status(rows_few(j, (cudaStream_t)stream));
  j.x = parts.rows_of(x, rows, c_in);
  j.w = parts.rows_of(w, (long long)groups * c_out, c_in);
  cudaError_t e = parts.copy((cudaStream_t)stream);
  if (e == cudaSuccess) e = rows_tc(j, false, (DcWsHeader *)workspace, (cudaStream_t)stream);
  return status(e);
}

extern "C" dc_status dc_group_backward(const void *dy, const void *x, long long rows, int c_in, const int *offsets, int groups,
                                       const void *w, int c_out, void *dx, void *dw, float *db, dc_dtype dtype, void *workspace,
                                       size_t workspace_bytes, dc_stream stream) {
  size_t need;
  const dc_status s = dc_group_workspace_bytes(rows, groups, c_in, c_out, dtype, &need);
  if (s != DC_OK) return s;
  if (!offsets || (rows && !dy) || (!dx && !dw && !db && rows) || (rows && dx && !w) || (rows && dw && !x)) return DC_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < need) return DC_ERR_WORKSPACE;
  if (!aligned({dy, x, w, dx, dw, db, workspace}) || (reinterpret_cast<uintptr_t>(offsets) & 3u)) return DC_ERR_ALIGNMENT;
  if (rows == 0 && !dw && !db) return DC_OK;
  const Runs runs = {offsets, nullptr, groups, (int)rows, groups, 0};
  Parts parts(workspace, dtype);
  RowsJob j = group_job(rows, c_in, c_out, offsets, groups, w, true, dtype);
  j.x = j.raw_x = dy;
  j.x_pitch = parts.pitch(c_out);
  j.w_pitch = parts.pitch(c_in);
  j.y = dx;
  const bool with_dx = dx && rows, fmas = with_dx && direct(j);
  const void *dy_at = dw || db || !fmas ? parts.rows_of(dy, rows, c_out) : nullptr, *x_at = dw ? parts.rows_of(x, rows, c_in) : nullptr;
  j.x = dy_at;
  if (with_dx && !fmas) j.w = parts.rows_of(w, (long long)groups * c_out, c_in);
  cudaError_t e = parts.copy((cudaStream_t)stream);
  if (with_dx && e == cudaSuccess) e = fmas ? rows_few(j, (cudaStream_t)stream) : rows_tc(j, false, (DcWsHeader *)workspace, (cudaStream_t)stream);
  if ((dw || db) && e == cudaSuccess) {
    GradJob j = {};
    j.p = dy_at;
    j.q = x_at;
    j.p_pitch = parts.pitch(c_out);
    j.q_pitch = parts.pitch(c_in);
    j.m = c_out;
    j.n = c_in;
    j.runs = runs;
    j.out = dw;
    j.sums = db;
    j.dtype = dtype;
    j.raw_p = dy;
    j.raw_q = x;
    e = grad_tc(j, with_dx, (DcWsHeader *)workspace, (cudaStream_t)stream);
  }
  return status(e);
}

extern "C" dc_status dc_adapter_saved_bytes(long long rows, int rank, dc_dtype dtype, size_t *bytes) {
  if (rows < 0 || rank < 1 || !bytes || (dtype != DC_F32 && dtype != DC_BF16)) return DC_ERR_INVALID_ARG;
  if (rows > kMaxRows || rank > kMaxRank) return DC_ERR_UNSUPPORTED;
  *bytes = saved_bytes(rows, rank, dtype);
  return DC_OK;
}

extern "C" dc_status dc_adapter_workspace_bytes(long long rows, int c_in, int c_out, const dc_adapters *adapters, dc_dtype dtype,
                                                size_t *bytes) {
  dc_status s = check_sizes(rows, c_in, c_out, dtype);
  if (s == DC_OK) s = check_adapters(adapters);
  if (s != DC_OK) return s;
  if (!bytes) return DC_ERR_INVALID_ARG;
  Parts need(nullptr, dtype);
  need.add(saved_bytes(rows, adapters->rank, dtype));   // u
  need.reserve(rows, c_in);
  need.reserve(rows, c_out);
  need.reserve(c_out, c_in);
  need.reserve((long long)adapters->count * adapters->rank, c_in);
  need.reserve((long long)adapters->count * c_out, adapters->rank);
  *bytes = need.bytes;
  return DC_OK;
}

namespace {
// what the two adapter calls check alike
dc_status check_adapter_call(long long rows, int c_in, int c_out, const void *w, const dc_adapters *ad, const int *offsets, const int *which,
                             int runs, dc_dtype dtype, void *workspace, size_t workspace_bytes) {
  size_t need;
  const dc_status s = dc_adapter_workspace_bytes(rows, c_in, c_out, ad, dtype, &need);
  if (s != DC_OK) return s;
  if (!ad->a || !ad->b || runs < 0 || !offsets || (runs && !which)) return DC_ERR_INVALID_ARG;
  if (runs > kMaxRuns) return DC_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < need) return DC_ERR_WORKSPACE;
  if (!aligned({w, ad->a, ad->b, workspace}) || (reinterpret_cast<uintptr_t>(offsets) & 3u) || (reinterpret_cast<uintptr_t>(which) & 3u) ||
      (reinterpret_cast<uintptr_t>(ad->scale) & 3u))
    return DC_ERR_ALIGNMENT;
  return DC_OK;
}
// Rows through the adapters' first matrices -- a, or in the backward pass b read across -- scaled, to `out`.
RowsJob narrow_job(const void *x, int x_pitch, int rows, int k, int m_pitch, bool backward, const dc_adapters *ad, const Runs &runs, void *out, dc_dtype dtype) {
  RowsJob j = {};
  j.x = j.raw_x = x;
  j.rows = rows;
  j.k = k;
  j.n = ad->rank;
  j.w = j.raw_w = backward ? ad->b : ad->a;
  j.w_across = backward;
  j.x_pitch = x_pitch;
  j.w_pitch = m_pitch;
  j.runs = runs;
  j.alpha = ad->scale;
  j.y = out;
  j.y_terms = 1;
  j.dtype = dtype;
  return j;
}
cudaError_t narrow(const RowsJob &j, void *workspace, cudaStream_t st) {
  if (j.runs.count == 0) return cudaSuccess;
  return narrow_apart(j) ? narrow_tc(j, st) : rows_tc(j, false, (DcWsHeader *)workspace, st);
}
}  // namespace

extern "C" dc_status dc_adapter_forward(const void *x, long long rows, int c_in, const void *w, int c_out, const dc_adapters *adapters,
                                        const int *offsets, const int *which, int runs, const float *bias, dc_act act,
                                        const void *residual, void *saved, void *y, dc_dtype dtype, void *workspace,
                                        size_t workspace_bytes, dc_stream stream) {
  const dc_status s = check_adapter_call(rows, c_in, c_out, w, adapters, offsets, which, runs, dtype, workspace, workspace_bytes);
  if (s != DC_OK) return s;
  if (act != DC_ACT_IDENTITY && act != DC_ACT_RELU6) return DC_ERR_INVALID_ARG;
  if (rows && (!x || !y || !saved)) return DC_ERR_INVALID_ARG;
  if (!aligned({x, bias, residual, saved, y})) return DC_ERR_ALIGNMENT;
  if (rows == 0) return DC_OK;
  const Runs of = {offsets, which, runs, (int)rows, adapters->count, 1}, all = {nullptr, nullptr, 1, (int)rows, 1, 0};
  const cudaStream_t st = (cudaStream_t)stream;
  Parts parts(workspace, dtype);
  const int in = parts.pitch(c_in), of_rank = parts.pitch(adapters->rank);
  RowsJob t = narrow_job(x, in, (int)rows, c_in, in, false, adapters, of, saved, dtype), j = {};
  j.x = j.raw_x = x;
  j.rows = (int)rows;
  j.k = c_in;
  j.n = c_out;
  j.w = j.raw_w = w;
  j.x_pitch = j.w_pitch = in;
  j.runs = all;
  j.t = runs ? saved : nullptr;
  j.e = j.raw_e = adapters->b;
  j.e_pitch = of_rank;
  j.rank = adapters->rank;
  j.ext = of;
  j.dtype = dtype;
  // what the kernels read is copied first, unless they read fp32 as it lies
  const bool fmas = direct(j), raw = dtype == DC_F32 && (!runs || narrow_apart(t));
  if (!fmas || !raw) j.x = t.x = parts.rows_of(x, rows, c_in);
  if (!raw) t.w = parts.rows_of(adapters->a, (long long)adapters->count * adapters->rank, c_in);
  if (!fmas) {
    j.w = parts.rows_of(w, c_out, c_in);
    j.e = parts.rows_of(adapters->b, (long long)adapters->count * c_out, adapters->rank);
  }
  cudaError_t e = parts.copy(st);
  if (e == cudaSuccess) e = narrow(t, workspace, st);
  if (e != cudaSuccess) return status(e);
  j.bias = bias;
  j.act = (int)act;
  j.residual = residual;
  j.y = y;
  return status(fmas ? rows_few(j, st) : rows_tc(j, runs > 0, (DcWsHeader *)workspace, st));
}

extern "C" dc_status dc_adapter_backward(const void *dy, const void *x, long long rows, int c_in, const void *w, int c_out,
                                         const dc_adapters *adapters, const int *offsets, const int *which, int runs, const void *saved,
                                         void *dx, void *da, void *db, dc_dtype dtype, void *workspace, size_t workspace_bytes,
                                         dc_stream stream) {
  const dc_status s = check_adapter_call(rows, c_in, c_out, w, adapters, offsets, which, runs, dtype, workspace, workspace_bytes);
  if (s != DC_OK) return s;
  if (rows && (!dy || (!dx && !da && !db) || (da && !x) || (db && !saved))) return DC_ERR_INVALID_ARG;
  if (!aligned({dy, x, saved, dx, da, db})) return DC_ERR_ALIGNMENT;
  if (rows == 0 && !da && !db) return DC_OK;
  const Runs of = {offsets, which, runs, (int)rows, adapters->count, 1}, all = {nullptr, nullptr, 1, (int)rows, 1, 0};
  const cudaStream_t st = (cudaStream_t)stream;
  Parts parts(workspace, dtype);
  void *u = parts.add(saved_bytes(rows, adapters->rank, dtype));
  const bool with_u = (dx || da) && rows;
  const int in = parts.pitch(c_in), out = parts.pitch(c_out), of_rank = parts.pitch(adapters->rank);
  RowsJob t = narrow_job(dy, out, (int)rows, c_out, of_rank, true, adapters, of, u, dtype), j = {};
  j.x = j.raw_x = dy;
  j.rows = (int)rows;
  j.k = c_out;
  j.n = c_in;
  j.w = j.raw_w = w;
  j.w_across = 1;
  j.x_pitch = out;
  j.w_pitch = in;
  j.runs = all;
  j.t = runs ? u : nullptr;
  j.e = j.raw_e = adapters->a;
  j.e_across = 1;
  j.e_pitch = in;
  j.rank = adapters->rank;
  j.ext = of;
  j.y = dx;
  j.dtype = dtype;
  const bool with_dx = dx && rows, fmas = with_dx && direct(j), raw = dtype == DC_F32 && (!with_u || !runs || narrow_apart(t));
  const void *dy_at = (with_dx && !fmas) || (with_u && !raw) || db ? parts.rows_of(dy, rows, c_out) : nullptr, *x_at = da ? parts.rows_of(x, rows, c_in) : nullptr;
  j.x = t.x = dy_at;
  if (with_u && !raw) t.w = parts.rows_of(adapters->b, (long long)adapters->count * c_out, adapters->rank);
  if (with_dx && !fmas) {
    j.w = parts.rows_of(w, c_out, c_in);
    j.e = parts.rows_of(adapters->a, (long long)adapters->count * adapters->rank, c_in);
  }
  // One behind the other: u, with db beside it; dx, with da beside it (which reads u from its start: not beside a dx that has not waited for u).
  const bool dx_early = !db && with_u && runs && !fmas;
  cudaError_t e = parts.copy(st);
  if (with_u && e == cudaSuccess) e = narrow(t, workspace, st);
  GradJob g = {};
  g.runs = of;
  g.dtype = dtype;
  g.q_terms = 1;
  g.n = adapters->rank;
  if (db && e == cudaSuccess) {
    g.p = dy_at;
    g.raw_p = dy;
    g.m = c_out;
    g.p_pitch = out;
    g.q = saved;
    g.out = db;
    e = grad_tc(g, with_u && runs, (DcWsHeader *)workspace, st);
  }
  if (with_dx && e == cudaSuccess) e = fmas ? rows_few(j, st) : rows_tc(j, dx_early, (DcWsHeader *)workspace, st);
  if (da && e == cudaSuccess) {                  // as x^T u, so that the long side is the instructions' 128 rows
    g.p = x_at;
    g.raw_p = x;
    g.m = c_in;
    g.p_pitch = in;
    g.q = u;
    g.out = da;
    g.out_across = 1;
    e = grad_tc(g, with_dx && !dx_early, (DcWsHeader *)workspace, st);
  }
  return status(e);
}

extern "C" dc_status dc_group_plan_query(long long rows, int runs, int c_in, int c_out, int rank, dc_dtype dtype, dc_group_part part,
                                         dc_group_plan *plan) {
  const dc_status s = check_sizes(rows, c_in, c_out, dtype);
  if (s != DC_OK) return s;
  if (rows < 1 || runs < 1 || rank < 0 || !plan || part < DC_GROUP_FORWARD || part > DC_GROUP_DW) return DC_ERR_INVALID_ARG;
  if (runs > kMaxRuns || rank > kMaxRank) return DC_ERR_UNSUPPORTED;
  // addresses that say what there is, and are not looked at
  int offsets = 0;
  const void *there = &offsets;
  const Runs of = {&offsets, rank ? &offsets : nullptr, runs, (int)rows, runs, rank > 0}, all = {nullptr, nullptr, 1, (int)rows, 1, 0};
  if (part == DC_GROUP_DW) {
    GradJob j = {};
    j.m = rank ? c_in : c_out;
    j.n = rank ? rank : c_in;
    j.q_terms = rank > 0;
    j.runs = of;
    j.out = &offsets;
    j.dtype = dtype;
    return grad_tc(j, false, nullptr, nullptr, plan) == cudaSuccess ? DC_OK : DC_ERR_CUDA;
  }
  RowsJob j = {};
  j.rows = (int)rows;
  j.k = part == DC_GROUP_DX ? c_out : c_in;
  j.n = part == DC_GROUP_DX ? c_in : c_out;
  j.w = there;
  j.w_across = j.e_across = part == DC_GROUP_DX;
  j.runs = rank ? all : of;
  j.t = rank ? there : nullptr;
  j.rank = rank;
  j.e_pitch = dtype == DC_BF16 && rank % 8 == 0 ? (part == DC_GROUP_DX ? c_in : rank) : 64;
  j.ext = of;
  j.dtype = dtype;
  j.raw_w = there;
  if (direct(j)) {
    *plan = {DC_GROUP_FMAS, rows_few_tile(j), rows_few_sets(j), 3};
    return DC_OK;
  }
  return rows_tc(j, false, nullptr, nullptr, plan) == cudaSuccess ? DC_OK : DC_ERR_CUDA;
}
