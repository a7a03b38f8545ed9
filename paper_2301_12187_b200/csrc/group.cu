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

size_t saved_bytes(long long rows, int rank) { return (size_t)rows * (size_t)rank_pad(rank) * 4; }

struct Need {
  size_t bytes = sizeof(DcWsHeader);
  size_t add(size_t n) {
    const size_t at = bytes;
    bytes += dc_round_up(n, 256);
    return at;
  }
};

}  // namespace

extern "C" dc_status dc_group_workspace_bytes(long long rows, int groups, int c_in, int c_out, dc_dtype dtype, size_t *bytes) {
  const dc_status s = check_sizes(rows, c_in, c_out, dtype);
  if (s != DC_OK) return s;
  if (!bytes || groups < 1) return DC_ERR_INVALID_ARG;
  if (groups > kMaxRuns) return DC_ERR_UNSUPPORTED;
  *bytes = Need().bytes;
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
  RowsJob j = {};
  j.x = x;
  j.rows = (int)rows;
  j.k = c_in;
  j.n = c_out;
  j.w = w;
  j.runs = {offsets, nullptr, groups, (int)rows, groups, 0};
  j.bias = bias;
  j.bias_each = 1;
  j.act = (int)act;
  j.y = y;
  j.dtype = dtype;
  return status(rows_any(j, (cudaStream_t)stream));
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
  cudaError_t e = cudaSuccess;
  if (dx && rows) {
    RowsJob j = {};
    j.x = dy;
    j.rows = (int)rows;
    j.k = c_out;
    j.n = c_in;
    j.w = w;
    j.w_across = 1;
    j.runs = runs;
    j.y = dx;
    j.dtype = dtype;
    e = rows_any(j, (cudaStream_t)stream);
  }
  if ((dw || db) && e == cudaSuccess) {
    GradJob j = {};
    j.p = dy;
    j.q = x;
    j.m = c_out;
    j.n = c_in;
    j.runs = runs;
    j.out = dw;
    j.sums = db;
    j.dtype = dtype;
    e = grad_any(j, (cudaStream_t)stream);
  }
  return status(e);
}

extern "C" dc_status dc_adapter_saved_bytes(long long rows, int rank, dc_dtype dtype, size_t *bytes) {
  if (rows < 0 || rank < 1 || !bytes || (dtype != DC_F32 && dtype != DC_BF16)) return DC_ERR_INVALID_ARG;
  if (rows > kMaxRows || rank > kMaxRank) return DC_ERR_UNSUPPORTED;
  *bytes = saved_bytes(rows, rank);
  return DC_OK;
}

extern "C" dc_status dc_adapter_workspace_bytes(long long rows, int c_in, int c_out, const dc_adapters *adapters, dc_dtype dtype,
                                                size_t *bytes) {
  dc_status s = check_sizes(rows, c_in, c_out, dtype);
  if (s == DC_OK) s = check_adapters(adapters);
  if (s != DC_OK) return s;
  if (!bytes) return DC_ERR_INVALID_ARG;
  Need n;
  n.add(saved_bytes(rows, adapters->rank));      // u
  *bytes = n.bytes;
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
// out = rows of x through the adapters' first matrices (a, or in the backward pass b read across), scaled
cudaError_t narrow(const void *x, int rows, int k, const dc_adapters *ad, bool backward, const Runs &runs, void *out, dc_dtype dtype,
                   cudaStream_t st) {
  if (runs.count == 0) return cudaSuccess;
  RowsJob j = {};
  j.x = x;
  j.rows = rows;
  j.k = k;
  j.n = ad->rank;
  j.w = backward ? ad->b : ad->a;
  j.w_across = backward;
  j.runs = runs;
  j.alpha = ad->scale;
  j.y = out;
  j.y_terms = 1;
  j.dtype = dtype;
  return rows_any(j, st);
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
  cudaError_t e = narrow(x, (int)rows, c_in, adapters, false, of, saved, dtype, (cudaStream_t)stream);
  if (e != cudaSuccess) return status(e);
  RowsJob j = {};
  j.x = x;
  j.rows = (int)rows;
  j.k = c_in;
  j.n = c_out;
  j.w = w;
  j.runs = all;
  j.t = runs ? saved : nullptr;
  j.e = adapters->b;
  j.rank = adapters->rank;
  j.ext = of;
  j.bias = bias;
  j.act = (int)act;
  j.residual = residual;
  j.y = y;
  j.dtype = dtype;
  return status(rows_any(j, (cudaStream_t)stream));
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
  void *u = (uint8_t *)workspace + sizeof(DcWsHeader);
  cudaError_t e = cudaSuccess;
  if ((dx || da) && rows) e = narrow(dy, (int)rows, c_out, adapters, true, of, u, dtype, st);
  if (dx && rows && e == cudaSuccess) {
    RowsJob j = {};
    j.x = dy;
    j.rows = (int)rows;
    j.k = c_out;
    j.n = c_in;
    j.w = w;
    j.w_across = 1;
    j.runs = all;
    j.t = runs ? u : nullptr;
    j.e = adapters->a;
    j.e_across = 1;
    j.rank = adapters->rank;
    j.ext = of;
    j.y = dx;
    j.dtype = dtype;
    e = rows_any(j, st);
  }
  GradJob g = {};
  g.runs = of;
  g.dtype = dtype;
  if (da && e == cudaSuccess) {
    g.p = u;
    g.p_terms = 1;
    g.m = adapters->rank;
    g.q = x;
    g.q_terms = 0;
    g.n = c_in;
    g.out = da;
    e = grad_any(g, st);
  }
  if (db && e == cudaSuccess) {
    g.p = dy;
    g.p_terms = 0;
    g.m = c_out;
    g.q = saved;
    g.q_terms = 1;
    g.n = adapters->rank;
    g.out = db;
    e = grad_any(g, st);
  }
  return status(e);
}
