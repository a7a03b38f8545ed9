// Grouped products and adapters on CUDA cores: fp32, and bf16 whose rows do not lie on 16 bytes.
//
// A CTA works out 64 x 64 results, 16 terms of their sums at a time through shared memory, 4 x 4 a thread.  Sums are fp32, those of 512 terms
// added to a second one: a sum of 16384 fp32 terms is otherwise 3 times as far from 64 bits as a library's product.
#include "group.cuh"

namespace {
using grp::GradJob;
using grp::Run;
using grp::RowsJob;
using grp::Runs;

constexpr int kTile = 64, kDepth = 16, kThreads = 256, kFlush = 32;      // kFlush: steps of kDepth terms

template <typename T>
__device__ __forceinline__ float value(const void *p, size_t i) { return (float)__ldg(reinterpret_cast<const T *>(p) + i); }
// number j of what row `row` keeps of an adapter
template <typename T>
__device__ __forceinline__ float term(const void *t, int row, int rank, int j) {
  const size_t pad = (size_t)grp::rank_pad(rank);
  const T *at = reinterpret_cast<const T *>(t) + (size_t)row * (sizeof(T) == 4 ? pad : 2 * pad) + (size_t)j;
  return sizeof(T) == 4 ? (float)at[0] : (float)at[0] + (float)at[pad];
}

struct Sums {
  float part[4][4], all[4][4];
  __device__ void zero() {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) part[i][j] = all[i][j] = 0.f;
  }
  __device__ void flush() {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) { all[i][j] += part[i][j]; part[i][j] = 0.f; }
  }
};
typedef float Stage[kDepth][kTile + 4];

__device__ __forceinline__ void multiply(Sums &s, const Stage &p, const Stage &q, int ti, int tj) {
#pragma unroll
  for (int k = 0; k < kDepth; ++k) {
    const float4 a = *reinterpret_cast<const float4 *>(&p[k][ti * 4]), b = *reinterpret_cast<const float4 *>(&q[k][tj * 4]);
    const float x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s.part[i][j] = fmaf(x[i], y[j], s.part[i][j]);
  }
}
// fills a stage; `first` runs fastest over neighbouring addresses: the terms (0) or the tile's rows (1)
template <typename F>
__device__ __forceinline__ void fill(Stage &s, int across, F at) {
#pragma unroll
  for (int u = 0; u < kTile * kDepth / kThreads; ++u) {
    const int v = (int)threadIdx.x + u * kThreads;
    const int k = across ? v / kTile : v % kDepth, i = across ? v % kTile : v / kDepth;
    s[k][i] = at(i, k);
  }
}

template <typename T>
__device__ void rows_tile(const RowsJob &j, Stage &p, Stage &q, int row0, int end, int weight, int col0) {
  const int ti = (int)threadIdx.x / 16, tj = (int)threadIdx.x % 16;
  Sums s;
  s.zero();
  int step = 0;
  if (j.w) {
    const size_t w0 = (size_t)weight * (size_t)j.n * (size_t)j.k;
    for (int k0 = 0; k0 < j.k; k0 += kDepth) {
      fill(p, 0, [&](int i, int k) { return row0 + i < end && k0 + k < j.k ? value<T>(j.x, (size_t)(row0 + i) * (size_t)j.k + (size_t)(k0 + k)) : 0.f; });
      fill(q, j.w_across, [&](int i, int k) {
        const int o = col0 + i, kk = k0 + k;
        if (o >= j.n || kk >= j.k) return 0.f;
        return value<T>(j.w, w0 + (j.w_across ? (size_t)kk * (size_t)j.n + (size_t)o : (size_t)o * (size_t)j.k + (size_t)kk));
      });
      __syncthreads();
      multiply(s, p, q, ti, tj);
      __syncthreads();
      if (++step % kFlush == 0) s.flush();
    }
    s.flush();
    if (j.alpha) {
      const float alpha = __ldg(j.alpha + weight);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) s.all[i][c] *= alpha;
    }
  }
  if (j.t)
    for (int r = grp::first_run_behind(j.ext, row0); r < j.ext.count; ++r) {
      const Run run = grp::run_at(j.ext, r);
      if (run.begin >= end) break;
      if (run.weight < 0) continue;
      const size_t e0 = (size_t)run.weight * (size_t)j.n * (size_t)j.rank;
      for (int k0 = 0; k0 < j.rank; k0 += kDepth) {
        fill(p, 0, [&](int i, int k) {
          const int row = row0 + i;
          return row < end && row >= run.begin && row < run.end && k0 + k < j.rank ? term<T>(j.t, row, j.rank, k0 + k) : 0.f;
        });
        fill(q, j.e_across, [&](int i, int k) {
          const int o = col0 + i, kk = k0 + k;
          if (o >= j.n || kk >= j.rank) return 0.f;
          return value<T>(j.e, e0 + (j.e_across ? (size_t)kk * (size_t)j.n + (size_t)o : (size_t)o * (size_t)j.rank + (size_t)kk));
        });
        __syncthreads();
        // rows of other runs: 0 times an infinity would be a NaN
        if (row0 + ti * 4 + 3 >= run.begin && row0 + ti * 4 < run.end) {
          Sums one;
          one.zero();
          multiply(one, p, q, ti, tj);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int row = row0 + ti * 4 + i;
            if (row >= run.begin && row < run.end) {
#pragma unroll
              for (int c = 0; c < 4; ++c) s.part[i][c] += one.part[i][c];
            }
          }
        }
        __syncthreads();
      }
    }
  s.flush();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = row0 + ti * 4 + i;
    if (row >= end) break;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int o = col0 + tj * 4 + c;
      float v = s.all[i][c];
      if (j.y_terms) {
        const int pad = grp::rank_pad(j.n);
        if (o >= pad) break;
        if (o >= j.n) v = 0.f;                   // what the padding holds
        T *y = reinterpret_cast<T *>(j.y) + (size_t)row * (size_t)(sizeof(T) == 4 ? pad : 2 * pad);
        const T high = (T)v;
        y[o] = high;
        if (sizeof(T) == 2) {
          const float low = v - (float)high;
          y[pad + o] = (T)(low == low ? low : 0.f);        // of an infinity: itself and 0
        }
        continue;
      }
      if (o >= j.n) break;
      const size_t at = (size_t)row * (size_t)j.n + (size_t)o;
      if (j.bias) v += __ldg(j.bias + (j.bias_each ? (size_t)weight * (size_t)j.n : 0) + (size_t)o);
      if (j.residual) v += (float)reinterpret_cast<const T *>(j.residual)[at];
      reinterpret_cast<T *>(j.y)[at] = (T)dc_act_apply(v, j.act);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_group_rows(const __grid_constant__ RowsJob j) {
  __shared__ Stage p, q;
  __shared__ int found_s[4];
  dc_pdl_enter();
  grp::Walk walk;
  walk.start();
  for (long long item = blockIdx.y;; item += gridDim.y) {
    if (threadIdx.x < 32) {
      Run run = {0, 0, -1};
      int index = 0;
      long long inside = 0;
      const bool found = walk.find(j.runs, kTile, 1, item, &run, &index, &inside);
      if (threadIdx.x == 0) {
        found_s[0] = found ? 1 : 0;
        found_s[1] = run.begin + (int)inside * kTile;
        found_s[2] = run.end;
        found_s[3] = run.weight;
      }
    }
    __syncthreads();
    if (!found_s[0]) return;
    const int row0 = found_s[1], end = min(found_s[2], row0 + kTile), weight = found_s[3];
    __syncthreads();
    rows_tile<T>(j, p, q, row0, end, weight, (int)blockIdx.x * kTile);
  }
}

template <typename T>
__device__ void grad_tile(const GradJob &j, Stage &p, Stage &q, int weight, int i0, int j0) {
  const int ti = (int)threadIdx.x / 16, tj = (int)threadIdx.x % 16;
  Sums s;
  s.zero();
  int step = 0;
  const int first = j.runs.mapped ? 0 : weight, last = j.runs.mapped ? j.runs.count : weight + 1;
  for (int r = first; r < last; ++r) {
    const Run run = grp::run_at(j.runs, r);
    if (run.weight != weight) continue;
    for (int r0 = run.begin; r0 < run.end; r0 += kDepth) {
      fill(p, 1, [&](int i, int k) {
        if (i0 + i >= j.m || r0 + k >= run.end) return 0.f;
        return j.p_terms ? term<T>(j.p, r0 + k, j.m, i0 + i) : value<T>(j.p, (size_t)(r0 + k) * (size_t)j.m + (size_t)(i0 + i));
      });
      fill(q, 1, [&](int i, int k) {
        if (j0 + i >= j.n || r0 + k >= run.end) return 0.f;
        return j.q_terms ? term<T>(j.q, r0 + k, j.n, j0 + i) : value<T>(j.q, (size_t)(r0 + k) * (size_t)j.n + (size_t)(j0 + i));
      });
      __syncthreads();
      multiply(s, p, q, ti, tj);
      __syncthreads();
      if (++step % kFlush == 0) s.flush();
    }
  }
  s.flush();
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int a = i0 + ti * 4 + i, b = j0 + tj * 4 + c;
      if (a < j.m && b < j.n) reinterpret_cast<T *>(j.out)[((size_t)weight * (size_t)j.m + (size_t)a) * (size_t)j.n + (size_t)b] = (T)s.all[i][c];
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_group_grad(const __grid_constant__ GradJob j, int tiles_m, int tiles_n) {
  __shared__ Stage p, q;
  dc_pdl_enter();
  const int per = tiles_m * tiles_n;
  for (long long item = blockIdx.x; item < (long long)per * j.runs.weights; item += gridDim.x) {
    const int weight = (int)(item / per), at = (int)(item - (long long)weight * per);
    grad_tile<T>(j, p, q, weight, at / tiles_n * kTile, at % tiles_n * kTile);
  }
}

// sums of p over each weight's rows: a CTA to 32 columns, eight rows at a time, added up in the order of the rows
template <typename T>
__global__ void __launch_bounds__(256) k_group_sums(const __grid_constant__ GradJob j) {
  __shared__ float part[8][33];
  dc_pdl_enter();
  const int lane = (int)threadIdx.x & 31, slice = (int)threadIdx.x >> 5, col = (int)blockIdx.x * 32 + lane;
  for (int weight = (int)blockIdx.y; weight < j.runs.weights; weight += (int)gridDim.y) {
    float all = 0.f;
    const int first = j.runs.mapped ? 0 : weight, last = j.runs.mapped ? j.runs.count : weight + 1;
    for (int r = first; r < last; ++r) {
      const Run run = grp::run_at(j.runs, r);
      if (run.weight != weight || col >= j.m) continue;
      for (int r0 = run.begin + slice; r0 < run.end; r0 += 8 * 64) {
        float some = 0.f;
#pragma unroll 8
        for (int k = 0; k < 64; ++k)
          if (r0 + 8 * k < run.end) some += value<T>(j.p, (size_t)(r0 + 8 * k) * (size_t)j.m + (size_t)col);
        all += some;
      }
    }
    part[slice][lane] = all;
    __syncthreads();
    if (slice == 0 && col < j.m) {
      for (int k = 1; k < 8; ++k) all += part[k][lane];
      j.sums[(size_t)weight * (size_t)j.m + (size_t)col] = all;
    }
    __syncthreads();
  }
}

}  // namespace

namespace grp {

// No more row tiles than this: every run may end inside one.
static long long row_tiles(const Runs &r, int tile) {
  const long long runs = r.offsets ? (r.count < r.rows ? r.count : r.rows) : 1;
  return r.rows / tile + runs;
}
static unsigned at_most(long long n, long long most) { return (unsigned)(n < most ? n : most); }

cudaError_t rows_any(const RowsJob &j, cudaStream_t st) {
  const dim3 grid((unsigned)dc_div_up(j.y_terms ? rank_pad(j.n) : j.n, kTile), at_most(row_tiles(j.runs, kTile), 65535));
  return j.dtype == DC_BF16 ? dc_launch_pdl(k_group_rows<__nv_bfloat16>, grid, dim3(kThreads), 0, st, j)
                            : dc_launch_pdl(k_group_rows<float>, grid, dim3(kThreads), 0, st, j);
}

cudaError_t grad_any(const GradJob &j, cudaStream_t st) {
  if (j.out) {
    const int tiles_m = dc_div_up(j.m, kTile), tiles_n = dc_div_up(j.n, kTile);
    const dim3 grid(at_most((long long)tiles_m * tiles_n * j.runs.weights, 1 << 20));
    const cudaError_t e = j.dtype == DC_BF16 ? dc_launch_pdl(k_group_grad<__nv_bfloat16>, grid, dim3(kThreads), 0, st, j, tiles_m, tiles_n)
                                             : dc_launch_pdl(k_group_grad<float>, grid, dim3(kThreads), 0, st, j, tiles_m, tiles_n);
    if (e != cudaSuccess) return e;
  }
  if (j.sums) {
    const dim3 grid((unsigned)dc_div_up(j.m, 32), at_most(j.runs.weights, 65535));
    return j.dtype == DC_BF16 ? dc_launch_pdl(k_group_sums<__nv_bfloat16>, grid, dim3(256), 0, st, j)
                              : dc_launch_pdl(k_group_sums<float>, grid, dim3(256), 0, st, j);
  }
  return cudaSuccess;
}

}  // namespace grp
