// Products of rows that belong to runs, each run with a weight matrix of its own, and low-rank adapters beside a shared matrix: what the
// kernels of both families share.  The operators are described in include/dc.h.
#pragma once

#include "common.cuh"

namespace grp {

constexpr int kMaxRank = 128;
constexpr int kMaxRuns = 1 << 20;

// Runs of rows: run s is rows [offsets[s], offsets[s + 1]), cut to [0, rows), and belongs to weight which[s] where runs are mapped, else to
// weight s.  Without offsets there is one run of all rows, of weight 0.
struct Runs {
  const int *offsets, *which;
  int count;
  int rows;
  int weights;               // a run whose weight is not one of them has none
  int mapped;
};
struct Run {
  int begin, end, weight;    // weight < 0: none
};
__device__ __forceinline__ Run run_at(const Runs &r, int s) {
  Run o;
  if (!r.offsets) {
    o.begin = 0;
    o.end = s == 0 ? r.rows : 0;
    o.weight = 0;
    return o;
  }
  o.begin = min(max(__ldg(r.offsets + s), 0), r.rows);
  o.end = min(max(__ldg(r.offsets + s + 1), o.begin), r.rows);
  o.weight = r.mapped ? __ldg(r.which + s) : s;
  if ((unsigned)o.weight >= (unsigned)r.weights) o.weight = -1;
  return o;
}

// Finds a row tile among the runs' tiles of `tile` rows each, for callers that ask in increasing order.  All lanes of a warp call it and get
// the same answer; 32 runs are looked at at a time.
struct Walk {
  int base;                  // runs before it are behind us
  long long before;          // items of theirs
  Run last;                  // the run of the last answer, and its items
  long long first, after;
  __device__ void start() { base = 0; before = first = after = 0; }
  // items of a run: row tiles x per_tile.  false: there is no such item
  __device__ bool find(const Runs &r, int tile, int per_tile, long long item, Run *run, long long *inside) {
    if (item < first || item >= after) {
      const int lane = (int)(threadIdx.x & 31u);
      for (;; base += 32) {
        if (base >= r.count) return false;
        Run o = {0, 0, -1};
        if (base + lane < r.count) o = run_at(r, base + lane);
        const int tiles = o.weight < 0 ? 0 : (int)(((unsigned)(o.end - o.begin) + (unsigned)tile - 1u) / (unsigned)tile);
        const long long mine = (long long)tiles * per_tile;
        long long upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const long long v = __shfl_up_sync(0xffffffffu, upto, d);
          if (lane >= d) upto += v;
        }
        const unsigned past = __ballot_sync(0xffffffffu, before + upto > item);
        if (past) {
          const int at = __ffs(past) - 1;
          last.begin = __shfl_sync(0xffffffffu, o.begin, at);
          last.end = __shfl_sync(0xffffffffu, o.end, at);
          last.weight = __shfl_sync(0xffffffffu, o.weight, at);
          after = before + __shfl_sync(0xffffffffu, upto, at);
          first = after - __shfl_sync(0xffffffffu, mine, at);
          break;
        }
        before += __shfl_sync(0xffffffffu, upto, 31);
      }
    }
    *run = last;
    *inside = item - first;
    return true;
  }
};

// The first run, of those between offsets, that ends behind `row` (runs in order: the one that holds it, or the next); runs.count: none.  One thread.
__device__ __forceinline__ int first_run_behind(const Runs &r, int row) {
  int lo = 0, hi = r.count;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(r.offsets + mid + 1) > row) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// For the runs with an adapter that have rows in [row0, end), all lanes together: each lane looks at its own run, `mine(run)`, then f(lane) for each of
// those that count.
template <typename G, typename F>
__device__ __forceinline__ void each_run(const Runs &r, int row0, int end, G mine, F f) {
  const int lane = (int)(threadIdx.x & 31u);
  // the first run that ends behind row0: 32 probes at a time
  int lo = 0, n = r.count;
  while (n > 32) {
    const int step = (n + 31) >> 5, probe = min((lane + 1) * step, n);
    const unsigned past = __ballot_sync(0xffffffffu, __ldg(r.offsets + lo + probe) > row0);
    if (!past) return;
    const int at = __ffs(past) - 1;
    lo += at * step;
    n = min(step, n - at * step);
  }
  for (int base = lo; base < r.count; base += 32) {
    Run o = {0, 0, -1};
    bool stop = base + lane >= r.count;
    if (!stop) {
      o = run_at(r, base + lane);
      stop = o.begin >= end;
    }
    const bool counts = !stop && o.weight >= 0 && o.end > row0 && o.end > o.begin;
    if (counts) mine(o);
    unsigned here = __ballot_sync(0xffffffffu, counts);
    while (here) {
      const int at = __ffs(here) - 1;
      here &= here - 1;
      f(at);
    }
    if (__any_sync(0xffffffffu, stop)) return;
  }
}
// What a row keeps of an adapter: `rank` numbers, padded with zeros to a multiple of 16, as terms of bf16 that add up to them: all high ones, then all
// low ones.  bf16 rows: two, 16 bits together (with one bf16 the adapter's part of a result would be as far off as the result's own rounding, 2^-9,
// and so would its gradients); fp32 rows: three.
__host__ __device__ static inline int rank_pad(int rank) { return (rank + 15) / 16 * 16; }

// y[r][o] = act(alpha_w * sum_k x[r][k] W_w(o, k) + sum_j t[r][j] E_e(o, j) + bias_w[o] + residual[r][o]) for the rows r of runs with a
// weight w; e is the weight of the run of `ext` that r is in.
struct RowsJob {
  const void *x;             // x, w and e as the kernels read them (Copy), their pitches below
  int rows, k, n;
  const void *w;             // [weights][n][k], or with w_across [weights][k][n]; NULL: no such sum
  int w_across;
  Runs runs;
  const float *alpha;        // one for each weight, or NULL
  const void *t;             // what rows keep, or NULL
  const void *e;             // [weights][n][rank], or with e_across [weights][rank][n]
  int rank, e_across;
  Runs ext;
  const float *bias;         // [n], or with bias_each [weights][n]
  int bias_each, act;
  const void *residual;
  void *y;                   // [rows][n], or with y_terms what rows keep of an adapter, n its rank
  int y_terms;
  dc_dtype dtype;
  int x_pitch, w_pitch, e_pitch;
  const void *raw_x, *raw_w, *raw_e;             // as the caller has them
};

// out_w(i, j) = sum over the rows r of the runs of weight w of p[r][i] q[r][j]; 0 without rows
struct GradJob {
  const void *p, *q;         // [rows][m], [rows][n], as the kernels read them; with q_terms q is what rows keep of an adapter, n its rank
  int m, n, q_terms;
  Runs runs;
  void *out;                 // [weights][m][n], or with out_across [weights][n][m]; NULL: sums alone
  float *sums;               // [weights][m]: sums of p over the rows, or NULL
  dc_dtype dtype;
  int out_across;
  int p_pitch, q_pitch;
  const void *raw_p, *raw_q;
};

// An array's rows for the tensor core's loads: bf16 ones beginning on 16 bytes (pitch: a multiple of 8 elements), fp32 ones as three rows of bf16 terms.
struct Copy {
  const void *from;
  void *to;
  long long rows;
  int cols, pitch;
};
constexpr int kMaxCopies = 5;

cudaError_t copies_tc(const Copy *c, int count, dc_dtype dtype, cudaStream_t st);
// early: the launch in front of this one, by narrow_tc, rows_tc or grad_tc, writes nothing of what this one reads but `t`, and nothing that it
// writes; nothing else of the caller's is between them.  Both then run side by side as far as there is room, and this one ends behind that one.
bool narrow_apart(const RowsJob &j);             // y_terms: by a kernel for short runs
cudaError_t narrow_tc(const RowsJob &j, cudaStream_t st);
// with `plan`: says how, and launches nothing; with `us`: how long tiles of 128 rows would take
cudaError_t rows_tc(const RowsJob &j, bool early, DcWsHeader *ws, cudaStream_t st, dc_group_plan *plan = nullptr, double *us = nullptr);
cudaError_t grad_tc(const GradJob &j, bool early, DcWsHeader *ws, cudaStream_t st, dc_group_plan *plan = nullptr);

// fp32 rows of short runs by FMAs, from the caller's arrays (group_few.cu); like those above it lets the next launch begin behind its own wait
double rows_few_us(const RowsJob &j);            // estimated
int rows_few_tile(const RowsJob &j);             // rows of its tiles
int rows_few_sets(const RowsJob &j);             // of four warps to a tile
cudaError_t rows_few(const RowsJob &j, cudaStream_t st);

}  // namespace grp
