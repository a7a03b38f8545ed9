// Grouped products and adapters of short runs in fp32: FMAs, each weight read once from memory as it lies.
//
// The tensor core's kernels want fp32 as three terms of bf16, which makes 16 bytes of traffic out of a weight's four.  Of a few rows to a weight FMAs keep
// up with memory; of 16 they, and what comes with them, take twice as long as the bytes (below), and still less than terms.  A CTA of four warps, or of H x four where there are
// fewer than two to an SM, works out R rows of a run x 32 columns, H x 128 numbers of the sum a step.
//   along   the sum runs along the matrix's rows: a warp to eight columns and 128 numbers of a step, its lanes share the sum.
//   across  it runs across them: eight lanes to the 32 columns, H x 16 such sets share the sum.
// The next step's weights are on their way into registers and two steps' rows into shared memory.  Partial sums meet by shuffles that halve what a
// lane holds, and in shared memory.  Two CTAs to an SM, as what they wait for is longer than what they add: 64 groups of 16 rows, 2048 -> 1408,
// take 241 us (one of eight warps: 348; rows read through L1: 332; by terms 554; 114 for the weights' bytes).  Weights that few rows share come
// at the rate of memory: 64 groups of 2 rows in 134 us (by terms 525).
#include <math.h>

#include "group.cuh"

namespace {
using grp::Run;
using grp::RowsJob;

constexpr int kCols = 32, kStages = 3;

// eight neighbours of what a row keeps
__device__ __forceinline__ void kept8(const __nv_bfloat16 *t, int row, int pad, int j, float *to) {
  const __nv_bfloat16 *at = t + (size_t)row * (size_t)(3 * pad) + (size_t)j;
  uint4 w[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) w[k] = *reinterpret_cast<const uint4 *>(at + k * pad);
  const uint32_t u[3][4] = {{w[0].x, w[0].y, w[0].z, w[0].w}, {w[1].x, w[1].y, w[1].z, w[1].w}, {w[2].x, w[2].y, w[2].z, w[2].w}};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    to[2 * i] = __uint_as_float(u[0][i] << 16) + (__uint_as_float(u[1][i] << 16) + __uint_as_float(u[2][i] << 16));
    to[2 * i + 1] = __uint_as_float(u[0][i] & 0xffff0000u) + (__uint_as_float(u[1][i] & 0xffff0000u) + __uint_as_float(u[2][i] & 0xffff0000u));
  }
}
// four values: neighbours from 4 * i on (VEC), or every STRIDE-th from i on; zeros from `end` on
template <bool VEC, int STRIDE>
__device__ __forceinline__ void load4(const float *__restrict__ at, int i, int end, float (&v)[4]) {
  if (VEC) {
    const float4 f = 4 * i < end ? __ldg(reinterpret_cast<const float4 *>(at) + i) : make_float4(0.f, 0.f, 0.f, 0.f);
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
  } else {
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = i + STRIDE * u < end ? __ldg(at + i + STRIDE * u) : 0.f;
  }
}
// What a lane holds in N registers is summed over the lanes that differ in the bits FROM, FROM / 2, ... TO: in each step half of it goes to the
// other lane, while there is more than one number.  `first`: which of the N the lane is left with.
template <int N, int FROM, int TO>
__device__ __forceinline__ void halve(float *v, int lane, int &first) {
  if constexpr (FROM >= TO) {
    if constexpr (N > 1) {
      const bool upper = lane & FROM;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const float give = upper ? v[i] : v[i + N / 2], keep = upper ? v[i + N / 2] : v[i];
        v[i] = keep + __shfl_xor_sync(0xffffffffu, give, FROM);
      }
      if (upper) first += N / 2;
      halve<N / 2, FROM / 2, TO>(v, lane, first);
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], FROM);
      halve<1, FROM / 2, TO>(v, lane, first);
    }
  }
}

// An adapter's part of a row's 32 columns, along the adapter's rows: a lane to a number of the rank, so that loads are neighbours, and the 32 columns' sums over
// the lanes by halving.  Each lane is left with column `first`.  (A column to a lane: 111 rows of rank 64, 224 -> 3279, 48 us for 39.)
__device__ __forceinline__ float of_adapter(const RowsJob &j, int a, const float *t, int o0, int cols, int lane, int &first) {
  const float *e = reinterpret_cast<const float *>(j.raw_e) + ((size_t)a * (size_t)j.n + (size_t)o0) * (size_t)j.rank;
  float v[kCols];
#pragma unroll
  for (int c = 0; c < kCols; ++c) v[c] = 0.f;
#pragma unroll 1
  for (int q = lane; q - lane < j.rank; q += 32) {
    const bool is = q < j.rank;
    const float f = is ? t[q] : 0.f;
    const float *at = e + min(q, j.rank - 1);
    float w[kCols];
#pragma unroll
    for (int c = 0; c < kCols; ++c) w[c] = __ldg(at + min(c, cols - 1) * j.rank);
#pragma unroll
    for (int c = 0; c < kCols; ++c) v[c] = fmaf(f, is ? w[c] : 0.f, v[c]);
  }
  first = 0;
  halve<kCols, 16, 1>(v, lane, first);
  return v[0];
}

__device__ __forceinline__ void deliver(const RowsJob &j, int row, int weight, int o, float v) {
  const size_t at = (size_t)row * (size_t)j.n + (size_t)o;
  if (j.bias) v += __ldg(j.bias + (j.bias_each ? (size_t)weight * (size_t)j.n : 0) + (size_t)o);
  if (j.residual) v += reinterpret_cast<const float *>(j.residual)[at];
  reinterpret_cast<float *>(j.y)[at] = dc_act_apply(v, j.act);
}

// Step `k0` of the rows to shared memory, [R][kStep], zeros behind the end; the last row again where there are no more.
template <int R, int H, bool VEC>
__device__ __forceinline__ void stage(const RowsJob &j, const float *x, int rows, int k0, float *to) {
  constexpr int kEach = VEC ? 4 : 1, kThreads = 128 * H, kStep = 128 * H;
  const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
#pragma unroll
  for (int i = (int)threadIdx.x * kEach; i < R * kStep; i += kThreads * kEach) {
    const int r = i / kStep, k = k0 + i % kStep;
    const float *from = x + (size_t)min(r, rows - 1) * (size_t)j.k + (size_t)min(k, j.k - kEach);
    const int bytes = k < j.k ? 4 * kEach : 0;
    if (VEC) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at + 4u * (uint32_t)i), "l"(from), "r"(bytes) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(at + 4u * (uint32_t)i), "l"(from), "r"(bytes) : "memory");
  }
}

template <int R, int H, bool ACROSS, bool VEC>
__device__ __forceinline__ void tile(const RowsJob &j, float *xs, float *parts, const float *ts, const int *adapter, int row0, int rows, int weight, int o0) {
  constexpr int kWarps = 4 * H, kThreads = 128 * H, kStep = 128 * H, kOwn = ACROSS ? 4 : 8;          // kOwn: a lane's columns
  const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int oct = lane & 7, set = warp * 4 + (lane >> 3);                // across: which columns, which numbers of the sum
  const int own = (warp & 3) * 8, half = (warp >> 2) * 128;              // along
  const float *x = reinterpret_cast<const float *>(j.raw_x) + (size_t)row0 * (size_t)j.k;
  const float *w = reinterpret_cast<const float *>(j.raw_w) + (size_t)weight * (size_t)j.n * (size_t)j.k;
  const int cols = min(kCols, j.n - o0);
  float acc[R][kOwn];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int c = 0; c < kOwn; ++c) acc[r][c] = 0.f;
  // eight times four numbers of the matrix: a column's four of the sum; across, a number's four columns
  auto load = [&](float (&m)[8][4], int k0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (ACROSS) {
        const int k = k0 + i / 4 * (64 * H) + 4 * set + i % 4;
        load4<VEC, 8>(w + (size_t)k * (size_t)j.n + (size_t)o0, oct, k < j.k ? cols : 0, m[i]);
      } else {
        load4<VEC, 32>(w + (size_t)(o0 + min(own + i, cols - 1)) * (size_t)j.k + (size_t)(k0 + half), lane, j.k - k0 - half, m[i]);
      }
    }
  };
  auto add = [&](const float (&m)[8][4], const float *at) {
#pragma unroll
    for (int p = 0; p < (ACROSS ? 2 : 1); ++p)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float f[4];
        if (ACROSS || VEC) {
          const float4 v = *reinterpret_cast<const float4 *>(at + r * kStep + (ACROSS ? 64 * H * p + 4 * set : half + 4 * lane));
          f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u) f[u] = at[r * kStep + half + lane + 32 * u];
        }
#pragma unroll
        for (int c = 0; c < kOwn; ++c)
#pragma unroll
          for (int u = 0; u < 4; ++u) acc[r][c] = fmaf(f[u], ACROSS ? m[4 * p + u][c] : m[c][u], acc[r][c]);
      }
  };
  if (j.w) {
    float m[2][8][4];
    const int steps = dc_div_up(j.k, kStep);
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) {
      if (s < steps) stage<R, H, VEC>(j, x, rows, s * kStep, xs + s * R * kStep);
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    load(m[0], 0);
    int at = 0, to = kStages - 1;
#pragma unroll 1
    for (int s = 0; s < steps; s += 2) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (s + h >= steps) break;
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncthreads();
        if (s + h + kStages - 1 < steps) stage<R, H, VEC>(j, x, rows, (s + h + kStages - 1) * kStep, xs + to * R * kStep);
        asm volatile("cp.async.commit_group;" ::: "memory");
        load(m[h ^ 1], (s + h + 1) * kStep);
        add(m[h], xs + at * R * kStep);
        at = at + 1 == kStages ? 0 : at + 1;
        to = to + 1 == kStages ? 0 : to + 1;
      }
    }
  }
  if (ACROSS && j.t) {                           // the adapters' rows are further numbers of the sum
    const float *e = reinterpret_cast<const float *>(j.raw_e);
#pragma unroll 1
    for (int q = set; q < j.rank; q += 16 * H) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const bool is = adapter[r] >= 0;         // t may be no number where there is no adapter
        float v[4];
        load4<VEC, 8>(e + ((size_t)max(adapter[r], 0) * (size_t)j.rank + (size_t)q) * (size_t)j.n + (size_t)o0, oct, is ? cols : 0, v);
        const float t = is ? ts[r * grp::rank_pad(j.rank) + q] : 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[r][c] = fmaf(t, v[c], acc[r][c]);
      }
    }
  }
  int first = 0;
  float *sums = &acc[0][0];
  if (ACROSS) {
    halve<4 * R, 16, 8>(sums, lane, first);
#pragma unroll
    for (int i = 0; i < R; ++i) parts[(warp * R + (first + i) / 4) * kCols + (VEC ? 4 * oct + (first + i) % 4 : oct + 8 * ((first + i) % 4))] = sums[i];
  } else {
    halve<8 * R, 16, 1>(sums, lane, first);
#pragma unroll
    for (int i = 0; i < R / 4; ++i) parts[((warp >> 2) * R + (first + i) / 8) * kCols + own + (first + i) % 8] = sums[i];
  }
  __syncthreads();
  if (!ACROSS && j.t) {
#pragma unroll 1
    for (int r = warp; r < rows; r += kWarps) {
      if (adapter[r] < 0) continue;              // t may be no number there
      const float sum = of_adapter(j, adapter[r], ts + r * grp::rank_pad(j.rank), o0, cols, lane, first);
      parts[r * kCols + first] += sum;
    }
    __syncthreads();
  }
#pragma unroll 1
  for (int i = tid; i < rows * kCols; i += kThreads) {
    const int r = i / kCols, o = i - r * kCols;
    float v = parts[i];
    if (ACROSS) {
#pragma unroll
      for (int p = 1; p < kWarps; ++p) v += parts[p * R * kCols + i];
    } else if (H == 2) {
      v += parts[R * kCols + i];
    }
    if (o >= cols) continue;
    deliver(j, row0 + r, weight, o0 + o, v);
  }
}

template <int R, int H, bool ACROSS, bool VEC>
__global__ void __launch_bounds__(128 * H, (R == 4 ? 4 : 2) / H) k_group_few_f32(const __grid_constant__ RowsJob j, const int most) {
  constexpr int kThreads = 128 * H;
  extern __shared__ __align__(16) float xs[];    // kStages steps of rows; the sums' parts; t
  float *parts = xs + kStages * R * 128 * H, *ts = parts + (ACROSS ? 4 : 1) * H * R * kCols;
  __shared__ int adapter[R], found[4];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  grp::Walk walk;
  walk.start();
  for (long long item = blockIdx.y; item < most; item += gridDim.y) {
    __syncthreads();
    if (threadIdx.x < 32) {
      Run run = {0, 0, -1};
      long long inside = 0;
      const bool is = walk.find(j.runs, R, 1, item, &run, &inside);
      if (threadIdx.x == 0) {
        found[0] = is ? 1 : 0;
        found[1] = run.begin + (int)inside * R;
        found[2] = run.end;
        found[3] = run.weight;
      }
    }
    __syncthreads();
    if (!found[0]) return;
    const int row0 = found[1], rows = min(R, found[2] - row0), weight = found[3];
    if (j.t) {
      const int pad = grp::rank_pad(j.rank);
      if (threadIdx.x < 32) {
        if ((int)threadIdx.x < R) adapter[threadIdx.x] = -1;
        __syncwarp();
        grp::each_run(j.ext, row0, row0 + rows, [&](const Run &run) {
          for (int i = max(run.begin - row0, 0); i < min(run.end - row0, rows); ++i) adapter[i] = run.weight;
        }, [](int) {});
      }
      for (int i = (int)threadIdx.x * 8; i < rows * pad; i += kThreads * 8) kept8(reinterpret_cast<const __nv_bfloat16 *>(j.t), row0 + i / pad, pad, i % pad, ts + i);
      __syncthreads();
    }
    tile<R, H, ACROSS, VEC>(j, xs, parts, ts, adapter, row0, rows, weight, (int)blockIdx.x * kCols);
  }
}

template <int R, int H, bool ACROSS, bool VEC>
cudaError_t launch(const RowsJob &j, dim3 grid, int most, cudaStream_t st) {
  constexpr int kBytes = R * (kStages * 128 * H + (ACROSS ? 4 : 1) * H * kCols + grp::kMaxRank) * 4;
  static unsigned char done[kDcMaxDevices];
  const cudaError_t e = dc_set_max_smem_once(k_group_few_f32<R, H, ACROSS, VEC>, kBytes, done);
  return e != cudaSuccess ? e : dc_launch_pdl(k_group_few_f32<R, H, ACROSS, VEC>, grid, dim3(128 * H), kBytes, st, j, most);
}
template <int R>
cudaError_t launch(const RowsJob &j, dim3 grid, int most, int sets, bool across, bool vec, cudaStream_t st) {
  if (!vec && across) return launch<R, 1, true, false>(j, grid, most, st);
  if (!vec) return sets == 2 ? launch<R, 2, false, false>(j, grid, most, st) : launch<R, 1, false, false>(j, grid, most, st);
  if (across) return sets == 2 ? launch<R, 2, true, true>(j, grid, most, st) : launch<R, 1, true, true>(j, grid, most, st);
  return sets == 2 ? launch<R, 2, false, true>(j, grid, most, st) : launch<R, 1, false, true>(j, grid, most, st);
}
int runs_of(const RowsJob &j) { return !j.runs.offsets ? 1 : j.runs.count < j.rows ? j.runs.count : j.rows; }
bool across_of(const RowsJob &j) { return j.w ? j.w_across : j.e_across; }
bool vec_of(const RowsJob &j) { return j.k % 4 == 0 && (!across_of(j) || j.n % 4 == 0); }
int most_tiles(const RowsJob &j) { return j.runs.offsets ? j.rows / grp::rows_few_tile(j) + runs_of(j) : dc_div_up(j.rows, grp::rows_few_tile(j)); }

}  // namespace

namespace grp {

int rows_few_tile(const RowsJob &j) {
  const int mean = j.rows / runs_of(j);
  return mean <= 3 ? 4 : mean <= 8 ? 8 : 16;
}

double rows_few_us(const RowsJob &j) {
  const double rows = rows_few_tile(j), runs = runs_of(j), whole = j.runs.offsets ? j.rows / rows + 0.5 * runs : dc_div_up(j.rows, (int)rows);
  const double tiles = whole < runs ? runs : whole, weights = j.w ? (double)j.n * j.k : 0.0;
  // FMAs and what comes with them; weights from memory once, adapters for each row; a CTA's steps one behind the other
  const double fma = tiles * weights * (0.45 + 0.057 * rows) * 1e-6;
  const double memory = (runs * weights + (j.t ? (double)j.rows * j.n * rank_pad(j.rank) : 0.0)) * 4 / 6e6;
  const double steps = j.w ? dc_div_up(j.k, 256) * (0.3 + 0.065 * rows) : 0.0;
  return 4.0 + (j.t ? 2.5 : 0.0) + fmax(fma, fmax(memory, steps));
}

// Two where there are fewer CTAs than two to an SM; of rows that begin anywhere, fewer than one (2 x 55: 32 us with one set, 25 with two; 35 x 5: 16 and 22),
// and across them never (2 x 84: 11 and 16).
int rows_few_sets(const RowsJob &j) {
  const long long tiles = (long long)dc_div_up(j.n, kCols) * most_tiles(j);
  return tiles < (vec_of(j) ? 2 : across_of(j) ? 0 : 1) * dc_sm_count() ? 2 : 1;
}

cudaError_t rows_few(const RowsJob &j, cudaStream_t st) {
  const int rows = rows_few_tile(j), most = most_tiles(j), sets = rows_few_sets(j);
  // A CTA finds its first tile by walking over the runs in front of it, 32 at a time: of many runs there are CTAs for one round, which walk on
  // (1000 groups of 16 rows, 256 -> 256, 153 us for 476; 256 of 16 rows, 512 -> 512, 186 for 156).
  const int columns = dc_div_up(j.n, kCols), round = dc_div_up((rows == 4 ? 4 : 2) / sets * dc_sm_count(), columns);
  const dim3 grid((unsigned)columns, (unsigned)(j.runs.count > 256 && most > round ? round : most < 65535 ? most : 65535));
  const bool across = across_of(j), vec = vec_of(j);
  return rows == 4 ? launch<4>(j, grid, most, sets, across, vec, st) : rows == 8 ? launch<8>(j, grid, most, sets, across, vec, st) : launch<16>(j, grid, most, sets, across, vec, st);
}

}  // namespace grp
