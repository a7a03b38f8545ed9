// Grouped products, adapters and their gradients on the tensor core, for bf16 rows that begin on 16 bytes (group.cu sees to that).
//
// tcgen05.mma multiplies 128 x N x 16 at a time; operands come by TMA in pieces of 64 along the sum (128-byte rows, swizzled), through a ring of
// stages.  One warp loads, one thread issues, eight warps read out the accumulators, of which there are two: a tile's results go out while
// the next is multiplied.  CTAs walk over tiles; which rows a tile has is found from the runs' offsets on the device, by each warp for itself.
// Matrices that the sum runs across ([k][n], and both operands of a gradient, [rows][...]) are read as they lie: pieces are then 64
// neighbouring columns of 64 rows, and the instruction takes them the other way round.
//   kTile   128 rows of a run x up to 256 columns of its matrix.
//   kFew    runs of few rows: 128 columns of the matrix take the place of the 128 rows, so that an instruction is as wide as there are rows and
//           the matrix streams through once.  Few tiles: a cluster shares a tile's sum.
//   kGrad   128 x up to 256 of a gradient: the sum runs over the rows of a weight's runs.  The last piece of a run holds rows of the next one, which a warp
//           sets to zero in both operands (0 times a NaN is a NaN).
// Adapters (kTile): each run's part is added to the same accumulator by instructions that leave the lanes of other rows alone, so that an
// infinity in one request's adapter stays in its own rows.  (kFew: by the warps that read out, while the matrix streams.)
#include <string.h>

#include "group.cuh"
#include "tc_ptx.cuh"

namespace {
using namespace tc;
using grp::Run;
using grp::Runs;

enum { kTile = 0, kFew = 1, kGrad = 2 };
constexpr int kEpi = 8;                          // warps reading out
template <int FORM>
constexpr int kThreadsOf = (2 + kEpi + (FORM == kGrad ? 1 : 0)) * 32;
constexpr int kMaxStages = 8, kMaxSplit = 8;
constexpr int kSmem = 220 * 1024;
constexpr int kPiece = 64;                       // of the sum, 128 bytes of bf16
constexpr int kP = 128 * 128;                    // bytes of the 128-row operand in a stage
constexpr int kBox = 64 * 128;                   // 64 columns of 64 rows
constexpr int kSuper = 16;                       // rows of tiles that are walked together: 16 x 9 tiles at once read a twelfth of what a row or column of them would
constexpr unsigned long long kLongNs = 20ull * 1000ull * 1000ull * 1000ull;      // a gradient's tile may take seconds: a sum over 2^30 rows
constexpr int kFewMost = 64;                     // rows of a tile of kFew

typedef __nv_bfloat16 bf16;

struct Params {
  int rows, k, n;            // kGrad: m in the place of k
  Runs runs, ext;
  const float *alpha, *bias;
  int bias_each, act;
  const bf16 *residual;
  bf16 *y;
  int y_terms, vec;          // vec: rows of y begin on 16 bytes
  int nt, acc;               // columns of an instruction; of an accumulator
  int tiles_m, tiles_n;      // kGrad: both of a weight; else tiles_n
  int pieces, pieces_per, split;
  long long most;            // items: one to a cluster
  int stages, q_bytes, tmem_cols;
  int maps;                  // bits of the tensor maps that there are
  int rank, rank_pieces;     // adapters: pieces of 64 of the rank
  const bf16 *t, *e;         // kFew: what the reading-out warps take of them
  int e_pitch;
  int early;                 // kFew: what is loaded by TMA was there before the launch in front of this one began
  int off_t;                 // kFew: t's numbers in shared memory
  // kGrad
  float *sums;
  int p_terms, q_terms;
  int out_across;            // out is [n][m]
};

__device__ __forceinline__ uint64_t desc_along(uint32_t a) {     // rows of 64 along the sum, 1024 bytes between groups of 8 rows
  return ((uint64_t)(64u | (1u << 14) | (2u << 29)) << 32) | (uint64_t)((a >> 4) & 0x3FFFu) | (1u << 16);
}
__device__ __forceinline__ uint64_t desc_across(uint32_t a) {    // rows of 64 across it: 1024 bytes between groups of 8 rows, kBox between blocks of 64 columns
  return ((uint64_t)(64u | (1u << 14) | (2u << 29)) << 32) | (uint64_t)((a >> 4) & 0x3FFFu) | ((uint64_t)(kBox >> 4) << 16);
}
template <bool ACROSS>
__device__ __forceinline__ uint64_t desc_of(uint32_t a) { return ACROSS ? desc_across(a) : desc_along(a); }
template <bool ACROSS>
constexpr uint32_t kStepOf = ACROSS ? 16 * 128 / 16 : 32 / 16;   // 16 terms further on, in units of 16 bytes
// D += A B with the lanes of `off` left as they are
__device__ __forceinline__ void umma_lanes(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, const uint32_t (&off)[4]) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, {%5, %6, %7, %8}, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(off[0]), "r"(off[1]), "r"(off[2]), "r"(off[3])
      : "memory");
}

// The tile of an item: tiles of a run are walked column by column in bands of kSuper rows of tiles.
struct Tile {
  int row0, end, weight, tn;
};
template <int FORM>
__device__ __forceinline__ bool find_tile(const Params &p, grp::Walk &walk, long long item, Tile *t) {
  Run run;
  int index;
  long long inside;
  const int tile = FORM == kFew ? p.nt : 128;
  if (!walk.find(p.runs, tile, p.tiles_n, item, &run, &index, &inside)) return false;
  const int tiles_m = (run.end - run.begin + tile - 1) / tile;
  const int band = (int)(inside / ((long long)kSuper * p.tiles_n)), rem = (int)(inside - (long long)band * kSuper * p.tiles_n);
  const int deep = min(kSuper, tiles_m - band * kSuper);
  t->tn = rem / deep;
  t->row0 = run.begin + (band * kSuper + rem - t->tn * deep) * tile;
  t->end = run.end;
  t->weight = run.weight;
  return true;
}

// Calls f(begin, end, weight) for the runs with an adapter that have rows in [row0, end), all lanes together.
template <typename F>
__device__ __forceinline__ void each_run(const Runs &r, int row0, int end, F f) {
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
      o = grp::run_at(r, base + lane);
      stop = o.begin >= end;
    }
    unsigned here = __ballot_sync(0xffffffffu, !stop && o.weight >= 0 && o.end > row0 && o.end > o.begin);
    while (here) {
      const int at = __ffs(here) - 1;
      here &= here - 1;
      f(__shfl_sync(0xffffffffu, o.begin, at), __shfl_sync(0xffffffffu, o.end, at), __shfl_sync(0xffffffffu, o.weight, at));
    }
    if (__any_sync(0xffffffffu, stop)) return;
  }
}

// Calls f(first row, rows, last) for the pieces of 64 rows of a weight's runs.
template <typename F>
__device__ __forceinline__ void each_piece(const Params &p, int weight, int rank, F f) {
  const int first = p.runs.mapped ? 0 : weight, last = p.runs.mapped ? p.runs.count : weight + 1;
  int turn = 0;                                  // pieces go round the CTAs of a cluster
  for (int s = first; s < last; ++s) {
    const Run run = grp::run_at(p.runs, s);
    if (run.weight != weight) continue;
    for (int r = run.begin; r < run.end; r += kPiece) {
      if (turn == rank && !f(r, min(kPiece, run.end - r))) return;
      if (++turn == p.split) turn = 0;
    }
  }
}

__device__ __forceinline__ void unpack8(uint4 w, float *v) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}
__device__ __forceinline__ uint4 pack8(const float *v) {
  return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
// what is left of a value behind its bf16; of an infinity or a NaN nothing
__device__ __forceinline__ float left_of(float v) {
  const float low = v - __bfloat162float(__float2bfloat16(v));
  return low == low ? low : 0.f;
}

enum { kFull = 0, kEmpty = kMaxStages, kDFull = 2 * kMaxStages, kDEmpty = kDFull + 2, kOnes = kDEmpty + 2, kAsk, kFixed, kBars };

template <int FORM, bool ACROSS>
__global__ void __launch_bounds__(kThreadsOf<FORM>, 1)
k_group_tc(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_t,
           const __grid_constant__ CUtensorMap map_e, const __grid_constant__ Params p, DcWsHeader *ws) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bar[kBars];
  __shared__ uint32_t tmem_s, abort_s;
  __shared__ int weight_s[kFewMost], ask_s[3];
  volatile uint32_t *abort_flag = &abort_s;
  const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sm = (smem_u32(smem_raw) + 1023u) & ~1023u;
  if (warp == 0) {
    for (int i = lane; i < kBars; i += 32) mbar_init(&bar[i], i >= kDEmpty && i < kDEmpty + 2 ? kEpi : 1);
    if (lane == 0) abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  } else if (warp == 1 && lane < 4) {
    if (p.maps >> lane & 1) prefetch_tensormap(lane == 0 ? &map_p : lane == 1 ? &map_q : lane == 2 ? &map_t : &map_e);
  }
  // Tensor memory only behind the wait for the launch before this one, whose CTAs may still have theirs to ask for; the one in front of an
  // early launch has none.
  if (FORM == kFew && p.early) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  else dc_pdl_enter();
  if (warp == 1) {
    tmem_alloc(&tmem_s, (uint32_t)p.tmem_cols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_s;
  const int rank = p.split > 1 ? (int)blockIdx.x % p.split : 0;
  const int team = (int)blockIdx.x / p.split, teams = (int)gridDim.x / p.split;
  const uint32_t stage_bytes = (uint32_t)(kP + p.q_bytes);
  const int c0 = rank * p.pieces_per, c1 = min(p.pieces, c0 + p.pieces_per);
  const int per_weight = p.tiles_m * p.tiles_n;  // kGrad; with sums a column of tiles more
  const uint32_t ones = sm + (uint32_t)p.stages * stage_bytes;
  int met = 0;                                   // meetings of the cluster that this thread was at: two, whatever happens

  if (warp == 0) {
    // ---------------------------------------------------------------- load
    const bool lead = elect_one();
    int stage = 0;
    uint32_t parity = 0;
    bool ok = true;
    auto next = [&]() { if (++stage == p.stages) { stage = 0; parity ^= 1u; } };
    if (FORM == kGrad) {
      for (long long item = team; ok && item < p.most; item += teams) {
        const int weight = (int)(item / per_weight), at = (int)(item - (long long)weight * per_weight), tm = at / p.tiles_n, tn = at - tm * p.tiles_n;
        const bool sums = p.sums && tn == p.tiles_n - 1;
        if (lead)
          each_piece(p, weight, rank, [&](int r, int) {
            ok = mbar_wait(&bar[kEmpty + stage], parity ^ 1u, abort_flag, ws, 0x10000u | (uint32_t)stage);
            if (!ok) return false;
            uint64_t *full = &bar[kFull + stage];
            const uint32_t a = sm + (uint32_t)stage * stage_bytes;
            mbar_arrive_expect_tx(full, sums ? (uint32_t)kP : stage_bytes);
            tma_load_2d(a, &map_p, full, tm * 128, r);
            tma_load_2d(a + kBox, &map_p, full, tm * 128 + 64, r);
            if (!sums)
              for (int b = 0; b < p.q_bytes / kBox; ++b) tma_load_2d(a + kP + (uint32_t)(b * kBox), &map_q, full, tn * p.nt + b * 64, r);
            next();
            return true;
          });
        ok = __all_sync(0xffffffffu, ok);
      }
    } else {
      grp::Walk walk;
      walk.start();
      Tile t;
      for (long long item = team; ok && item < p.most && find_tile<FORM>(p, walk, item, &t); item += teams) {
        if (lead) {
          for (int c = c0; c < c1; ++c, next()) {
            ok = mbar_wait(&bar[kEmpty + stage], parity ^ 1u, abort_flag, ws, 0x10000u | (uint32_t)stage);
            if (!ok) break;
            uint64_t *full = &bar[kFull + stage];
            const uint32_t a = sm + (uint32_t)stage * stage_bytes, rows_at = FORM == kFew ? a + kP : a, w_at = FORM == kFew ? a : a + kP;
            mbar_arrive_expect_tx(full, stage_bytes);
            tma_load_2d(rows_at, &map_p, full, c * kPiece, t.row0);
            const int n0 = t.tn * (FORM == kFew ? 128 : p.nt);
            if (ACROSS) {
              for (int b = 0; b < (FORM == kFew ? 2 : p.q_bytes / kBox); ++b)
                tma_load_3d(w_at + (uint32_t)(b * kBox), &map_q, full, n0 + b * 64, c * kPiece, t.weight);
            } else {
              tma_load_3d(w_at, &map_q, full, c * kPiece, n0, t.weight);
            }
          }
        } else {
          for (int c = c0; c < c1; ++c) next();
        }
        __syncwarp();
        if (FORM == kTile && p.rank)
          each_run(p.ext, t.row0, min(t.end, t.row0 + 128), [&](int, int, int weight) {
            for (int c = 0; c < 2 * p.rank_pieces; ++c, next()) {
              if (!lead || !ok) continue;
              ok = mbar_wait(&bar[kEmpty + stage], parity ^ 1u, abort_flag, ws, 0x20000u | (uint32_t)stage);
              if (!ok) continue;
              const int cc = c % p.rank_pieces;
              uint64_t *full = &bar[kFull + stage];
              const uint32_t a = sm + (uint32_t)stage * stage_bytes;
              mbar_arrive_expect_tx(full, stage_bytes);
              tma_load_2d(a, &map_t, full, (c < p.rank_pieces ? 0 : grp::rank_pad(p.rank)) + cc * kPiece, t.row0);
              if (ACROSS) {
                for (int b = 0; b < p.q_bytes / kBox; ++b) tma_load_3d(a + kP + (uint32_t)(b * kBox), &map_e, full, t.tn * p.nt + b * 64, cc * kPiece, weight);
              } else {
                tma_load_3d(a + kP, &map_e, full, cc * kPiece, t.tn * p.nt, weight);
              }
            }
          });
        ok = __all_sync(0xffffffffu, ok);
      }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- multiply: one lane issues, without the others
    const bool lead = elect_one();
    int stage = 0, buf = 0;
    uint32_t parity = 0, use = 0, fixed = 0;     // fixed: pieces with rows that were set to zero
    bool ok = true;
    auto next = [&]() { if (++stage == p.stages) { stage = 0; parity ^= 1u; } };
    auto next_item = [&]() { if (++buf == 2) { buf = 0; ++use; } };
    const uint32_t base = (1u << 4) | (1u << 7) | (1u << 10) | (8u << 24) | ((uint32_t)(p.nt >> 3) << 17);
    if (FORM == kGrad) {
      for (long long item = team; ok && item < p.most; item += teams) {
        const int weight = (int)(item / per_weight), at = (int)(item - (long long)weight * per_weight), tm = at / p.tiles_n;
        const bool sums = p.sums && at - tm * p.tiles_n == p.tiles_n - 1;
        if (lead) {
          bool any = false;
          if (p.sums) ok = mbar_wait(&bar[kOnes], 0, abort_flag, ws, 0x90000u);
          if (ok) ok = mbar_wait(&bar[kDEmpty + buf], (use & 1u) ^ 1u, abort_flag, ws, 0x30000u | (uint32_t)buf);
          tc_fence_after();
          const uint32_t d = tmem + (uint32_t)(buf * p.acc), idesc = (sums ? (base & ~(0x3Fu << 17)) | (2u << 17) : base) | (1u << 15) | (1u << 16);
          if (ok)
            each_piece(p, weight, rank, [&](int, int rows) {
              ok = mbar_wait(&bar[kFull + stage], parity, abort_flag, ws, 0x40000u | (uint32_t)stage);
              if (ok && rows < kPiece) {         // rows of the next run
                ask_s[0] = stage;
                ask_s[1] = rows;
                ask_s[2] = 2 + (sums ? 0 : p.q_bytes / kBox);
                mbar_arrive(&bar[kAsk]);
                ok = mbar_wait(&bar[kFixed], fixed & 1u, abort_flag, ws, 0x50000u | (uint32_t)stage);
                ++fixed;
              }
              if (!ok) return false;
              tc_fence_after();
              const uint32_t a = sm + (uint32_t)stage * stage_bytes;
              const uint64_t ad = desc_across(a), bd = desc_across(sums ? ones : a + kP);
              const int steps = (rows + 15) / 16;
              for (int k = 0; k < steps; ++k, any = true) umma_bf16(d, ad + kStepOf<true> * k, bd + kStepOf<true> * k, idesc, any ? 1u : 0u);
              umma_commit(&bar[kEmpty + stage]);
              next();
              return true;
            });
          if (ok) {
            if (any) umma_commit(&bar[kDFull + buf]);
            else mbar_arrive(&bar[kDFull + buf]);
          }
        }
        next_item();
        ok = __all_sync(0xffffffffu, ok);
      }
      if (lead) {                                // no more
        ask_s[0] = -1;
        mbar_arrive(&bar[kAsk]);
      }
    } else {
      grp::Walk walk;
      walk.start();
      Tile t;
      const uint32_t idesc = base | (!ACROSS ? 0u : FORM == kFew ? 1u << 15 : 1u << 16);
      for (long long item = team; ok && item < p.most && find_tile<FORM>(p, walk, item, &t); item += teams) {
        bool any = false;
        const uint32_t d = tmem + (uint32_t)(buf * p.acc);
        if (lead) {
          ok = mbar_wait(&bar[kDEmpty + buf], (use & 1u) ^ 1u, abort_flag, ws, 0x30000u | (uint32_t)buf);
          tc_fence_after();
          uint32_t ready = 0;
          for (int c = c0; ok && c < c1; ++c) {
            if (!ready) ok = mbar_wait(&bar[kFull + stage], parity, abort_flag, ws, 0x40000u | (uint32_t)stage);
            if (!ok) break;
            ready = stage + 1 < p.stages ? mbar_test(&bar[kFull + stage + 1], parity) : mbar_test(&bar[kFull], parity ^ 1u);
            tc_fence_after();
            const uint32_t a = sm + (uint32_t)stage * stage_bytes;
            const uint64_t ad = FORM == kFew ? desc_of<ACROSS>(a) : desc_along(a), bd = FORM == kFew ? desc_along(a + kP) : desc_of<ACROSS>(a + kP);
            constexpr uint32_t kStepA = FORM == kFew ? kStepOf<ACROSS> : kStepOf<false>, kStepB = FORM == kFew ? kStepOf<false> : kStepOf<ACROSS>;
            const int steps = min(4, (p.k - c * kPiece + 15) / 16);
            if (steps == 4) {
#pragma unroll
              for (int k = 0; k < 4; ++k) umma_bf16(d, ad + kStepA * k, bd + kStepB * k, idesc, any || k > 0 ? 1u : 0u);
            } else {
              for (int k = 0; k < steps; ++k) umma_bf16(d, ad + kStepA * k, bd + kStepB * k, idesc, any || k > 0 ? 1u : 0u);
            }
            any = true;
            umma_commit(&bar[kEmpty + stage]);
            next();
          }
        } else {
          for (int c = c0; c < c1; ++c) next();
        }
        __syncwarp();
        if (FORM == kTile && p.rank)
          each_run(p.ext, t.row0, min(t.end, t.row0 + 128), [&](int begin, int end, int) {
            uint32_t off[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {        // lanes of other rows
              const int lo = max(begin - t.row0 - 32 * i, 0), hi = min(end - t.row0 - 32 * i, 32);
              off[i] = lo >= hi ? 0xffffffffu : ~((hi - lo == 32 ? 0xffffffffu : (1u << (hi - lo)) - 1u) << lo);
            }
            bool first = c0 >= c1;               // without a shared matrix the run's first instruction sets its lanes
            for (int c = 0; c < 2 * p.rank_pieces; ++c, next()) {
              if (!lead || !ok) continue;
              ok = mbar_wait(&bar[kFull + stage], parity, abort_flag, ws, 0x60000u | (uint32_t)stage);
              if (!ok) continue;
              tc_fence_after();
              const uint32_t a = sm + (uint32_t)stage * stage_bytes;
              const uint64_t ad = desc_along(a), bd = desc_of<ACROSS>(a + kP);
              const int steps = min(4, (p.rank - c % p.rank_pieces * kPiece + 15) / 16);
              for (int k = 0; k < steps; ++k, first = false) umma_lanes(d, ad + kStepOf<false> * k, bd + kStepOf<ACROSS> * k, idesc, first ? 0u : 1u, off);
              any = true;
              umma_commit(&bar[kEmpty + stage]);
            }
          });
        if (lead && ok) {
          if (any) umma_commit(&bar[kDFull + buf]);
          else mbar_arrive(&bar[kDFull + buf]);
        }
        next_item();
        ok = __all_sync(0xffffffffu, ok);
      }
    }
  } else if (warp < 2 + kEpi) {
    // ---------------------------------------------------------------- read out
    const int quad = warp & 3, set = (warp - 2) >> 2, own = quad * 32 + lane;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    int buf = 0;
    uint32_t use = 0;
    bool ok = true;
    auto next_item = [&]() { if (++buf == 2) { buf = 0; ++use; } };
    auto release = [&]() {
      tc_fence_before();
      __syncwarp();
      if (elect_one()) mbar_arrive(&bar[kDEmpty + buf]);
      __syncwarp();
    };
    if (FORM == kGrad) {
      if (p.sums) {                              // a block of ones: sums are products with it
        for (int i = (warp - 2) * 32 + lane; i < kBox / 16; i += kEpi * 32) sts_u4(ones + (uint32_t)(i * 16), make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u));
        fence_proxy_async();
        bar_sync(1, kEpi * 32);
        if (warp == 2 && lane == 0) mbar_arrive(&bar[kOnes]);
      }
      for (long long item = team; ok && item < p.most; item += teams) {
        const int weight = (int)(item / per_weight), at = (int)(item - (long long)weight * per_weight), tm = at / p.tiles_n, tn = at - tm * p.tiles_n;
        const bool sums = p.sums && tn == p.tiles_n - 1;
        ok = warp_wait(&bar[kDFull + buf], use & 1u, abort_flag, ws, 0x70000u | (uint32_t)buf, kLongNs);
        if (!ok) break;
        tc_fence_after();
        // whether there is anything to read: with none of this CTA's pieces nothing was multiplied
        int have = 0;
        each_piece(p, weight, rank, [&](int, int) { have = 1; return false; });
        const int i = tm * 128 + own, cols = sums ? 16 : p.nt, pad = p.nt / 2;
        const uint32_t d = tmem + (uint32_t)(buf * p.acc) + lanes;
        bf16 *out = p.y + (size_t)weight * (size_t)p.k * (size_t)p.n;
        auto deliver = [&](int c, const float (&v)[16]) {            // columns c on of this thread's row
          if (i >= p.k) return;
          if (sums) {
            if (c == 0) p.sums[(size_t)weight * (size_t)p.k + (size_t)i] = v[0];
            return;
          }
          const int j0 = tn * p.nt + c;
          if (p.out_across) {
#pragma unroll
            for (int x = 0; x < 16; ++x)
              if (j0 + x < p.n) out[(size_t)(j0 + x) * (size_t)p.k + (size_t)i] = __float2bfloat16(v[x]);
            return;
          }
          bf16 *to = out + (size_t)i * (size_t)p.n + (size_t)j0;
          if (p.vec) {
#pragma unroll
            for (int x = 0; x < 16; x += 8)
              if (j0 + x < p.n) *reinterpret_cast<uint4 *>(to + x) = pack8(v + x);
          } else {
#pragma unroll
            for (int x = 0; x < 16; ++x)
              if (j0 + x < p.n) to[x] = __float2bfloat16(v[x]);
          }
        };
        if (p.split == 1) {
          const int half = p.q_terms ? pad : cols;
          for (int c = set * 16; c < half; c += 32) {
            float v[16], w[16];
            __syncwarp();
            tmem_ld16(d + (uint32_t)c, reinterpret_cast<uint32_t *>(v));
            if (p.q_terms && !sums) tmem_ld16(d + (uint32_t)(pad + c), reinterpret_cast<uint32_t *>(w));
            tmem_ld_wait();
#pragma unroll
            for (int x = 0; x < 16; ++x) {
              if (p.q_terms && !sums) v[x] += w[x];
              if (!have) v[x] = 0.f;
            }
            deliver(c, v);
          }
          release();
        } else {
          // the part to shared memory, [columns][128]; the ring is not in use any more
          for (int c = set * 16; c < cols; c += 32) {
            uint32_t v[16];
            __syncwarp();
            tmem_ld16(d + (uint32_t)c, v);
            tmem_ld_wait();
#pragma unroll
            for (int x = 0; x < 16; ++x) asm volatile("st.shared.b32 [%0], %1;" ::"r"(sm + (uint32_t)(((c + x) * 128 + own) * 4)), "r"(have ? v[x] : 0u) : "memory");
          }
          __syncwarp();
          cluster_sync();
          ++met;
          const int half = p.q_terms && !sums ? pad : cols, blocks = half / 16;
          for (int b = rank + set * p.split; b < blocks; b += 2 * p.split) {
            float v[16];
#pragma unroll
            for (int x = 0; x < 16; ++x) v[x] = 0.f;
            for (int k = 0; k < p.split; ++k) {
              const uint32_t from = map_cluster(sm, (uint32_t)k);
#pragma unroll
              for (int x = 0; x < 16; ++x) {
                v[x] += lds_cluster_f(from + (uint32_t)(((b * 16 + x) * 128 + own) * 4));
                if (p.q_terms && !sums) v[x] += lds_cluster_f(from + (uint32_t)(((pad + b * 16 + x) * 128 + own) * 4));
              }
            }
            deliver(b * 16, v);
          }
          release();
        }
        next_item();
      }
    } else if (FORM == kTile) {
      grp::Walk walk;
      walk.start();
      Tile t;
      for (long long item = team; ok && item < p.most && find_tile<FORM>(p, walk, item, &t); item += teams) {
        const int row = t.row0 + own;
        const bool mine = row < t.end;
        float alpha = p.alpha ? __ldg(p.alpha + t.weight) : 1.f;
        bool filled = true;                      // without a shared matrix: whether an adapter has set this lane
        if (p.rank && c0 >= c1) {
          const int s = mine ? grp::first_run_behind(p.ext, row) : p.ext.count;
          filled = false;
          for (int r = s; r < p.ext.count; ++r) {      // empty runs in between
            const Run run = grp::run_at(p.ext, r);
            if (run.begin > row) break;
            if (run.end > row) { filled = run.weight >= 0; break; }
          }
        }
        const float *bias = p.bias ? p.bias + (p.bias_each ? (size_t)t.weight * (size_t)p.n : 0) : nullptr;
        const uint32_t d = tmem + (uint32_t)(buf * p.acc) + lanes;
        ok = warp_wait(&bar[kDFull + buf], use & 1u, abort_flag, ws, 0x70000u | (uint32_t)buf);
        if (!ok) break;
        tc_fence_after();
        const int o0 = t.tn * p.nt;
#pragma unroll 1
        for (int c = set * 32; c < p.nt; c += 64) {
          float v[32];
          __syncwarp();
          tmem_ld32(d + (uint32_t)c, reinterpret_cast<uint32_t *>(v));
          tmem_ld_wait();
          if (c + 64 >= p.nt) release();
          if (!mine) continue;
#pragma unroll
          for (int x = 0; x < 32; ++x) v[x] = filled ? v[x] * alpha : 0.f;
          if (p.y_terms) {
            const int pad = grp::rank_pad(p.n);
            bf16 *to = p.y + (size_t)row * (size_t)(2 * pad) + (size_t)(o0 + c);
#pragma unroll
            for (int x = 0; x < 32; x += 8) {
              if (o0 + c + x >= pad) break;
              float low[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                if (o0 + c + x + i >= p.n) v[x + i] = 0.f;         // what the padding holds
                low[i] = left_of(v[x + i]);
              }
              *reinterpret_cast<uint4 *>(to + x) = pack8(v + x);
              *reinterpret_cast<uint4 *>(to + pad + x) = pack8(low);
            }
            continue;
          }
          const size_t at = (size_t)row * (size_t)p.n + (size_t)(o0 + c);
          if (p.vec) {
#pragma unroll
            for (int x = 0; x < 32; x += 8) {
              if (o0 + c + x >= p.n || c + x >= p.nt) break;
              if (bias) {
                const float4 b0 = __ldg(reinterpret_cast<const float4 *>(bias + o0 + c + x)), b1 = __ldg(reinterpret_cast<const float4 *>(bias + o0 + c + x + 4));
                v[x] += b0.x; v[x + 1] += b0.y; v[x + 2] += b0.z; v[x + 3] += b0.w;
                v[x + 4] += b1.x; v[x + 5] += b1.y; v[x + 6] += b1.z; v[x + 7] += b1.w;
              }
              if (p.residual) {
                float r[8];
                unpack8(*reinterpret_cast<const uint4 *>(p.residual + at + x), r);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[x + i] += r[i];
              }
#pragma unroll
              for (int i = 0; i < 8; ++i) v[x + i] = dc_act_apply(v[x + i], p.act);
              *reinterpret_cast<uint4 *>(p.y + at + x) = pack8(v + x);
            }
          } else {
#pragma unroll
            for (int x = 0; x < 32; ++x) {
              if (o0 + c + x >= p.n || c + x >= p.nt) break;
              if (bias) v[x] += __ldg(bias + o0 + c + x);
              if (p.residual) v[x] += __bfloat162float(p.residual[at + x]);
              p.y[at + x] = __float2bfloat16(dc_act_apply(v[x], p.act));
            }
          }
        }
        if (set * 32 >= p.nt) release();
        next_item();
      }
    } else {
      if (p.early) asm volatile("griddepcontrol.wait;" ::: "memory");
      grp::Walk walk;
      walk.start();
      Tile t;
      const int half = p.nt / 2;                 // of a set of four warps: rows of x
      for (long long item = team; item < p.most && find_tile<FORM>(p, walk, item, &t); item += teams) {
        const int o = t.tn * 128 + own, count = min(p.nt, t.end - t.row0);
        float part[kFewMost / 2];
#pragma unroll
        for (int i = 0; i < kFewMost / 2; ++i) part[i] = 0.f;
        if (p.rank) {
          // the adapters' part of the rows that this CTA delivers, while the shared matrix is multiplied
          const uint32_t ts = sm + (uint32_t)p.off_t;
          const int pad = grp::rank_pad(p.rank), u = (warp - 2) * 32 + lane;
          bar_sync(1, kEpi * 32);                // the last item's are read
          if (u < p.nt) {
            int w = -1;
            const int row = t.row0 + u;
            if (u < count)
              for (int r = grp::first_run_behind(p.ext, row); r < p.ext.count; ++r) {
                const Run run = grp::run_at(p.ext, r);
                if (run.begin > row) break;
                if (run.end > row) { w = run.weight; break; }
              }
            weight_s[u] = w;
          }
          for (int i = u; i < count * pad; i += kEpi * 32) {
            const int r = i / pad, jj = i - r * pad;
            const bf16 *at = p.t + (size_t)(t.row0 + r) * (size_t)(2 * pad) + (size_t)jj;
            const float v = __bfloat162float(at[0]) + __bfloat162float(at[pad]);
            asm volatile("st.shared.f32 [%0], %1;" ::"r"(ts + (uint32_t)(i * 4)), "f"(v) : "memory");
          }
          bar_sync(1, kEpi * 32);
          if (o < p.n) {
            const int o_of = o;
#pragma unroll
            for (int i0 = 0; i0 < kFewMost / 2; i0 += 4) {
              if (i0 >= half) break;
              int w[4];
              bool any = false;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int r = set * half + i0 + i;
                w[i] = r < count && (p.split == 1 || r % p.split == rank) ? weight_s[r] : -1;
                any |= w[i] >= 0;
              }
              if (!any) continue;
              for (int j0 = 0; j0 < p.rank; j0 += 8) {
                float e[4][8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  if (ACROSS) {
#pragma unroll
                    for (int x = 0; x < 8; ++x)
                      e[i][x] = w[i] >= 0 && j0 + x < p.rank ? __bfloat162float(p.e[((size_t)w[i] * (size_t)p.rank + (size_t)(j0 + x)) * (size_t)p.e_pitch + (size_t)o_of]) : 0.f;
                  } else {
                    uint4 raw = make_uint4(0, 0, 0, 0);
                    if (w[i] >= 0) raw = __ldg(reinterpret_cast<const uint4 *>(p.e + ((size_t)w[i] * (size_t)p.n + (size_t)o_of) * (size_t)p.e_pitch + (size_t)j0));
                    unpack8(raw, e[i]);
                  }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  if (w[i] < 0) continue;
                  const uint32_t at = ts + (uint32_t)(((set * half + i0 + i) * pad + j0) * 4);
                  const uint4 t0 = lds_u4(at), t1 = lds_u4(at + 16);
                  const uint32_t tv[8] = {t0.x, t0.y, t0.z, t0.w, t1.x, t1.y, t1.z, t1.w};
#pragma unroll
                  for (int x = 0; x < 8; ++x) part[i0 + i] = fmaf(__uint_as_float(tv[x]), e[i][x], part[i0 + i]);
                }
              }
            }
          }
        }
        const float b = p.bias && o < p.n ? __ldg(p.bias + (p.bias_each ? (size_t)t.weight * (size_t)p.n : 0) + (size_t)o) : 0.f;
        const uint32_t d = tmem + (uint32_t)(buf * p.acc) + lanes;
        // a wait that ran out does not end the loop: the barriers above are of all these warps
        if (!warp_wait(&bar[kDFull + buf], use & 1u, abort_flag, ws, 0x70000u | (uint32_t)buf)) {
          next_item();
          continue;
        }
        tc_fence_after();
        auto deliver = [&](int r, float v) {     // row r of the tile: its part of the sum
          if (r >= count || o >= p.n) return;
          const size_t at = (size_t)(t.row0 + r) * (size_t)p.n + (size_t)o;
          v += b;
          if (p.residual) v += __bfloat162float(p.residual[at]);
          p.y[at] = __float2bfloat16(dc_act_apply(v, p.act));
        };
        if (p.split == 1) {
#pragma unroll
          for (int i0 = 0; i0 < kFewMost / 2; i0 += 8) {
            if (i0 >= half) break;
            float v[8];
            __syncwarp();
            tmem_ld8(d + (uint32_t)(set * half + i0), reinterpret_cast<uint32_t *>(v));
            tmem_ld_wait();
            if (i0 + 8 >= half) release();
#pragma unroll
            for (int i = 0; i < 8; ++i) deliver(set * half + i0 + i, (p.pieces ? v[i] : 0.f) + part[i0 + i]);
          }
        } else {
          // parts to shared memory, [rows][128]; the ring is not in use any more
          for (int i0 = 0; i0 < half; i0 += 8) {
            uint32_t v[8];
            __syncwarp();
            tmem_ld8(d + (uint32_t)(set * half + i0), v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 8; ++i) asm volatile("st.shared.b32 [%0], %1;" ::"r"(sm + (uint32_t)(((set * half + i0 + i) * 128 + own) * 4)), "r"(v[i]) : "memory");
          }
          __syncwarp();
          cluster_sync();
          ++met;
#pragma unroll
          for (int i = 0; i < kFewMost / 2; ++i) {
            const int r = set * half + i;
            if (i >= half || r % p.split != rank || r >= count) continue;
            float v = part[i];
            for (int k = 0; k < p.split; ++k) v += lds_cluster_f(map_cluster(sm, (uint32_t)k) + (uint32_t)((r * 128 + own) * 4));
            deliver(r, v);
          }
          release();
        }
        next_item();
      }
    }
  } else {
    // ---------------------------------------------------------------- kGrad: rows behind the end of a run are set to zero
    for (uint32_t asked = 0;; ++asked) {
      if (!warp_wait(&bar[kAsk], asked & 1u, abort_flag, ws, 0x80000u, kLongNs)) break;
      const int stage = ask_s[0], rows = ask_s[1], boxes = ask_s[2], per = (kPiece - rows) * 8;       // 16 bytes each
      if (stage < 0) break;
      const uint32_t a = sm + (uint32_t)stage * stage_bytes;
      for (int b = 0; b < boxes; ++b)
        for (int i = lane; i < per; i += 32) sts_u4(a + (uint32_t)(b * kBox + rows * 128 + i * 16), make_uint4(0, 0, 0, 0));
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar[kFixed]);
    }
  }
  __syncwarp();
  if (p.split > 1)
    for (; met < 2; ++met) cluster_sync();       // the parts are there; and read
  if (warp == 1 && *abort_flag) {                // copies and products may still be in flight: give them time to end
    const unsigned long long t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 20ull * 1000ull * 1000ull) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, (uint32_t)p.tmem_cols);
}

// x [rows][cols], bf16 -> rows that begin on 16 bytes, zeros behind them
__global__ void __launch_bounds__(256) k_group_pitch(const bf16 *__restrict__ x, bf16 *__restrict__ y, long long rows, int cols, int pitch) {
  dc_pdl_enter();
  const int per = pitch / 8;
  for (long long u = (long long)blockIdx.x * 256 + threadIdx.x; u < rows * per; u += (long long)gridDim.x * 256) {
    const long long row = u / per;
    const int c = (int)(u - row * per) * 8;
    const unsigned short *from = reinterpret_cast<const unsigned short *>(x) + (size_t)row * (size_t)cols + (size_t)c;
    uint32_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? from[i] : 0;
    *reinterpret_cast<uint4 *>(y + (size_t)row * (size_t)pitch + (size_t)c) =
        make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
  }
}

// What rows keep of their adapters where runs are short: a warp to two numbers of a row, the adapter's rows read straight through.
// The next launch starts only behind the wait for the one before this: what that one wrote is there for it.
__global__ void __launch_bounds__(256) k_adapter_narrow(const bf16 *__restrict__ x, int x_pitch, const bf16 *__restrict__ a, int a_pitch, int k, int rank,
                                                        const __grid_constant__ Runs runs, const float *__restrict__ scale, bf16 *__restrict__ t) {
  __shared__ int weight_s;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int row = (int)blockIdx.x, warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
  if (warp == 0) {
    int w = -1;
    each_run(runs, row, row + 1, [&](int begin, int end, int weight) { if (begin <= row && row < end) w = weight; });
    if (lane == 0) weight_s = w;
  }
  __syncthreads();
  const int w = weight_s;
  if (w < 0) return;
  const int j = (int)blockIdx.y * 16 + warp * 2, pad = grp::rank_pad(rank);
  float s[2] = {0.f, 0.f};
  const bf16 *xr = x + (size_t)row * (size_t)x_pitch, *ar = a + ((size_t)w * (size_t)rank + (size_t)j) * (size_t)a_pitch;
  const bool two = j + 1 < rank;
  if (j < rank) {
    constexpr int kAhead = 4;
    for (int i0 = lane * 8; i0 < k; i0 += kAhead * 256) {
      uint4 xv[kAhead], av[kAhead], bv[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int i = i0 + u * 256;
        xv[u] = av[u] = bv[u] = make_uint4(0, 0, 0, 0);
        if (i < k) {
          xv[u] = *reinterpret_cast<const uint4 *>(xr + i);
          av[u] = *reinterpret_cast<const uint4 *>(ar + i);
          if (two) bv[u] = *reinterpret_cast<const uint4 *>(ar + (size_t)a_pitch + i);
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        float xf[8], af[8], bf_[8];
        unpack8(xv[u], xf);
        unpack8(av[u], af);
        unpack8(bv[u], bf_);
#pragma unroll
        for (int i = 0; i < 8; ++i) { s[0] = fmaf(xf[i], af[i], s[0]); s[1] = fmaf(xf[i], bf_[i], s[1]); }
      }
    }
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    s[0] += __shfl_xor_sync(0xffffffffu, s[0], d);
    s[1] += __shfl_xor_sync(0xffffffffu, s[1], d);
  }
  if (lane == 0) {
    const float f = scale ? __ldg(scale + w) : 1.f;
    bf16 *to = t + (size_t)row * (size_t)(2 * pad) + (size_t)j;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float v = j + i < rank ? s[i] * f : 0.f;
      to[i] = __float2bfloat16(v);
      to[pad + i] = __float2bfloat16(left_of(v));
    }
  }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn get_encode_fn() {
  static EncodeTiledFn fn = nullptr;
  if (!fn) {
    void *ptr = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &qres) == cudaSuccess &&
        qres == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeTiledFn>(ptr);
  }
  return fn;
}
// [outer][rows][cols] with rows `pitch` elements apart: boxes of 64 columns x `box` rows, zeros outside
bool map_of(CUtensorMap *map, const void *at, long long cols, long long rows, long long outer, long long pitch, int box) {
  EncodeTiledFn encode = get_encode_fn();
  if (!encode) return false;
  const cuuint64_t dim[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)outer}, str[2] = {(cuuint64_t)pitch * 2, (cuuint64_t)pitch * 2 * (cuuint64_t)rows};
  const cuuint32_t bx[3] = {kPiece, (cuuint32_t)box, 1}, es[3] = {1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, outer ? 3 : 2, const_cast<void *>(at), dim, str, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int FORM, bool ACROSS>
cudaError_t launch(const Params &p, int grid, const CUtensorMap (&m)[4], DcWsHeader *ws, cudaStream_t st) {
  static unsigned char attr_done[kDcMaxDevices];
  const cudaError_t e = dc_set_max_smem_once(k_group_tc<FORM, ACROSS>, kSmem, attr_done);
  if (e != cudaSuccess) return e;
  return dc_launch_pdl_cluster(k_group_tc<FORM, ACROSS>, dim3((unsigned)grid), dim3(kThreadsOf<FORM>), (size_t)kSmem, st, p.split, m[0], m[1], m[2], m[3], p, ws);
}

// Shared and tensor memory; `apart`: bytes beside the ring
void lay_out(Params *p, int apart) {
  p->acc = (int)dc_round_up((size_t)p->nt, 32);
  p->tmem_cols = 32;
  while (p->tmem_cols < 2 * p->acc) p->tmem_cols *= 2;
  p->stages = (kSmem - 1024 - apart) / (kP + p->q_bytes);
  if (p->stages > kMaxStages) p->stages = kMaxStages;
  p->off_t = p->stages * (kP + p->q_bytes);
}
// CTAs that share a tile's sum of `pieces`: as many as keep all SMs busy, each with `least` pieces at least
int split_of(long long items, int pieces, int least, int n_sm) {
  int s = items > 0 ? (int)(n_sm / items) : 1;
  if (s > kMaxSplit) s = kMaxSplit;
  if (s > pieces / least) s = pieces / least;
  if (s < 1) s = 1;
  return s;
}
// columns to a tile: the fewest rounds of tiles, each as long as its instructions (narrower ones wait for shared memory)
int columns_of(int n, double tiles_m, int n_sm) {
  static constexpr struct { int nt; double cost; } kinds[3] = {{256, 1.0}, {128, 0.58}, {64, 0.42}};
  int best = 256;
  double least = 1e30;
  for (const auto &k : kinds) {
    if (k.nt > 64 && n <= k.nt / 2) continue;
    const double rounds = tiles_m * dc_div_up(n, k.nt) / n_sm, time = (rounds < 1 ? 1 : rounds + 0.5) * k.cost;
    if (time < least) { least = time; best = k.nt; }
  }
  return best;
}

}  // namespace

namespace grp {

static long long row_tiles(const Runs &r, int tile) {
  const long long runs = r.offsets ? (r.count < r.rows ? r.count : r.rows) : 1;
  return r.rows / tile + runs;
}

cudaError_t pitch_tc(const void *x, void *y, long long rows, int cols, int pitch, cudaStream_t st) {
  const long long blocks = (rows * (pitch / 8) + 255) / 256;
  return dc_launch_pdl(k_group_pitch, dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20))), dim3(256), 0, st, (const bf16 *)x, (bf16 *)y, rows, cols, pitch);
}

// Rows whose runs are this short go by kFew (rows through it again for each tile of 64; 128 columns of a matrix are a tile's whatever its rows).
static bool few(const RowsJob &j) {
  if (j.y_terms) return false;
  if (!j.runs.offsets) return j.rows <= 128;
  const int runs = j.runs.count < j.rows ? j.runs.count : j.rows;
  return j.rows / runs <= 48;
}
bool narrow_apart(const RowsJob &j) { return j.y_terms && !j.w_across && j.rows <= 1024 && j.rows / (j.runs.count < j.rows ? j.runs.count : j.rows) <= 8; }

cudaError_t narrow_tc(const RowsJob &j, cudaStream_t st) {
  return dc_launch_pdl(k_adapter_narrow, dim3((unsigned)j.rows, (unsigned)dc_div_up(rank_pad(j.n), 16)), dim3(256), 0, st, (const bf16 *)j.x, j.x_pitch, (const bf16 *)j.w,
                       j.w_pitch, j.k, j.n, j.runs, j.alpha, (bf16 *)j.y);
}

cudaError_t rows_tc(const RowsJob &j, bool behind_narrow, DcWsHeader *ws, cudaStream_t st) {
  const int n_sm = dc_sm_count();
  Params p = {};
  p.rows = j.rows;
  p.k = j.k;
  p.n = j.n;
  p.runs = j.runs;
  p.alpha = j.alpha;
  p.bias = j.bias;
  p.bias_each = j.bias_each;
  p.act = j.act;
  p.residual = (const bf16 *)j.residual;
  p.y = (bf16 *)j.y;
  p.y_terms = j.y_terms;
  p.vec = j.n % 8 == 0;
  p.pieces = j.w ? dc_div_up(j.k, kPiece) : 0;
  p.split = 1;
  if (j.t) {
    p.ext = j.ext;
    p.rank = j.rank;
    p.rank_pieces = dc_div_up(j.rank, kPiece);
    p.t = (const bf16 *)j.t;
    p.e = (const bf16 *)j.e;
    p.e_pitch = j.e_pitch;
  }
  const bool by_few = few(j);
  long long items;
  if (by_few) {
    const int runs = j.runs.offsets ? (j.runs.count < j.rows ? j.runs.count : j.rows) : 1, mean = j.rows / runs;
    p.nt = mean <= (runs == 1 ? 16 : 12) ? 16 : mean <= (runs == 1 ? 32 : 24) ? 32 : 64;
    p.q_bytes = p.nt * 128;
    p.tiles_n = dc_div_up(j.n, 128);
    items = row_tiles(j.runs, p.nt) * p.tiles_n;
    if (runs == 1) items = (long long)dc_div_up(j.rows, p.nt) * p.tiles_n;
    p.split = split_of(items, p.pieces, 4, n_sm);
    p.early = behind_narrow && !j.runs.offsets;
    lay_out(&p, p.rank ? p.nt * rank_pad(p.rank) * 4 : 0);
  } else {
    const int runs = j.runs.offsets ? (j.runs.count < j.rows ? j.runs.count : j.rows) : 1;
    p.nt = j.y_terms ? rank_pad(j.n) : columns_of(j.n, j.rows / 128.0 + 0.5 * runs, n_sm);
    p.q_bytes = j.w_across ? dc_div_up(p.nt, 64) * kBox : p.nt * 128;
    p.tiles_n = dc_div_up(j.n, p.nt);
    items = row_tiles(j.runs, 128) * p.tiles_n;
    lay_out(&p, 0);
  }
  p.pieces_per = dc_div_up(p.pieces, p.split);
  while (p.split > 1 && p.pieces_per * (p.split - 1) >= p.pieces) { --p.split; p.pieces_per = dc_div_up(p.pieces, p.split); }
  CUtensorMap m[4] = {};
  p.maps = (j.w ? 3 : 0) | (j.t && !by_few ? 12 : 0);
  const int of_w = j.w_across ? 64 : by_few ? 128 : p.nt;
  if (j.w) {
    if (!map_of(&m[0], j.x, j.k, j.rows, 0, j.x_pitch, by_few ? p.nt : 128)) return cudaErrorNotSupported;
    if (!(j.w_across ? map_of(&m[1], j.w, j.n, j.k, j.runs.weights, j.w_pitch, of_w) : map_of(&m[1], j.w, j.k, j.n, j.runs.weights, j.w_pitch, of_w)))
      return cudaErrorNotSupported;
  }
  if (j.t && !by_few) {
    if (!map_of(&m[2], j.t, 2 * rank_pad(j.rank), j.rows, 0, 2 * rank_pad(j.rank), 128)) return cudaErrorNotSupported;
    if (!(j.e_across ? map_of(&m[3], j.e, j.n, j.rank, j.ext.weights, j.e_pitch, 64) : map_of(&m[3], j.e, j.rank, j.n, j.ext.weights, j.e_pitch, p.nt)))
      return cudaErrorNotSupported;
  }
  const long long teams = items < n_sm / p.split ? items : n_sm / p.split;
  const int grid = (int)teams * p.split;
  p.most = p.split > 1 ? teams : 1ll << 62;
  const bool across = j.w ? j.w_across : j.e_across;
  if (by_few) return across ? launch<kFew, true>(p, grid, m, ws, st) : launch<kFew, false>(p, grid, m, ws, st);
  return across ? launch<kTile, true>(p, grid, m, ws, st) : launch<kTile, false>(p, grid, m, ws, st);
}

// out_w = p^T q of the rows of each weight.  p plain, q plain or what rows keep of an adapter; out [m][n], or [n][m] with out_across.
cudaError_t grad_tc(const GradJob &j, DcWsHeader *ws, cudaStream_t st) {
  const int n_sm = dc_sm_count();
  Params p = {};
  p.rows = j.runs.rows;
  p.k = j.m;
  p.n = j.n;
  p.runs = j.runs;
  p.y = (bf16 *)j.out;
  p.sums = j.sums;
  p.q_terms = j.q_terms;
  p.out_across = j.out_across;
  p.vec = j.n % 8 == 0;
  const int pad = rank_pad(j.n), weights = j.runs.weights;
  p.tiles_m = dc_div_up(j.m, 128);
  p.nt = !j.out ? 64 : j.q_terms ? 2 * pad : columns_of(j.n, (double)p.tiles_m * weights, n_sm);
  p.q_bytes = dc_div_up(p.nt, 64) * kBox;
  p.tiles_n = (j.out ? dc_div_up(j.q_terms ? 1 : j.n, j.q_terms ? 1 : p.nt) : 0) + (j.sums ? 1 : 0);
  const long long items = (long long)p.tiles_m * p.tiles_n * weights;
  const int pieces = j.runs.rows / kPiece / weights;
  p.split = split_of(items, pieces, 4, n_sm);
  lay_out(&p, j.sums ? kBox : 0);
  CUtensorMap m[4] = {};
  p.maps = j.runs.rows ? (j.out ? 3 : 1) : 0;
  if (j.runs.rows) {                             // without rows nothing is loaded
    if (!map_of(&m[0], j.p, j.m, j.runs.rows, 0, j.p_pitch, 64)) return cudaErrorNotSupported;
    if (j.out && !map_of(&m[1], j.q, j.q_terms ? 2 * pad : j.n, j.runs.rows, 0, j.q_terms ? 2 * pad : j.q_pitch, 64)) return cudaErrorNotSupported;
  }
  const long long teams = items < n_sm / p.split ? items : n_sm / p.split;
  p.most = items;
  return launch<kGrad, true>(p, (int)teams * p.split, m, ws, st);
}

}  // namespace grp
