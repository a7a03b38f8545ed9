// Grouped products, adapters and their gradients on the tensor core.
//
// tcgen05.mma multiplies 128 x N x 16 at a time; operands come by TMA in pieces of 64 along the sum (128-byte rows, swizzled), through a ring of
// stages.  One warp loads, one thread issues, eight warps read out the accumulators, of which there are two or more: a tile's results go out
// while the next is multiplied.  CTAs walk over tiles; which rows a tile has is found from the runs' offsets on the device, by each warp for itself.
// Matrices that the sum runs across ([k][n], and both operands of a gradient, [rows][...]) are read as they lie: pieces are then 64
// neighbouring columns of 64 rows, and the instruction takes them the other way round.
//   kTile   128 rows of a run x up to 256 columns of its matrix.
//   kFew    runs of few rows (bf16): 128 columns of the matrix take the place of the 128 rows, so that an instruction is as wide as there are rows and
//           the matrix streams through once.  Adapters' parts of those columns, a row's after a row's, come through a ring of their own.
//   kGrad   128 x up to 256 of a gradient: the sum runs over the rows of a weight's runs.  Where a run ends inside a piece, rows of other weights in it are set to zero by
//           a warp, in both operands (0 times a NaN is a NaN).
// kTile and kGrad in pairs (cta_group::2): two CTAs multiply 256 x 256, each loads half of either operand.
// Few tiles: a cluster shares a tile's sum, and adds up its parts through its shared memory.
// Adapters (kTile): each run's part is added to the same accumulator by instructions that leave the lanes of other rows alone, so that an
// infinity in one request's adapter stays in its own rows.  (kFew: by the warps that read out, while the matrix streams.)
//
// fp32: a value is three bf16 terms that add up to it (split_tc), laid out one behind the other, and a stage holds all three of both operands: six of
// their nine products are above 2^-24 of the result, small ones first.  The tensor core cuts its sums instead of rounding them, so a piece's
// sum is read out and added up in fp32 registers.  A result that is a NaN is worked out again by FMAs: an infinity, or a value
// beyond the largest bf16, has a NaN among its terms.
//
// What bounds it: many rows, the tensor core under the power cap (8192 rows, 4096 -> 4096 in one group 184 us, 1.49 PFLOP/s; 16384 ragged rows of 16
// groups 401 us a launch by itself, 486 one behind the other); few rows, the weights' bytes (256 rows of 64 groups, 2048 -> 2048, 82 to 85 us, 6.4 TB/s); fp32,
// its six products and what an SM takes in, 45 bytes a cycle (a piece of 128 x 128: 0.8 us of products, 96 KB, 1.2 in all; in pairs of 256 x 256, for half the
// bytes, 2048 x 2048 x 2048 took 96 us for 98, but 16 groups of 256 rows, 512 -> 512, 40 for 26); single rows, a chain of launch, offsets, loads and a
// cluster's meeting (4 rows of 8 groups, 1024 -> 1024, 6.7 us).
#include <math.h>
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
constexpr int kThreadsOf = (2 + kEpi + (FORM == kTile ? 0 : 1)) * 32;
constexpr int kMaxStages = 8, kMaxSplit = 8, kMaxSlots = 8, kMaxAccs = 4;
constexpr int kSmem = 226 * 1024;                // what the static arrays leave
constexpr int kPiece = 64;                       // of the sum, 128 bytes of bf16
constexpr int kP = 128 * 128;                    // bytes of the 128-row operand in a stage
constexpr int kBox = 64 * 128;                   // 64 columns of 64 rows
constexpr int kOut = kEpi * 32 * 128;            // staged results: 32 rows x 32 sums a warp
constexpr int kSuper = 16;                       // rows of tiles that are walked together: of 128 x 256, 16 x 9 at once read a quarter of what a column of as many would, a ninth of a row
constexpr int kFewMost = 64, kFewWide = 32;     // rows of a tile of kFew; of adapters of a rank above 64, each of which takes more shared memory
// A gradient's tile may take seconds (2^30 rows are 17 million pieces), and so may results that are worked out again by FMAs: 0.8 s a million rows of one weight.
constexpr unsigned long long kLongNs = 20ull * 1000ull * 1000ull * 1000ull;

typedef __nv_bfloat16 bf16;
template <typename T>
constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;
template <typename T>
constexpr int kAccs = sizeof(T) == 4 ? 4 : 2;   // accumulators: fp32 takes one for each piece, so that four of the next tile's are multiplied while results go out

struct Params {
  int k, n;                  // kGrad: m in the place of k
  Runs runs, ext;
  const float *alpha, *bias;
  int bias_each, act;
  const void *residual;
  void *y;
  int y_terms, vec;          // vec: rows of y begin on 16 bytes
  int nt, acc;               // columns of an instruction; of an accumulator
  int tiles_m, tiles_n;      // kGrad: both of a weight; else tiles_n
  int pieces, pieces_per, split;
  long long most;            // items: one to a cluster
  int stages, q_bytes, tmem_cols;
  int maps;                  // bits of the tensor maps that there are
  int rank, rank_pieces;     // adapters: pieces of 64 of the rank
  int t_bytes, e_bytes, e_wide;      // kTile: bytes of a stage's rows of t and e; numbers of the rank in a row (e across: rows)
  const bf16 *t;             // what rows keep
  const void *e;             // kFew: the adapters' matrices; fp32: as the caller has them
  int e_pitch;
  int slots, slot_rows, row_bytes;       // kFew: of adapters' parts of the tile's columns in shared memory, slot_rows rows' to a slot
  int early;                 // all but t was there before the launch in front of this one began, and that one writes nothing that this one does
  int off_out, off_t;        // staged results; kFew: t's numbers in shared memory
  // kGrad
  float *sums;
  int q_terms, out_across;   // out_across: out is [n][m]
  const void *raw_p, *raw_q; // fp32: the operands themselves
};

__device__ __forceinline__ uint64_t desc_along(uint32_t a) {     // rows of 64 along the sum, 1024 bytes between groups of 8 rows
  return ((uint64_t)(64u | (1u << 14) | (2u << 29)) << 32) | (uint64_t)((a >> 4) & 0x3FFFu) | (1u << 16);
}
__device__ __forceinline__ uint64_t desc_across(uint32_t a) {    // rows of 64 across it: 1024 bytes between groups of 8 rows, kBox between blocks of 64 columns
  return ((uint64_t)(64u | (1u << 14) | (2u << 29)) << 32) | (uint64_t)((a >> 4) & 0x3FFFu) | ((uint64_t)(kBox >> 4) << 16);
}
// the same for rows of 16, 32 or 64 along the sum (swizzled over as many bytes), and for blocks of `rows` rows across it
__device__ __forceinline__ uint64_t desc_narrow(uint32_t a, uint32_t row_bytes) {
  const uint32_t swizzle = row_bytes == 128u ? 2u : row_bytes == 64u ? 4u : 6u;
  return ((uint64_t)(row_bytes / 2u | (1u << 14) | (swizzle << 29)) << 32) | (uint64_t)((a >> 4) & 0x3FFFu) | (1u << 16);
}
__device__ __forceinline__ uint64_t desc_short(uint32_t a, uint32_t rows) {
  return ((uint64_t)(64u | (1u << 14) | (2u << 29)) << 32) | (uint64_t)((a >> 4) & 0x3FFFu) | ((uint64_t)(rows * 8u) << 16);
}
template <bool ACROSS>
__device__ __forceinline__ uint64_t desc_of(uint32_t a) { return ACROSS ? desc_across(a) : desc_along(a); }
template <bool ACROSS>
constexpr uint32_t kStepOf = ACROSS ? 16 * 128 / 16 : 32 / 16;   // 16 terms further on, in units of 16 bytes

template <bool P>
__device__ __forceinline__ void umma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if (P)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
  else
    umma_bf16(d, a, b, idesc, accumulate);
}
// D += A B with the lanes of `off` left as they are
template <bool P>
__device__ __forceinline__ void umma_lanes(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, const uint32_t (&off)[8]) {
  if (P)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, {%5, %6, %7, %8, %9, %10, %11, %12}, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(off[0]), "r"(off[1]), "r"(off[2]), "r"(off[3]), "r"(off[4]), "r"(off[5]), "r"(off[6]), "r"(off[7])
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, {%5, %6, %7, %8}, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(off[0]), "r"(off[1]), "r"(off[2]), "r"(off[3])
        : "memory");
}
// arrives at the barrier (of both CTAs of a pair) once all that this thread has issued is done
template <bool P>
__device__ __forceinline__ void commit(uint64_t *bar) {
  if (P)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)), "h"((uint16_t)3)
                 : "memory");
  else
    umma_commit(bar);
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// The same for what orders no memory: as a release it would wait for this thread's stores, 1500 cycles where results are on their way.  Of an accumulator that is given back
// nothing but what was read passes, and that is in registers: tcgen05.wait::ld stands before it, and the fence for the other thread's instructions.
__device__ __forceinline__ void arrive_cluster_relaxed(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// a phase that has been seen to end: what the cluster's threads wrote before they arrived is visible behind this
__device__ __forceinline__ void mbar_acquire_cluster(uint64_t *bar, uint32_t parity) {
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%0], %1;\n\t}" ::"r"(smem_u32(bar)), "r"(parity) : "memory");
}
// columns from c0 on of term `term`, rows from `row` on, of matrix `outer`; a pair's loads report to its first CTA (cluster address `bar`)
template <bool P>
__device__ __forceinline__ void load_box(uint32_t to, const CUtensorMap *map, uint32_t bar, int c0, int term, int row, int outer) {
  if (P)
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(to), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(term), "r"(row), "r"(outer) : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(to), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(term), "r"(row), "r"(outer) : "memory");
}
__device__ __forceinline__ void sts_f(uint32_t a, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(a), "f"(v) : "memory"); }

// The tile of an item: tiles of a run are walked column by column in bands of kSuper rows of tiles.
struct Tile {
  int row0, end, weight, tn;
};
__device__ __forceinline__ bool find_tile(const Params &p, int tile, grp::Walk &walk, long long item, Tile *t) {
  Run run;
  long long inside;
  if (!walk.find(p.runs, tile, p.tiles_n, item, &run, &inside)) return false;
  const int tiles_m = (run.end - run.begin + tile - 1) / tile;
  const int band = (int)(inside / ((long long)kSuper * p.tiles_n)), rem = (int)(inside - (long long)band * kSuper * p.tiles_n);
  const int deep = min(kSuper, tiles_m - band * kSuper);
  t->tn = rem / deep;
  t->row0 = run.begin + (band * kSuper + rem - t->tn * deep) * tile;
  t->end = run.end;
  t->weight = run.weight;
  return true;
}

// the adapter of a row, -1: none.  One thread.
__device__ __forceinline__ int adapter_of(const Runs &r, int row) {
  for (int s = grp::first_run_behind(r, row); s < r.count; ++s) {        // empty runs in between
    const Run run = grp::run_at(r, s);
    if (run.begin > row) break;
    if (run.end > row) return run.weight;
  }
  return -1;
}

// Calls f(begin, end) for the runs of a weight that have rows, all lanes together; of mapped runs 32 are looked at at a time.
template <typename F>
__device__ __forceinline__ void each_run_of(const Runs &r, int weight, F f) {
  if (!r.mapped) {
    const Run run = grp::run_at(r, weight);
    if (run.end > run.begin) f(run.begin, run.end);
    return;
  }
  const int lane = (int)(threadIdx.x & 31u);
  for (int base = 0; base < r.count; base += 32) {
    Run o = {0, 0, -1};
    if (base + lane < r.count) o = grp::run_at(r, base + lane);
    unsigned here = __ballot_sync(0xffffffffu, o.weight == weight && o.end > o.begin);
    while (here) {
      const int at = __ffs(here) - 1;
      here &= here - 1;
      f(__shfl_sync(0xffffffffu, o.begin, at), __shfl_sync(0xffffffffu, o.end, at));
    }
  }
}
// Calls f(first row, rows, mask) for this CTA's pieces of a weight's runs, all lanes together: 64 rows from the first one on, of which those in the mask are the
// weight's, the last of them row `rows` - 1.  What a run leaves of 64 rows shares a piece with the runs that begin inside it (single rows of many requests
// are 64 to a piece then, not one).  Pieces go round the CTAs of a cluster that share a sum.
__device__ __forceinline__ uint64_t row_bits(int lo, int hi) { return (hi - lo >= 64 ? ~0ull : (1ull << (hi - lo)) - 1ull) << lo; }
template <typename F>
__device__ __forceinline__ void each_piece(const Params &p, int weight, int share, F f) {
  int turn = 0, first = 0;
  bool open = false;
  uint64_t mask = 0;
  auto close = [&]() {
    if (turn == share) f(first, 64 - __clzll((long long)mask), mask);
    if (++turn == p.split) turn = 0;
    open = false;
  };
  each_run_of(p.runs, weight, [&](int begin, int end) {
    if (open) {
      if (begin < first + kPiece) {
        const int lo = max(begin - first, 0), hi = min(end - first, kPiece);
        if (hi > lo) mask |= row_bits(lo, hi);
        if (end < first + kPiece) return;
        begin = first + kPiece;
      }
      close();
    }
    const int whole = (end - begin) / kPiece;
    int k = share - turn;
    if (k < 0) k += p.split;
    for (; k < whole; k += p.split) f(begin + k * kPiece, kPiece, ~0ull);
    turn = (turn + whole) % p.split;
    first = begin + whole * kPiece;
    if (first < end) {
      open = true;
      mask = row_bits(0, end - first);
    }
  });
  if (open) close();
  __syncwarp();
}
// whether rows that the instructions of a piece take have to be set to zero
__device__ __forceinline__ bool has_holes(int rows, uint64_t mask) { return mask != row_bits(0, (rows + 15) / 16 * 16); }
__device__ __forceinline__ int count_pieces(const Params &p, int weight, int share) {
  int all = 0;
  each_piece(p, weight, share, [&](int, int, uint64_t) { ++all; });
  return all;
}

__device__ __forceinline__ void unpack8(uint4 w, float *v) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}
__device__ __forceinline__ uint4 pack8(const float *v) {
  return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
// What a row keeps, as terms of bf16 that add up: two, or of fp32 rows three.
// Two: the first is cut off, not rounded, and one step less where nothing is left, so that both have the number's sign and neither is 0 (numbers below 2^-118
// aside): an infinity times the number is then the infinity of both products.  (Rounded, with a low term of 0 or of the other sign, their sum was a NaN.)  What is left is
// below 2^-7 of the number and rounded to 2^-9 of itself: 16 bits.  Of an infinity or a NaN both are itself.
// Three: rounded, 24 bits.  Of an infinity or a NaN the first is itself, the others 0; of a number that would round to an infinity the first is the largest bf16.
template <typename T>
__device__ __forceinline__ void terms_of(float v, float (&t)[3]) {
  if (sizeof(T) == 2) {
    uint32_t u = __float_as_uint(v) & 0xffff0000u;
    if (u == __float_as_uint(v) && v != 0.f) u -= 0x10000u;
    const bool finite = v - v == 0.f;
    t[0] = finite ? __uint_as_float(u) : v;
    t[1] = finite ? v - t[0] : v;                // stored rounded
    t[2] = 0.f;
    return;
  }
  constexpr float kLargest = 3.38953138925153547e38f;
  t[0] = __bfloat162float(__float2bfloat16(v));
  if (fabsf(v) > kLargest && fabsf(v) <= 3.402823466e38f) t[0] = copysignf(kLargest, v);
  float left = v - t[0];
  left = left - left == 0.f ? left : 0.f;
  t[1] = __bfloat162float(__float2bfloat16(left));
  t[2] = left - t[1];
}
template <typename T>
__device__ __forceinline__ float kept(const bf16 *t, int row, int pad, int j) {
  constexpr int N = sizeof(T) == 4 ? 3 : 2;
  const bf16 *at = t + (size_t)row * (size_t)(N * pad) + (size_t)j;
  float v = __bfloat162float(at[0]), low = __bfloat162float(at[pad]);
  if (N == 3) low += __bfloat162float(at[2 * pad]);
  return v + low;
}
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16 v) { return __bfloat162float(v); }

__device__ __forceinline__ bool any_nan(const float (&v)[32]) {
  bool nan = false;
#pragma unroll
  for (int i = 0; i < 32; ++i) nan |= !(v[i] == v[i]);
  return nan;
}
// Results that came out as NaN, by FMAs: a warp together, 32 rows, one to a lane, x 8 columns at a time, results of a lane as it put them to its 128 bytes of shared
// memory (in registers they, and more columns at a time, would cost what the usual way needs).  A term's 8 numbers that all lanes multiply by are asked for by 8 lanes, 4
// terms to a load.  It ends as soon as all that is wanted is a NaN.  65536 rows with an infinity, gradients of 128 x 128: 55 ms (each element by its own lane 880 to
// 1120, which of two million rows is more than waits allow); 512 rows, 4096 -> 1024, one of them with an infinity: 2.2 ms (9.8).
constexpr int kAgain = 8;                        // columns, and terms, at once
struct Again {
  uint32_t wanted;
  float s[kAgain];
  __device__ __forceinline__ bool start(uint32_t at, bool valid, int count) {
    wanted = 0;
#pragma unroll
    for (int x = 0; x < kAgain; ++x) {
      const float v = lds_f(at + (uint32_t)(x * 4));
      if (valid && x < count && !(v == v)) wanted |= 1u << x;
      s[x] = 0.f;
    }
    return __any_sync(0xffffffffu, wanted != 0) != 0;
  }
  __device__ __forceinline__ bool open() const {
    bool is = false;
#pragma unroll
    for (int x = 0; x < kAgain; ++x) is |= (wanted >> x & 1u) && s[x] == s[x];
    return __any_sync(0xffffffffu, is) != 0;
  }
  // a: this lane's row, kAgain terms; b: terms lane / 8 and lane / 8 + 4 of column lane % 8
  __device__ __forceinline__ void add(const float (&a)[kAgain], const float (&b)[2]) {
#pragma unroll
    for (int u = 0; u < kAgain; ++u)
#pragma unroll
      for (int x = 0; x < kAgain; ++x) s[x] = fmaf(a[u], __shfl_sync(0xffffffffu, b[u >> 2], (u & 3) * 8 + x), s[x]);
  }
  __device__ __forceinline__ void end(uint32_t at) const {
#pragma unroll
    for (int x = 0; x < kAgain; ++x)
      if (wanted >> x & 1u) sts_f(at + (uint32_t)(x * 4), s[x]);
  }
};
template <bool ACROSS>
static __device__ __noinline__ void again(const Params &p, uint32_t at, int row, int end, int weight, int o0, int count) {
  const int lane = (int)(threadIdx.x & 31u);
  const bool valid = row < end;
  row = min(row, end - 1);
#pragma unroll 1
  for (; count > 0; count -= kAgain, o0 += kAgain, at += kAgain * 4) {
    Again f;
    if (!f.start(at, valid, count)) continue;
    if (p.pieces) {
      const size_t o = (size_t)min(o0 + (lane & 7), p.n - 1), step = ACROSS ? (size_t)p.n : 1;
      const float *x = reinterpret_cast<const float *>(p.raw_p) + (size_t)row * (size_t)p.k;
      const float *w = reinterpret_cast<const float *>(p.raw_q) + (size_t)weight * (size_t)p.n * (size_t)p.k + (ACROSS ? o : o * (size_t)p.k);
#pragma unroll 1
      for (int i0 = 0; i0 < p.k && f.open(); i0 += kAgain) {
        float a[kAgain], b[2];
#pragma unroll
        for (int u = 0; u < kAgain; ++u) a[u] = i0 + u < p.k ? x[i0 + u] : 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int i = i0 + u * 4 + (lane >> 3);
          b[u] = i < p.k ? w[(size_t)i * step] : 0.f;
        }
        f.add(a, b);
      }
    }
    if (p.alpha) {
      const float alpha = __ldg(p.alpha + weight);
#pragma unroll
      for (int x = 0; x < kAgain; ++x) f.s[x] *= alpha;
    }
    const int adapter = p.rank && f.wanted ? adapter_of(p.ext, row) : -1;
    if (adapter >= 0) {                          // each lane's own
      const float *e = reinterpret_cast<const float *>(p.e) + (size_t)adapter * (size_t)p.n * (size_t)p.rank + (ACROSS ? (size_t)o0 : (size_t)o0 * (size_t)p.rank);
      const size_t column = ACROSS ? 1 : (size_t)p.rank, step = ACROSS ? (size_t)p.n : 1;
#pragma unroll 1
      for (int j = 0; j < p.rank; ++j) {
        const float t = kept<float>(p.t, row, grp::rank_pad(p.rank), j);
#pragma unroll
        for (int x = 0; x < kAgain; ++x) f.s[x] = fmaf(t, e[(size_t)min(x, p.n - 1 - o0) * column + (size_t)j * step], f.s[x]);
      }
    }
    f.end(at);
  }
}
// The same of a gradient, from row i (a lane's own) and column j0 on; `sums`: its first column is the sum of p.
static __device__ __noinline__ void again_grad(const Params &p, uint32_t at, int weight, int i, int j0, bool sums, int count) {
  const int lane = (int)(threadIdx.x & 31u), pad = grp::rank_pad(p.n);
  const float *a_at = reinterpret_cast<const float *>(p.raw_p) + (size_t)min(i, p.k - 1);
#pragma unroll 1
  for (; count > 0; count -= kAgain, j0 += kAgain, at += kAgain * 4) {
    Again f;
    if (!f.start(at, i < p.k, count)) continue;
    const int j = min(j0 + (lane & 7), p.n - 1);
    const float *b_at = reinterpret_cast<const float *>(p.raw_q) + (size_t)j;
    each_run_of(p.runs, weight, [&](int begin, int end) {
#pragma unroll 1
      for (int r0 = begin; r0 < end && f.open(); r0 += kAgain) {
        float a[kAgain], b[2];
#pragma unroll
        for (int u = 0; u < kAgain; ++u) a[u] = r0 + u < end ? a_at[(size_t)(r0 + u) * (size_t)p.k] : 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int row = r0 + u * 4 + (lane >> 3);
          b[u] = row >= end ? 0.f : sums ? 1.f : p.q_terms ? kept<float>(p.t, row, pad, j) : b_at[(size_t)row * (size_t)p.n];
        }
        f.add(a, b);
      }
    });
    f.end(at);
  }
}
// 32 results of a lane to its 128 bytes, and back
__device__ __forceinline__ void put_lane(uint32_t at, const float (&v)[32]) {
  __syncwarp();                                  // others have read what was there
#pragma unroll
  for (int i = 0; i < 8; ++i)
    sts_u4(at + (uint32_t)(i * 16), make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])));
}
__device__ __forceinline__ void get_lane(uint32_t at, float (&v)[32]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint4 u = lds_u4(at + (uint32_t)(i * 16));
    v[4 * i] = __uint_as_float(u.x); v[4 * i + 1] = __uint_as_float(u.y); v[4 * i + 2] = __uint_as_float(u.z); v[4 * i + 3] = __uint_as_float(u.w);
  }
}

// What a lane delivers of a block of 32 rows x 32 columns: 4 columns of every fourth row.  bf16: its part of the residual, asked for ahead (fp32 has no registers
// to spare: what it asks for ahead is nothing).
template <typename T>
struct Ahead { uint2 v[sizeof(T) == 4 ? 1 : 8]; };
template <typename T>
__device__ __forceinline__ void ask_block(Ahead<T> &a, const T *residual, size_t pitch, int rows, int cols) {
  const int lane = (int)(threadIdx.x & 31u), piece = lane & 7, r0 = lane >> 3;
  const T *at = residual + (size_t)r0 * pitch + (size_t)(piece * 4);
#pragma unroll
  for (int i = 0; i < 8; ++i, at += 4 * pitch)
    if (sizeof(T) == 2) a.v[sizeof(T) == 2 ? i : 0] = i * 4 + r0 < rows && piece * 4 < cols ? *reinterpret_cast<const uint2 *>(at) : make_uint2(0, 0);
}
// 32 sums of each lane's row -> rows of y, `rows` x `cols` of them, through shared memory: a row's results then go out side by side
template <typename T>
__device__ __forceinline__ void store_block(const Params &p, uint32_t stage, const float (&v)[32], T *y, size_t pitch, int rows, int cols, const float *bias, const T *residual,
                                            const Ahead<T> &ahead) {
  const int lane = (int)(threadIdx.x & 31u);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i)
    sts_u4(stage + (uint32_t)(lane * 128 + ((i ^ (lane & 7)) * 16)),
           make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])));
  __syncwarp();
  if (p.vec) {
    const int piece = lane & 7, r0 = lane >> 3;
    if (piece * 4 >= cols) return;
    const float4 b = bias ? __ldg(reinterpret_cast<const float4 *>(bias) + piece) : make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int kAtOnce = sizeof(T) == 4 ? 4 : 8;
    T *at = y + (size_t)r0 * pitch + (size_t)(piece * 4);
    const T *res = residual + (size_t)r0 * pitch + (size_t)(piece * 4);
#pragma unroll
    for (int i0 = 0; i0 < 8; i0 += kAtOnce) {
      uint4 w[kAtOnce], r[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int row = (i0 + i) * 4 + r0;
        w[i] = lds_u4(stage + (uint32_t)(row * 128 + ((piece ^ (row & 7)) * 16)));
        if (sizeof(T) == 4 && residual) {
          r[i] = row < rows ? *reinterpret_cast<const uint4 *>(res) : make_uint4(0, 0, 0, 0);
          res += 4 * pitch;
        }
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i, at += 4 * pitch) {
        float f[4] = {__uint_as_float(w[i].x), __uint_as_float(w[i].y), __uint_as_float(w[i].z), __uint_as_float(w[i].w)};
        if (bias) { f[0] += b.x; f[1] += b.y; f[2] += b.z; f[3] += b.w; }
        if (residual) {
          if (sizeof(T) == 4) {
            f[0] += __uint_as_float(r[i].x); f[1] += __uint_as_float(r[i].y); f[2] += __uint_as_float(r[i].z); f[3] += __uint_as_float(r[i].w);
          } else {
            const uint2 u = ahead.v[sizeof(T) == 2 ? i : 0];
            f[0] += __uint_as_float(u.x << 16); f[1] += __uint_as_float(u.x & 0xffff0000u);
            f[2] += __uint_as_float(u.y << 16); f[3] += __uint_as_float(u.y & 0xffff0000u);
          }
        }
        if (p.act) {
#pragma unroll
          for (int x = 0; x < 4; ++x) f[x] = dc_act_apply(f[x], DC_ACT_RELU6);
        }
        if ((i0 + i) * 4 + r0 < rows) {
          if (sizeof(T) == 4) *reinterpret_cast<float4 *>(at) = make_float4(f[0], f[1], f[2], f[3]);
          else *reinterpret_cast<uint2 *>(at) = make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]));
        }
      }
    }
    return;
  }
  if (lane >= cols) return;
  const float b = bias ? __ldg(bias + lane) : 0.f;
#pragma unroll 1
  for (int i0 = 0; i0 < rows; i0 += 8) {         // eight rows at once, so that what one waits for the others do not add to
    float f[8], r[8];
    const size_t at = (size_t)i0 * pitch + (size_t)lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      f[i] = lds_f(stage + (uint32_t)((i0 + i) * 128 + (((lane >> 2) ^ i) * 16) + (lane & 3) * 4));
      r[i] = residual && i0 + i < rows ? to_float(residual[at + (size_t)i * pitch]) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = dc_act_apply(f[i] + b + r[i], p.act);
      if (i0 + i < rows) y[at + (size_t)i * pitch] = (T)v;
    }
  }
}

enum { kFull = 0, kEmpty = kMaxStages, kTail = 2 * kMaxStages, kReady = 3 * kMaxStages, kDFull = 4 * kMaxStages, kDEmpty = kDFull + kMaxAccs, kParts = kDEmpty + kMaxAccs, kEFull, kEEmpty = kEFull + kMaxSlots, kBars = kEEmpty + kMaxSlots };

// P: in pairs.  ACROSS: the matrices' sums run across their rows (of both operands of a gradient always).
template <int FORM, bool ACROSS, typename T, bool P>
__global__ void __launch_bounds__(kThreadsOf<FORM>, 1)
k_group_tc(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_t,
           const __grid_constant__ CUtensorMap map_e, const __grid_constant__ Params p, DcWsHeader *ws) {
  constexpr int N = kTerms<T>;
  constexpr bool kShort = N == 3;                // sums of a piece
  constexpr uint32_t kAcc = kAccs<T> - 1, kAccLog = kShort ? 2 : 1;
  constexpr unsigned long long kLimit = FORM == kGrad || kShort ? kLongNs : kWaitLimitNs;
  // products of terms, small ones first
  constexpr int kPairs = N == 3 ? 6 : 1;
  constexpr int kTermP[6] = {N == 3 ? 2 : 0, 0, 1, 1, 0, 0}, kTermQ[6] = {0, 2, 1, 0, 1, 0};
  constexpr int kRows = P ? 256 : 128;           // of a tile
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bar[kBars];
  __shared__ uint32_t tmem_s, abort_s;
  __shared__ int weight_s[kFewMost], list_s[kFewMost], listed_s;        // kFew: the rows' adapters, and which of this CTA's rows have one
  volatile uint32_t *abort_flag = &abort_s;
  const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sm = (smem_u32(smem_raw) + 1023u) & ~1023u;
  if (warp == 0) {
    for (int i = lane; i < kBars; i += 32) mbar_init(&bar[i], i >= kDEmpty && i < kDEmpty + kMaxAccs ? (P ? 2 : 1) * kEpi : i >= kReady && i < kReady + kMaxStages && P ? 2 : i == kParts ? p.split * kEpi : i >= kEEmpty ? kEpi / 2 : 1);
    if (lane == 0) abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  } else if (warp == 1 && lane < 4) {
    if (p.maps >> lane & 1) prefetch_tensormap(lane == 0 ? &map_p : lane == 1 ? &map_q : lane == 2 ? &map_t : &map_e);
  }
  if (FORM == kFew && p.split > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");   // this CTA is there, its barriers too: waited for before parts go out
  // The next launch may start once this one has waited for the one before it: an early launch, which does not wait at its start, then finds
  // all that was written before this one.  Tensor memory only behind that wait, since CTAs of the launch before may still have theirs to ask for; those of the one in
  // front of an early launch, one to an SM, have it, or need none.
  if (!p.early) asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (warp == 1) {
    if (P) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"((uint32_t)p.tmem_cols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      tmem_alloc(&tmem_s, (uint32_t)p.tmem_cols);
      tmem_relinquish();
    }
  }
  const uint32_t stage_bytes = (uint32_t)(N * (kP + p.q_bytes)), ones = sm + (uint32_t)p.stages * stage_bytes;
  if (FORM == kGrad && p.sums) {                 // a block of ones: sums are products with it
    for (int i = tid; i < kBox / 16; i += kThreadsOf<FORM>) sts_u4(ones + (uint32_t)(i * 16), make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u));
    fence_proxy_async();
  }
  tc_fence_before();
  __syncthreads();
  if (P) cluster_sync();                         // the barriers of both CTAs are there
  tc_fence_after();
  const uint32_t tmem = tmem_s;
  const int group = P ? 2 : p.split;             // CTAs to an item
  const int rank = group > 1 ? (int)blockIdx.x % group : 0;
  const int share = P ? 0 : rank, half = P ? rank : 0;             // of a split sum; of a pair's tile
  const int team = (int)blockIdx.x / group, teams = (int)gridDim.x / group;
  const int c0 = share * p.pieces_per, c1 = min(p.pieces, c0 + p.pieces_per), own_pieces = max(c1 - c0, 0);
  const int per_weight = p.tiles_m * p.tiles_n;  // kGrad; with sums a column of tiles more
  const int tile_rows = FORM == kFew ? p.nt : kRows;
  int met = 0;                                   // meetings of a cluster that shares a sum: two, whatever happens
  int stage = 0;
  uint32_t parity = 0, turn = 0;                 // of the ring; of the accumulators
  bool ok = true;
  auto next = [&]() { if (++stage == p.stages) { stage = 0; parity ^= 1u; } };
  // ring uses of an adapter's part: both terms of up to 32 numbers at once, else 64 numbers of one term at a time; fp32 all terms of 64
  const bool adapters = FORM == kTile && p.rank && share == 0;     // of a shared sum one CTA's
  const int ext_uses = N == 3 ? p.rank_pieces : p.rank <= 32 ? 1 : 2 * p.rank_pieces;

  if (warp == 0) {
    // ---------------------------------------------------------------- load
    const bool lead = elect_one();
    // waits for the next stage: its barrier's address for loads, or 0
    auto open = [&](uint32_t bytes, uint32_t site, bool tail = false) -> uint32_t {
      ok = mbar_wait(&bar[kEmpty + stage], parity ^ 1u, abort_flag, ws, site | (uint32_t)stage, kLimit);
      if (!ok) return 0u;
      if (FORM == kGrad && tail) {               // passed on by a warp of this CTA
        mbar_arrive_expect_tx(&bar[kTail + stage], bytes);
        return P ? map_cluster(smem_u32(&bar[kTail + stage]), (uint32_t)rank) : smem_u32(&bar[kTail + stage]);
      }
      if (!P || rank == 0) mbar_arrive_expect_tx(&bar[kFull + stage], (P ? 2u : 1u) * bytes);
      return P ? map_cluster(smem_u32(&bar[kFull + stage]), 0) : smem_u32(&bar[kFull + stage]);
    };
    if (FORM == kGrad) {
      for (long long item = team; ok && item < p.most; item += teams) {
        const int weight = (int)(item / per_weight), at = (int)(item - (long long)weight * per_weight), tm = at / p.tiles_n, tn = at - tm * p.tiles_n;
        const bool sums = p.sums && tn == p.tiles_n - 1;
        const int i0 = tm * kRows + half * 128, j0 = tn * p.nt + half * (p.nt / 2);
        each_piece(p, weight, share, [&](int r, int rows, uint64_t mask) {
          const uint32_t full = lead && ok ? open(sums ? (uint32_t)(N * kP) : stage_bytes, 0x10000u, has_holes(rows, mask)) : 0u;
          if (full) {
            uint32_t a = sm + (uint32_t)stage * stage_bytes;
            for (int t = 0; t < N; ++t)
              for (int b = 0; b < 2; ++b, a += kBox) load_box<P>(a, &map_p, full, i0 + b * 64, t, r, 0);
            if (!sums)
              for (int t = 0; t < N; ++t)
                for (int b = 0; b < p.q_bytes / kBox; ++b, a += kBox) load_box<P>(a, &map_q, full, j0 + b * 64, t, r, 0);
          }
          next();
        });
        ok = __all_sync(0xffffffffu, ok);
      }
    } else {
      grp::Walk walk;
      walk.start();
      Tile t;
      for (long long item = team; ok && item < p.most && find_tile(p, tile_rows, walk, item, &t); item += teams) {
        const int n0 = t.tn * (FORM == kFew ? 128 : p.nt) + half * (p.nt / 2), row0 = t.row0 + half * 128;
        auto load_w = [&](const CUtensorMap *map, uint32_t at, uint32_t full, int c, int term, int weight) {
          if (ACROSS) {
            for (int b = 0; b < (FORM == kFew ? 2 : p.q_bytes / kBox); ++b) load_box<P>(at + (uint32_t)(b * kBox), map, full, n0 + b * 64, term, c, weight);
          } else {
            load_box<P>(at, map, full, c, term, n0, weight);
          }
        };
        for (int c = c0; c < c1; ++c, next()) {
          if (!lead || !ok) continue;
          const uint32_t full = open(stage_bytes, 0x10000u);
          if (!full) continue;
          const uint32_t a = sm + (uint32_t)stage * stage_bytes, b = a + (uint32_t)(N * kP);
          for (int term = 0; term < N; ++term) {
            if (FORM == kFew) {
              load_box<P>(b + (uint32_t)(term * p.q_bytes), &map_p, full, c * kPiece, term, row0, 0);
              load_w(&map_q, a + (uint32_t)(term * kP), full, c * kPiece, term, t.weight);
            } else {
              load_box<P>(a + (uint32_t)(term * kP), &map_p, full, c * kPiece, term, row0, 0);
              load_w(&map_q, b + (uint32_t)(term * p.q_bytes), full, c * kPiece, term, t.weight);
            }
          }
        }
        __syncwarp();
        if (adapters && p.early && item == team) asm volatile("griddepcontrol.wait;" ::: "memory");
        int run_weight = 0;
        if (adapters)
          grp::each_run(p.ext, t.row0, min(t.end, t.row0 + kRows), [&](const Run &run) { run_weight = run.weight; }, [&](int from) {
            const int weight = __shfl_sync(0xffffffffu, run_weight, from);
            for (int c = 0; c < ext_uses; ++c, next()) {
              if (!lead || !ok) continue;
              const uint32_t full = open((uint32_t)(N * (p.t_bytes + p.e_bytes)), 0x20000u);
              if (!full) continue;
              const int cc = c < p.rank_pieces ? c : c - p.rank_pieces;
              const uint32_t a = sm + (uint32_t)stage * stage_bytes, b = a + (uint32_t)(N * kP);
              for (int term = 0; term < N; ++term) {
                load_box<P>(a + (uint32_t)(term * kP), &map_t, full, (c < p.rank_pieces ? 0 : grp::rank_pad(p.rank)) + cc * kPiece, term, row0, 0);
                const uint32_t to = b + (uint32_t)(term * p.q_bytes);
                if (ACROSS) {
                  for (int x = 0; x < p.q_bytes / kBox; ++x) load_box<P>(to + (uint32_t)(x * p.e_wide * 128), &map_e, full, n0 + x * 64, term, cc * kPiece, weight);
                } else {
                  load_box<P>(to, &map_e, full, cc * kPiece, term, n0, weight);
                }
              }
            }
          });
        ok = __all_sync(0xffffffffu, ok);
      }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- multiply: one lane issues, without the others (of a pair, the first CTA's)
    const bool lead = elect_one() && (!P || rank == 0);
    uint32_t fulls = 0, tails = 0;               // kGrad: phases of each stage's barriers, of whole pieces and of those at a run's end
    const uint32_t base = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kRows >> 4) << 24) | ((uint32_t)(p.nt >> 3) << 17);
    uint32_t d = 0;
    auto begin = [&]() {                         // the next accumulator
      ok = ok && mbar_wait(&bar[kDEmpty + (turn & kAcc)], (turn >> kAccLog & 1u) ^ 1u, abort_flag, ws, 0x30000u | (turn & kAcc), kLimit);
      tc_fence_after();
      d = tmem + (turn & kAcc) * (uint32_t)p.acc;
    };
    auto end = [&](bool any) {
      if (any) {
        commit<P>(&bar[kDFull + (turn & kAcc)]);
      } else {
        mbar_arrive(&bar[kDFull + (turn & kAcc)]);
        if (P) arrive_cluster(map_cluster(smem_u32(&bar[kDFull + (turn & kAcc)]), 1));
      }
      ++turn;
    };
    if (FORM == kGrad) {
      for (long long item = team; ok && item < p.most; item += teams) {
        const int weight = (int)(item / per_weight), at = (int)(item - (long long)weight * per_weight), tm = at / p.tiles_n;
        const bool sums = p.sums && at - tm * p.tiles_n == p.tiles_n - 1;
        bool any = false;
        if (lead) begin();
        const uint32_t idesc = (sums ? (base & ~(0x3Fu << 17)) | (uint32_t)(kRows / 64) << 17 : base) | (1u << 15) | (1u << 16);
        each_piece(p, weight, share, [&](int, int rows, uint64_t mask) {
          if (!lead || !ok) {
            next();
            return;
          }
          if (kShort && any) {
            end(true);
            begin();
            any = false;
          }
          if (has_holes(rows, mask)) {           // rows of other weights: set to zero before the piece is passed on
            const uint32_t phase = tails >> stage & 1u;
            ok = ok && mbar_wait(&bar[kReady + stage], phase, abort_flag, ws, 0x50000u | (uint32_t)stage, kLimit);
            if (P && ok) mbar_acquire_cluster(&bar[kReady + stage], phase);
            tails ^= 1u << stage;
          } else {
            ok = ok && mbar_wait(&bar[kFull + stage], fulls >> stage & 1u, abort_flag, ws, 0x40000u | (uint32_t)stage, kLimit);
            fulls ^= 1u << stage;
          }
          if (!ok) return;
          tc_fence_after();
          const uint32_t a = sm + (uint32_t)stage * stage_bytes, b = a + (uint32_t)(N * kP);
          const int steps = (rows + 15) / 16;
#pragma unroll
          for (int x = 0; x < kPairs; ++x) {
            if (sums && kTermQ[x] != 0) continue;                  // of the block of ones there is one term
            const uint64_t ad = desc_across(a + (uint32_t)(kTermP[x] * kP)), bd = desc_across(sums ? ones : b + (uint32_t)(kTermQ[x] * p.q_bytes));
            if (steps == 4) {
#pragma unroll
              for (int k = 0; k < 4; ++k) umma<P>(d, ad + kStepOf<true> * k, bd + kStepOf<true> * k, idesc, any || k > 0 ? 1u : 0u);
            } else {
              for (int k = 0; k < steps; ++k) umma<P>(d, ad + kStepOf<true> * k, bd + kStepOf<true> * k, idesc, any || k > 0 ? 1u : 0u);
            }
            any = true;
          }
          commit<P>(&bar[kEmpty + stage]);
          next();
        });
        if (lead && ok) end(any);
        ok = __all_sync(0xffffffffu, ok);
      }
    } else {
      grp::Walk walk;
      walk.start();
      Tile t;
      const uint32_t idesc = base | (!ACROSS ? 0u : FORM == kFew ? 1u << 15 : 1u << 16);
      constexpr bool kA = FORM == kFew && ACROSS, kB = FORM != kFew && ACROSS;     // operands that the sum runs across
      for (long long item = team; ok && item < p.most && find_tile(p, tile_rows, walk, item, &t); item += teams) {
        bool any = false;
        if (lead) {
          begin();
          uint32_t ready = 0;
          for (int c = c0; ok && c < c1; ++c) {
            if (kShort && any) {
              end(true);
              begin();
              any = false;
            }
            if (ok && !ready) ok = mbar_wait(&bar[kFull + stage], parity, abort_flag, ws, 0x40000u | (uint32_t)stage, kLimit);
            if (!ok) break;
            ready = stage + 1 < p.stages ? mbar_test(&bar[kFull + stage + 1], parity) : mbar_test(&bar[kFull], parity ^ 1u);
            tc_fence_after();
            const uint32_t a = sm + (uint32_t)stage * stage_bytes, b = a + (uint32_t)(N * kP);
            const int steps = min(4, (p.k - c * kPiece + 15) / 16);
#pragma unroll
            for (int x = 0; x < kPairs; ++x) {
              // the matrix is the first operand of kFew
              const int tp = FORM == kFew ? kTermQ[x] : kTermP[x], tq = FORM == kFew ? kTermP[x] : kTermQ[x];
              const uint64_t ad = desc_of<kA>(a + (uint32_t)(tp * kP)), bd = desc_of<kB>(b + (uint32_t)(tq * p.q_bytes));
              if (steps == 4) {
#pragma unroll
                for (int k = 0; k < 4; ++k) umma<P>(d, ad + kStepOf<kA> * k, bd + kStepOf<kB> * k, idesc, any || k > 0 ? 1u : 0u);
              } else {
                for (int k = 0; k < steps; ++k) umma<P>(d, ad + kStepOf<kA> * k, bd + kStepOf<kB> * k, idesc, any || k > 0 ? 1u : 0u);
              }
              any = true;
            }
            commit<P>(&bar[kEmpty + stage]);
            next();
          }
        } else {
          for (int c = c0; c < c1; ++c) next();
        }
        __syncwarp();
        uint32_t run_off[8];
        if (adapters)
          grp::each_run(p.ext, t.row0, min(t.end, t.row0 + kRows), [&](const Run &run) {
#pragma unroll
            for (int i = 0; i < 2 * kRows / 64; ++i) {
              const int lo = max(run.begin - t.row0 - 32 * i, 0), hi = min(run.end - t.row0 - 32 * i, 32);
              run_off[i] = lo >= hi ? 0xffffffffu : ~((hi - lo == 32 ? 0xffffffffu : (1u << (hi - lo)) - 1u) << lo);
            }
          }, [&](int from) {
            uint32_t off[8];                     // lanes of other rows
#pragma unroll
            for (int i = 0; i < 8; ++i) off[i] = i < 2 * kRows / 64 ? __shfl_sync(0xffffffffu, run_off[i], from) : 0u;
            bool first = own_pieces == 0;        // without a shared matrix the run's first instruction sets its lanes
            for (int c = 0; c < ext_uses; ++c, next()) {
              if (!lead || !ok) continue;
              ok = mbar_wait(&bar[kFull + stage], parity, abort_flag, ws, 0x60000u | (uint32_t)stage, kLimit);
              if (!ok) continue;
              tc_fence_after();
              const uint32_t a = sm + (uint32_t)stage * stage_bytes, b = a + (uint32_t)(N * kP);
              const int steps = min(4, (p.rank - (c < p.rank_pieces ? c : c - p.rank_pieces) * kPiece + 15) / 16);
              const uint32_t t_row = (uint32_t)p.t_bytes / 128u;
              auto e_desc = [&](uint32_t at) { return ACROSS ? desc_short(at, (uint32_t)p.e_wide) : desc_narrow(at, (uint32_t)p.e_wide * 2u); };
              if (N == 3) {
#pragma unroll
                for (int x = 0; x < kPairs; ++x)
                  for (int k = 0; k < steps; ++k, first = false)
                    umma_lanes<P>(d, desc_narrow(a + (uint32_t)(kTermP[x] * kP), t_row) + kStepOf<false> * k, e_desc(b + (uint32_t)(kTermQ[x] * p.q_bytes)) + kStepOf<kB> * k, idesc, first ? 0u : 1u, off);
              } else {
                const uint64_t ad = desc_narrow(a, t_row), bd = e_desc(b);
                for (int k = 0; k < steps; ++k, first = false) umma_lanes<P>(d, ad + kStepOf<false> * k, bd + kStepOf<kB> * k, idesc, first ? 0u : 1u, off);
                if (p.rank <= 32)                // the low terms lie behind the high ones
                  for (int k = 0; k < steps; ++k) umma_lanes<P>(d, ad + kStepOf<false> * (steps + k), bd + kStepOf<kB> * k, idesc, 1u, off);
              }
              any = true;
              commit<P>(&bar[kEmpty + stage]);
            }
          });
        if (lead && ok) end(any);
        ok = __all_sync(0xffffffffu, ok);
      }
    }
  } else if (warp < 2 + kEpi) {
    // ---------------------------------------------------------------- read out
    const int quad = warp & 3, set = (warp - 2) >> 2, own = quad * 32 + lane, unit = (warp - 2) * 32 + lane;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16, staged = sm + (uint32_t)(p.off_out + (warp - 2) * 32 * 128);
    const uint32_t freed = P ? map_cluster(smem_u32(&bar[kDEmpty]), 0) : 0u;
    auto wait_sums = [&]() {
      const bool there = warp_wait(&bar[kDFull + (turn & kAcc)], turn >> kAccLog & 1u, abort_flag, ws, 0x70000u | (turn & kAcc), kLimit);
      tc_fence_after();
      return there;
    };
    auto sums_at = [&]() { return tmem + (turn & kAcc) * (uint32_t)p.acc + lanes; };
    auto release = [&]() {                       // the accumulator is read
      tc_fence_before();
      __syncwarp();
      if (elect_one()) {
        if (P) arrive_cluster_relaxed(freed + (turn & kAcc) * 8u);
        else mbar_arrive(&bar[kDEmpty + (turn & kAcc)]);
      }
      __syncwarp();
    };
    constexpr int kBlocks = kShort ? 2 : 4;      // of 32 columns, of a set
    // parts of a tile's sum in shared memory, [columns][128]; the ring is not in use any more
    auto part_at = [&](uint32_t from, int c) { return from + (uint32_t)((c * 128 + own) * 4); };
    float all[kShort ? kBlocks : 1][32];         // fp32: pieces' sums added up
    // Reads a tile's sums block by block: got(block's first column, sums).  `pieces` of them where they are short; `zero`: nothing was multiplied.
    // `low`: columns from there on hold a second part of each sum.
    auto read_out = [&](int pieces, bool zero, int cols, int low, auto got) -> bool {
      if (kShort) {
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int x = 0; x < 32; ++x) all[b < (kShort ? kBlocks : 1) ? b : 0][x] = 0.f;
        for (int i = 0; i < pieces; ++i) {
          if (!wait_sums()) return false;
          const uint32_t d = sums_at();
#pragma unroll
          for (int b = 0; b < kBlocks; ++b) {
            const int c = set * 32 + b * 64;
            if (c >= cols) break;
            float v[32];
            tmem_ld32(d + (uint32_t)c, reinterpret_cast<uint32_t *>(v));
            tmem_ld_wait();
#pragma unroll
            for (int x = 0; x < 32; ++x) all[b < (kShort ? kBlocks : 1) ? b : 0][x] += zero ? 0.f : v[x];
          }
          release();
          ++turn;
        }
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
          const int c = set * 32 + b * 64;
          if (c >= cols) break;
          __syncwarp();
          got(c, all[b < (kShort ? kBlocks : 1) ? b : 0]);
        }
        return true;
      }
      if (!wait_sums()) return false;
      const uint32_t d = sums_at();
      bool held = true;
#pragma unroll 1
      for (int c = set * 32; c < cols; c += 64) {
        float v[32];
        __syncwarp();
        tmem_ld32(d + (uint32_t)c, reinterpret_cast<uint32_t *>(v));
        if (low) {
          float w[32];
          tmem_ld32(d + (uint32_t)(low + c), reinterpret_cast<uint32_t *>(w));
          tmem_ld_wait();
#pragma unroll
          for (int x = 0; x < 32; ++x) v[x] += w[x];
        } else {
          tmem_ld_wait();
        }
        if (c + 64 >= cols) { release(); held = false; }
        if (zero) {
#pragma unroll
          for (int x = 0; x < 32; ++x) v[x] = 0.f;
        }
        got(c, v);
      }
      if (held) release();
      ++turn;
      return true;
    };
    // the cluster's parts of block c: added up in the order of their CTAs
    auto add_parts = [&](int c, int low, float (&v)[32]) {
#pragma unroll
      for (int x = 0; x < 32; ++x) v[x] = 0.f;
      for (int k = 0; k < p.split; ++k) {
        const uint32_t from = map_cluster(sm, (uint32_t)k);
#pragma unroll
        for (int x = 0; x < 32; ++x) v[x] += lds_cluster_f(part_at(from, c + x));
        if (low) {
#pragma unroll
          for (int x = 0; x < 32; ++x) v[x] += lds_cluster_f(part_at(from, low + c + x));
        }
      }
    };
    auto put_part = [&](int c, const float (&v)[32]) {
#pragma unroll
      for (int x = 0; x < 32; ++x) sts_f(part_at(sm, c + x), v[x]);
    };
    if (FORM == kGrad) {
      for (long long item = team; item < p.most; item += teams) {
        const int weight = (int)(item / per_weight), at = (int)(item - (long long)weight * per_weight), tm = at / p.tiles_n, tn = at - tm * p.tiles_n;
        const bool sums = p.sums && tn == p.tiles_n - 1;
        const int mine = count_pieces(p, weight, share);
        const int i0 = tm * kRows + half * 128 + quad * 32, i = i0 + lane, low = p.q_terms && !kShort && !sums ? p.nt / 2 : 0;
        const int cols = sums ? 16 : low ? low : p.nt;
        T *out = reinterpret_cast<T *>(p.y) + (size_t)weight * (size_t)p.k * (size_t)p.n;
        auto deliver = [&](int c, float (&v)[32]) {                 // columns c on of this thread's row
          const int j0 = tn * p.nt + c;
          if (kShort && __any_sync(0xffffffffu, any_nan(v))) {
            const uint32_t at = staged + (uint32_t)(lane * 128);
            put_lane(at, v);
            again_grad(p, at, weight, i, j0, sums, sums ? (c == 0 ? 1 : 0) : min(min(32, cols - c), p.n - j0));
            get_lane(at, v);
          }
          if (sums) {
            if (c == 0 && i < p.k) p.sums[(size_t)weight * (size_t)p.k + (size_t)i] = v[0];
          } else if (p.out_across) {
            if (i < p.k) {
#pragma unroll
              for (int x = 0; x < 32; ++x)
                if (j0 + x < p.n && c + x < cols) out[(size_t)(j0 + x) * (size_t)p.k + (size_t)i] = (T)v[x];
            }
          } else if (i0 < p.k) {
            store_block<T>(p, staged, v, out + (size_t)i0 * (size_t)p.n + (size_t)j0, (size_t)p.n, min(32, p.k - i0), min(min(32, cols - c), p.n - j0), nullptr, (const T *)nullptr, Ahead<T>());
          }
        };
        if (P || p.split == 1) {
          ok = read_out(max(mine, 1), mine == 0, cols, low, deliver);
          if (!ok) break;
        } else {
          ok = read_out(max(mine, 1), mine == 0, sums ? 16 : p.nt, 0, put_part);
          __syncwarp();
          cluster_sync();
          ++met;
          if (!ok) break;
          for (int c = (rank + set * p.split) * 32; c < cols; c += 64 * p.split) {
            float v[32];
            add_parts(c, low, v);
            deliver(c, v);
          }
        }
      }
    } else if (FORM == kTile) {
      grp::Walk walk;
      walk.start();
      Tile t;
      for (long long item = team; item < p.most && find_tile(p, tile_rows, walk, item, &t); item += teams) {
        const int row0 = t.row0 + half * 128 + quad * 32, row = row0 + lane;
        const float alpha = p.alpha ? __ldg(p.alpha + t.weight) : 1.f;
        bool filled = p.pieces > 0;              // without a shared matrix: whether an adapter has set this lane
        if (p.rank && p.pieces == 0) filled = row < t.end && adapter_of(p.ext, row) >= 0;
        const float *bias = p.bias ? p.bias + (p.bias_each ? (size_t)t.weight * (size_t)p.n : 0) : nullptr;
        Ahead<T> next_residual;
        const bool residual = p.residual && p.vec;
        auto ask = [&](int c) {
          const int o0 = t.tn * p.nt + c;
          if (sizeof(T) == 2 && residual && row0 < t.end && c < p.nt && o0 < p.n)
            ask_block<T>(next_residual, reinterpret_cast<const T *>(p.residual) + (size_t)row0 * (size_t)p.n + (size_t)o0, (size_t)p.n, min(32, t.end - row0), min(min(32, p.nt - c), p.n - o0));
        };
        const int c_first = p.split > 1 ? (rank + set * p.split) * 32 : set * 32, c_step = 64 * p.split;
        if (residual && row < t.end)             // to L2, while the tile is multiplied
          for (int c = set * 64; c < p.nt; c += 128)
            if (t.tn * p.nt + c < p.n) asm volatile("prefetch.global.L2 [%0];" ::"l"(reinterpret_cast<const T *>(p.residual) + (size_t)row * (size_t)p.n + (size_t)(t.tn * p.nt + c)));
        ask(c_first);
        auto deliver = [&](int c, float (&v)[32]) {
          const int o0 = t.tn * p.nt + c;
          const Ahead<T> now = next_residual;
          ask(c + c_step);
          if (row0 >= t.end) return;
          if (p.alpha || p.pieces == 0) {
#pragma unroll
            for (int x = 0; x < 32; ++x) v[x] = filled ? v[x] * alpha : 0.f;
          }
          if (kShort && __any_sync(0xffffffffu, any_nan(v))) {
            const uint32_t at = staged + (uint32_t)(lane * 128);
            put_lane(at, v);
            again<ACROSS>(p, at, row, t.end, t.weight, o0, min(min(32, p.nt - c), p.n - o0));
            get_lane(at, v);
          }
          if (p.y_terms) {
            constexpr int kKept = N == 3 ? 3 : 2;
            const int pad = grp::rank_pad(p.n);
            bf16 *to = reinterpret_cast<bf16 *>(p.y) + (size_t)row * (size_t)(kKept * pad) + (size_t)o0;
            if (row < t.end) {
#pragma unroll
              for (int x = 0; x < 32; x += 8) {
                if (o0 + x >= pad) break;
                float term[3][8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                  float f[3];
                  terms_of<T>(o0 + x + i < p.n ? v[x + i] : 0.f, f);         // what the padding holds: zeros
#pragma unroll
                  for (int k = 0; k < 3; ++k) term[k][i] = f[k];
                }
#pragma unroll
                for (int k = 0; k < kKept; ++k) *reinterpret_cast<uint4 *>(to + k * pad + x) = pack8(term[k]);
              }
            }
            return;
          }
          const size_t at = (size_t)row0 * (size_t)p.n + (size_t)o0;
          store_block<T>(p, staged, v, reinterpret_cast<T *>(p.y) + at, (size_t)p.n, min(32, t.end - row0), min(min(32, p.nt - c), p.n - o0), bias ? bias + o0 : nullptr,
                         p.residual ? reinterpret_cast<const T *>(p.residual) + at : nullptr, now);
        };
        if (P || p.split == 1) {
          ok = read_out(max(own_pieces, 1), false, p.nt, 0, deliver);
          if (!ok) break;
        } else {
          ok = read_out(max(own_pieces, 1), false, p.nt, 0, put_part);
          __syncwarp();
          cluster_sync();
          ++met;
          if (!ok) break;
          for (int c = c_first; c < p.nt; c += c_step) {
            float v[32];
            add_parts(c, 0, v);
            deliver(c, v);
          }
        }
      }
    } else {
      bool waited = !p.early;                    // for the launch in front of this one
      grp::Walk walk;
      walk.start();
      Tile t;
      const int half_rows = p.nt / 2;            // of a set of four warps
      const int pad = grp::rank_pad(p.rank);
      const uint32_t ts = sm + (uint32_t)p.off_t, es = ts + (uint32_t)(p.nt * pad * 4), parts = es + (uint32_t)(p.rank ? p.nt * 512 : 0);
      const int part_rows = (p.nt + p.split - 1) / p.split;
      const uint32_t ring = parts + (uint32_t)(p.split > 1 ? p.split * part_rows * 512 : 0);
      int groups = 0;                            // slots of the ring so far
      for (long long item = team; item < p.most && find_tile(p, tile_rows, walk, item, &t); item += teams) {
        // Of a cluster's CTAs each has every split-th row of the tile; of those each set of four warps every second one.
        const int o = t.tn * 128 + own, count = min(p.nt, t.end - t.row0), here = count > share ? (count - share - 1) / p.split + 1 : 0;
        if (p.rank) {
          // the adapters' part of those rows, while the shared matrix is multiplied
          bar_sync(1, kEpi * 32 + 32);           // the last item's are read
          bar_sync(1, kEpi * 32 + 32);           // the rows' adapters are there
          if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
          waited = true;
#pragma unroll 1
          for (int i = unit; i < count * pad; i += kEpi * 32) {
            const int r = i / pad;
            sts_f(ts + (uint32_t)(i * 4), kept<T>(p.t, t.row0 + r, pad, i - r * pad));
          }
          bar_sync(2, kEpi * 32);
          {
            // Slots go to the sets of warps in turn.  Rows of a slot would lie in the same banks for neighbouring lanes: each lane begins with another piece of 8 numbers.
            const int chunks = (p.rank + 7) / 8, turned = own * (p.e_pitch / 8) / 8 % chunks, listed = listed_s;
            for (int q = set; q < here; q += 2) sts_f(part_at(es, share + p.split * q), 0.f);
            bar_sync(2, kEpi * 32);
            for (int i0 = set * p.slot_rows; i0 < listed; i0 += 2 * p.slot_rows) {
              const int group = groups + i0 / p.slot_rows, slot = group % p.slots;
              const uint32_t e0 = ring + (uint32_t)(slot * p.slot_rows * p.row_bytes);
              const bool there = warp_wait(&bar[kEFull + slot], (uint32_t)(group / p.slots) & 1u, abort_flag, ws, 0xA0000u | (uint32_t)slot);
#pragma unroll 2
              for (int i = i0; i < min(listed, i0 + p.slot_rows); ++i) {
                const int r = list_s[i];
                const uint32_t e = e0 + (uint32_t)((i - i0) * p.row_bytes), tr = ts + (uint32_t)(r * pad * 4);
                float some[4] = {0.f, 0.f, 0.f, 0.f};
                if (ACROSS) {
#pragma unroll 1
                  for (int j0 = 0; j0 < p.rank; j0 += 8) {
                    const uint4 t0 = lds_u4(tr + (uint32_t)(j0 * 4)), t1 = lds_u4(tr + (uint32_t)(j0 * 4 + 16));
                    const uint32_t tv[8] = {t0.x, t0.y, t0.z, t0.w, t1.x, t1.y, t1.z, t1.w};
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                      uint16_t h;
                      asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(e + (uint32_t)(min(j0 + x, p.rank - 1) * 256 + own * 2)) : "memory");
                      if (j0 + x < p.rank) some[x & 3] = fmaf(__uint_as_float(tv[x]), __uint_as_float((uint32_t)h << 16), some[x & 3]);
                    }
                  }
                } else {
                  int c = turned;
#pragma unroll 2
                  for (int y = 0; y < chunks; ++y) {
                    const uint4 raw = lds_u4(e + (uint32_t)(own * p.e_pitch * 2 + c * 16)), t0 = lds_u4(tr + (uint32_t)(c * 32)), t1 = lds_u4(tr + (uint32_t)(c * 32 + 16));
                    const uint32_t tv[8] = {t0.x, t0.y, t0.z, t0.w, t1.x, t1.y, t1.z, t1.w};
                    float v[8];
                    unpack8(raw, v);
#pragma unroll
                    for (int x = 0; x < 8; ++x) some[x & 3] = fmaf(__uint_as_float(tv[x]), v[x], some[x & 3]);
                    c = c + 1 == chunks ? 0 : c + 1;
                  }
                }
                if (there) sts_f(part_at(es, r), (some[0] + some[1]) + (some[2] + some[3]));
              }
              __syncwarp();
              if (lane == 0) mbar_arrive(&bar[kEEmpty + slot]);
            }
            groups += (listed + p.slot_rows - 1) / p.slot_rows;
            if (p.split > 1) bar_sync(2, kEpi * 32);        // rows are delivered by others than those who worked their parts out
          }
          if (p.split == 1) bar_sync(2, kEpi * 32);       // rows are then delivered by whom their sums lie with
        }
        const float b = p.bias && o < p.n ? __ldg(p.bias + (p.bias_each ? (size_t)t.weight * (size_t)p.n : 0) + (size_t)o) : 0.f;
        auto deliver = [&](int r, float v) {     // row r of the tile: its sum
          if (r >= count || o >= p.n) return;
          const size_t at = (size_t)(t.row0 + r) * (size_t)p.n + (size_t)o;
          if (p.rank) v += lds_f(part_at(es, r));
          v += b;
          if (p.residual) v += to_float(reinterpret_cast<const T *>(p.residual)[at]);
          reinterpret_cast<T *>(p.y)[at] = (T)dc_act_apply(v, p.act);
        };
        // a block of eight rows' sums goes to whom they are delivered by
        auto hand_on = [&](int i0, const float *v) {
          if (p.split == 1) {
#pragma unroll
            for (int i = 0; i < 8; ++i) deliver(set * half_rows + i0 + i, v[i]);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int r = set * half_rows + i0 + i, q = r / p.split;
              asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(map_cluster(part_at(parts, share * part_rows + q), (uint32_t)(r - q * p.split))), "f"(v[i]) : "memory");
            }
          }
        };
        if (p.split > 1 && met++ == 0) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");         // the other CTAs are there
        // a wait that ran out does not end the loop: the barriers above are of all these warps
        {
          ok = wait_sums();
          const uint32_t d = sums_at() + (uint32_t)(set * half_rows);
#pragma unroll 1
          for (int i0 = 0; ok && i0 < half_rows; i0 += 8) {
            float v[8];
            __syncwarp();
            tmem_ld8(d + (uint32_t)i0, reinterpret_cast<uint32_t *>(v));
            tmem_ld_wait();
            if (i0 + 8 >= half_rows) release();
            if (!own_pieces) {
#pragma unroll
              for (int i = 0; i < 8; ++i) v[i] = 0.f;
            }
            hand_on(i0, v);
          }
          ++turn;
        }
        if (p.split > 1) {
          __syncwarp();
          if (lane < p.split) arrive_cluster(map_cluster(smem_u32(&bar[kParts]), (uint32_t)lane));
          if (warp_wait(&bar[kParts], 0, abort_flag, ws, 0x90000u, kLimit) && ok) {
            mbar_acquire_cluster(&bar[kParts], 0);
#pragma unroll 1
            for (int q0 = set; q0 < here; q0 += 8) {
              float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
              for (int k = 0; k < p.split; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += q0 + 2 * i < here ? lds_f(part_at(parts, k * part_rows + q0 + 2 * i)) : 0.f;
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (q0 + 2 * i < here) deliver(share + p.split * (q0 + 2 * i), v[i]);
            }
          }
        }
      }
      if (p.split > 1 && met == 0) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
  } else if (FORM == kFew) {
    // ---------------------------------------------------------------- kFew: which adapters rows have, and their parts of the tile's columns
    const uint32_t ring = sm + (uint32_t)(p.off_t + p.nt * grp::rank_pad(p.rank) * 4 + p.nt * 512 + (p.split > 1 ? p.split * ((p.nt + p.split - 1) / p.split) * 512 : 0));
    grp::Walk walk;
    walk.start();
    Tile t;
    int group = 0;                               // slots of the ring so far
    if (p.rank)
      for (long long item = team; item < p.most && find_tile(p, tile_rows, walk, item, &t); item += teams) {
        const int count = min(p.nt, t.end - t.row0), here = count > share ? (count - share - 1) / p.split + 1 : 0, o0 = t.tn * 128;
        bar_sync(1, kEpi * 32 + 32);
        for (int i = lane; i < p.nt; i += 32) weight_s[i] = -1;
        __syncwarp();
        grp::each_run(p.ext, t.row0, t.row0 + count, [&](const Run &run) {
          for (int i = max(run.begin - t.row0, 0); i < min(run.end - t.row0, count); ++i) weight_s[i] = run.weight;
        }, [](int) {});
        __syncwarp();
        int listed = 0;
        for (int q0 = 0; q0 < here; q0 += 32) {
          const int r = share + p.split * (q0 + lane);
          const bool has = q0 + lane < here && weight_s[r] >= 0;
          const unsigned all = __ballot_sync(0xffffffffu, has);
          if (has) list_s[listed + __popc(all & ((1u << lane) - 1u))] = r;
          listed += __popc(all);
        }
        if (lane == 0) listed_s = listed;
        __syncwarp();
        bar_sync(1, kEpi * 32 + 32);
        for (int i0 = 0; i0 < listed; i0 += p.slot_rows, ++group) {
          const int slot = group % p.slots, rows = min(p.slot_rows, listed - i0);
          ok = ok && warp_wait(&bar[kEEmpty + slot], ((uint32_t)(group / p.slots) & 1u) ^ 1u, abort_flag, ws, 0xB0000u | (uint32_t)slot);
          if (!ok) continue;
          const uint32_t to = ring + (uint32_t)(slot * p.slot_rows * p.row_bytes);
          const bf16 *e = reinterpret_cast<const bf16 *>(p.e);
          if (ACROSS) {                        // `rank` rows of the tile's columns (row by row, 14 rows' adapters of rank 64, 192 -> 2224, took 41 us for 16)
            if (lane == 0) mbar_arrive_expect_tx(&bar[kEFull + slot], (uint32_t)(p.row_bytes * rows));
            __syncwarp();
            if (lane < rows) load_box<false>(to + (uint32_t)(lane * p.row_bytes), &map_e, smem_u32(&bar[kEFull + slot]), o0, 0, 0, weight_s[list_s[i0 + lane]]);
          } else {                             // the columns' rows, one piece
            const uint32_t bytes = (uint32_t)(min(128, p.n - o0) * p.e_pitch) * 2u;
            if (lane == 0) mbar_arrive_expect_tx(&bar[kEFull + slot], bytes * (uint32_t)rows);
            __syncwarp();
            if (lane < rows)
              bulk_load(to + (uint32_t)(lane * p.row_bytes), e + ((size_t)weight_s[list_s[i0 + lane]] * (size_t)p.n + (size_t)o0) * (size_t)p.e_pitch, bytes, &bar[kEFull + slot]);
          }
          __syncwarp();
        }
      }
  } else {
    // ---------------------------------------------------------------- kGrad: pieces with rows of other weights are passed on once those are zeros.  (Asked for by
    // the warp that multiplies, where it came to such a piece, this took a tile 1.6 us: 131 us in the place of 109 for 8 groups of 1041 or 1007 rows.)
    uint32_t tails = 0;
    for (long long item = team; ok && item < p.most; item += teams) {
      const int weight = (int)(item / per_weight), at = (int)(item - (long long)weight * per_weight), tm = at / p.tiles_n;
      const bool sums = p.sums && at - tm * p.tiles_n == p.tiles_n - 1;
      each_piece(p, weight, share, [&](int, int rows, uint64_t mask) {
        if (has_holes(rows, mask)) {
          ok = ok && warp_wait(&bar[kTail + stage], tails >> stage & 1u, abort_flag, ws, 0x80000u | (uint32_t)stage, kLimit);
          tails ^= 1u << stage;
          if (ok) {
            const uint32_t a = sm + (uint32_t)stage * stage_bytes;
            const int boxes = N * (2 + (sums ? 0 : p.q_bytes / kBox));
            for (int r = lane >> 3; r < (rows + 15) / 16 * 16; r += 4)       // 16 bytes each
              if (!(mask >> r & 1ull))
                for (int b = 0; b < boxes; ++b) sts_u4(a + (uint32_t)(b * kBox + r * 128 + (lane & 7) * 16), make_uint4(0, 0, 0, 0));
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
              if (P) arrive_cluster(map_cluster(smem_u32(&bar[kReady + stage]), 0));
              else mbar_arrive(&bar[kReady + stage]);
            }
          }
        }
        next();
      });
    }
  }
  __syncwarp();
  if (p.early) asm volatile("griddepcontrol.wait;" ::: "memory");        // this launch does not end before the one in front of it
  if (FORM == kFew) {
    if (p.split > 1) {
      if (warp < 2 || warp >= 2 + kEpi) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
      if (*abort_flag) {                         // parts may still be on their way here: until the other CTAs are done too, or 20 ms
        const unsigned long long t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 20ull * 1000ull * 1000ull) __nanosleep(1000);
      }
    }
  } else if (!P && p.split > 1) {
    for (; met < 2; ++met) cluster_sync();       // the parts are there; and read
  }
  if (warp == 1 && *abort_flag) {                // copies and products may still be in flight: give them time to end
    const unsigned long long t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 20ull * 1000ull * 1000ull) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (P) {
    cluster_sync();                              // neither CTA's memory is touched by the other's instructions any more
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)p.tmem_cols) : "memory");
  } else if (warp == 1) {
    tmem_dealloc(tmem, (uint32_t)p.tmem_cols);
  }
}

// Rows as the tensor core's kernels read them: bf16 rows begin on 16 bytes, with zeros behind them; fp32 rows are three terms of bf16, one row of
// each behind the other.  (Two rounded, what is left has 8 bits: tc_ptx.cuh.)  Several arrays in one launch.
struct Copies {
  int count;
  grp::Copy c[grp::kMaxCopies];
  long long units[grp::kMaxCopies];              // of 8 columns, with those of the arrays before
};
template <typename T>
__global__ void __launch_bounds__(256) k_group_rows_of(const __grid_constant__ Copies all) {
  dc_pdl_enter();
  const long long total = all.units[all.count - 1];
  for (long long u = (long long)blockIdx.x * 256 + threadIdx.x; u < total; u += (long long)gridDim.x * 256) {
    int k = 0;
    while (u >= all.units[k]) ++k;
    const grp::Copy &j = all.c[k];
    const long long v = k ? u - all.units[k - 1] : u;
    const int per = j.pitch / 8;
    const long long row = v / per;
    const int c = (int)(v - row * per) * 8;
    const T *from = reinterpret_cast<const T *>(j.from) + (size_t)row * (size_t)j.cols + (size_t)c;
    if (sizeof(T) == 2) {
      const unsigned short *at = reinterpret_cast<const unsigned short *>(from);
      uint32_t x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = c + i < j.cols ? at[i] : 0;
      *reinterpret_cast<uint4 *>(reinterpret_cast<bf16 *>(j.to) + (size_t)row * (size_t)j.pitch + (size_t)c) =
          make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
    } else {
      float x[8];
      if (j.cols % 4 == 0) {
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
          float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
          if (c + i < j.cols) f = *reinterpret_cast<const float4 *>(from + i);
          x[i] = f.x; x[i + 1] = f.y; x[i + 2] = f.z; x[i + 3] = f.w;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = c + i < j.cols ? to_float(from[i]) : 0.f;
      }
      uint4 h, m, l;
      bf16_terms8(x, h, m, l);
      uint4 *to = reinterpret_cast<uint4 *>(reinterpret_cast<bf16 *>(j.to) + (size_t)row * (size_t)(3 * j.pitch) + (size_t)c);
      to[0] = h;
      to[per] = m;
      to[2 * per] = l;
    }
  }
}

// What rows keep of their adapters where runs are short: a warp to a number of a row, the adapter's row read straight through.
// The next launch starts only behind the wait for the one before this: what that one wrote is there for it.
template <typename T>
__global__ void __launch_bounds__(256) k_adapter_narrow(const T *__restrict__ x, int x_pitch, const T *__restrict__ a, int a_pitch, int k, int rank,
                                                        const __grid_constant__ Runs runs, const float *__restrict__ scale, bf16 *__restrict__ t) {
  constexpr int kPer = 16 / (int)sizeof(T), kAhead = 8, kStep = 32 * kPer;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int row = (int)blockIdx.x, warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31, j = (int)blockIdx.y * 8 + warp, pad = grp::rank_pad(rank);
  const T *xr = x + (size_t)row * (size_t)x_pitch;
  uint4 xv[kAhead], av[kAhead];
  auto ask = [&](const T *from, uint4 (&to)[kAhead], int i0) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) to[u] = i0 + u * kStep < k ? *reinterpret_cast<const uint4 *>(from + i0 + u * kStep) : make_uint4(0, 0, 0, 0);
  };
  ask(xr, xv, lane * kPer);                      // while the run is looked for
  int w = -1;
  each_run(runs, row, row + 1, [&](const Run &run) { if (run.begin <= row && row < run.end) w = run.weight; }, [](int) {});
  w = __reduce_max_sync(0xffffffffu, w);
  if (w < 0) return;
  float s = 0.f;
  if (j < rank) {
    const T *ar = a + ((size_t)w * (size_t)rank + (size_t)j) * (size_t)a_pitch;
    for (int i0 = lane * kPer; i0 < k; i0 += kAhead * kStep) {
      ask(ar, av, i0);
      if (i0 >= kAhead * kStep) ask(xr, xv, i0);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        float f[2][8];
        if (sizeof(T) == 2) {
          unpack8(xv[u], f[0]);
          unpack8(av[u], f[1]);
        } else {
          f[0][0] = __uint_as_float(xv[u].x); f[0][1] = __uint_as_float(xv[u].y); f[0][2] = __uint_as_float(xv[u].z); f[0][3] = __uint_as_float(xv[u].w);
          f[1][0] = __uint_as_float(av[u].x); f[1][1] = __uint_as_float(av[u].y); f[1][2] = __uint_as_float(av[u].z); f[1][3] = __uint_as_float(av[u].w);
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) s = fmaf(f[0][i], f[1][i], s);
      }
    }
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
  if (lane == 0 && j < pad) {
    constexpr int kKept = sizeof(T) == 4 ? 3 : 2;
    float term[3];
    terms_of<T>(j < rank ? s * (scale ? __ldg(scale + w) : 1.f) : 0.f, term);
    bf16 *to = t + (size_t)row * (size_t)(kKept * pad) + (size_t)j;
#pragma unroll
    for (int y = 0; y < kKept; ++y) to[y * pad] = __float2bfloat16(term[y]);
  }
}

// The same for u = dy B, B read across: a CTA to a row, its eight warps to as many parts of the sum; a lane takes 8 of the rank's numbers (and as many lanes
// as that needs the whole rank) of every 32 / lanes-th row of B.
template <typename T>
__global__ void __launch_bounds__(256) k_adapter_narrow_across(const T *__restrict__ x, int x_pitch, const T *__restrict__ b, int b_pitch, int k, int rank,
                                                               const __grid_constant__ Runs runs, const float *__restrict__ scale, bf16 *__restrict__ t) {
  __shared__ float part[8][grp::kMaxRank];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int row = (int)blockIdx.x, warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31, pad = grp::rank_pad(rank), groups = (rank + 7) / 8;
  int across = 1;                                // lanes to a row of B
  while (across < groups) across *= 2;
  int w = -1;
  each_run(runs, row, row + 1, [&](const Run &run) { if (run.begin <= row && row < run.end) w = run.weight; }, [](int) {});
  w = __reduce_max_sync(0xffffffffu, w);
  if (w < 0) return;
  const int g = lane & (across - 1), step = 32 / across;
  const T *xr = x + (size_t)row * (size_t)x_pitch, *br = b + (size_t)w * (size_t)k * (size_t)b_pitch + (size_t)(g * 8);
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  constexpr int kAhead = 4;
  if (g < groups)
    for (int i0 = warp * step + lane / across; i0 < k; i0 += kAhead * 8 * step) {
      float xv[kAhead], v[kAhead][8];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int i = i0 + u * 8 * step;
        const bool here = i < k;
        xv[u] = here ? to_float(xr[i]) : 0.f;
        const T *at = br + (size_t)i * (size_t)b_pitch;
        if (sizeof(T) == 2) {
          const uint4 raw = here ? *reinterpret_cast<const uint4 *>(at) : make_uint4(0, 0, 0, 0);
          unpack8(raw, v[u]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; j += 4) {
            const float4 f = here && g * 8 + j < rank ? *reinterpret_cast<const float4 *>(at + j) : make_float4(0.f, 0.f, 0.f, 0.f);
            v[u][j] = f.x; v[u][j + 1] = f.y; v[u][j + 2] = f.z; v[u][j + 3] = f.w;
          }
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = fmaf(xv[u], v[u][j], s[j]);
    }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    for (int d = across; d < 32; d *= 2) s[j] += __shfl_xor_sync(0xffffffffu, s[j], d);
  if (lane < groups) {
#pragma unroll
    for (int j = 0; j < 8; ++j) part[warp][lane * 8 + j] = s[j];
  }
  __syncthreads();
  const int j = (int)threadIdx.x;
  if (j < pad) {
    constexpr int kKept = sizeof(T) == 4 ? 3 : 2;
    float all = 0.f, term[3];
    if (j < rank) {
      for (int u = 0; u < 8; ++u) all += part[u][j];
      if (scale) all *= __ldg(scale + w);
    }
    terms_of<T>(all, term);
    bf16 *to = t + (size_t)row * (size_t)(kKept * pad) + (size_t)j;
#pragma unroll
    for (int y = 0; y < kKept; ++y) to[y * pad] = __float2bfloat16(term[y]);
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
// [outer][rows][terms][cols], rows of a term `pitch` elements: boxes of `wide` columns (16, 32 or 64) x `box` rows, zeros outside
bool map_of(CUtensorMap *map, const void *at, long long cols, int terms, long long rows, long long outer, long long pitch, int box, int wide = kPiece) {
  EncodeTiledFn encode = get_encode_fn();
  if (!encode) return false;
  const cuuint64_t one = (cuuint64_t)pitch * 2;
  const cuuint64_t dim[4] = {(cuuint64_t)cols, (cuuint64_t)terms, (cuuint64_t)rows, (cuuint64_t)outer}, str[3] = {one, one * (cuuint64_t)terms, one * (cuuint64_t)terms * (cuuint64_t)rows};
  const cuuint32_t bx[4] = {(cuuint32_t)wide, 1, (cuuint32_t)box, 1}, es[4] = {1, 1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(at), dim, str, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                wide == 128 ? CU_TENSOR_MAP_SWIZZLE_NONE : wide == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : wide == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int FORM, bool ACROSS, typename T, bool P>
cudaError_t launch(Params &p, long long items, int n_sm, const CUtensorMap (&m)[4], DcWsHeader *ws, cudaStream_t st) {
  static unsigned char attr_done[kDcMaxDevices];
  const cudaError_t e = dc_set_max_smem_once(k_group_tc<FORM, ACROSS, T, P>, kSmem, attr_done);
  if (e != cudaSuccess) return e;
  if (p.tmem_cols > 512 || p.stages < 1) return cudaErrorNotSupported;        // no such form: a rule above would be wrong
  const int group = P ? 2 : p.split;
  const long long teams = items < n_sm / group ? items : n_sm / group;
  p.most = FORM == kGrad ? items : group > 1 && !P ? teams : 1ll << 62;
  return dc_launch_pdl_cluster(k_group_tc<FORM, ACROSS, T, P>, dim3((unsigned)(teams * group)), dim3(kThreadsOf<FORM>), (size_t)kSmem, st, group, m[0], m[1], m[2], m[3], p, ws);
}
template <int FORM, bool ACROSS>
cudaError_t launch_any(Params &p, bool wide, bool pair, long long items, int n_sm, const CUtensorMap (&m)[4], DcWsHeader *ws, cudaStream_t st) {
  if constexpr (FORM != kFew) {
    if (wide) return launch<FORM, ACROSS, float, false>(p, items, n_sm, m, ws, st);
    if (pair) return launch<FORM, ACROSS, bf16, true>(p, items, n_sm, m, ws, st);
  }
  return launch<FORM, ACROSS, bf16, false>(p, items, n_sm, m, ws, st);
}

// Shared and tensor memory; `apart`: bytes beside the ring and the staged results
void lay_out(Params *p, int terms, int apart) {
  // An accumulator is read 32 columns at a time, and of a bf16 gradient with terms each half so, from its own first column on: what is read
  // belongs to it, beyond its last column too (rank 16: 16 + 16 columns, of which 16 to 47 are the second read).
  const int half = p->q_terms && terms == 1 ? p->nt / 2 : 0;
  p->acc = (int)dc_round_up((size_t)(half ? half + (int)dc_round_up((size_t)half, 32) : p->nt), 32);
  p->tmem_cols = 32;
  while (p->tmem_cols < (terms == 3 ? kAccs<float> : kAccs<bf16>) * p->acc) p->tmem_cols *= 2;
  const int stage = terms * (kP + p->q_bytes);
  p->stages = (kSmem - 1024 - apart) / stage;
  if (p->stages > kMaxStages) p->stages = kMaxStages;
  p->off_out = p->off_t = p->stages * stage;
}
// Clusters of so many CTAs, one to an SM, that run at once on 148 SMs.
int clusters_at_once(int split, int n_sm) {
  static constexpr int kAt148[kMaxSplit + 1] = {0, 148, 74, 45, 33, 26, 22, 15, 15};
  return kAt148[split] * n_sm / 148;
}
// CTAs that share a tile's sum of `pieces`: as many as keep all SMs busy at once, each with `least` pieces at least
int split_of(long long items, int pieces, int least, int n_sm) {
  int s = kMaxSplit;
  while (s > 1 && (items > clusters_at_once(s, n_sm) || s > pieces / least)) --s;
  return s;
}
struct Shape { int nt; bool pair; int split; double us; };
// Columns to a tile, whether CTAs work in pairs, and how many share a tile's sum, by an estimate in cycles: a piece of 64 terms takes its loads (an SM takes in some 45
// bytes a cycle; two stages of fp32 terms wait for them) or its instructions; results go out beside the next tile's pieces, and of the last tile behind
// them; a cluster meets twice, and reads each other's parts.  `matrices`: bytes that come from memory (at 4.4 TB/s with the rows that come with them); `more`: cycles
// that a tile's adapters take.
Shape shape_of(int n, double rows, double runs, double pieces, double matrices, double more, bool wide, int n_sm) {
  static constexpr struct { int nt; bool pair; } kinds[4] = {{256, true}, {256, false}, {128, false}, {64, false}};
  Shape best = {64, false, 1, 1e30};
  for (const auto &k : kinds) {
    if ((wide && k.nt > 128) || (k.nt > 64 && n <= k.nt / 2)) continue;
    const double tiles = (rows / (k.pair ? 256 : 128) + 0.5 * runs) * dc_div_up(n, k.nt), most = (floor(rows / 128) + runs) * dc_div_up(n, k.nt);
    const double bytes = (128 + (k.pair ? k.nt / 2 : k.nt)) * 128.0 * (wide ? 3 : 1), sums = k.nt * 2.0 * (wide ? 6 : 1);
    double piece = bytes / 45 > sums ? bytes / 45 : sums;
    if (wide && piece < (sums + 1000 + bytes / 45) / 2) piece = (sums + 1000 + bytes / 45) / 2;
    for (int split = 1; split <= (k.pair ? 1 : kMaxSplit); ++split) {
      if (split > 1 && (most > clusters_at_once(split, n_sm) || pieces < 4 * split)) break;
      const double rounds = tiles * split / (k.pair ? n_sm / 2 : n_sm), main = pieces / split * piece + more, out = (800 + k.nt * 14.0) / split + (split > 1 ? 3000 + k.nt * 8.0 : 0);
      double cycles = (rounds < 1 ? 1 : rounds + 0.4) * (main > out ? main : out) + (main > out ? out : main) + (k.pair ? 800 : 0);
      if (cycles < matrices / 2.3e3) cycles = matrices / 2.3e3;
      if (cycles / 1.9e3 < best.us) best = {k.nt, k.pair, split, cycles / 1.9e3};
    }
  }
  return best;
}
// The same for short runs: rows to a tile, and CTAs to its sum, in microseconds.  The matrix comes once for each tile of rows (82 GB/s to an SM), the rows'
// adapters 0.3 a row or at 40 GB/s, in two sets of warps; a cluster meets.
Shape few_shape_of(const grp::RowsJob &j, int runs, long long (*row_tiles)(const Runs &, int), int pieces, double matrices, int n_sm) {
  const int mean = j.rows / runs;
  Shape best = {16, false, 1, 1e30};
  for (int nt = 16; nt <= (j.rank > 64 && j.t ? kFewWide : kFewMost); nt *= 2) {
    if (runs > 1 && nt > 16 && mean <= nt * 3 / 8) break;
    const long long all = row_tiles(j.runs, nt) * dc_div_up(j.n, 128);
    const double tiles = ((double)j.rows / nt + (runs > 1 ? 0.7 : 0.5) * runs) * dc_div_up(j.n, 128);
    for (int split = 1; split <= kMaxSplit; ++split) {
      if (split > 1 && (all > clusters_at_once(split, n_sm) || (pieces ? split > pieces / 4 : !j.t || split > nt / 4))) break;
      const double rounds = (runs > 1 && split == 1 ? tiles : (double)all) * split / n_sm, rows = (double)(j.rows < nt ? j.rows : nt) / split / 2;
      const double stream = (double)dc_div_up(pieces, split) * (kP + nt * 128) / 82e3, memory = matrices / 6.5e6;
      const double row = 256.0 * grp::rank_pad(j.rank) / 40e3, ext = j.t ? 2.0 + rows * (row > 0.3 ? row : 0.3) : 0.0;
      const double work = stream > ext ? stream : ext, out = 0.6 + nt * 0.02;
      const double all_of = (rounds < 1 ? 1 : rounds + 0.3) * (work > out ? work : out) + 0.3 * (memory < work ? memory : work) + (split > 1 ? 1.2 : 0.5);
      const double us = all_of > memory ? all_of : memory;
      if (us < best.us) best = {nt, false, split, us};
    }
  }
  return best;
}

}  // namespace

namespace grp {

static int runs_with_rows(const Runs &r) { return !r.offsets ? 1 : r.count < r.rows ? r.count : r.rows; }
// no more row tiles than this: every run may end inside one
static long long row_tiles(const Runs &r, int tile) { return r.offsets ? r.rows / tile + runs_with_rows(r) : (r.rows + tile - 1) / tile; }

cudaError_t copies_tc(const Copy *c, int count, dc_dtype dtype, cudaStream_t st) {
  Copies all = {};
  long long units = 0;
  for (int i = 0; i < count; ++i) {
    if (c[i].rows == 0) continue;
    units += c[i].rows * (c[i].pitch / 8);
    all.c[all.count] = c[i];
    all.units[all.count++] = units;
  }
  if (!all.count) return cudaSuccess;
  const long long blocks = (units + 255) / 256;
  const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)));
  return dtype == DC_BF16 ? dc_launch_pdl(k_group_rows_of<bf16>, grid, dim3(256), 0, st, all) : dc_launch_pdl(k_group_rows_of<float>, grid, dim3(256), 0, st, all);
}

// By the kernels for short runs: each row reads all of its adapter's matrix, 3 us, 2.5 for each eight CTAs of an SM, and what they take from L2 at 3 MB a us; tiles take 6 us, the last two of them for a cluster's
// parts, and 0.25 for a piece.
bool narrow_apart(const RowsJob &j) {
  if (!j.y_terms || (j.dtype == DC_F32 && (j.w_across ? j.n % 4 : j.k % 4) != 0)) return false;
  const int n_sm = dc_sm_count(), pieces = dc_div_up(j.k, kPiece);
  const double wide = j.dtype == DC_F32 ? 2.0 : 1.0, apart = 3.0 + (double)j.rows * (j.w_across ? 1.0 : rank_pad(j.n) / 8) / (8.0 * n_sm) * 2.5 + (double)j.rows * rank_pad(j.n) * j.k * 2.0 * wide / 3e6;
  const long long items = row_tiles(j.runs, 128);
  const int split = split_of(items, pieces, 4, n_sm);
  const double tiles = 6.0 + dc_div_up((int)(items < (1 << 20) ? items : 1 << 20) * split, n_sm) * (double)dc_div_up(pieces, split) * 0.25 * (wide > 1.0 ? 4.0 : 1.0);
  return apart < tiles;
}
cudaError_t narrow_tc(const RowsJob &j, cudaStream_t st) {
  const dim3 grid((unsigned)j.rows, j.w_across ? 1u : (unsigned)(rank_pad(j.n) / 8));
  bf16 *y = (bf16 *)j.y;
  if (j.dtype == DC_BF16) {
    if (j.w_across) return dc_launch_pdl(k_adapter_narrow_across<bf16>, grid, dim3(256), 0, st, (const bf16 *)j.x, j.x_pitch, (const bf16 *)j.w, j.w_pitch, j.k, j.n, j.runs, j.alpha, y);
    return dc_launch_pdl(k_adapter_narrow<bf16>, grid, dim3(256), 0, st, (const bf16 *)j.x, j.x_pitch, (const bf16 *)j.w, j.w_pitch, j.k, j.n, j.runs, j.alpha, y);
  }
  const float *x = (const float *)j.raw_x, *w = (const float *)j.raw_w;
  if (j.w_across) return dc_launch_pdl(k_adapter_narrow_across<float>, grid, dim3(256), 0, st, x, j.k, w, j.n, j.k, j.n, j.runs, j.alpha, y);
  return dc_launch_pdl(k_adapter_narrow<float>, grid, dim3(256), 0, st, x, j.k, w, j.k, j.k, j.n, j.runs, j.alpha, y);
}

cudaError_t rows_tc(const RowsJob &j, bool early, DcWsHeader *ws, cudaStream_t st, dc_group_plan *plan, double *us) {
  const int n_sm = dc_sm_count();
  const bool wide = j.dtype == DC_F32;
  const int terms = wide ? 3 : 1;
  Params p = {};
  p.k = j.k;
  p.n = j.n;
  p.runs = j.runs;
  p.alpha = j.alpha;
  p.bias = j.bias;
  p.bias_each = j.bias_each;
  p.act = j.act;
  p.residual = j.residual;
  p.y = j.y;
  p.y_terms = j.y_terms;
  p.vec = j.n % 4 == 0;
  p.raw_p = j.raw_x;
  p.raw_q = j.raw_w;
  p.pieces = j.w ? dc_div_up(j.k, kPiece) : 0;
  p.split = 1;
  if (j.t) {
    p.ext = j.ext;
    p.rank = j.rank;
    p.rank_pieces = dc_div_up(j.rank, kPiece);
    p.t = (const bf16 *)j.t;
    p.e = wide ? j.raw_e : j.e;
    p.e_pitch = j.e_pitch;
  }
  const int runs = runs_with_rows(j.runs);
  const double matrices = j.w ? (double)runs * j.n * j.k * 2 * terms : 0.0;
  // an adapter's instructions, and the way to the next one, of the runs that a tile has rows of
  const double per_tile = j.t ? 1.0 + 128.0 * j.ext.count / j.rows : 0.0, more = 850.0 * (per_tile < 129.0 ? per_tile : 129.0) * (wide ? 2.0 : 1.0);
  const Shape tile = j.y_terms ? Shape{rank_pad(j.n), false, 1, 0.0} : shape_of(j.n, j.rows, runs, p.pieces, matrices, more, wide, n_sm);
  if (us) {
    *us = tile.us;
    return cudaSuccess;
  }
  // runs of up to 128 rows: 128 columns of a matrix in the place of 128 rows, where that is faster
  Shape shape = tile;
  bool by_few = false;
  if (!j.y_terms && !wide && j.rows / runs <= 128) {
    const Shape f = few_shape_of(j, runs, row_tiles, p.pieces, matrices, n_sm);
    by_few = f.us <= tile.us;
    if (by_few) shape = f;
  }
  long long items;
  const bool pair = shape.pair;
  p.nt = shape.nt;
  p.split = shape.split;
  p.early = early;
  if (by_few) {
    p.q_bytes = p.nt * 128;
    p.tiles_n = dc_div_up(j.n, 128);
    items = row_tiles(j.runs, p.nt) * p.tiles_n;
    int apart = (p.rank ? p.nt * (rank_pad(p.rank) * 4 + 512) : 0) + (p.split > 1 ? (p.nt + p.split) * 512 : 0);
    if (p.rank) {
      p.row_bytes = j.e_across ? p.rank * 256 : 128 * p.e_pitch * 2;
      p.slot_rows = 16384 / p.row_bytes < 1 ? 1 : 16384 / p.row_bytes < 8 ? 16384 / p.row_bytes : 8;
      p.slots = 65536 / (p.slot_rows * p.row_bytes) < kMaxSlots ? 65536 / (p.slot_rows * p.row_bytes) : kMaxSlots;
      apart += p.slots * p.slot_rows * p.row_bytes;
    }
    lay_out(&p, terms, apart);
  } else {
    const int wide_nt = pair ? p.nt / 2 : p.nt;  // of a CTA
    p.q_bytes = j.w_across || (!j.w && j.e_across) ? dc_div_up(wide_nt, 64) * kBox : wide_nt * 128;
    p.tiles_n = dc_div_up(j.n, p.nt);
    items = row_tiles(j.runs, pair ? 256 : 128) * p.tiles_n;
    if (j.y_terms) p.split = split_of(items, p.pieces, 4, n_sm);
    lay_out(&p, terms, kOut);
  }
  p.pieces_per = dc_div_up(p.pieces, p.split);
  while (p.split > 1 && p.pieces && p.pieces_per * (p.split - 1) >= p.pieces) { --p.split; p.pieces_per = dc_div_up(p.pieces, p.split); }
  if (plan) {
    *plan = {by_few ? DC_GROUP_FEW_ROWS : pair ? DC_GROUP_PAIRS : DC_GROUP_TILES, p.nt, p.split, p.stages};
    return cudaSuccess;
  }
  CUtensorMap m[4] = {};
  p.maps = (j.w ? 3 : 0) | (j.t && !by_few ? 12 : 0) | (j.t && by_few && j.e_across ? 8 : 0);
  const int box = pair ? p.nt / 2 : p.nt;
  if (j.w) {
    if (!map_of(&m[0], j.x, j.k, terms, j.rows, 1, j.x_pitch, by_few ? p.nt : 128)) return cudaErrorNotSupported;
    if (!(j.w_across ? map_of(&m[1], j.w, j.n, terms, j.k, j.runs.weights, j.w_pitch, 64) : map_of(&m[1], j.w, j.k, terms, j.n, j.runs.weights, j.w_pitch, by_few ? 128 : box)))
      return cudaErrorNotSupported;
  }
  if (j.t && by_few && j.e_across && !map_of(&m[3], j.e, j.n, 1, j.rank, j.ext.weights, j.e_pitch, j.rank, 128)) return cudaErrorNotSupported;
  if (j.t && !by_few) {
    // Rows no wider than the rank: what lies outside a box costs a load as much as what is there (16 numbers a row in boxes of 64: 1100 cycles a run).
    const int pad = rank_pad(j.rank), row = pad <= 16 ? 16 : pad <= 32 ? 32 : 64;
    p.e_wide = row;
    p.e_bytes = j.e_across ? p.q_bytes / kBox * row * 128 : box * row * 2;
    const int t_wide = wide ? row : pad <= 16 ? 32 : 64;             // bf16: both terms as one row
    p.t_bytes = 128 * t_wide * 2;
    if (!(wide ? map_of(&m[2], j.t, pad, 3, j.rows, 1, pad, 128, t_wide) : map_of(&m[2], j.t, 2 * pad, 1, j.rows, 1, 2 * pad, 128, t_wide))) return cudaErrorNotSupported;
    if (!(j.e_across ? map_of(&m[3], j.e, j.n, terms, j.rank, j.ext.weights, j.e_pitch, row) : map_of(&m[3], j.e, j.rank, terms, j.n, j.ext.weights, j.e_pitch, box, row)))
      return cudaErrorNotSupported;
  }
  const bool across = j.w ? j.w_across : j.e_across;
  if (by_few) return across ? launch_any<kFew, true>(p, wide, false, items, n_sm, m, ws, st) : launch_any<kFew, false>(p, wide, false, items, n_sm, m, ws, st);
  return across ? launch_any<kTile, true>(p, wide, pair, items, n_sm, m, ws, st) : launch_any<kTile, false>(p, wide, pair, items, n_sm, m, ws, st);
}

cudaError_t grad_tc(const GradJob &j, bool early, DcWsHeader *ws, cudaStream_t st, dc_group_plan *plan) {
  const int n_sm = dc_sm_count();
  const bool wide = j.dtype == DC_F32;
  if (wide && j.out && j.sums && !plan) {                 // two stages of fp32 terms leave no room for the block of ones
    GradJob apart = j;
    apart.out = nullptr;
    const cudaError_t e = grad_tc(apart, early, ws, st);
    if (e != cudaSuccess) return e;
    apart = j;
    apart.sums = nullptr;
    return grad_tc(apart, true, ws, st);
  }
  const int terms = wide ? 3 : 1, pad = rank_pad(j.n), weights = j.runs.weights;
  Params p = {};
  p.k = j.m;
  p.n = j.n;
  p.runs = j.runs;
  p.y = j.out;
  p.sums = j.sums;
  p.q_terms = j.q_terms;
  p.t = (const bf16 *)j.q;
  p.out_across = j.out_across;
  p.vec = j.n % 4 == 0;
  p.raw_p = j.raw_p;
  p.raw_q = j.raw_q;
  bool pair = false;
  if (!j.out) {
    p.nt = 64;
  } else if (j.q_terms) {
    p.nt = wide ? pad : 2 * pad;
  } else {
    const Shape s = shape_of(j.n, (double)dc_div_up(j.m, 128) * 128 * weights, 0, (double)j.runs.rows / kPiece / weights + 0.5, 0.0, 0.0, wide, n_sm);
    p.nt = s.nt;
    pair = s.pair && j.m > 128;
    p.split = s.split;
  }
  p.tiles_m = dc_div_up(j.m, pair ? 256 : 128);
  p.q_bytes = dc_div_up(pair ? p.nt / 2 : p.nt, 64) * kBox;
  p.tiles_n = (j.out ? (j.q_terms ? 1 : dc_div_up(j.n, p.nt)) : 0) + (j.sums ? 1 : 0);
  const long long items = (long long)p.tiles_m * p.tiles_n * weights;
  if (!j.out || j.q_terms) p.split = split_of(items, j.runs.rows / kPiece / weights, 4, n_sm);
  else if (pair) p.split = 1;
  else while (p.split > 1 && items > clusters_at_once(p.split, n_sm)) --p.split;
  p.early = early;
  lay_out(&p, terms, kOut + (j.sums ? kBox : 0));
  if (j.sums) p.off_out += kBox;
  if (plan) {
    *plan = {pair ? DC_GROUP_PAIRS : DC_GROUP_TILES, p.nt, p.split, p.stages};
    return cudaSuccess;
  }
  CUtensorMap m[4] = {};
  p.maps = j.runs.rows ? (j.out ? 3 : 1) : 0;
  if (j.runs.rows) {                             // without rows nothing is loaded
    if (!map_of(&m[0], j.p, j.m, terms, j.runs.rows, 1, j.p_pitch, 64)) return cudaErrorNotSupported;
    if (j.out && !(!j.q_terms ? map_of(&m[1], j.q, j.n, terms, j.runs.rows, 1, j.q_pitch, 64)
                   : wide     ? map_of(&m[1], j.q, pad, 3, j.runs.rows, 1, pad, 64)
                              : map_of(&m[1], j.q, 2 * pad, 1, j.runs.rows, 1, 2 * pad, 64)))
      return cudaErrorNotSupported;
  }
  return launch_any<kGrad, true>(p, wide, pair, items, n_sm, m, ws, st);
}

}  // namespace grp
