// Products of matrices in microscaled 4 bits on the tensor core (dc_q4_product, dc_q4_forward).
//
// tcgen05.mma.block_scale multiplies 64 columns of 128 rows x nt rows at a time: codes from shared memory (rows of 128 bytes, 256 codes, with
// the 128-byte swizzle), scales from tensor memory, where tcgen05.cp puts them from the tiles in which a quantised matrix keeps them
// (32 lanes x 4 columns, one for each 32 rows of the tile; four bytes a column, which are four blocks).  DC_NV4: a tile is one instruction's
// scales; DC_MX4: two instructions', told apart by the descriptor's scale id.  Sums are fp32 in tensor memory.
//
// A stage of the ring is 256 columns: codes of both operands and their scale tiles; its scales have columns of tensor memory of their own, so a
// slot's scales are written over only behind the products that read them.  One warp loads, one issues, eight or twelve read out the accumulators.
// CTAs walk over tiles.  The forms:
//   kOne     both operands by TMA.  Few tiles: a cluster shares a tile's reduction.  Each of its CTAs owns some columns of the result; all send their
//            parts of them to its shared memory, and it adds them up in rank order.  (Parts left where they were would take two meetings of the
//            cluster and reads from afar.)  Tensor memory is given back without waiting for a CTA that may be waiting for
//            some.  One column of tiles to a CTA and few stages: w stays in shared memory.
//            Narrow tiles, of 32 or 64 columns: the products are those of 128 rows of w around the tile's, of which only the tile's are there; the rest is
//            what lies around them in shared memory, and is not read out.
//            (6272 x 320 -> 1280 in mx4 8.8 us, a fill of as many bytes as its results 5.1; 128 x 4096 -> 4096 in nv4 9.5.)
//   kPair    two CTAs multiply 256 x 256 (cta_group::2): each loads half of either operand, which halves what an SM has to fetch of w.  8192^3 in nv4 242 to
//            246 us, 4.5 PFLOP/s, in calls one behind the other, the clock falls under the power cap; 203 to 212 in short runs (178 without loads of codes).
//   kRows    up to 32 rows of bf16 or fp32: quantised by the reading-out warps into shared memory, where all of them stay.  One row of 4096 -> 4096 7.5 us:
//            3.2 until the first products, four stages, the cluster's meeting.
//   kStream  many rows of bf16 or fp32 and one column of tiles: four more warps quantise them, a stage at a time.
//            200704 x 24 -> 144 21.2 us (quantised apart 26.2; a fill of as many bytes as its results 15.9).
#include <string.h>

#include "q4.cuh"
#include "tc_ptx.cuh"

namespace {
using namespace tc;
using q4::kAtom;

enum { kOne = DC_Q4_TILES, kPair = DC_Q4_PAIRS, kRows = DC_Q4_FEW_ROWS, kStream = DC_Q4_STREAM };
template <int FORM>
constexpr int kEpi = FORM == kOne || FORM == kStream ? 12 : 8;                 // warps reading out
constexpr int kCutWarps = 4;                     // quantising, form kStream
template <int FORM>
constexpr int kThreadsOf = (2 + kEpi<FORM> + (FORM == kStream ? kCutWarps : 0)) * 32;
constexpr int kMaxStages = 8, kMaxSplit = 8, kMaxAcc = 3;
template <int FORM>
constexpr int kSmemOf = (FORM == kPair ? 224 : 214) * 1024;    // what the static arrays leave
constexpr int kStageCols = 256;                  // columns of a stage: 128 bytes of codes
constexpr int kOutBytes = 32 * 128;              // of a reading-out warp: 32 rows of 128 bytes of results
template <typename T>
constexpr int kOut = 128 / (int)sizeof(T);       // ... which are so many columns
constexpr int kMaxRows = 32;                     // of form kRows

struct Params {
  long long rows;
  int c_in, c_out, act;
  float scale;
  float g, r6;               // kRows, kStream: x's tensor scale
  int nt, nb;                // rows of w in a tile, 128-row scale tiles that they touch
  int acc;                   // columns of an accumulator: nt, or 128 around a narrow tile's
  int tiles_m, tiles_n, items;
  int chunks;                // stages of a row
  int columns;               // CTAs keep to a column of tiles: item = row of tiles
  int split, chunks_per;     // CTAs that share an item, stages of each
  int stages, acc_bufs;
  int stage_bytes, sf_cols;  // of a stage: shared memory, and tensor memory of its scales
  int w_stays, w_bytes;      // w's stages stay in shared memory; bytes of one
  int a_bytes;               // of x's codes in a stage: 128 rows, or fewer where x has fewer
  int off_sfa, off_ring, off_out, out_bufs;
  int part_rows, part_cols;  // of a part that a CTA of a cluster sends to another (columns: whole 16-byte pieces of y)
  int vec;                   // rows of y begin on 16 bytes
  int vec_x;                 // kRows: rows of x do
};

constexpr int kA = 128 * 128;                    // bytes that a product reads of x's codes in a stage
template <int F>
constexpr int kAtomsOf = F == DC_NV4 ? 4 : 2;    // scale tiles of a stage, for 128 rows

__device__ __forceinline__ uint64_t operand_desc(uint32_t a) {   // K-major, 128-byte swizzle, 1024 bytes between groups of 8 rows
  return ((uint64_t)((64u) | (1u << 14) | (2u << 29)) << 32) | (uint64_t)((a >> 4) & 0x3FFFu) | (1u << 16);
}
__device__ __forceinline__ uint64_t scales_desc(uint32_t a) {    // a scale tile: 32 rows of 16 bytes, 128 between groups of 8
  return ((uint64_t)((8u) | (1u << 14)) << 32) | (uint64_t)((a >> 4) & 0x3FFFu) | (1u << 16);
}
// the pair's forms act in both CTAs: each copies from its own shared to its own tensor memory, and multiplies its own 128 rows
template <bool P>
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
  if (P) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
  else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
#define Q4_MMA(GROUP, KIND)                                                                            \
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"                                       \
               "tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %1, %2, %3, [%4], [%5], p;\n\t}" \
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory")
template <int F, bool P>
__device__ __forceinline__ void mma_q4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  if (F == DC_NV4) {
    if (P) Q4_MMA("2", "mxf4nvf4.block_scale.scale_vec::4X");
    else Q4_MMA("1", "mxf4nvf4.block_scale.scale_vec::4X");
  } else {
    if (P) Q4_MMA("2", "mxf4.block_scale.scale_vec::2X");
    else Q4_MMA("1", "mxf4.block_scale.scale_vec::2X");
  }
}
#undef Q4_MMA
// instruction descriptor: e2m1 x e2m1, N, M, type of the scales
template <int F>
__device__ __forceinline__ uint32_t q4_idesc(int n, int m) {
  return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((F == DC_MX4 ? 1u : 0u) << 23) | ((uint32_t)(m >> 7) << 27);
}
// ... with the half of a scale word that product k of a stage takes (DC_MX4)
template <int F>
__device__ __forceinline__ uint32_t with_id(uint32_t idesc, int k) {
  return F == DC_MX4 && (k & 1) ? idesc | (2u << 4) | (2u << 29) : idesc;
}
// A stage: its scales to tensor memory (columns from `ta`), then its products.  One thread issues all of it, and the tensor core takes 512 cycles for
// 256 columns of w: with descriptors worked out in loops the issuing thread was what bound large products (8192^3 in nv4 389 us).
template <int F, bool P, int NB, int STEPS>
__device__ __forceinline__ void multiply(uint32_t d, uint32_t a, uint32_t b, uint32_t sfa, uint32_t sfb, uint32_t ta, uint32_t idesc, bool accumulate) {
  constexpr int kAtoms = kAtomsOf<F>;
  const uint64_t da = scales_desc(sfa), db = scales_desc(sfb), ad = operand_desc(a), bd = operand_desc(b);
  const uint32_t tb = ta + 4u * kAtoms;
#pragma unroll
  for (int i = 0; i < (F == DC_NV4 ? STEPS : (STEPS + 1) / 2); ++i) {
    copy_scales<P>(ta + 4u * i, da + (uint64_t)(i * (kAtom / 16)));
#pragma unroll
    for (int j = 0; j < NB; ++j) copy_scales<P>(tb + 4u * (i * NB + j), db + (uint64_t)((j * kAtoms + i) * (kAtom / 16)));
  }
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    const uint32_t atom = F == DC_NV4 ? (uint32_t)k : (uint32_t)(k >> 1);
    mma_q4<F, P>(d, ad + 2u * k, bd + 2u * k, with_id<F>(idesc, k), ta + 4u * atom, tb + 4u * NB * atom, accumulate || k > 0 ? 1u : 0u);
  }
}
template <int F, bool P, int NB>
__device__ __forceinline__ void multiply_steps(int steps, uint32_t d, uint32_t a, uint32_t b, uint32_t sfa, uint32_t sfb, uint32_t ta, uint32_t idesc, bool accumulate) {
  if (steps == 4) multiply<F, P, NB, 4>(d, a, b, sfa, sfb, ta, idesc, accumulate);
  else if (steps == 1) multiply<F, P, NB, 1>(d, a, b, sfa, sfb, ta, idesc, accumulate);
  else if (steps == 2) multiply<F, P, NB, 2>(d, a, b, sfa, sfb, ta, idesc, accumulate);
  else multiply<F, P, NB, 3>(d, a, b, sfa, sfb, ta, idesc, accumulate);
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
// loads that report to a barrier of the pair's first CTA (cluster address `bar`)
__device__ __forceinline__ void pair_load_2d(uint32_t sdst, const CUtensorMap *map, uint32_t bar, int c0, int c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4}], [%2];"
      ::"r"(sdst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void pair_load_3d(uint32_t sdst, const CUtensorMap *map, uint32_t bar, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(sdst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void sts_cluster_f4(uint32_t a, float x, float y, float z, float w) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(a), "f"(x), "f"(y), "f"(z), "f"(w) : "memory");
}
// a phase that has been seen to end: what the cluster's threads wrote before they arrived is visible behind this
__device__ __forceinline__ void mbar_acquire_cluster(uint64_t *bar, uint32_t parity) {
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%0], %1;\n\t}" ::"r"(smem_u32(bar)), "r"(parity) : "memory");
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// What a lane delivers: N neighbouring results of a row, 16 bytes of y.
template <typename T>
constexpr int kPer = 16 / (int)sizeof(T);
template <typename T>
__device__ __forceinline__ void unpack16(uint4 w, float *r) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (sizeof(T) == 2) { r[2 * j % kPer<T>] = __uint_as_float(u[j] << 16); r[(2 * j + 1) % kPer<T>] = __uint_as_float(u[j] & 0xffff0000u); }
    else r[j] = __uint_as_float(u[j]);
  }
}
template <typename T>
__device__ __forceinline__ uint4 pack16(const float *v) {
  constexpr int N = kPer<T>;
  if (N == 8) return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4 % N], v[5 % N]), pack_bf16x2(v[6 % N], v[7 % N]));
  return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ void load_bias(const float *__restrict__ bias, int o, int n, float *b) {
#pragma unroll
  for (int i = 0; i < n; i += 4) *reinterpret_cast<float4 *>(b + i) = bias ? __ldg(reinterpret_cast<const float4 *>(bias + o + i)) : make_float4(0.f, 0.f, 0.f, 0.f);
}
// The activation of a result of type T.  In bf16 the minimum comes first, and a NaN becomes 6, as it does in relu6_fast: which form a call takes, and with it
// which of the two is used, is not to be seen in its results.
template <typename T>
__device__ __forceinline__ float act_of(float t, int act) {
  if (sizeof(T) == 2) return act == DC_ACT_RELU6 ? fmaxf(fminf(t, 6.f), 0.f) : t;
  return dc_act_apply(t, act);
}
template <typename T>
__device__ __forceinline__ uint4 finish16(const Params &p, const float *b, bool has_residual, uint4 residual, float *v) {
  constexpr int N = kPer<T>;
  float r[N];
  if (has_residual) unpack16<T>(residual, r);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float t = fmaf(v[i], p.scale, b[i]);
    if (has_residual) t += r[i];
    v[i] = act_of<T>(t, p.act);
  }
  return pack16<T>(v);
}
// two FMAs in one instruction
__device__ __forceinline__ void fma2(float &lo, float &hi, uint64_t s, uint64_t b) { q4::unpair(q4::fma2(q4::pair(lo, hi), s, b), lo, hi); }
// ReLU6 of two values with one instruction behind the conversion: packed minima and maxima run at half rate and are much of the read-out (with a maximum
// ahead, for which a NaN becomes 0, 6272 x 320 -> 1280 takes 9.1 us in the place of 8.9, 50176 x 64 -> 256 from bf16 15.6 in the place of 15.2).  A NaN becomes 6.
__device__ __forceinline__ uint32_t relu6_fast(float lo, float hi) { return min_bf16x2(pack_bf16x2_relu(lo, hi), 0x40C040C0u); }
// 32 sums of a thread's row -> values of y in its staged row, 16-byte pieces from `first` on at i ^ swap: scale and bias (shared memory, the same
// for all lanes), residual (in place), activation
template <typename T, bool RES, bool RELU6>
__device__ __forceinline__ void finish32(float scale, uint32_t bias, float *v, uint32_t row, uint32_t swap, uint32_t first) {
  constexpr int N = kPer<T>, K = 32 / N;
  uint4 b[8], res[K];
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = lds_u4(bias + (uint32_t)(i * 16));
  if (RES) {
#pragma unroll
    for (int i = 0; i < K; ++i) res[i] = lds_u4(row + ((first + (uint32_t)i) ^ swap) * 16u);
  }
  const uint64_t s = q4::pair(scale, scale);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    fma2(v[4 * i], v[4 * i + 1], s, q4::pair(__uint_as_float(b[i].x), __uint_as_float(b[i].y)));
    fma2(v[4 * i + 2], v[4 * i + 3], s, q4::pair(__uint_as_float(b[i].z), __uint_as_float(b[i].w)));
  }
#pragma unroll
  for (int i = 0; i < K; ++i) {
    float *u = v + i * N;
    if (RES) {
      float r[N];
      unpack16<T>(res[i], r);
#pragma unroll
      for (int j = 0; j < N; ++j) u[j] += r[j];
    }
    uint4 w;
    if (RELU6 && N == 8) {
      w = make_uint4(relu6_fast(u[0], u[1]), relu6_fast(u[2], u[3]), relu6_fast(u[4 % N], u[5 % N]), relu6_fast(u[6 % N], u[7 % N]));
    } else {
      if (RELU6) {
#pragma unroll
        for (int j = 0; j < N; ++j) u[j] = dc_act_apply(u[j], DC_ACT_RELU6);
      }
      w = pack16<T>(u);
    }
    sts_u4(row + ((first + (uint32_t)i) ^ swap) * 16u, w);
  }
}
// H times as many; columns beyond the end of a row are left out
template <typename T, int H, bool RES, bool RELU6>
__device__ __forceinline__ void finish(float scale, uint32_t bias, float (*v)[32], uint32_t row, uint32_t swap, int halves) {
  finish32<T, RES, RELU6>(scale, bias, v[0], row, swap, 0);
  if (H > 1 && halves > 1) finish32<T, RES, RELU6>(scale, bias + 128u, v[H - 1], row, swap, 32 / kPer<T>);
}
template <typename T>
__device__ __forceinline__ void finish_any(const Params &p, bool residual, uint32_t bias, float *v, uint32_t row, uint32_t swap, uint32_t first) {
  if (residual) {
    if (p.act == DC_ACT_RELU6) finish32<T, true, true>(p.scale, bias, v, row, swap, first);
    else finish32<T, true, false>(p.scale, bias, v, row, swap, first);
  } else {
    if (p.act == DC_ACT_RELU6) finish32<T, false, true>(p.scale, bias, v, row, swap, first);
    else finish32<T, false, false>(p.scale, bias, v, row, swap, first);
  }
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, uint32_t ssrc, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(ssrc), "r"(c0),
               "r"(c1)
               : "memory");
}
// columns one by one, where rows of y do not begin on 16 bytes
template <typename T>
__device__ __forceinline__ void deliver_one(const Params &p, float t, float b, const T *residual, T *y, size_t at) {
  t = fmaf(t, p.scale, b);
  if (residual) t += (float)residual[at];
  y[at] = (T)act_of<T>(t, p.act);
}
// the same of a part's sum (split tiles)
template <typename T>
__device__ __forceinline__ void deliver(const Params &p, const float *__restrict__ bias, const T *residual, T *y, long long row, int o, float *v) {
  constexpr int N = kPer<T>;
  const size_t at = (size_t)row * (size_t)p.c_out + (size_t)o;
  if (p.vec) {                                   // rows then have whole pieces
    float b[N];
    load_bias(bias, o, N, b);
    uint4 r = make_uint4(0, 0, 0, 0);
    if (residual) r = *reinterpret_cast<const uint4 *>(residual + at);
    *reinterpret_cast<uint4 *>(y + at) = finish16<T>(p, b, residual != nullptr, r, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (o + i < p.c_out) deliver_one<T>(p, v[i], bias ? __ldg(bias + o + i) : 0.f, residual, y, at + i);
}
// a lane to a column, where rows of y do not begin on 16 bytes; eight rows at once, so that what one waits for the others do not add to
template <typename T, bool RES>
__device__ __forceinline__ void deliver_columns(const Params &p, float b, const T *residual, T *y, int rows, uint32_t sm, int lane) {
  const size_t pitch = (size_t)p.c_out;
  const uint32_t at = sm + (uint32_t)((lane & 3) * 4), piece = (uint32_t)lane >> 2;
#pragma unroll 1
  for (int r0 = 0; r0 < rows; r0 += 8, y += 8 * pitch) {
    float t[8], r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = lds_f(at + (uint32_t)((r0 + i) * 128) + ((piece ^ (uint32_t)i) << 4));
    if (RES) {
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = r0 + i < rows ? (float)residual[i * pitch] : 0.f;
      residual += 8 * pitch;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      t[i] = fmaf(t[i], p.scale, b);
      if (RES) t[i] += r[i];
      t[i] = act_of<T>(t[i], p.act);
    }
    if (r0 + 8 <= rows) {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i * pitch] = (T)t[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r0 + i < rows) y[i * pitch] = (T)t[i];
    }
  }
}

// largest magnitude of 16 values, its bits as fp32
template <typename T>
__device__ __forceinline__ uint32_t largest16(const uint4 *raw) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 16 / kPer<T>; ++i) {
    const uint32_t u[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) top = sizeof(T) == 2 ? __vmaxu2(top, u[j] & 0x7fff7fffu) : max(top, u[j] & 0x7fffffffu);
  }
  return sizeof(T) == 2 ? max(top & 0xffff0000u, top << 16) : top;
}
// 16 columns, piece `seg` of a row, -> codes in an operand's rows and the block's scale in its tile.
template <int F, typename T>
__device__ __forceinline__ void put_x16(float *v, const Params &p, uint32_t a, uint32_t sfa, int row, int seg, bool valid) {
  uint32_t top = q4::largest16(v);
  if (F == DC_MX4) top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  const q4::BlockScale s = q4::block_scale<F>(top, p.g, p.r6);
  const uint2 code = q4::codes16<F, sizeof(T) == 2>(v, s);
  if (valid) {
    const uint32_t at = a + (uint32_t)((row >> 3) * 1024 + (row & 7) * 128 + ((((seg & 15) >> 1) ^ (row & 7)) * 16) + (seg & 1) * 8);
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(code.x), "r"(code.y) : "memory");
    if (F == DC_NV4 || (seg & 1) == 0) {
      const uint32_t b = (uint32_t)(F == DC_NV4 ? seg : seg >> 1);
      asm volatile("st.shared.b8 [%0], %1;" ::"r"(sfa + (b >> 2) * kAtom + q4::scale_at((uint32_t)row, b)), "r"(s.byte) : "memory");
    }
  }
}

enum { kFull = 0, kEmpty = kMaxStages, kDFull = 2 * kMaxStages, kDEmpty = kDFull + kMaxAcc, kXFull = kDEmpty + kMaxAcc, kWFull, kParts, kRes, kBars = kRes + kEpi<kOne> };

template <int F, typename T, int FORM>
__global__ void __launch_bounds__(kThreadsOf<FORM>, 1)
k_q4_product(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_sx, const __grid_constant__ CUtensorMap map_w,
             const __grid_constant__ CUtensorMap map_sw, const __grid_constant__ CUtensorMap map_y, const __grid_constant__ CUtensorMap map_res,
             const T *__restrict__ x, const float *__restrict__ bias, const T *residual, T *y,
             const __grid_constant__ Params p, DcWsHeader *ws) {
  constexpr int kAtoms = kAtomsOf<F>;
  constexpr bool P = FORM == kPair;
  constexpr uint32_t kTmemCols = 512;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bar[kBars];
  __shared__ __align__(16) float bias_s[kEpi<FORM>][P ? 64 : 256];                // of a warp's tile; of a pair, whose stages want the room, of the columns at hand
  __shared__ uint32_t tmem_s, abort_s;
  volatile uint32_t *abort_flag = &abort_s;
  const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sm = (smem_u32(smem_raw) + 1023u) & ~1023u;
  if (warp == 0) {
    // a lane to a barrier: one after the other they took 0.4 us
    for (int i = lane; i < kBars; i += 32) {
      const uint32_t arrivals = i < kEmpty ? (FORM == kStream ? kCutWarps + (p.w_stays ? 0 : 1) : 1)
                                : i >= kDEmpty && i < kXFull ? (P ? 2 : 1) * kEpi<FORM> / p.acc_bufs
                                : i == kXFull ? kEpi<FORM> : i == kParts ? p.split * kEpi<FORM> : 1;
      mbar_init(&bar[i], arrivals);
    }
    if (lane == 0) abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncwarp();
  } else if (warp == 1 && lane < 4) {
    if (lane < 2) prefetch_tensormap(lane ? &map_sw : &map_w);
    else if (FORM == kOne || P) prefetch_tensormap(lane == 2 ? &map_x : &map_sx);
  }
  const bool parts = FORM != kPair && FORM != kStream && p.split > 1;
  if (parts) asm volatile("barrier.cluster.arrive.release;" ::: "memory");     // this CTA is there, its barriers too: waited for before the parts go out
  // Tensor memory only behind the wait for the launch before this one, whose CTAs may still have theirs to ask for.
  dc_pdl_enter();
  if (warp == 1) {
    if (P) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"(kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      tmem_alloc(&tmem_s, kTmemCols);
      tmem_relinquish();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (P) cluster_sync();                         // the barriers of both CTAs are there
  tc_fence_after();
  const uint32_t tmem = tmem_s;

  const int team = P ? 2 : p.split;              // CTAs that share an item
  const int rank = team > 1 ? (int)(blockIdx.x % (unsigned)team) : 0;
  const int team_id = (int)blockIdx.x / team, teams = (int)gridDim.x / team;
  const int first = p.columns ? team_id / p.tiles_n : team_id, step = p.columns ? teams / p.tiles_n : teams;
  const int items = p.columns ? p.tiles_m : p.items, own_tn = p.columns ? team_id % p.tiles_n : 0;
  auto column_of = [&](int item) { return p.columns || p.tiles_n == 1 ? own_tn : item / p.tiles_m; };
  const int c0 = P ? 0 : rank * p.chunks_per, c1 = P ? p.chunks : min(p.chunks, c0 + p.chunks_per);
  const uint32_t sf_base = tmem + (uint32_t)(p.acc_bufs * p.acc);
  auto inside = [&](int tn) { return !P && p.nt < p.acc ? tn * p.nt & 127 : 0; };          // a narrow tile's place among its scale tile's rows
  const uint32_t ring = sm + (uint32_t)p.off_ring, w_base = ring + (uint32_t)(p.stages * p.stage_bytes);
  const int b_rows = P ? p.nt / 2 : p.nt;
  const uint32_t w_codes = (uint32_t)b_rows * 128u;

  if (warp == 0) {
    // ---------------------------------------------------------------- load
    if (p.w_stays && elect_one()) {
      mbar_arrive_expect_tx(&bar[kWFull], (uint32_t)(p.chunks * p.w_bytes));
      for (int ch = 0; ch < p.chunks; ++ch) {
        const uint32_t b = w_base + (uint32_t)(ch * p.w_bytes);
        tma_load_2d(b, &map_w, &bar[kWFull], ch * 128, own_tn * p.nt);
        tma_load_3d(b + w_codes, &map_sw, &bar[kWFull], 0, ch * kAtoms, own_tn * p.nt / 128);
      }
    }
    __syncwarp();
    int stage = 0;
    uint32_t parity = 0;
    bool ok = true;
    if (!(FORM == kStream && p.w_stays))
      for (int item = first; ok && item < items; item += step) {
        const int tn = column_of(item), tm = p.columns ? item : item - tn * p.tiles_m, x_tile = P ? tm * 2 + rank : tm;
        for (int ch = c0; ch < c1; ++ch) {
          ok = warp_wait(&bar[kEmpty + stage], parity ^ 1u, abort_flag, ws, 0x10000u | (uint32_t)stage);
          if (!ok) break;
          if (elect_one()) {
            uint64_t *full = &bar[kFull + stage];
            const uint32_t at = ring + (uint32_t)(stage * p.stage_bytes);
            const uint32_t sfa = at + (uint32_t)p.a_bytes, b = FORM == kRows ? at : sfa + kAtoms * kAtom;
            const uint32_t kX = FORM == kOne || P ? (uint32_t)(p.a_bytes + kAtoms * kAtom) : 0u;
            const uint32_t bytes = kX + (p.w_stays ? 0u : w_codes + (uint32_t)(p.nb * kAtoms * kAtom));
            if (P) {
              const uint32_t to = map_cluster(smem_u32(full), 0);
              if (rank == 0) mbar_arrive_expect_tx(full, 2 * bytes);
              pair_load_2d(at, &map_x, to, ch * 128, x_tile * 128);
              pair_load_3d(sfa, &map_sx, to, 0, ch * kAtoms, x_tile);
              pair_load_2d(b, &map_w, to, ch * 128, tn * p.nt + rank * b_rows);
              pair_load_3d(b + w_codes, &map_sw, to, 0, ch * kAtoms, tn * p.nt / 128);
            } else {
              mbar_arrive_expect_tx(full, bytes);
              if (FORM == kOne) {
                tma_load_2d(at, &map_x, full, ch * 128, x_tile * 128);
                tma_load_3d(sfa, &map_sx, full, 0, ch * kAtoms, x_tile);
              }
              if (!p.w_stays) {
                tma_load_2d(b, &map_w, full, ch * 128, tn * p.nt);
                tma_load_3d(b + w_codes, &map_sw, full, 0, ch * kAtoms, tn * p.nt / 128);
              }
            }
          }
          __syncwarp();
          if (++stage == p.stages) { stage = 0; parity ^= 1u; }
        }
      }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- multiply
    int stage = 0, buf = 0;
    uint32_t parity = 0, use = 0;                // use: of the accumulators, how many times round
    bool ok = !P || rank == 0;
    if (FORM == kRows && ok) ok = warp_wait(&bar[kXFull], 0, abort_flag, ws, 0x50000u);
    if (p.w_stays && ok) ok = warp_wait(&bar[kWFull], 0, abort_flag, ws, 0x60000u);
    // One lane, without the others: with a meeting of the warp for each stage a stage of 128 x 128 took 750 cycles, of which the products are 264.  The next
    // stage's barrier is asked for ahead of this one's instructions.
    if (elect_one()) {
      uint32_t ready = 0;
      for (int item = first; ok && item < items; item += step) {
        ok = mbar_wait(&bar[kDEmpty + buf], (use & 1u) ^ 1u, abort_flag, ws, 0x20000u | (uint32_t)buf);
        if (!ok) break;
        tc_fence_after();
        const uint32_t d = tmem + (uint32_t)(buf * p.acc), idesc = q4_idesc<F>(p.acc, P ? 256 : 128);
        const uint32_t shift = (uint32_t)inside(p.nt < p.acc ? column_of(item) : 0) * 128u;
        for (int ch = c0; ch < c1; ++ch) {
          if (!ready) ok = mbar_wait(&bar[kFull + stage], parity, abort_flag, ws, 0x30000u | (uint32_t)stage);
          if (!ok) break;
          ready = stage + 1 < p.stages ? mbar_test(&bar[kFull + stage + 1], parity) : mbar_test(&bar[kFull], parity ^ 1u);
          const uint32_t at = ring + (uint32_t)(stage * p.stage_bytes);
          const uint32_t a = FORM == kRows ? sm + (uint32_t)((ch - c0) * p.a_bytes) : at;
          const uint32_t sfa = FORM == kRows ? sm + (uint32_t)(p.off_sfa + (ch - c0) * kAtoms * kAtom) : at + (uint32_t)p.a_bytes;
          const uint32_t b = p.w_stays ? w_base + (uint32_t)(ch * p.w_bytes) : (FORM == kRows ? at : at + (uint32_t)p.a_bytes + kAtoms * kAtom), sfb = b + w_codes;
          const uint32_t ta = sf_base + (uint32_t)(stage * p.sf_cols);
          const int steps = min(4, dc_div_up(p.c_in - ch * kStageCols, 64));
          if (p.nb == 2) multiply_steps<F, P, 2>(steps, d, a, b, sfa, sfb, ta, idesc, ch > c0);
          else multiply_steps<F, P, 1>(steps, d, a, b - shift, sfa, sfb, ta, idesc, ch > c0);
          commit<P>(&bar[kEmpty + stage]);
          if (ch == c1 - 1) commit<P>(&bar[kDFull + buf]);
          if (++stage == p.stages) { stage = 0; parity ^= 1u; }
        }
        if (++buf == p.acc_bufs) { buf = 0; ++use; }
      }
    }
    __syncwarp();
  } else if (warp < 2 + kEpi<FORM>) {
    // ---------------------------------------------------------------- read out
    const int quad = warp & 3, set = (warp - 2) >> 2;
    if (FORM == kRows) {
      // the whole rows, as far as this CTA multiplies them, in pieces of 16 columns
      const int segs = (min(p.c_in - c0 * kStageCols, (c1 - c0) * kStageCols) + 63) / 64 * 4, total = (int)p.rows * segs;
      constexpr int kRaw = 16 / kPer<T>, kStep = kEpi<FORM> * 32;
      uint4 next[2][kRaw];                       // the next two pieces of this thread, on their way
      auto ask = [&](int k, int u) {
        const int row = u / segs, col = c0 * kStageCols + (u - row * segs) * 16;
        const uint4 *at = reinterpret_cast<const uint4 *>(x + (size_t)row * (size_t)p.c_in + col);
#pragma unroll
        for (int i = 0; i < kRaw; ++i) next[k][i] = u < total && col + i * kPer<T> < p.c_in ? __ldg(at + i) : make_uint4(0, 0, 0, 0);
      };
      const int u_first = (warp - 2) * 32 + lane;
      if (p.vec_x) {
        ask(0, u_first);
        ask(1, u_first + kStep);
      }
#pragma unroll 1
      for (int u = u_first; u - lane < total; u += 2 * kStep) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int uk = u + k * kStep, row = uk / segs, seg = uk - row * segs;
          if (uk - lane >= total) break;         // the same for all lanes
          float v[16];
          if (p.vec_x) {
#pragma unroll
            for (int i = 0; i < kRaw; ++i) unpack16<T>(next[k][i], v + i * kPer<T>);
            ask(k, uk + 2 * kStep);
          } else {
            const int col = c0 * kStageCols + seg * 16;
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = uk < total && col + i < p.c_in ? (float)x[(size_t)row * (size_t)p.c_in + col + i] : 0.f;
          }
          put_x16<F, T>(v, p, sm + (uint32_t)((seg >> 4) * p.a_bytes), sm + (uint32_t)p.off_sfa, row, seg, uk < total);
        }
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar[kXFull]);
    }
    constexpr int kCols = kOut<T>, kHalves = kCols / 32;
    const uint32_t out0 = sm + (uint32_t)(p.off_out + (warp - 2) * p.out_bufs * kOutBytes), bias_w = smem_u32(bias_s[warp - 2]);
    const uint32_t swap = (uint32_t)lane & 7u;   // 16-byte pieces of a row lie at i ^ swap
    uint32_t turn = 0;
    const uint32_t freed = P ? map_cluster(smem_u32(&bar[kDEmpty]), 0) : 0u;
    // sets of four warps: each takes every acc_bufs-th tile, an accumulator of its own, and shares its columns with the other sets on it
    const int buf = set % p.acc_bufs, c_first = set / p.acc_bufs * kCols, c_step = kEpi<FORM> / 4 / p.acc_bufs * kCols;
    uint32_t use = 0, res_parity = 0;
    int bias_tn = -1;
    bool met = false;                            // the cluster's other CTAs
    for (int item = first + buf * step; item < items; item += p.acc_bufs * step, ++use) {
      const int tn = column_of(item), tm = p.columns ? item : item - tn * p.tiles_m;
      const long long row0 = (long long)(P ? tm * 2 + rank : tm) * 128 + quad * 32;
      const int cols = min(p.nt, p.c_out - tn * p.nt);
      const bool work = row0 < p.rows && c_first < cols, staged = work && !parts && p.vec;
      const uint32_t d = tmem + (uint32_t)(buf * p.acc + inside(tn)) + ((uint32_t)(quad * 32) << 16);
      if (!P && work && !parts && tn != bias_tn) {
        bias_tn = tn;
        __syncwarp();
        for (int i = lane; i < p.nt; i += 32) bias_s[warp - 2][i] = bias && i < cols ? __ldg(bias + tn * p.nt + i) : 0.f;
        __syncwarp();
      }
      bool ok = true;
      auto release = [&](int c) {                // the columns from c on are read: where they are the last of this warp, the next tile may have the accumulator
        constexpr int kRead = P ? 128 / kCols : 1;
        if (c + kRead * c_step < cols) return;
        tc_fence_before();
        __syncwarp();
        if (elect_one()) {
          if (P) arrive_cluster(freed + (uint32_t)(buf * 8));
          else mbar_arrive(&bar[kDEmpty + buf]);
        }
        __syncwarp();
      };
      // A pair reads all of a warp's columns before it works on them: its one accumulator is then free for the next tile's products.  These are 128 sums a
      // lane, of 168 registers: 336 to 352 bytes of them are spilled (66 in the bf16 kernels of single tiles, at 128 registers).
      constexpr int kAhead = P ? 128 / kCols : 1;
#pragma unroll 1
      for (int cc = c_first; cc < cols || cc == c_first; cc += kAhead * c_step) {
        constexpr int kNow = FORM == kStream ? 1 : kHalves;    // 32 columns at a time where registers are few
        float va[kAhead][kNow][32];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int c = cc + k * c_step, col = tn * p.nt + c;
          const bool here = work && c < cols;
          float (*v)[32] = va[k];
          const uint32_t out = out0 + turn * kOutBytes, mine = out + (uint32_t)lane * 128u;
          auto wait_out = [&]() {                // what this buffer held is read
            if (p.out_bufs == 2) bulk_wait_read1();
            else bulk_wait_read0();
          };
          if (P && here) {
            const float b0 = bias && c + lane < cols ? __ldg(bias + col + lane) : 0.f, b1 = bias && c + 32 + lane < cols ? __ldg(bias + col + 32 + lane) : 0.f;
            bias_s[warp - 2][lane] = b0;
            bias_s[warp - 2][lane + 32] = b1;
            __syncwarp();
          }
          if (staged && c < cols && residual) {  // the results before these have been read: the residual to their place
            if (elect_one()) {
              wait_out();
              mbar_arrive_expect_tx(&bar[kRes + warp - 2], kOutBytes);
              tma_load_2d(out, &map_res, &bar[kRes + warp - 2], col, (int)row0);
            }
            __syncwarp();
          }
          if (k == 0) {
            if (cc == c_first) {
              ok = warp_wait(&bar[kDFull + buf], use & 1u, abort_flag, ws, 0x40000u | (uint32_t)buf);
              if (!ok) break;
              tc_fence_after();
            }
            if (work) {
#pragma unroll
              for (int a = 0; a < kAhead; ++a)
#pragma unroll
                for (int h = 0; h < kNow; ++h)
                  if (cc + a * c_step + h * 32 < cols) tmem_ld32(d + (uint32_t)(cc + a * c_step + h * 32), reinterpret_cast<uint32_t *>(va[a][h]));
              tmem_ld_wait();
            }
            if (FORM != kStream || !work) release(cc);
          }
          if (!here) continue;
          if (parts) {
            if (!met) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
            met = true;
            if (row0 + lane < p.rows) {
              // columns to the CTA that owns them
              constexpr int N = kPer<T>;
              const uint32_t from = sm + (uint32_t)(p.off_out + (rank * p.part_rows + quad * 32 + lane) * p.part_cols * 4);
              int owner = c / p.part_cols, at = c - owner * p.part_cols;         // of the next columns: whose, and their place there
#pragma unroll
              for (int i = 0; i < kCols / N; ++i, at += N)
                if (c + i * N < p.nt) {
                  if (at == p.part_cols) { at = 0; ++owner; }
                  const uint32_t to = map_cluster(from + (uint32_t)(at * 4), (uint32_t)owner);
#pragma unroll
                  for (int j = 0; j < N; j += 4) {
                    const float *u = v[(i * N + j) / 32] + (i * N + j) % 32;
                    sts_cluster_f4(to + (uint32_t)(j * 4), u[0], u[1], u[2], u[3]);
                  }
                }
            }
          } else if (p.vec) {
            const uint32_t bias_c = bias_w + (P ? 0u : (uint32_t)(c * 4));
            const int halves = c + 32 < cols ? 2 : 1;
            if (residual) {
              ok = warp_wait(&bar[kRes + warp - 2], res_parity, abort_flag, ws, 0xA0000u | (uint32_t)warp);
              if (!ok) break;
              res_parity ^= 1u;
            } else {
              if (elect_one()) wait_out();
              __syncwarp();
            }
            if (FORM == kStream) {
#pragma unroll
              for (int h = 0; h < kHalves; ++h) {
                if (h > 0 && halves > 1) {
                  tmem_ld32(d + (uint32_t)(c + 32), reinterpret_cast<uint32_t *>(v[0]));
                  tmem_ld_wait();
                }
                if (h == kHalves - 1) release(c);
                if (h > 0 && halves < 2) break;
                finish_any<T>(p, residual != nullptr, bias_c + (uint32_t)(h * 128), v[0], mine, swap, (uint32_t)(h * 32 / kPer<T>));
              }
            } else if (residual) {
              if (p.act == DC_ACT_RELU6) finish<T, kHalves, true, true>(p.scale, bias_c, v, mine, swap, halves);
              else finish<T, kHalves, true, false>(p.scale, bias_c, v, mine, swap, halves);
            } else {
              if (p.act == DC_ACT_RELU6) finish<T, kHalves, false, true>(p.scale, bias_c, v, mine, swap, halves);
              else finish<T, kHalves, false, false>(p.scale, bias_c, v, mine, swap, halves);
            }
            fence_proxy_async();
            __syncwarp();
            if (elect_one()) {
              tma_store_2d(&map_y, out, col, (int)row0);
              bulk_commit();
            }
            __syncwarp();
            if (p.out_bufs == 2) turn ^= 1u;
          } else if (FORM != kStream) {            // (which is for rows of y that begin on 16 bytes)
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float *u = v[h] + i * 4;
                sts_u4(mine + ((uint32_t)i ^ swap) * 16u, make_uint4(__float_as_uint(u[0]), __float_as_uint(u[1]), __float_as_uint(u[2]), __float_as_uint(u[3])));
              }
              __syncwarp();
              const int o = c + h * 32 + lane;
              if (o < cols) {
                const size_t to = (size_t)row0 * (size_t)p.c_out + (size_t)(tn * p.nt + o);
                const int rows = p.rows - row0 < 32 ? (int)(p.rows - row0) : 32;
                const float b = bias_s[warp - 2][P ? o - c : o];
                if (residual) deliver_columns<T, true>(p, b, residual + to, y + to, rows, out, lane);
                else deliver_columns<T, false>(p, b, nullptr, y + to, rows, out, lane);
              }
              __syncwarp();
            }
          }
        }
        if (!ok) break;
      }
      if (!ok) break;
    }
    if (parts) {
      if (!met) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");       // nothing was to be sent
      __syncwarp();
      if (lane < p.split) arrive_cluster(map_cluster(smem_u32(&bar[kParts]), (uint32_t)lane));
      const int tn = first / p.tiles_m, tm = first - tn * p.tiles_m;
      const long long row0 = (long long)tm * 128;
      const int rows = p.rows - row0 < 128 ? (int)(p.rows - row0) : 128, pieces = p.part_cols / kPer<T>;
      const int col0 = rank * p.part_cols, end = min(p.nt, p.c_out - tn * p.nt);
      if (warp_wait(&bar[kParts], 0, abort_flag, ws, 0xB0000u)) {
        mbar_acquire_cluster(&bar[kParts], 0);
        for (int u = (warp - 2) * 32 + lane; u < rows * pieces; u += kEpi<FORM> * 32) {
          const int r = u / pieces, c = (u - r * pieces) * kPer<T>;
          if (col0 + c >= end) continue;
          float v[kPer<T>];
#pragma unroll
          for (int i = 0; i < kPer<T>; ++i) v[i] = 0.f;
          uint32_t at = sm + (uint32_t)(p.off_out + (r * p.part_cols + c) * 4);
          for (int k = 0; k < p.split; ++k, at += (uint32_t)(p.part_rows * p.part_cols * 4)) {
#pragma unroll
            for (int i = 0; i < kPer<T>; i += 4) {
              const uint4 w = lds_u4(at + (uint32_t)(i * 4));
              v[i] += __uint_as_float(w.x); v[i + 1] += __uint_as_float(w.y); v[i + 2] += __uint_as_float(w.z); v[i + 3] += __uint_as_float(w.w);
            }
          }
          deliver<T>(p, bias, residual, y, row0 + r, tn * p.nt + col0 + c, v);
        }
      }
    } else {
      if (elect_one()) bulk_wait_all();          // the last results are read, and written
      __syncwarp();
    }
  } else {
    // ---------------------------------------------------------------- quantise (kStream): a thread to a row, 32 of its up to 64 columns at a time.  The next
    // kDeep runs of 32, of the next tiles, are on their way: with one the loads' latency was a tile's time (200704 x 24 -> 48 20.0 us).
    const int r = (warp - 2 - kEpi<FORM>) * 32 + lane;
    constexpr int kRaw = 32 / kPer<T>, kDeep = sizeof(T) == 2 ? 3 : 2;
    uint4 next[kDeep][kRaw];
    int ask_item = first, ask_c = 0;
    auto ask = [&](uint4 *to) {
      const long long row = (long long)ask_item * 128 + r;
      const uint4 *at = reinterpret_cast<const uint4 *>(x + (size_t)row * (size_t)p.c_in + ask_c);
      const bool here = ask_item < items && row < p.rows;
#pragma unroll
      for (int i = 0; i < kRaw; ++i) to[i] = here && ask_c + i * kPer<T> < p.c_in ? __ldg(at + i) : make_uint4(0, 0, 0, 0);
      ask_c += 32;
      if (ask_c >= p.c_in) { ask_c = 0; ask_item += step; }
    };
#pragma unroll
    for (int k = 0; k < kDeep; ++k) ask(next[k]);
    int item = first, c = 0, stage = 0;
    uint32_t parity = 0;
    bool ok = true;
    while (ok && item < items) {
#pragma unroll
      for (int k = 0; k < kDeep; ++k) {
        if (!ok || item >= items) break;         // the same for all lanes
        if (c == 0) ok = warp_wait(&bar[kEmpty + stage], parity ^ 1u, abort_flag, ws, 0x70000u | (uint32_t)stage);
        if (!ok) break;
        const uint32_t at = ring + (uint32_t)(stage * p.stage_bytes), a = at + (uint32_t)((r >> 3) * 1024 + (r & 7) * 128), sfa = at + kA;
        auto put = [&](int col, uint4 code, uint32_t byte) {
          sts_u4(a + (uint32_t)(((col >> 5) ^ (r & 7)) * 16), code);
          const uint32_t to = sfa + q4::scale_at((uint32_t)r, (uint32_t)(F == DC_NV4 ? col >> 4 : col >> 5));
          if (F == DC_NV4) asm volatile("st.shared.b16 [%0], %1;" ::"r"(to), "h"((uint16_t)byte) : "memory");
          else asm volatile("st.shared.b8 [%0], %1;" ::"r"(to), "r"(byte) : "memory");
        };
        uint32_t top[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) top[h] = largest16<T>(next[k] + h * kRaw / 2);
        if (F == DC_MX4) top[0] = top[1] = max(top[0], top[1]);
        uint2 code[2];
        uint32_t byte = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float v[16];
#pragma unroll
          for (int i = 0; i < kRaw / 2; ++i) unpack16<T>(next[k][h * kRaw / 2 + i], v + i * kPer<T>);
          const q4::BlockScale s = q4::block_scale<F>(top[h], p.g, p.r6);
          code[h] = q4::codes16<F, sizeof(T) == 2>(v, s);
          byte |= F == DC_NV4 ? s.byte << (8 * h) : s.byte;
        }
        ask(next[k]);
        put(c, make_uint4(code[0].x, code[0].y, code[1].x, code[1].y), byte);
        if (c == 0 && p.c_in <= 32) put(32, make_uint4(0, 0, 0, 0), 0);        // what a run of 64 columns has behind the last one is 0
        c += 32;
        if (c < p.c_in) continue;
        c = 0;
        item += step;
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar[kFull + stage]);
        if (++stage == p.stages) { stage = 0; parity ^= 1u; }
      }
    }
  }
  if (parts && warp == 1) {                      // read out: tensor memory goes back while the parts are on their way
    warp_wait(&bar[kDEmpty], 0, abort_flag, ws, 0xC0000u);
    if (*abort_flag) {
      const unsigned long long t0 = globaltimer_ns();
      while (globaltimer_ns() - t0 < 20ull * 1000ull * 1000ull) __nanosleep(1000);
    }
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  } else if (warp == 1 && *abort_flag) {         // copies and products may still be in flight: give them time to end
    const unsigned long long t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 20ull * 1000ull * 1000ull) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (P) {
    cluster_sync();                              // neither CTA's memory is touched by the other's instructions any more
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    return;
  }
  if (parts) {
    if (warp < 2) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    if (*abort_flag) cluster_sync();             // parts may still be on their way here: until the other CTAs are here as well, or gone
  } else if (warp == 1) {
    tmem_dealloc(tmem, kTmemCols);
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
// codes as rows of bytes: boxes of 128 bytes x `box` rows, zeros outside
bool codes_map(EncodeTiledFn encode, CUtensorMap *map, const void *q, size_t pitch, long long rows, int box) {
  const cuuint64_t dim[2] = {(cuuint64_t)pitch, (cuuint64_t)rows}, str[1] = {(cuuint64_t)pitch};
  const cuuint32_t bx[2] = {128, (cuuint32_t)box}, es[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(q), dim, str, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// scale tiles: boxes of one stage of `tiles` x 128 rows
bool scales_map(EncodeTiledFn encode, CUtensorMap *map, const void *q, const q4::Layout &l, long long rows, int atoms, int tiles) {
  const cuuint64_t dim[3] = {kAtom / 4, (cuuint64_t)l.tiles, (cuuint64_t)((rows + 127) / 128)}, str[2] = {kAtom, (cuuint64_t)l.tiles * kAtom};
  const cuuint32_t bx[3] = {kAtom / 4, (cuuint32_t)atoms, (cuuint32_t)tiles}, es[3] = {1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, (char *)const_cast<void *>(q) + l.scale_offset, dim, str, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// y, or the residual: boxes of what a warp reads out at a time
template <typename T>
bool results_map(EncodeTiledFn encode, CUtensorMap *map, const void *y, const Params &p) {
  const cuuint64_t dim[2] = {(cuuint64_t)p.c_out, (cuuint64_t)p.rows}, str[1] = {(cuuint64_t)p.c_out * sizeof(T)};
  const cuuint32_t bx[2] = {(cuuint32_t)kOut<T>, 32}, es[2] = {1, 1};
  return encode(map, sizeof(T) == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, const_cast<void *>(y), dim, str, bx, es,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Call {
  const void *x, *w;
  const q4::Layout *lx, *lw;
  const float *bias;
  const void *residual;
  void *y;
  DcWsHeader *ws;
  int n_sm;
  cudaStream_t st;
};
template <int F, typename T, int FORM>
cudaError_t launch(Params &p, const Call &c) {
  static unsigned char attr_done[kDcMaxDevices];
  const cudaError_t e = dc_set_max_smem_once(k_q4_product<F, T, FORM>, kSmemOf<FORM>, attr_done);
  if (e != cudaSuccess) return e;
  EncodeTiledFn encode = get_encode_fn();
  if (!encode) return cudaErrorNotSupported;
  CUtensorMap map_x = {}, map_sx = {}, map_w, map_sw, map_y = {}, map_res = {};
  constexpr int kAtoms = kAtomsOf<F>;
  if (!codes_map(encode, &map_w, c.w, c.lw->pitch, p.c_out, FORM == kPair ? p.nt / 2 : p.nt) || !scales_map(encode, &map_sw, c.w, *c.lw, p.c_out, kAtoms, p.nb))
    return cudaErrorNotSupported;
  if ((FORM == kOne || FORM == kPair) &&
      (!codes_map(encode, &map_x, c.x, c.lx->pitch, p.rows, p.a_bytes / 128) || !scales_map(encode, &map_sx, c.x, *c.lx, p.rows, kAtoms, 1)))
    return cudaErrorNotSupported;
  if (p.vec && (!results_map<T>(encode, &map_y, c.y, p) || (c.residual && !results_map<T>(encode, &map_res, c.residual, p)))) return cudaErrorNotSupported;
  const int team = FORM == kPair ? 2 : p.split;
  const int columns = p.columns ? c.n_sm / p.tiles_n * p.tiles_n : 0;
  const int grid = columns ? columns : team > 1 ? (p.items * team < c.n_sm / team * team ? p.items * team : c.n_sm / team * team) : (p.items < c.n_sm ? p.items : c.n_sm);
  // all of a CTA's shared memory is asked for: two CTAs on an SM would each want all of its tensor memory
  return dc_launch_pdl_cluster(k_q4_product<F, T, FORM>, dim3((unsigned)grid), dim3(kThreadsOf<FORM>), (size_t)kSmemOf<FORM>, c.st, team, map_x, map_sx, map_w,
                               map_sw, map_y, map_res, FORM == kRows || FORM == kStream ? (const T *)c.x : (const T *)nullptr, c.bias, (const T *)c.residual, (T *)c.y, p, c.ws);
}

// Shared and tensor memory of a form, tile width and split; false: it does not fit.
bool lay_out(Params *p, int form, int format, int dtype, int n_sm) {
  const int atoms = format == DC_NV4 ? 4 : 2;
  p->nb = p->nt > 128 ? 2 : 1;
  p->w_bytes = (form == kPair ? p->nt / 2 : p->nt) * 128 + p->nb * atoms * kAtom;
  p->sf_cols = 4 * atoms * (1 + p->nb);
  const int epi = form == kOne || form == kStream ? kEpi<kOne> : kEpi<kPair>, at_once = form == kPair ? n_sm / 2 : n_sm;
  const bool many = p->split == 1 && p->items > at_once;       // CTAs have several tiles
  p->acc_bufs = many && epi / 4 * p->nt + 3 * p->sf_cols <= 512 ? epi / 4 : 1;
  const bool narrow = p->tiles_n > 1 && p->nt < 128;
  if (narrow && (many || p->split > 1)) return false;
  p->acc = narrow ? 128 : p->nt;
  if (narrow) p->vec = 0;
  // a column of tiles to a CTA, where that leaves none idle for long: w is loaded once, and 148 SMs do not all ask for the same part of it
  p->columns = 0;
  if (many && form != kPair && p->tiles_n <= at_once) {
    const int rows_at_once = at_once / p->tiles_n;
    const double kept = (double)p->tiles_m / (dc_div_up(p->tiles_m, rows_at_once) * (double)rows_at_once) * (rows_at_once * p->tiles_n) / at_once;
    p->columns = p->tiles_n == 1 || kept > 0.8;
  }
  // x's codes: few rows are loaded alone, and the products read on into what lies behind them, sums that nobody reads
  p->a_bytes = form == kOne || form == kRows ? (p->rows < 128 ? (int)dc_round_up((size_t)p->rows, 8) * 128 : kA) : kA;
  const int x_bytes = form == kRows ? 0 : p->a_bytes + atoms * kAtom, smem = form == kPair ? kSmemOf<kPair> : kSmemOf<kOne>;
  p->out_bufs = form == kOne || form == kStream ? (p->chunks <= 4 && many ? 2 : 1) : 1;
  // the staged results, or the parts from a cluster's CTAs, lie last; an operand is read on into them
  const int per = dtype == DC_F32 ? 4 : 8;
  p->part_rows = p->rows < 128 ? (int)p->rows : 128;
  p->part_cols = dc_div_up(dc_div_up(p->nt, per), p->split) * per;
  int last = p->split > 1 ? p->split * p->part_rows * p->part_cols * 4 : epi * p->out_bufs * kOutBytes;
  if (last < kA) last = kA;
  int room = smem - 1024 - last;
  p->off_sfa = p->off_ring = 0;
  if (form == kRows) {
    p->off_sfa = p->chunks_per * p->a_bytes;
    p->off_ring = p->off_sfa + p->chunks_per * atoms * kAtom;                  // a multiple of 1024
  }
  if (narrow && p->off_ring < (128 - p->nt) * 128) p->off_ring = (128 - p->nt) * 128;     // what a narrow tile's products read in front of its codes
  room -= p->off_ring;
  p->w_stays = p->columns && (form == kOne || form == kStream) && (long long)p->chunks * p->w_bytes + 4ll * x_bytes <= room;
  if (p->w_stays) room -= p->chunks * p->w_bytes;
  p->stage_bytes = x_bytes + (p->w_stays ? 0 : p->w_bytes);    // multiples of 1024: nt is one of 16, a stage's scales are of 1024
  p->stages = room / p->stage_bytes;
  if (p->stages > kMaxStages) p->stages = kMaxStages;
  if (p->acc_bufs * p->acc + p->stages * p->sf_cols > 512) p->stages = (512 - p->acc_bufs * p->acc) / p->sf_cols;
  p->off_out = p->off_ring + p->stages * p->stage_bytes + (p->w_stays ? p->chunks * p->w_bytes : 0);
  return p->stages >= 2;
}

// Estimated time of a form in microseconds, fitted to products in all their forms (1 to 200704 rows, 16 to 8192 columns of either operand): of 106
// calls timed in all their forms (1 to 401408 rows; products and forward calls) the chosen one took 1.2 % longer than the best on average, 14 % at most.
// A stage takes its products or its loads; a tile's results go out beside the next tile's products where they have an accumulator of their own.
// A cluster costs its meetings, and its parts their way between SMs.  Of the start 3.2 us, launch and first loads.
double estimate(const Params &p, int form, int dtype, int n_sm) {
  static constexpr int kClusters[kMaxSplit + 1] = {0, 148, 74, 45, 33, 26, 22, 15, 15};    // of that many CTAs that run at once, on 148 SMs
  const bool narrow = p.nt < p.acc;
  const double wide = p.acc / 128.0, type = dtype == DC_F32 ? 1.8 : 1.0;
  const double stage = form == kPair ? (p.nt > 128 ? 0.47 : 0.43) : p.nt > 128 ? 0.44 + 0.16 * (wide - 1) : 0.3 + 0.14 * wide;
  const double w_total = (double)p.tiles_n * p.w_bytes * p.chunks * (form == kPair ? 2 : 1) / 4.5e6;
  double cut = form == kRows ? 256.0 * p.rows * p.chunks_per * 115e-6 - 1.0 : 0;      // quantising; beside the first loads
  if (cut < 0) cut = 0;
  if (p.split > 1) {
    const double main = p.chunks_per * stage, waves = dc_div_up(p.items, kClusters[p.split]);
    return 3.2 + waves * ((main > w_total ? main : w_total) + 1.2 + 0.4 * p.split + p.part_rows * p.nt * 4 / 16e3) +
           cut;
  }
  const int at_once = form == kPair ? n_sm / 2 : n_sm;
  const double waves = p.columns ? dc_div_up(p.tiles_m, at_once / p.tiles_n) : dc_div_up(p.items, at_once);
  double main = p.chunks * stage, out = (form == kPair ? (p.nt > 128 ? 2.2 : 2.0) : wide) * type;
  main += cut;
  if (narrow) out = 0.7 + (dtype == DC_F32 ? 0.2 : 0.7) * p.nt / 32;
  else if (!p.vec) out *= dtype == DC_F32 ? 1.5 : 2.3;
  if (form == kStream) return 3.2 + waves * ((dtype == DC_F32 ? 1.2 : 0.65) * dc_div_up(p.c_in, 32) + 0.95 * out);   // fitted as a sum: the two take turns on a tile, no pipe is busy for more than a third of the time
  const double total = 3.2 + (p.acc_bufs > 1 ? waves * (main > out ? main : out) : waves * (main + out));
  return total > 3.2 + w_total ? total : 3.2 + w_total;
}

// Fills p for the form that takes the least of the estimates.  Tiles of fewer than all of w's rows begin where a scale tile does, with 128 or
// 256 rows, or are narrow, a part of one: where few tiles leave SMs idle and reading out is most of the time, more CTAs then read out (1001 x 1000 -> 1003
// in fp32 7.1 us; tiles of 128 columns 9.2, halves of their reductions in a cluster 14).
int choose(Params *p, bool raw, int format, int dtype, int n_sm, double *us_of) {
  double best = 1e30;
  Params best_p = *p;
  int best_form = -1;
  const int whole = (int)dc_round_up((size_t)p->c_out, 16);
  auto look = [&](int form, int nt, int split) {
    Params q = *p;
    q.nt = nt;
    q.split = split;
    q.chunks_per = dc_div_up(q.chunks, split);
    q.tiles_n = dc_div_up(q.c_out, nt);
    q.tiles_m = (int)(form == kPair ? (q.rows + 255) / 256 : (q.rows + 127) / 128);
    if ((long long)q.tiles_m * q.tiles_n > 0x3fffffffll) return;
    q.items = q.tiles_m * q.tiles_n;
    if (split > 1 && (q.chunks_per * (split - 1) >= q.chunks || (long long)q.items * split > n_sm)) return;     // no CTA without a stage
    if (!lay_out(&q, form, format, dtype, n_sm)) return;
    const double us = estimate(q, form, dtype, n_sm);
    if (us < best) { best = us; best_p = q; best_form = form; }
  };
  if (raw && p->rows <= kMaxRows) {
    for (int s = 1; s <= kMaxSplit; ++s) look(kRows, whole < 128 ? whole : 128, s);
  } else if (raw) {
    if (p->c_in <= 64 && whole <= 256 && p->vec_x && p->vec) look(kStream, whole, 1);
  } else {
    for (int n = 128; n <= 256; n += 128) {
      for (int s = 1; s <= kMaxSplit; ++s) look(kOne, whole < n ? whole : n, s);
      if (whole <= n) break;
    }
    for (int n = 32; n < 128 && n < whole; n *= 2) look(kOne, n, 1);
    if (p->rows > 128 && whole > 128) {
      look(kPair, 256, 1);
      look(kPair, 128, 1);
    }
  }
  *p = best_p;
  *us_of = best;
  return best_form;
}

template <int F, typename T>
cudaError_t launch_form(int form, Params &p, const Call &c) {
  switch (form) {
    case kOne: return launch<F, T, kOne>(p, c);
    case kPair: return launch<F, T, kPair>(p, c);
    case kRows: return launch<F, T, kRows>(p, c);
    default: return launch<F, T, kStream>(p, c);
  }
}
dc_status run(int form, Params &p, dc_q4_format format, dc_dtype dtype, Call &c) {
  if (form < 0) return DC_ERR_UNSUPPORTED;
  cudaError_t e;
  if (format == DC_MX4) e = dtype == DC_BF16 ? launch_form<DC_MX4, __nv_bfloat16>(form, p, c) : launch_form<DC_MX4, float>(form, p, c);
  else e = dtype == DC_BF16 ? launch_form<DC_NV4, __nv_bfloat16>(form, p, c) : launch_form<DC_NV4, float>(form, p, c);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? DC_OK : DC_ERR_CUDA;
}

dc_status check(const void *x, long long rows, int c_in, const void *w, int c_out, dc_q4_format format, const void *bias, dc_act act,
                const void *residual, const void *y, dc_dtype dtype, const void *workspace, size_t workspace_bytes, q4::Layout *lx, q4::Layout *lw) {
  dc_status s = q4::layout_of(rows, c_in, format, lx);
  if (s == DC_OK) s = q4::layout_of(c_out, c_in, format, lw);
  if (s != DC_OK) return s;
  if (!x || !w || !y || (dtype != DC_F32 && dtype != DC_BF16) || (act != DC_ACT_IDENTITY && act != DC_ACT_RELU6)) return DC_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < sizeof(DcWsHeader)) return DC_ERR_WORKSPACE;
  if (!dc_aligned16(x) || !dc_aligned16(w) || !dc_aligned16(y) || !dc_aligned16(bias) || !dc_aligned16(residual) || !dc_aligned16(workspace))
    return DC_ERR_ALIGNMENT;
  return DC_OK;
}

Params params_of(long long rows, int c_in, int c_out, dc_act act, dc_dtype dtype, float scale) {
  Params p = {};
  p.rows = rows;
  p.c_in = c_in;
  p.c_out = c_out;
  p.act = (int)act;
  p.scale = scale;
  p.g = 1.f;
  p.r6 = 1.f / 6.f;
  p.chunks = dc_div_up(c_in, kStageCols);
  const size_t es = dtype == DC_F32 ? 4 : 2;
  p.vec = (size_t)c_out * es % 16 == 0;
  p.vec_x = (size_t)c_in * es % 16 == 0;
  return p;
}

// Whether a forward call quantises in the product's launch (p, form) or in one of its own before it (q, apart: 2 us, and its bytes at what it moves of them).
bool in_one_launch(Params *p, Params *q, dc_q4_format format, dc_dtype dtype, int n_sm, int *form, int *apart) {
  double us, us_apart;
  *form = choose(p, true, format, dtype, n_sm, &us);
  *apart = choose(q, false, format, dtype, n_sm, &us_apart);
  const double row = p->c_in * (dtype == DC_F32 ? 4.0 : 2.0) + (p->c_in < 64 ? 36.0 : p->c_in * 0.57);
  // a product that keeps all of w waits 2 us for it behind the launch that quantised
  return *form >= 0 && us <= us_apart + (q->w_stays && q->tiles_n == 1 ? 4.0 : 2.0) + (double)p->rows * row / 3.5e6;
}

}  // namespace

extern "C" dc_status dc_q4_plan_query(long long rows, int c_in, int c_out, dc_q4_format format, dc_dtype dtype, int forward, dc_q4_plan *plan) {
  q4::Layout lx, lw;
  dc_status s = q4::layout_of(rows, c_in, format, &lx);
  if (s == DC_OK) s = q4::layout_of(c_out, c_in, format, &lw);
  if (s != DC_OK) return s;
  if (!plan || (dtype != DC_F32 && dtype != DC_BF16)) return DC_ERR_INVALID_ARG;
  const int n_sm = dc_sm_count();
  Params p = params_of(rows, c_in, c_out, DC_ACT_IDENTITY, dtype, 1.f), q = p;
  int form = -1, apart;
  double us;
  if (!forward || !in_one_launch(&p, &q, format, dtype, n_sm, &form, &apart)) {
    p = params_of(rows, c_in, c_out, DC_ACT_IDENTITY, dtype, 1.f);
    form = choose(&p, false, format, dtype, n_sm, &us);
  }
  if (form < 0) return DC_ERR_UNSUPPORTED;
  plan->form = (dc_q4_form)form;
  plan->launches = forward && form != kRows && form != kStream ? 2 : 1;
  plan->tile_cols = p.nt;
  plan->split = p.split;
  plan->stages = p.stages;
  plan->accumulators = p.acc_bufs;
  plan->columns = p.columns;
  plan->w_stays = p.w_stays;
  return DC_OK;
}

extern "C" dc_status dc_q4_workspace_bytes(long long rows, int c_in, dc_q4_format format, size_t *bytes) {
  q4::Layout l;
  const dc_status s = q4::layout_of(rows, c_in, format, &l);
  if (s != DC_OK) return s;
  if (!bytes) return DC_ERR_INVALID_ARG;
  *bytes = sizeof(DcWsHeader) + l.bytes;
  return DC_OK;
}

extern "C" dc_status dc_q4_product(const void *x, long long rows, int c_in, const void *w, int c_out, dc_q4_format format, float scale,
                                   const float *bias, dc_act act, const void *residual, void *y, dc_dtype dtype, void *workspace,
                                   size_t workspace_bytes, dc_stream stream) {
  q4::Layout lx, lw;
  const dc_status s = check(x, rows, c_in, w, c_out, format, bias, act, residual, y, dtype, workspace, workspace_bytes, &lx, &lw);
  if (s != DC_OK) return s;
  if (!(scale - scale == 0.f)) return DC_ERR_INVALID_ARG;
  Params p = params_of(rows, c_in, c_out, act, dtype, scale);
  Call c = {x, w, &lx, &lw, bias, residual, y, (DcWsHeader *)workspace, dc_sm_count(), (cudaStream_t)stream};
  double us;
  const int form = choose(&p, false, format, dtype, c.n_sm, &us);
  return run(form, p, format, dtype, c);
}

extern "C" dc_status dc_q4_forward(const void *x, long long rows, int c_in, const void *w, int c_out, dc_q4_format format, float x_scale,
                                   float w_scale, const float *bias, dc_act act, const void *residual, void *y, dc_dtype dtype,
                                   void *workspace, size_t workspace_bytes, dc_stream stream) {
  q4::Layout lx, lw;
  dc_status s = check(x, rows, c_in, w, c_out, format, bias, act, residual, y, dtype, workspace, workspace_bytes, &lx, &lw);
  if (s != DC_OK) return s;
  if (!q4::tensor_scale_ok(x_scale, format) || !q4::tensor_scale_ok(w_scale, format)) return DC_ERR_INVALID_ARG;
  const float scale = x_scale * w_scale;
  if (!(scale - scale == 0.f) || scale == 0.f) return DC_ERR_INVALID_ARG;         // powers of two: exact from 2^-149 on
  if (workspace_bytes < sizeof(DcWsHeader) + lx.bytes) return DC_ERR_WORKSPACE;
  Params p = params_of(rows, c_in, c_out, act, dtype, scale);
  p.g = x_scale;
  p.r6 = 1.f / (6.f * x_scale);
  Call c = {x, w, &lx, &lw, bias, residual, y, (DcWsHeader *)workspace, dc_sm_count(), (cudaStream_t)stream};
  Params q = params_of(rows, c_in, c_out, act, dtype, scale);
  int form, apart;
  if (in_one_launch(&p, &q, format, dtype, c.n_sm, &form, &apart)) return run(form, p, format, dtype, c);
  uint8_t *xq = (uint8_t *)workspace + sizeof(DcWsHeader);
  s = dc_q4_quantize(x, rows, c_in, c_in, dtype, format, x_scale, xq, stream);
  if (s != DC_OK) return s;
  c.x = xq;
  return run(apart, q, format, dtype, c);
}
