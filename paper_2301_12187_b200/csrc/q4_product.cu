// Products of matrices in microscaled 4 bits on the tensor core (dc_q4_product, dc_q4_forward).
//
// tcgen05.mma.block_scale multiplies 64 columns of 128 rows x NT rows at a time: codes from shared memory (rows of 128 bytes, 256 codes, TMA
// with the 128-byte swizzle), scales from tensor memory, where tcgen05.cp puts them from the tiles in which a quantised matrix keeps them
// (32 lanes x 4 columns, one for each 32 rows of the tile; four bytes a column, which are four blocks).  DC_NV4: a tile is one instruction's
// scales; DC_MX4: two instructions', told apart by the descriptor's scale id.  Sums are fp32 in tensor memory.
//
// A stage of the ring is 256 columns: codes of both operands and their scale tiles; its scales have columns of tensor memory of their own, so a
// slot's scales are written over only behind the products that read them.  One warp loads, one issues, eight read out the accumulators
// (two sets where they fit), each thread one row.  A CTA walks over tiles; few tiles: a cluster shares a tile's columns and adds the parts
// up in rank order, through shared memory.  Tensor memory is given back before the CTAs of a cluster wait for one another: who holds
// some never waits for a CTA that may be waiting for some.
#include <string.h>

#include "q4.cuh"
#include "tc_ptx.cuh"

namespace {
using namespace tc;
using q4::kAtom;

constexpr int kEpiWarps = 8, kThreads = (2 + kEpiWarps) * 32;
constexpr int kMaxStages = 8, kMaxSplit = 8;
constexpr int kSmemMax = 225 * 1024;
constexpr int kStageCols = 256;                  // columns of a stage: 128 bytes of codes

struct Params {
  long long rows;
  int c_in, c_out, act;
  float scale;
  int tiles_m, tiles_n, items;
  int chunks, atoms;         // stages of a row; scale tiles of a row of them
  int split, chunks_per;     // CTAs that share an item, stages of each
  int stages, acc_bufs;
  int vec;                   // rows of y begin on 16 bytes
  const uint8_t *sx, *sw;    // scale tiles
};

template <int F, int NT>
struct Shape {
  static constexpr int kAtoms = F == DC_NV4 ? 4 : 2;             // scale tiles of a stage, for 128 rows
  static constexpr int kNb = NT > 128 ? 2 : 1;                   // 128-row tiles that NT rows touch
  static constexpr int kA = 128 * 128, kB = NT * 128, kSfa = kAtoms * kAtom, kSfb = kNb * kAtoms * kAtom;
  static constexpr int kStage = kA + kB + kSfa + kSfb;
  static constexpr int kSfCols = 4 * kAtoms * (1 + kNb);         // tensor memory of a stage's scales
  static_assert(kStage % 1024 == 0, "operands begin on 1024 bytes");
};

__device__ __forceinline__ uint64_t operand_desc(uint32_t a) {   // K-major, 128-byte swizzle, 1024 bytes between groups of 8 rows
  return ((uint64_t)((64u) | (1u << 14) | (2u << 29)) << 32) | (uint64_t)((a >> 4) & 0x3FFFu) | (1u << 16);
}
__device__ __forceinline__ uint64_t scales_desc(uint32_t a) {    // a scale tile: 32 rows of 16 bytes, 128 between groups of 8
  return ((uint64_t)((8u) | (1u << 14)) << 32) | (uint64_t)((a >> 4) & 0x3FFFu) | (1u << 16);
}
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
template <int F>
__device__ __forceinline__ void mma_q4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  if (F == DC_NV4)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
// instruction descriptor: e2m1 x e2m1, N, M = 128, type of the scales; `id`: which half of a scale word (DC_MX4)
template <int F>
__device__ __forceinline__ uint32_t q4_idesc(int n, uint32_t id) {
  return (id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((F == DC_MX4 ? 1u : 0u) << 23) | (1u << 27) | (id << 29);
}

// 16 results of a row, from column `o`: bias, residual, activation, store
template <typename T>
__device__ __forceinline__ void deliver16(const Params &p, const float *__restrict__ bias, const T *residual, T *y, long long row, int o, float *v) {
  const size_t at = (size_t)row * (size_t)p.c_out + (size_t)o;
  if (o + 16 <= p.c_out && p.vec) {
    float r[16];
    if (residual) {
      if (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint4 w = reinterpret_cast<const uint4 *>(residual + at)[i];
          const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) { r[8 * i + 2 * j] = __uint_as_float(u[j] << 16); r[8 * i + 2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u); }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<float4 *>(r + 4 * i) = reinterpret_cast<const float4 *>(residual + at)[i];
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float s = v[i] * p.scale;
      if (bias) s += __ldg(bias + o + i);
      if (residual) s += r[i];
      v[i] = dc_act_apply(s, p.act);
    }
    if (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        reinterpret_cast<uint4 *>(y + at)[i] = make_uint4(pack_bf16x2(v[8 * i], v[8 * i + 1]), pack_bf16x2(v[8 * i + 2], v[8 * i + 3]),
                                                          pack_bf16x2(v[8 * i + 4], v[8 * i + 5]), pack_bf16x2(v[8 * i + 6], v[8 * i + 7]));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) reinterpret_cast<float4 *>(y + at)[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (o + i < p.c_out) {
      float s = v[i] * p.scale;
      if (bias) s += __ldg(bias + o + i);
      if (residual) s += sizeof(T) == 2 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(residual)[at + i]) : reinterpret_cast<const float *>(residual)[at + i];
      s = dc_act_apply(s, p.act);
      if (sizeof(T) == 2) reinterpret_cast<__nv_bfloat16 *>(y)[at + i] = __float2bfloat16_rn(s);
      else reinterpret_cast<float *>(y)[at + i] = s;
    }
}

enum { kFull = 0, kEmpty = kMaxStages, kDFull = 2 * kMaxStages, kDEmpty = kDFull + 2, kBars = kDEmpty + 2 };

template <int F, int NT, typename T>
__global__ void __launch_bounds__(kThreads, 1)
k_q4_product(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const float *__restrict__ bias,
             const T *residual, T *y, const __grid_constant__ Params p, DcWsHeader *ws) {
  using S = Shape<F, NT>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bar[kBars];
  __shared__ uint32_t tmem_s, abort_s;
  volatile uint32_t *abort_flag = &abort_s;
  const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sm = (smem_u32(smem_raw) + 1023u) & ~1023u;
  constexpr uint32_t kTmemCols = 512;
  if (warp == 0) {
    if (lane == 0) {
      abort_s = 0;
      for (int i = 0; i < kMaxStages; ++i) { mbar_init(&bar[kFull + i], 1); mbar_init(&bar[kEmpty + i], 1); }
      for (int i = 0; i < 2; ++i) { mbar_init(&bar[kDFull + i], 1); mbar_init(&bar[kDEmpty + i], kEpiWarps); }
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      prefetch_tensormap(&map_x);
      prefetch_tensormap(&map_w);
    }
    __syncwarp();
  } else if (warp == 1) {
    tmem_alloc(&tmem_s, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_s;
  dc_pdl_enter();

  const int rank = p.split > 1 ? (int)(blockIdx.x % (unsigned)p.split) : 0;
  const int first = (int)blockIdx.x / p.split, step = (int)gridDim.x / p.split;
  const int c0 = rank * p.chunks_per, c1 = min(p.chunks, c0 + p.chunks_per);
  const uint32_t sf_base = tmem + (uint32_t)(p.acc_bufs * NT);

  if (warp == 0) {
    int stage = 0;
    uint32_t parity = 0;
    bool ok = true;
    for (int item = first; ok && item < p.items; item += step) {
      const int tm = item % p.tiles_m, tn = item / p.tiles_m;
      for (int ch = c0; ch < c1; ++ch) {
        ok = warp_wait(&bar[kEmpty + stage], parity ^ 1u, abort_flag, ws, 0x10000u | (uint32_t)stage);
        if (!ok) break;
        if (elect_one()) {
          const uint32_t a = sm + (uint32_t)stage * S::kStage, b = a + S::kA, sfa = b + S::kB, sfb = sfa + S::kSfa;
          const int na = min(S::kAtoms, p.atoms - ch * S::kAtoms);
          const int wt0 = tn * NT / 128, nb = min(S::kNb, dc_div_up(p.c_out, 128) - wt0);
          uint64_t *full = &bar[kFull + stage];
          mbar_arrive_expect_tx(full, (uint32_t)(S::kA + S::kB + na * kAtom * (1 + nb)));
          tma_load_2d(a, &map_x, full, ch * 128, tm * 128);
          tma_load_2d(b, &map_w, full, ch * 128, tn * NT);
          bulk_load(sfa, p.sx + ((size_t)tm * p.atoms + (size_t)ch * S::kAtoms) * kAtom, (uint32_t)(na * kAtom), full);
          for (int i = 0; i < nb; ++i)
            bulk_load(sfb + (uint32_t)(i * S::kAtoms * kAtom), p.sw + ((size_t)(wt0 + i) * p.atoms + (size_t)ch * S::kAtoms) * kAtom, (uint32_t)(na * kAtom), full);
        }
        __syncwarp();
        if (++stage == p.stages) { stage = 0; parity ^= 1u; }
      }
    }
  } else if (warp == 1) {
    int stage = 0, n = 0;
    uint32_t parity = 0;
    bool ok = true;
    for (int item = first; ok && item < p.items; item += step, ++n) {
      const int buf = p.acc_bufs == 2 ? n & 1 : 0;
      const uint32_t use = (uint32_t)(p.acc_bufs == 2 ? n >> 1 : n);
      ok = warp_wait(&bar[kDEmpty + buf], (use & 1u) ^ 1u, abort_flag, ws, 0x20000u | (uint32_t)buf);
      if (!ok) break;
      tc_fence_after();
      const uint32_t d = tmem + (uint32_t)(buf * NT);
      for (int ch = c0; ch < c1; ++ch) {
        ok = warp_wait(&bar[kFull + stage], parity, abort_flag, ws, 0x30000u | (uint32_t)stage);
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
          const uint32_t a = sm + (uint32_t)stage * S::kStage, b = a + S::kA, sfa = b + S::kB, sfb = sfa + S::kSfa;
          const uint32_t ta = sf_base + (uint32_t)(stage * S::kSfCols), tb = ta + 4u * S::kAtoms;
          const int na = min(S::kAtoms, p.atoms - ch * S::kAtoms), steps = min(4, dc_div_up(p.c_in - ch * kStageCols, 64));
          for (int i = 0; i < na; ++i) {
            copy_scales(ta + 4u * i, scales_desc(sfa + (uint32_t)(i * kAtom)));
#pragma unroll
            for (int j = 0; j < S::kNb; ++j) copy_scales(tb + 4u * (uint32_t)(i * S::kNb + j), scales_desc(sfb + (uint32_t)((j * S::kAtoms + i) * kAtom)));
          }
          const uint64_t ad = operand_desc(a), bd = operand_desc(b);
          for (int k = 0; k < steps; ++k) {
            const uint32_t atom = F == DC_NV4 ? (uint32_t)k : (uint32_t)(k >> 1), id = F == DC_NV4 ? 0u : (uint32_t)(k & 1) * 2u;
            mma_q4<F>(d, ad + 2u * k, bd + 2u * k, q4_idesc<F>(NT, id), ta + 4u * atom, tb + 4u * S::kNb * atom, ch > c0 || k > 0 ? 1u : 0u);
          }
          umma_commit(&bar[kEmpty + stage]);
          if (ch == c1 - 1) umma_commit(&bar[kDFull + buf]);
        }
        __syncwarp();
        if (++stage == p.stages) { stage = 0; parity ^= 1u; }
      }
    }
  } else {
    const int quad = warp & 3, half = (warp - 2) >> 2, r = quad * 32 + lane;
    int n = 0;
    for (int item = first; item < p.items; item += step, ++n) {
      const int buf = p.acc_bufs == 2 ? n & 1 : 0;
      const uint32_t use = (uint32_t)(p.acc_bufs == 2 ? n >> 1 : n);
      const int tm = item % p.tiles_m, tn = item / p.tiles_m;
      const long long row = (long long)tm * 128 + r;
      if (!warp_wait(&bar[kDFull + buf], use & 1u, abort_flag, ws, 0x40000u | (uint32_t)buf)) break;
      tc_fence_after();
      const uint32_t d = tmem + (uint32_t)(buf * NT) + ((uint32_t)(quad * 32) << 16);
#pragma unroll 1
      for (int c = half * (NT / 2); c < (half + 1) * (NT / 2); c += 16) {
        float v[16];
        tmem_ld16(d + (uint32_t)c, reinterpret_cast<uint32_t *>(v));
        tmem_ld_wait();
        if (p.split > 1) {
          if (row < p.rows) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              asm volatile("st.shared.f32 [%0], %1;" ::"r"(sm + (uint32_t)(((c + i) * 128 + r) * 4)), "f"(v[i]) : "memory");
          }
        } else if (row < p.rows) {
          deliver16<T>(p, bias, residual, y, row, tn * NT + c, v);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar[kDEmpty + buf]);
    }
  }
  if (warp == 1 && *abort_flag) {                // copies and products may still be in flight: give them time to end
    const unsigned long long t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 20ull * 1000ull * 1000ull) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, kTmemCols);
  if (p.split > 1) {
    // the parts, [column][row], added up in rank order; each CTA delivers a share of the columns, 16 at a time
    cluster_sync();
    const int tm = first % p.tiles_m, tn = first / p.tiles_m;
    if (abort_s == 0) {
      for (int u = tid; u < 128 * (NT / 16); u += kThreads) {
        const int c = (u >> 7) * 16, r = u & 127;
        const long long row = (long long)tm * 128 + r;
        if ((u >> 7) % p.split != rank || row >= p.rows) continue;
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = 0.f;
        for (int k = 0; k < p.split; ++k) {
          const uint32_t at = map_cluster(sm + (uint32_t)((c * 128 + r) * 4), (uint32_t)k);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] += lds_cluster_f(at + (uint32_t)(i * 512));
        }
        deliver16<T>(p, bias, residual, y, row, tn * NT + c, v);
      }
    }
    cluster_sync();                              // nobody leaves while its part may still be read
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

template <int F, int NT, typename T>
cudaError_t launch(Params &p, const void *x, const void *w, const q4::Layout &lx, const q4::Layout &lw, const float *bias, const void *residual,
                   void *y, DcWsHeader *ws, int n_sm, cudaStream_t st) {
  using S = Shape<F, NT>;
  static unsigned char attr_done[kDcMaxDevices];
  const cudaError_t e = dc_set_max_smem_once(k_q4_product<F, NT, T>, kSmemMax, attr_done);
  if (e != cudaSuccess) return e;
  EncodeTiledFn encode = get_encode_fn();
  if (!encode) return cudaErrorNotSupported;
  CUtensorMap map_x, map_w;
  if (!codes_map(encode, &map_x, x, lx.pitch, p.rows, 128) || !codes_map(encode, &map_w, w, lw.pitch, p.c_out, NT)) return cudaErrorNotSupported;
  p.acc_bufs = 2 * NT + 2 * S::kSfCols <= 512 ? 2 : 1;
  p.stages = (kSmemMax - 1024) / S::kStage;
  if (p.stages > kMaxStages) p.stages = kMaxStages;
  while (p.acc_bufs * NT + p.stages * S::kSfCols > 512) --p.stages;
  const int grid = p.split > 1 ? p.items * p.split : (p.items < n_sm ? p.items : n_sm);
  // all of a CTA's shared memory is asked for: two CTAs on an SM would each want all of its tensor memory
  return dc_launch_pdl_cluster(k_q4_product<F, NT, T>, dim3((unsigned)grid), dim3(kThreads), (size_t)kSmemMax, st, p.split, map_x, map_w, bias,
                               (const T *)residual, (T *)y, p, ws);
}

// Tile width and the CTAs that share a tile: the least of an estimate in cycles.  A stage takes its products or its loads, whichever is longer.
void choose(const Params &p, int n_sm, int *nt, int *split) {
  static constexpr int kClusters[kMaxSplit + 1] = {0, 148, 74, 45, 33, 26, 22, 15, 15};    // of that many CTAs that run at once, on 148 SMs
  double best = 1e30;
  for (int n = 128; n <= 256; n *= 2) {
    if (n > 128 && p.c_out <= 128) break;
    const long long items = (long long)p.tiles_m * dc_div_up(p.c_out, n);
    for (int s = 1; s <= kMaxSplit && s <= p.chunks; ++s) {
      const int per = dc_div_up(p.chunks, s);
      if (s > 1 && (per * (s - 1) >= p.chunks || items * s > n_sm)) continue;     // no CTA without a stage
      const double stage = (128 + n) * 140 / 45.0, main = per * (stage > 2.0 * n ? stage : 2.0 * n), out = 6.0 * n;
      const double waves = s > 1 ? (double)((items + kClusters[s] - 1) / kClusters[s]) : (double)((items + n_sm - 1) / n_sm);
      const double cycles = 3000 + waves * (n == 128 && s == 1 ? (main > out ? main : out) : main + out) + (s > 1 ? 1500 : 0);
      if (cycles < best) { best = cycles; *nt = n; *split = s; }
    }
  }
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

template <int F, typename T>
cudaError_t launch_nt(int nt, Params &p, const void *x, const void *w, const q4::Layout &lx, const q4::Layout &lw, const float *bias,
                      const void *residual, void *y, DcWsHeader *ws, int n_sm, cudaStream_t st) {
  switch (nt) {
    case 128: return launch<F, 128, T>(p, x, w, lx, lw, bias, residual, y, ws, n_sm, st);
    default: return launch<F, 256, T>(p, x, w, lx, lw, bias, residual, y, ws, n_sm, st);
  }
}

}  // namespace

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
  const int n_sm = dc_sm_count();
  Params p = {};
  p.rows = rows;
  p.c_in = c_in;
  p.c_out = c_out;
  p.act = (int)act;
  p.scale = scale;
  p.tiles_m = (int)((rows + 127) / 128);
  p.chunks = dc_div_up(c_in, kStageCols);
  p.atoms = (int)lx.tiles;
  p.vec = (size_t)c_out * (dtype == DC_F32 ? 4 : 2) % 16 == 0;
  p.sx = (const uint8_t *)x + lx.scale_offset;
  p.sw = (const uint8_t *)w + lw.scale_offset;
  int nt = 128;
  choose(p, n_sm, &nt, &p.split);
  p.tiles_n = dc_div_up(c_out, nt);
  if ((long long)p.tiles_m * p.tiles_n * p.split > 0x3fffffffll) return DC_ERR_UNSUPPORTED;
  p.items = p.tiles_m * p.tiles_n;
  p.chunks_per = dc_div_up(p.chunks, p.split);
  cudaStream_t st = (cudaStream_t)stream;
  DcWsHeader *ws = (DcWsHeader *)workspace;
  cudaError_t e;
  if (format == DC_MX4)
    e = dtype == DC_BF16 ? launch_nt<DC_MX4, __nv_bfloat16>(nt, p, x, w, lx, lw, bias, residual, y, ws, n_sm, st)
                         : launch_nt<DC_MX4, float>(nt, p, x, w, lx, lw, bias, residual, y, ws, n_sm, st);
  else
    e = dtype == DC_BF16 ? launch_nt<DC_NV4, __nv_bfloat16>(nt, p, x, w, lx, lw, bias, residual, y, ws, n_sm, st)
                         : launch_nt<DC_NV4, float>(nt, p, x, w, lx, lw, bias, residual, y, ws, n_sm, st);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? DC_OK : DC_ERR_CUDA;
}

extern "C" dc_status dc_q4_forward(const void *x, long long rows, int c_in, const void *w, int c_out, dc_q4_format format, float x_scale,
                                   float w_scale, const float *bias, dc_act act, const void *residual, void *y, dc_dtype dtype,
                                   void *workspace, size_t workspace_bytes, dc_stream stream) {
  q4::Layout lx, lw;
  dc_status s = check(x, rows, c_in, w, c_out, format, bias, act, residual, y, dtype, workspace, workspace_bytes, &lx, &lw);
  if (s != DC_OK) return s;
  if (!q4::tensor_scale_ok(x_scale, format) || !q4::tensor_scale_ok(w_scale, format)) return DC_ERR_INVALID_ARG;
  if (workspace_bytes < sizeof(DcWsHeader) + lx.bytes) return DC_ERR_WORKSPACE;
  uint8_t *xq = (uint8_t *)workspace + sizeof(DcWsHeader);
  s = dc_q4_quantize(x, rows, c_in, c_in, dtype, format, x_scale, xq, stream);
  if (s != DC_OK) return s;
  return dc_q4_product(xq, rows, c_in, w, c_out, format, x_scale * w_scale, bias, act, residual, y, dtype, workspace, workspace_bytes, stream);
}
