// Quantising matrices to microscaled 4 bits and reading them back (dc_q4_quantize, dc_q4_dequantize).
//
// A thread takes 16 columns of a row: a block of DC_NV4, half of one of DC_MX4 (the other half is in the neighbouring lane).  A CTA takes up to 256
// columns of 128 rows, whole scale tiles, whose bytes it collects in shared memory and writes 16 at a time -- or, where that gives too few CTAs,
// of the 32 rows that share a word of every 16 bytes of a scale tile.
#include <string.h>

#include "q4.cuh"

namespace {
using namespace q4;

constexpr int kThreads = 256;
constexpr int kCols = 256;                       // columns of a CTA, at most

struct Params {
  long long rows, stride;
  int cols;
  int segs, segs_log2;       // 16-column pieces of a row that a CTA takes; their log2 where rows go through shared memory
  int vec;                   // rows begin on 16 bytes: whole pieces are loaded and stored in 16-byte words
  int groups;                // CTAs that share 128 rows: 1 or 4
  float g, r6;
  uint32_t pitch, tiles, col_tiles;
  size_t scale_offset;
};

template <typename T>
constexpr int kPer = 16 / (int)sizeof(T);        // values in 16 bytes
template <typename T>
__device__ __forceinline__ void unpack(uint4 w, float *v) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (sizeof(T) == 2) { v[2 * j % kPer<T>] = __uint_as_float(u[j] << 16); v[(2 * j + 1) % kPer<T>] = __uint_as_float(u[j] & 0xffff0000u); }
    else v[j] = __uint_as_float(u[j]);
  }
}
template <typename T>
__device__ __forceinline__ uint4 pack(const float *v) {
  constexpr int N = kPer<T>;
  if (N == 4) return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i % N], v[(2 * i + 1) % N]);
    w[i] = *reinterpret_cast<const uint32_t *>(&t);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Rows that do not begin on 16 bytes go through shared memory, 4096 columns at a time: neighbouring threads then load and store neighbouring
// columns.  One word of padding behind 16 keeps the threads, 16 columns apart, out of one another's banks.
struct Staged {
  float at[4096 + 256];
  __device__ __forceinline__ float &operator()(int row, int col, int span_log2) { return at[(row << span_log2) + (row << (span_log2 - 4)) + col + (col >> 4)]; }
};

template <int F, typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, VEC ? 4 : 3) k_q4_quantize(const T *__restrict__ x, uint8_t *__restrict__ q, const Params p) {
  __shared__ __align__(16) uint8_t scales[4 * kAtom];
  extern __shared__ uint8_t staged_s[];            // Staged, where !VEC
  dc_pdl_enter();
  const int tid = (int)threadIdx.x, segs = VEC ? p.segs : 1 << p.segs_log2, span_log2 = p.segs_log2 + 4, span = segs * 16;
  const uint32_t strip = blockIdx.x / p.col_tiles, col_tile = blockIdx.x - strip * p.col_tiles;
  const uint32_t tile = strip / (uint32_t)p.groups, group = strip - tile * (uint32_t)p.groups;
  const int mine = VEC ? tid / segs : tid >> p.segs_log2, seg = tid - mine * segs, step = kThreads / segs;     // this thread's row of the `step` at a time
  const int c0 = (int)col_tile * span, c = c0 + seg * 16;
  const int most = 128 / p.groups, in_tile = (int)group * most;                  // rows of this CTA, and the first one's place in its scale tile
  const long long row0 = (long long)tile * 128 + in_tile;
  const int rows = p.rows - row0 < most ? (int)(p.rows - row0) : most;           // none or fewer: the scales of such rows are 0
  constexpr int kBlock = F == DC_MX4 ? 32 : 16, kPieces = 16 / kPer<T>;
  // scale tiles of this CTA; the bytes that no row or block writes are 0
  const int atoms = (span + 4 * kBlock - 1) / (4 * kBlock);
  for (int i = tid; i < atoms * (kAtom / 16); i += kThreads) reinterpret_cast<uint4 *>(scales)[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();
  const bool wanted = c < (int)(p.pitch * 2) && mine < step;
  auto put = [&](int r, uint32_t top, float *v) {
    if (F == DC_MX4) top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const BlockScale s = block_scale<F>(top, p.g, p.r6);
    const uint2 code = codes16<F, sizeof(T) == 2>(v, s);
    if (r < rows && wanted) {
      *reinterpret_cast<uint2 *>(q + (size_t)(row0 + r) * p.pitch + (c >> 1)) = code;
      if (c < p.cols && (F == DC_NV4 || (seg & 1) == 0)) {
        const uint32_t b = (uint32_t)(seg * 16 / kBlock);
        scales[(b >> 2) * kAtom + scale_at((uint32_t)(in_tile + r), b)] = (uint8_t)s.byte;
      }
    }
  };
  if (VEC) {
    constexpr int U = 2;                         // rows of a thread at once, so that their loads overlap
    const bool whole = c + 16 <= p.cols && wanted;
#pragma unroll 1
    for (int r = mine; r - mine < rows; r += U * step) {
      uint4 raw[U][kPieces];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int ru = r + u * step;
        const T *at = x + (row0 + ru) * p.stride + c;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          raw[u][i] = make_uint4(0, 0, 0, 0);
          if (whole) {
            if (ru < rows) raw[u][i] = __ldg(reinterpret_cast<const uint4 *>(at) + i);
          } else if (ru < rows && wanted) {
            const int left = p.cols - (c + i * kPer<T>);
            if (left >= kPer<T>) {
              raw[u][i] = __ldg(reinterpret_cast<const uint4 *>(at) + i);
            } else if (left > 0) {               // the last columns
              float t[kPer<T>];
#pragma unroll
              for (int j = 0; j < kPer<T>; ++j) t[j] = j < left ? (float)at[i * kPer<T> + j] : 0.f;
              raw[u][i] = pack<T>(t);
            }
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (u > 0 && r + u * step - mine >= most) break;       // the same for all threads
        float v[16];
#pragma unroll
        for (int i = 0; i < kPieces; ++i) unpack<T>(raw[u][i], v + i * kPer<T>);
        put(r + u * step, largest16(v), v);
      }
    }
  } else {
    Staged &staged = *reinterpret_cast<Staged *>(staged_s);
#pragma unroll 1
    for (int r0 = 0; r0 < rows; r0 += step) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int at = tid + i * kThreads, r = at >> span_log2, col = at & ((1 << span_log2) - 1);
        float v = 0.f;
        if (r0 + r < rows && c0 + col < p.cols) v = (float)x[(row0 + r0 + r) * p.stride + c0 + col];
        staged(r, col, span_log2) = v;
      }
      __syncthreads();
      float v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = staged(mine, seg * 16 + i, span_log2);
      put(r0 + mine, largest16(v), v);
      __syncthreads();
    }
  }
  __syncthreads();
  const uint32_t atom0 = col_tile * (uint32_t)atoms;
  const uint32_t left = p.tiles - atom0, n = left < (uint32_t)atoms ? left : (uint32_t)atoms;
  uint8_t *out = q + p.scale_offset + ((size_t)tile * p.tiles + atom0) * kAtom;
  if (p.groups == 1) {
    for (uint32_t i = tid; i < n * (kAtom / 16); i += kThreads) reinterpret_cast<uint4 *>(out)[i] = reinterpret_cast<const uint4 *>(scales)[i];
  } else {
    for (uint32_t i = tid; i < n * (kAtom / 16); i += kThreads)
      reinterpret_cast<uint32_t *>(out)[i * 4 + group] = reinterpret_cast<const uint32_t *>(scales)[i * 4 + group];
  }
}

template <int F, typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, VEC ? 4 : 3) k_q4_dequantize(const uint8_t *__restrict__ q, T *__restrict__ y, const Params p) {
  extern __shared__ uint8_t staged_s[];            // Staged, where !VEC
  dc_pdl_enter();
  const int tid = (int)threadIdx.x, segs = VEC ? p.segs : 1 << p.segs_log2, span_log2 = p.segs_log2 + 4, span = segs * 16;
  const uint32_t strip = blockIdx.x / p.col_tiles, col_tile = blockIdx.x - strip * p.col_tiles;
  const uint32_t tile = strip / (uint32_t)p.groups, group = strip - tile * (uint32_t)p.groups;
  const int mine = VEC ? tid / segs : tid >> p.segs_log2, seg = tid - mine * segs, step = kThreads / segs;     // this thread's row of the `step` at a time
  const int c0 = (int)col_tile * span, c = c0 + seg * 16;
  const int most = 128 / p.groups, in_tile = (int)group * most;                  // rows of this CTA, and the first one's place in its scale tile
  const long long row0 = (long long)tile * 128 + in_tile;
  const int rows = p.rows - row0 < most ? (int)(p.rows - row0) : most;           // none or fewer: the scales of such rows are 0
  constexpr int kBlock = F == DC_MX4 ? 32 : 16;
  const bool wanted = c < p.cols && mine < step;
  const uint32_t b = (uint32_t)(c / kBlock);
  const uint8_t *scales = q + p.scale_offset + ((size_t)tile * p.tiles + (b >> 2)) * kAtom;
  auto codes_of = [&](int r) { return wanted && r < rows ? __ldg(reinterpret_cast<const uint2 *>(q + (size_t)(row0 + r) * p.pitch + (c >> 1))) : make_uint2(0, 0); };
  auto values = [&](int r, uint2 code, float *v) {
    const float s = scale_value(__ldg(scales + scale_at((uint32_t)(in_tile + r), b)), F, p.g);
    uint32_t h[8];
    values8(code.x, h);
    values8(code.y, h + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[i]));
      v[2 * i] = f.x * s;
      v[2 * i + 1] = f.y * s;
    }
  };
  if (VEC) {
    if (!wanted) return;
#pragma unroll 1
    for (int r = mine; r < rows; r += step) {
      float v[16];
      values(r, codes_of(r), v);
      T *at = y + (row0 + r) * p.stride + c;
      if (c + 16 <= p.cols) {
#pragma unroll
        for (int i = 0; i < 16 / kPer<T>; ++i) reinterpret_cast<uint4 *>(at)[i] = pack<T>(v + i * kPer<T>);
        continue;
      }
#pragma unroll
      for (int i = 0; i < 16 / kPer<T>; ++i) {
        const int left = p.cols - (c + i * kPer<T>);
        if (left >= kPer<T>) {
          reinterpret_cast<uint4 *>(at)[i] = pack<T>(v + i * kPer<T>);
        } else {
#pragma unroll
          for (int j = 0; j < kPer<T>; ++j)
            if (j < left) at[i * kPer<T> + j] = (T)v[i * kPer<T> + j];
        }
      }
    }
  } else {
    Staged &staged = *reinterpret_cast<Staged *>(staged_s);
#pragma unroll 1
    for (int r0 = 0; r0 < rows; r0 += step) {
      const uint2 code = codes_of(r0 + mine);
      __syncthreads();
      if (wanted && r0 + mine < rows) {
        float v[16];
        values(r0 + mine, code, v);
#pragma unroll
        for (int i = 0; i < 16; ++i) staged(mine, seg * 16 + i, span_log2) = v[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int at = tid + i * kThreads, r = at >> span_log2, col = at & ((1 << span_log2) - 1);
        if (r0 + r < rows && c0 + col < p.cols) y[(row0 + r0 + r) * p.stride + c0 + col] = (T)staged(r, col, span_log2);
      }
    }
  }
}

// checks shared by the two calls; fills the launch's parameters
dc_status prepare(const void *x, long long rows, int cols, long long stride, dc_dtype dtype, dc_q4_format format, float g, const void *q,
                  Params *p, dim3 *grid) {
  Layout l;
  const dc_status s = layout_of(rows, cols, format, &l);
  if (s != DC_OK) return s;
  if (!x || !q || (dtype != DC_F32 && dtype != DC_BF16) || stride < cols || !tensor_scale_ok(g, format)) return DC_ERR_INVALID_ARG;
  if (!dc_aligned16(x) || !dc_aligned16(q)) return DC_ERR_ALIGNMENT;
  const size_t es = dtype == DC_F32 ? 4 : 2;
  p->rows = rows;
  p->stride = stride;
  p->cols = cols;
  p->segs_log2 = 2;          // pitch: whole runs of 64 columns
  while ((16 << p->segs_log2) < kCols && (16 << p->segs_log2) < cols) ++p->segs_log2;
  p->vec = stride % (long long)(16 / es) == 0;
  p->g = g;
  p->r6 = 1.f / (6.f * g);
  p->pitch = (uint32_t)l.pitch;
  p->tiles = (uint32_t)l.tiles;
  p->scale_offset = l.scale_offset;
  p->segs = p->vec ? (l.pitch < kCols / 2 ? (int)(l.pitch / 8) : kCols / 16) : 1 << p->segs_log2;
  p->col_tiles = (uint32_t)dc_div_up(cols, 16 * p->segs);
  const long long tiles = (rows + 127) / 128 * p->col_tiles;
  p->groups = tiles < 4ll * dc_sm_count() ? 4 : 1;
  const long long ctas = tiles * p->groups;
  if (ctas > 0x7fffffffll) return DC_ERR_UNSUPPORTED;
  *grid = dim3((unsigned)ctas);
  return DC_OK;
}

}  // namespace

extern "C" dc_status dc_q4_query(long long rows, int cols, dc_q4_format format, dc_q4_layout *layout) {
  Layout l;
  const dc_status s = layout_of(rows, cols, format, &l);
  if (s != DC_OK) return s;
  if (!layout) return DC_ERR_INVALID_ARG;
  *layout = {l.pitch, l.tiles, l.scale_offset, l.bytes};
  return DC_OK;
}

template <int F, typename T>
static cudaError_t quantize(const void *x, void *q, const Params &p, dim3 grid, cudaStream_t st) {
  return p.vec ? dc_launch_pdl(k_q4_quantize<F, T, true>, grid, dim3(kThreads), 0, st, (const T *)x, (uint8_t *)q, p)
               : dc_launch_pdl(k_q4_quantize<F, T, false>, grid, dim3(kThreads), sizeof(Staged), st, (const T *)x, (uint8_t *)q, p);
}
template <int F, typename T>
static cudaError_t dequantize(const void *q, void *y, const Params &p, dim3 grid, cudaStream_t st) {
  return p.vec ? dc_launch_pdl(k_q4_dequantize<F, T, true>, grid, dim3(kThreads), 0, st, (const uint8_t *)q, (T *)y, p)
               : dc_launch_pdl(k_q4_dequantize<F, T, false>, grid, dim3(kThreads), sizeof(Staged), st, (const uint8_t *)q, (T *)y, p);
}

extern "C" dc_status dc_q4_quantize(const void *x, long long rows, int cols, long long stride, dc_dtype dtype, dc_q4_format format,
                                    float tensor_scale, void *q, dc_stream stream) {
  Params p;
  dim3 grid;
  const dc_status s = prepare(x, rows, cols, stride, dtype, format, tensor_scale, q, &p, &grid);
  if (s != DC_OK) return s;
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e;
  if (format == DC_MX4) e = dtype == DC_BF16 ? quantize<DC_MX4, __nv_bfloat16>(x, q, p, grid, st) : quantize<DC_MX4, float>(x, q, p, grid, st);
  else e = dtype == DC_BF16 ? quantize<DC_NV4, __nv_bfloat16>(x, q, p, grid, st) : quantize<DC_NV4, float>(x, q, p, grid, st);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? DC_OK : DC_ERR_CUDA;
}

extern "C" dc_status dc_q4_dequantize(const void *q, long long rows, int cols, dc_q4_format format, float tensor_scale, void *y,
                                      long long stride, dc_dtype dtype, dc_stream stream) {
  Params p;
  dim3 grid;
  const dc_status s = prepare(y, rows, cols, stride, dtype, format, tensor_scale, q, &p, &grid);
  if (s != DC_OK) return s;
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e;
  if (format == DC_MX4) e = dtype == DC_BF16 ? dequantize<DC_MX4, __nv_bfloat16>(q, y, p, grid, st) : dequantize<DC_MX4, float>(q, y, p, grid, st);
  else e = dtype == DC_BF16 ? dequantize<DC_NV4, __nv_bfloat16>(q, y, p, grid, st) : dequantize<DC_NV4, float>(q, y, p, grid, st);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? DC_OK : DC_ERR_CUDA;
}
