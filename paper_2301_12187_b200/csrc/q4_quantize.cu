// Quantising matrices to microscaled 4 bits and reading them back (dc_q4_quantize, dc_q4_dequantize).
//
// A thread takes 16 columns of a row: a block of DC_NV4, half of one of DC_MX4 (the other half is in the neighbouring lane).  A CTA takes 128
// rows x up to 256 columns, the rows of whole scale tiles, collects their scale bytes in shared memory and writes them as 16-byte words.
#include <string.h>

#include "q4.cuh"

namespace {
using namespace q4;

constexpr int kThreads = 256;
constexpr int kCols = 256;                       // columns of a CTA, at most

struct Params {
  long long rows, stride;
  int cols;
  int segs_log2;             // log2 of the 16-column pieces of a row that a CTA takes
  int vec;                   // rows begin on 16 bytes: whole pieces are loaded and stored in 16-byte words
  float g, g6;
  uint32_t pitch, tiles, col_tiles;
  size_t scale_offset;
};

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

template <int F, typename T>
__global__ void __launch_bounds__(kThreads) k_q4_quantize(const T *__restrict__ x, uint8_t *__restrict__ q, const Params p) {
  __shared__ __align__(16) uint8_t scales[4 * kAtom];
  dc_pdl_enter();
  const int tid = (int)threadIdx.x, segs = 1 << p.segs_log2;
  const uint32_t tile = blockIdx.x / p.col_tiles, col_tile = blockIdx.x - tile * p.col_tiles;
  const int seg = tid & (segs - 1), c = (int)(col_tile << (p.segs_log2 + 4)) + seg * 16;
  const long long row0 = (long long)tile * 128;
  constexpr int kBlock = F == DC_MX4 ? 32 : 16;
  // scale tiles of this CTA; the bytes that no row or block writes are 0
  const int atoms = (1 << (p.segs_log2 + 4)) <= 4 * kBlock ? 1 : (1 << (p.segs_log2 + 4)) / (4 * kBlock);
  for (int i = tid; i < atoms * (kAtom / 16); i += kThreads) reinterpret_cast<uint4 *>(scales)[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();
#pragma unroll 1
  for (int r = tid >> p.segs_log2; r < 128; r += kThreads >> p.segs_log2) {
    const long long row = row0 + r;
    const bool in = row < p.rows && c < (int)(p.pitch * 2);
    float v[16];
    if (in) {
      const T *at = x + row * p.stride + c;
      if (p.vec && c + 16 <= p.cols) {
        if (sizeof(T) == 2) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint4 w = __ldg(reinterpret_cast<const uint4 *>(at) + i);
            v[8 * i] = bf16_lo(w.x); v[8 * i + 1] = bf16_hi(w.x); v[8 * i + 2] = bf16_lo(w.y); v[8 * i + 3] = bf16_hi(w.y);
            v[8 * i + 4] = bf16_lo(w.z); v[8 * i + 5] = bf16_hi(w.z); v[8 * i + 6] = bf16_lo(w.w); v[8 * i + 7] = bf16_hi(w.w);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 w = __ldg(reinterpret_cast<const float4 *>(at) + i);
            v[4 * i] = w.x; v[4 * i + 1] = w.y; v[4 * i + 2] = w.z; v[4 * i + 3] = w.w;
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          v[i] = 0.f;
          if (c + i < p.cols) v[i] = sizeof(T) == 2 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(at)[i]) : reinterpret_cast<const float *>(at)[i];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = 0.f;
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    if (F == DC_MX4) top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const BlockScale s = block_scale<F>(top, p.g, p.g6);
    const uint2 code = codes16<F>(v, s);
    if (in) {
      *reinterpret_cast<uint2 *>(q + (size_t)row * p.pitch + (c >> 1)) = code;
      if (c < p.cols && (F == DC_NV4 || (seg & 1) == 0)) {
        const uint32_t b = (uint32_t)(seg * 16 / kBlock);
        scales[(b >> 2) * kAtom + scale_at((uint32_t)r, b)] = (uint8_t)s.byte;
      }
    }
  }
  __syncthreads();
  const uint32_t atom0 = col_tile * (uint32_t)atoms;
  const uint32_t left = p.tiles - atom0, n = left < (uint32_t)atoms ? left : (uint32_t)atoms;
  uint4 *out = reinterpret_cast<uint4 *>(q + p.scale_offset + ((size_t)tile * p.tiles + atom0) * kAtom);
  for (uint32_t i = tid; i < n * (kAtom / 16); i += kThreads) out[i] = reinterpret_cast<const uint4 *>(scales)[i];
}

template <int F, typename T>
__global__ void __launch_bounds__(kThreads) k_q4_dequantize(const uint8_t *__restrict__ q, T *__restrict__ y, const Params p) {
  dc_pdl_enter();
  const int tid = (int)threadIdx.x, segs = 1 << p.segs_log2;
  const uint32_t tile = blockIdx.x / p.col_tiles, col_tile = blockIdx.x - tile * p.col_tiles;
  const int c = (int)(col_tile << (p.segs_log2 + 4)) + (tid & (segs - 1)) * 16;
  if (c >= p.cols) return;
  constexpr int kBlock = F == DC_MX4 ? 32 : 16;
  const uint32_t b = (uint32_t)(c / kBlock);
#pragma unroll 1
  for (int r = tid >> p.segs_log2; r < 128; r += kThreads >> p.segs_log2) {
    const long long row = (long long)tile * 128 + r;
    if (row >= p.rows) return;
    const uint2 code = __ldg(reinterpret_cast<const uint2 *>(q + (size_t)row * p.pitch + (c >> 1)));
    const uint32_t byte = __ldg(q + p.scale_offset + ((size_t)tile * p.tiles + (b >> 2)) * kAtom + scale_at((uint32_t)r, b));
    const float s = scale_value(byte, F, p.g);
    uint32_t h[8];
    values8(code.x, h);
    values8(code.y, h + 4);
    float v[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[i]));
      v[2 * i] = f.x * s;
      v[2 * i + 1] = f.y * s;
    }
    T *at = y + row * p.stride + c;
    if (p.vec && c + 16 <= p.cols) {
      if (sizeof(T) == 2) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
          w[i] = *reinterpret_cast<const uint32_t *>(&t);
        }
        reinterpret_cast<uint4 *>(at)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4 *>(at)[1] = make_uint4(w[4], w[5], w[6], w[7]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<float4 *>(at)[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (c + i < p.cols) {
          if (sizeof(T) == 2) reinterpret_cast<__nv_bfloat16 *>(at)[i] = __float2bfloat16_rn(v[i]);
          else reinterpret_cast<float *>(at)[i] = v[i];
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
  p->g6 = 6.f * g;
  p->pitch = (uint32_t)l.pitch;
  p->tiles = (uint32_t)l.tiles;
  p->scale_offset = l.scale_offset;
  p->col_tiles = (uint32_t)dc_div_up(cols, 16 << p->segs_log2);
  const long long ctas = (rows + 127) / 128 * p->col_tiles;
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

extern "C" dc_status dc_q4_quantize(const void *x, long long rows, int cols, long long stride, dc_dtype dtype, dc_q4_format format,
                                    float tensor_scale, void *q, dc_stream stream) {
  Params p;
  dim3 grid;
  const dc_status s = prepare(x, rows, cols, stride, dtype, format, tensor_scale, q, &p, &grid);
  if (s != DC_OK) return s;
  cudaStream_t st = (cudaStream_t)stream;
  uint8_t *out = (uint8_t *)q;
  cudaError_t e;
  if (dtype == DC_BF16) {
    const __nv_bfloat16 *in = (const __nv_bfloat16 *)x;
    e = format == DC_MX4 ? dc_launch_pdl(k_q4_quantize<DC_MX4, __nv_bfloat16>, grid, dim3(kThreads), 0, st, in, out, p)
                         : dc_launch_pdl(k_q4_quantize<DC_NV4, __nv_bfloat16>, grid, dim3(kThreads), 0, st, in, out, p);
  } else {
    const float *in = (const float *)x;
    e = format == DC_MX4 ? dc_launch_pdl(k_q4_quantize<DC_MX4, float>, grid, dim3(kThreads), 0, st, in, out, p)
                         : dc_launch_pdl(k_q4_quantize<DC_NV4, float>, grid, dim3(kThreads), 0, st, in, out, p);
  }
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? DC_OK : DC_ERR_CUDA;
}

extern "C" dc_status dc_q4_dequantize(const void *q, long long rows, int cols, dc_q4_format format, float tensor_scale, void *y,
                                      long long stride, dc_dtype dtype, dc_stream stream) {
  Params p;
  dim3 grid;
  const dc_status s = prepare(y, rows, cols, stride, dtype, format, tensor_scale, q, &p, &grid);
  if (s != DC_OK) return s;
  cudaStream_t st = (cudaStream_t)stream;
  const uint8_t *in = (const uint8_t *)q;
  cudaError_t e;
  if (dtype == DC_BF16) {
    __nv_bfloat16 *out = (__nv_bfloat16 *)y;
    e = format == DC_MX4 ? dc_launch_pdl(k_q4_dequantize<DC_MX4, __nv_bfloat16>, grid, dim3(kThreads), 0, st, in, out, p)
                         : dc_launch_pdl(k_q4_dequantize<DC_NV4, __nv_bfloat16>, grid, dim3(kThreads), 0, st, in, out, p);
  } else {
    float *out = (float *)y;
    e = format == DC_MX4 ? dc_launch_pdl(k_q4_dequantize<DC_MX4, float>, grid, dim3(kThreads), 0, st, in, out, p)
                         : dc_launch_pdl(k_q4_dequantize<DC_NV4, float>, grid, dim3(kThreads), 0, st, in, out, p);
  }
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? DC_OK : DC_ERR_CUDA;
}
