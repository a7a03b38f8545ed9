// Quantising matrices to microscaled 4 bits and reading them back (dc_q4_quantize, dc_q4_dequantize).
//
// Quantising, a thread takes 16 columns of a row: a block of DC_NV4, half of one of DC_MX4 (the other half is in the neighbouring lane).  A CTA takes
// up to 256 columns of 128 rows, whole scale tiles, whose bytes it collects in shared memory and writes 16 at a time -- or, where that gives too few
// CTAs, of the 32 rows that share a word of every 16 bytes of a scale tile (2048 x 4096: 6.0 us).  In all sizes that many CTAs would cost what
// the scales' 4-byte pieces do (16384 x 8192 71 us in the place of 61); reading back has no such cost.
#include <string.h>

#include "q4.cuh"

namespace {
using namespace q4;

constexpr int kThreads = 256;
constexpr int kCols = 256;                       // columns of a CTA, at most

struct Params {
  long long rows, stride;
  int cols;
  int segs;                  // threads' pieces of a row that a CTA takes
  int vec;                   // rows begin on 16 bytes
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
// Words that hold 16 values from byte `off` of the first on -> the values (off: below 16, a multiple of a value's size).  Rows that do not begin on
// 16 bytes are loaded in aligned words, one more than they fill, and shifted in registers.  (Through shared memory, loaded value by value: 5001 x 1003
// in fp32 10.9 us.)
template <typename T>
__device__ __forceinline__ void shift16(uint32_t *w, uint32_t off) {
  constexpr int N = 4 * (int)sizeof(T);
#pragma unroll
  for (int i = 0; i < N + 2; ++i) w[i] = off & 8u ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < N + 1; ++i) w[i] = off & 4u ? w[i + 1] : w[i];
  if (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (off & 2u) * 8u);
  }
}

// A row at a time, so that six CTAs fit an SM: 16001 x 4096 in fp32 52.2 us, 100352 x 192 in bf16 11.9, 16384 x 8192 61.2 (344 MB: 53 at the rate of a
// copy).  Two rows at once and four CTAs: 57.4, 13.5, 61.6.  Eight CTAs, of 32 registers a thread: 49.7, 15.2, 57.5.  The next row asked for ahead: 51.5,
// 13.0, 59.2, and narrow maps 1 us more.
template <int F, typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, VEC ? 6 : 5) k_q4_quantize(const T *__restrict__ x, uint8_t *__restrict__ q, const Params p) {
  __shared__ __align__(16) uint8_t scales[4 * kAtom];
  dc_pdl_enter();
  const int tid = (int)threadIdx.x, segs = p.segs, span = segs * 16;
  const uint32_t strip = blockIdx.x / p.col_tiles, col_tile = blockIdx.x - strip * p.col_tiles;
  const uint32_t tile = strip / (uint32_t)p.groups, group = strip - tile * (uint32_t)p.groups;
  const int mine = tid / segs, seg = tid - mine * segs, step = kThreads / segs;  // this thread's row of the `step` at a time
  const int c = (int)col_tile * span + seg * 16;
  const int most = 128 / p.groups, in_tile = (int)group * most;                  // rows of this CTA, and the first one's place in its scale tile
  const long long row0 = (long long)tile * 128 + in_tile;
  const int rows = p.rows - row0 < most ? (int)(p.rows - row0) : most;           // none or fewer: the scales of such rows are 0
  constexpr int kBlock = F == DC_MX4 ? 32 : 16, kPieces = 16 / kPer<T> + (VEC ? 0 : 1);
  // scale tiles of this CTA; the bytes that no row or block writes are 0
  const int atoms = (span + 4 * kBlock - 1) / (4 * kBlock);
  for (int i = tid; i < atoms * (kAtom / 16); i += kThreads) reinterpret_cast<uint4 *>(scales)[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();
  const bool wanted = c < (int)(p.pitch * 2) && mine < step;
  const int some = wanted ? (p.cols - c < 16 ? p.cols - c : 16) : 0;             // values of this thread's pieces; none or fewer: codes 0
  const long long end = (p.rows - 1) * p.stride + p.cols;                        // of x
  auto offset = [&](long long row) { return VEC ? 0u : (uint32_t)((row * p.stride + c) * (long long)sizeof(T)) & 15u; };   // of the first value in its word
#pragma unroll 1
  for (int r = mine; r - mine < rows; r += step) {
    uint4 raw[kPieces];
    const long long row = row0 + r;
    const int lead = VEC ? 0 : (int)offset(row) / (int)sizeof(T);                // values of the first word that come before this thread's
    const T *at = x + row * p.stride + c - lead;
    const int to = r < rows ? lead + some : 0;                                   // `lead` to here: of the values from `at` on
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      raw[i] = make_uint4(0, 0, 0, 0);
      if (i * kPer<T> >= to) continue;
      if ((i + 1) * kPer<T> <= to || (!VEC && (i + 1) * kPer<T> <= end - (row * p.stride + c - lead))) {      // a whole word of x
        raw[i] = __ldg(reinterpret_cast<const uint4 *>(at) + i);
      } else {
        float t[kPer<T>];
#pragma unroll
        for (int j = 0; j < kPer<T>; ++j) t[j] = i * kPer<T> + j >= lead && i * kPer<T> + j < to ? (float)at[i * kPer<T> + j] : 0.f;
        raw[i] = pack<T>(t);
      }
    }
    if (!VEC) shift16<T>(reinterpret_cast<uint32_t *>(raw), offset(row));
    float v[16];
#pragma unroll
    for (int i = 0; i < 16 / kPer<T>; ++i) unpack<T>(raw[i], v + i * kPer<T>);
    if (!VEC && some < 16) {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = i < some ? v[i] : 0.f;
    }
    uint32_t top = largest16(v);
    if (F == DC_MX4) top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const BlockScale s = block_scale<F>(top, p.g, p.r6);
    const uint2 code = codes16<F, sizeof(T) == 2>(v, s);
    if (r < rows && wanted) {
      *reinterpret_cast<uint2 *>(q + (size_t)row * p.pitch + (c >> 1)) = code;
      if (some > 0 && (F == DC_NV4 || (seg & 1) == 0)) {
        const uint32_t b = (uint32_t)(seg * 16 / kBlock);
        scales[(b >> 2) * kAtom + scale_at((uint32_t)(in_tile + r), b)] = (uint8_t)s.byte;
      }
    }
  }
  __syncthreads();
  const uint32_t atom0 = col_tile * (uint32_t)atoms;
  const uint32_t left = p.tiles - atom0, n = left < (uint32_t)atoms ? left : (uint32_t)atoms;
  if (blockIdx.x == 0) {                         // between the codes and the scales: up to 14 pieces of 16 bytes
    const size_t at = (size_t)p.rows * p.pitch + (size_t)tid * 16;
    if (at < p.scale_offset) *reinterpret_cast<uint4 *>(q + at) = make_uint4(0, 0, 0, 0);
  }
  uint8_t *out = q + p.scale_offset + ((size_t)tile * p.tiles + atom0) * kAtom;
  if (p.groups == 1) {
    for (uint32_t i = tid; i < n * (kAtom / 16); i += kThreads) reinterpret_cast<uint4 *>(out)[i] = reinterpret_cast<const uint4 *>(scales)[i];
  } else {
    for (uint32_t i = tid; i < n * (kAtom / 16); i += kThreads)
      reinterpret_cast<uint32_t *>(out)[i * 4 + group] = reinterpret_cast<const uint32_t *>(scales)[i * 4 + group];
  }
}

// Bound by what goes out: 8192 x 8192 to bf16 35.9 us, 16001 x 4096 to fp32 69.7 (a fill of as many bytes: 34.5, 67).  A thread writes 32 bytes of
// a row: with 64, which fp32's 16 columns are, the second took 84.7.  Rows of y that do not begin on 16 bytes: its columns begin up to 7 earlier, where they do, with codes and a
// scale of the piece before its own.  (Through shared memory, stored value by value: 5001 x 1003 in fp32 12.1 us.)
template <typename T>
constexpr int kTake = 32 / (int)sizeof(T);
template <int F, typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, 4) k_q4_dequantize(const uint8_t *__restrict__ q, T *__restrict__ y, const Params p) {
  dc_pdl_enter();
  const int tid = (int)threadIdx.x, segs = p.segs;
  const uint32_t strip = blockIdx.x / p.col_tiles, col_tile = blockIdx.x - strip * p.col_tiles;
  const uint32_t tile = strip / (uint32_t)p.groups, group = strip - tile * (uint32_t)p.groups;
  const int mine = tid / segs, seg = tid - mine * segs, step = kThreads / segs;  // this thread's row of the `step` at a time
  constexpr int N = kTake<T>, kBlock = F == DC_MX4 ? 32 : 16;
  const int c0 = ((int)col_tile * segs + seg) * N;
  const int most = 128 / p.groups, in_tile = (int)group * most;                  // rows of this CTA, and the first one's place in its scale tile
  const long long row0 = (long long)tile * 128 + in_tile;
  const int rows = p.rows - row0 < most ? (int)(p.rows - row0) : most;
  const bool own = c0 < p.cols;
  if (mine >= step || (VEC && !own)) return;
  const uint8_t *scales = q + p.scale_offset + (size_t)tile * p.tiles * kAtom;
  auto scales_of = [&](int col) { return scales + (size_t)(col / kBlock >> 2) * kAtom + (col / kBlock & 3); };       // of the block of a column
  const uint8_t *scales_own = scales_of(c0), *scales_before = VEC || c0 == 0 ? scales : scales_of(c0 - 1);
#pragma unroll 1
  for (int r = mine; r < rows; r += step) {
    const long long row = row0 + r;
    const int lead = VEC ? 0 : (int)((uint32_t)(row * p.stride * (long long)sizeof(T)) & 15u) / (int)sizeof(T);
    const int c = c0 - lead;
    if (!VEC && c >= p.cols) continue;
    const uint8_t *codes = q + (size_t)row * p.pitch + (c0 >> 1);
    const uint32_t at_row = scale_at((uint32_t)(in_tile + r), 0);
    uint32_t code[2] = {0, 0};
    float s = 0.f;
    if (VEC || own) {
      if (N == 16) {
        const uint2 w = __ldg(reinterpret_cast<const uint2 *>(codes));
        code[0] = w.x;
        code[1] = w.y;
      } else {
        code[0] = __ldg(reinterpret_cast<const uint32_t *>(codes));
      }
      s = scale_value(__ldg(scales_own + at_row), F, p.g);
    }
    float before = s;
    if (!VEC && lead > 0) {
      uint32_t w = 0;
      if (c0 > 0) {
        w = __ldg(reinterpret_cast<const uint32_t *>(codes) - 1);
        before = scale_value(__ldg(scales_before + at_row), F, p.g);
      }
      const uint32_t by = 32u - 4u * (uint32_t)lead;
      code[1] = __funnelshift_r(code[0], code[1], by);
      code[0] = __funnelshift_r(w, code[0], by);
    }
    uint32_t h[N / 2];
    values8(code[0], h);
    if (N == 16) values8(code[1], h + N / 2 - 4);
    float v[N];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[i]));
      v[2 * i] = f.x * (!VEC && 2 * i < lead ? before : s);
      v[2 * i + 1] = f.y * (!VEC && 2 * i + 1 < lead ? before : s);
    }
    T *at = y + row * p.stride + c;
    if (c >= 0 && c + N <= p.cols) {
#pragma unroll
      for (int i = 0; i < 2; ++i) reinterpret_cast<uint4 *>(at)[i] = pack<T>(v + i * kPer<T>);
      continue;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int first = c + i * kPer<T>;
      if (first >= 0 && first + kPer<T> <= p.cols) {
        reinterpret_cast<uint4 *>(at)[i] = pack<T>(v + i * kPer<T>);
      } else {
#pragma unroll
        for (int j = 0; j < kPer<T>; ++j)
          if (first + j >= 0 && first + j < p.cols) at[i * kPer<T> + j] = (T)v[i * kPer<T> + j];
      }
    }
  }
}

// checks shared by the two calls; fills the launch's parameters
dc_status prepare(const void *x, long long rows, int cols, long long stride, dc_dtype dtype, dc_q4_format format, float g, const void *q,
                  bool reads, Params *p, dim3 *grid) {
  Layout l;
  const dc_status s = layout_of(rows, cols, format, &l);
  if (s != DC_OK) return s;
  if (!x || !q || (dtype != DC_F32 && dtype != DC_BF16) || stride < cols || !tensor_scale_ok(g, format)) return DC_ERR_INVALID_ARG;
  if (!dc_aligned16(x) || !dc_aligned16(q)) return DC_ERR_ALIGNMENT;
  const size_t es = dtype == DC_F32 ? 4 : 2;
  p->rows = rows;
  p->stride = stride;
  p->cols = cols;
  p->vec = stride % (long long)(16 / es) == 0;
  p->g = g;
  p->r6 = 1.f / (6.f * g);
  p->pitch = (uint32_t)l.pitch;
  p->tiles = (uint32_t)l.tiles;
  p->scale_offset = l.scale_offset;
  if (reads) {               // pieces that begin up to 15 bytes early, in as few CTAs a row as hold them, alike
    const int take = 32 / (int)es, all = dc_div_up(p->vec ? cols : cols + (int)(16 / es) - 1, take);
    p->col_tiles = (uint32_t)dc_div_up(all, kCols / take);
    p->segs = dc_div_up(all, (int)p->col_tiles);
  } else {                   // whole scale tiles; pitch: whole runs of 64 columns
    p->segs = l.pitch < kCols / 2 ? (int)(l.pitch / 8) : kCols / 16;
    p->col_tiles = (uint32_t)dc_div_up(cols, 16 * p->segs);
  }
  const long long tiles = (rows + 127) / 128 * p->col_tiles;
  p->groups = tiles < (reads ? 8ll : 4ll) * dc_sm_count() ? 4 : 1;
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
               : dc_launch_pdl(k_q4_quantize<F, T, false>, grid, dim3(kThreads), 0, st, (const T *)x, (uint8_t *)q, p);
}
template <int F, typename T>
static cudaError_t dequantize(const void *q, void *y, const Params &p, dim3 grid, cudaStream_t st) {
  return p.vec ? dc_launch_pdl(k_q4_dequantize<F, T, true>, grid, dim3(kThreads), 0, st, (const uint8_t *)q, (T *)y, p)
               : dc_launch_pdl(k_q4_dequantize<F, T, false>, grid, dim3(kThreads), 0, st, (const uint8_t *)q, (T *)y, p);
}

extern "C" dc_status dc_q4_quantize(const void *x, long long rows, int cols, long long stride, dc_dtype dtype, dc_q4_format format,
                                    float tensor_scale, void *q, dc_stream stream) {
  Params p;
  dim3 grid;
  const dc_status s = prepare(x, rows, cols, stride, dtype, format, tensor_scale, q, false, &p, &grid);
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
  const dc_status s = prepare(y, rows, cols, stride, dtype, format, tensor_scale, q, true, &p, &grid);
  if (s != DC_OK) return s;
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e;
  if (format == DC_MX4) e = dtype == DC_BF16 ? dequantize<DC_MX4, __nv_bfloat16>(q, y, p, grid, st) : dequantize<DC_MX4, float>(q, y, p, grid, st);
  else e = dtype == DC_BF16 ? dequantize<DC_NV4, __nv_bfloat16>(q, y, p, grid, st) : dequantize<DC_NV4, float>(q, y, p, grid, st);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? DC_OK : DC_ERR_CUDA;
}
