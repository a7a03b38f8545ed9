// Microscaled 4-bit matrices: layout, and a block's scale and codes.  The formats are described in include/dc.h.
#pragma once

#include "common.cuh"

namespace q4 {

constexpr int kAtom = 512;                       // bytes of a scale tile: 128 rows x 4 blocks

struct Layout {
  size_t pitch, tiles, scale_offset, bytes;
};
__host__ __device__ static inline int block_of(int format) { return format == DC_MX4 ? 32 : 16; }
// columns that a scale tile spans
__host__ __device__ static inline int atom_cols(int format) { return 4 * block_of(format); }

static inline dc_status layout_of(long long rows, int cols, dc_q4_format format, Layout *l) {
  if (rows < 1 || cols < 1 || (format != DC_MX4 && format != DC_NV4)) return DC_ERR_INVALID_ARG;
  if (rows > 0x7fffff00ll || cols > (1 << 24)) return DC_ERR_UNSUPPORTED;
  l->pitch = dc_round_up((size_t)cols, 64) / 2;
  l->tiles = dc_round_up((size_t)cols, atom_cols(format)) / atom_cols(format);
  l->scale_offset = dc_round_up((size_t)rows * l->pitch, 256);
  l->bytes = l->scale_offset + dc_round_up((size_t)rows, 128) / 128 * l->tiles * kAtom;
  return DC_OK;
}
static inline bool tensor_scale_ok(float g, dc_q4_format format) {
  if (format == DC_MX4) return g == 1.0f;
  uint32_t b;
  memcpy(&b, &g, 4);
  return (b & 0x807fffffu) == 0 && b >= (27u << 23) && b <= (227u << 23);      // 2^-100 .. 2^100
}

// place of a scale inside its tile
__device__ __forceinline__ uint32_t scale_at(uint32_t row, uint32_t block) {
  return (row & 31u) * 16u + ((row & 127u) >> 5) * 4u + (block & 3u);
}

// eight values -> eight codes, the first in the lowest 4 bits
__device__ __forceinline__ uint32_t codes8(const float *v) {
  uint32_t d;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
      "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
      : "=r"(d)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return d;
}
// eight codes -> eight values as four pairs of fp16
__device__ __forceinline__ void values8(uint32_t c, uint32_t *h) {
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(c));
}
__device__ __forceinline__ uint32_t e4m3_of(float v) {       // v >= 0; 448 at most
  uint16_t d;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(0.f), "f"(v));
  return d & 0xffu;
}
__device__ __forceinline__ float e4m3_value(uint32_t b) {
  uint32_t h;
  const uint16_t s = (uint16_t)b;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(s));
  float f;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.f32.f16 %0, lo;\n\t}" : "=f"(f) : "r"(h));
  return f;
}
// what a scale byte stands for (with the tensor scale)
__device__ __forceinline__ float scale_value(uint32_t b, int format, float g) {
  if (format == DC_NV4) return e4m3_value(b) * g;
  if (b == 0xffu) return __uint_as_float(0x7fffffffu);
  return b ? __uint_as_float(b << 23) : __uint_as_float(1u << 22);              // 2^-127 is a subnormal number
}

// The scale of a block whose largest magnitude has the bits `top`, as its byte, and what codes16 needs of it.
struct BlockScale {
  uint32_t byte;
  float p, r;                // DC_MX4: r = 1 / scale.  DC_NV4: p = scale, r = 1 / p rounded (0 for scale 0)
  bool cut;                  // values beyond 7 p: cut them before the division, which would overflow
};
template <int F>
__device__ __forceinline__ BlockScale block_scale(uint32_t top, float g, float r6) {
  BlockScale s;
  if (F == DC_MX4) {
    const uint32_t e = top >> 23;
    s.byte = e == 255u ? 255u : (e > 2u ? e - 2u : 0u);
    s.p = 0.f;
    s.r = e == 255u ? 0.f : __uint_as_float((254u - s.byte) << 23);
    s.cut = false;
  } else {
    // A product with 1 / (6 g), rounded, in the place of a division.  6 g is three times a power of two, and the rounded third is 2^-25 of it above a
    // third: where `top` is 6 g times a border of e4m3 the product rounds to the border itself, and the tie is seen as one.  Of bf16 values every
    // scale is so the one of real arithmetic (other quotients are 2^-8 from a border), of fp32 values those further than 2^-23 from one.
    // value / (s g) is divided: its quotient, rounded to fp32, lies on the same side of every border of e2m1 as the exact one, or on the border with
    // it, since a border times s g has at most 7 significant bits and the value 24.
    const bool odd = top >= 0x7f800000u;
    s.byte = odd ? 0x7fu : e4m3_of(__uint_as_float(top) * r6);
    s.p = odd ? 0.f : e4m3_value(s.byte) * g;
    s.r = s.p > 0.f ? __frcp_rn(s.p) : 0.f;
    s.cut = __uint_as_float(top) > 7.f * s.p;
  }
  return s;
}
// the largest magnitude of three numbers, NaN if one of them is
__device__ __forceinline__ float largest3(float a, float b, float c) {
  float d;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// of sixteen values; its bits
__device__ __forceinline__ uint32_t largest16(const float *v) {
  const float a = largest3(v[0], v[1], v[2]), b = largest3(v[3], v[4], v[5]), c = largest3(v[6], v[7], v[8]), d = largest3(v[9], v[10], v[11]),
              e = largest3(v[12], v[13], v[14]);
  return __float_as_uint(largest3(largest3(a, b, c), largest3(d, e, v[15]), 0.f));
}
// pairs of floats in one instruction
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ void unpair(uint64_t d, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(d)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
// sixteen values -> their codes, in two words.  Values of a block whose scale is NaN get some code.  BF16: they are bf16 numbers.
template <int F, bool BF16>
__device__ __forceinline__ uint2 codes16(float *v, const BlockScale &s) {
  if (F == DC_NV4 && s.cut) {
    const float m = 7.f * s.p;
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = fminf(fmaxf(v[i], -m), m);
  }
  const uint64_t r = pair(s.r, s.r), p = pair(-s.p, -s.p);
#pragma unroll
  for (int i = 0; i < 16; i += 2) {
    const uint64_t x = pair(v[i], v[i + 1]);
    uint64_t u;
    if (F == DC_MX4) {
      u = mul2(x, r);                            // exact
    } else if (BF16) {
      // x r on a grid of 2^-14 (768 has that unit in its last place): a quotient is a border of e2m1, which the grid has, or at least 2^-11 from all
      u = add2(fma2(x, r, pair(768.f, 768.f)), pair(-768.f, -768.f));
    } else {
      u = mul2(x, r);                            // x / p rounded: one step of Newton's method from x r
      u = fma2(fma2(u, p, x), r, u);
    }
    unpair(u, v[i], v[i + 1]);
  }
  return make_uint2(codes8(v), codes8(v + 8));
}

}  // namespace q4
