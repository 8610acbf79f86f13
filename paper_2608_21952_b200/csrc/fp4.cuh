// Matrices in four bits (ssdi8_fp4_t): conversions, and a block's scale and codes from its values.
#pragma once
#include "block.cuh"

namespace ssdi8 {

// scales stand in tiles of 128 rows x 4 blocks, 512 bytes each, all of a row block beside one another: row 32 i + j of a tile has its
// four bytes at 16 j + 4 i (as the tensor cores' scale operands lie in tensor memory: 32 lanes of four words)
constexpr int kTileBytes = 512;
__host__ __device__ __forceinline__ int fp4_tiles(int width, int block) { return (width / block + 3) / 4; }
__device__ __forceinline__ i64 fp4_scale_at(i64 row, int tile, int tiles) {
  return ((row >> 7) * tiles + tile) * kTileBytes + ((row & 31) << 4) + ((row >> 5 & 3) << 2);
}

// e2m1 codes of eight values, the first in the lowest four bits; nearest, ties to even, beyond 6 the largest, NaN +6
__device__ __forceinline__ uint32_t e2m1_of8(const float (&v)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}
// the values of eight codes
__device__ __forceinline__ void e2m1_to8(uint32_t r, float (&v)[8]) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(r));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}
// e4m3 of a value >= 0 that is not NaN (nearest, ties to even, at most 448), and its value
__device__ __forceinline__ uint32_t e4m3_of(float v) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(v));
  return r;
}
__device__ __forceinline__ float e4m3_to(uint32_t b) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)b));
  return __half2float(__ushort_as_half((unsigned short)(h & 0xffffu)));
}
__device__ __forceinline__ float power_of_two(uint32_t b) {   // 2^(b - 127), b < 255
  return __uint_as_float(b == 0u ? 0x00400000u : b << 23);
}
__device__ __forceinline__ float e8m0_to(uint32_t b) {   // the same, of 255 a NaN
  uint32_t h;
  asm("cvt.rn.bf16x2.ue8m0x2 %0, %1;" : "=r"(h) : "h"((uint16_t)b));
  return __uint_as_float(h << 16);
}

// Blocks of 16 of a row with absmax m: the row's step size g is fdiv(m, 2688) (the largest code times the largest scale) with the low eight bits of its
// significand cleared; 1 if that is 0.  With 16 bits in g and 4 in a scale, what lies in the middle of two codes or of two scales is a
// binary32 number (the middles have 3 and 5 bits of their own), and a value that is not such a middle b d is 2^-24 of it away at least.
// Quotients are formed as the product t with an approximate reciprocal y (2^-23) and one correction, t + (p - t d) y (Markstein, IBM J. Res. Dev. 34, 1990):
// what is rounded is p / d up to 1.5 x 2^-46 of it.  That is b for p = b d, and for the p next to it 2^-44 off where it would round to b
// (b = 1/4, the only power of two among the middles, and a significand of p up to 2 - 2^-19, as d has 20 bits; 2^-28 and more elsewhere): codes
// and scales are those of the exact quotients.  Rows whose step size leaves [1e-25, 1e25] take divisions, which keep to the
// side of b as well, down to an absmax of 2e-32, below which d is subnormal.
struct Fp4Row {
  float g, unit, y;   // step size, 6 g, its reciprocal (approximate)
  bool safe;
};
__device__ __forceinline__ Fp4Row fp4_row(float m) {
  Fp4Row r;
  constexpr float c = 1.0f / 2688.0f;
  // (the correctly rounded quotient: for all 2^23 significands of m)
  const float t = __fmul_rn(m, c);
  float g = __fmaf_rn(__fmaf_rn(-t, 2688.0f, m), c, t);
  r.safe = g >= 1e-25f && g <= 1e25f;
  if (!r.safe) g = __fdiv_rn(m, 2688.0f);
  g = __uint_as_float(__float_as_uint(g) & 0xffffff00u);
  r.g = g > 0.f ? g : 1.0f;
  r.unit = __fmul_rn(6.0f, r.g);
  r.y = rcp_approx(r.unit);
  return r;
}
// scale byte of a block of 16 with absmax m: e4m3 of m / (6 g), at least the smallest e4m3 above 0 (inf / inf too)
template <bool SAFE>
__device__ __forceinline__ uint32_t fp4_scale16(float m, const Fp4Row& r) {
  float q = __fmul_rn(m, r.y);
  q = SAFE ? __fmaf_rn(__fmaf_rn(-q, r.unit, m), r.y, q) : __fdiv_rn(m, r.unit);
  return e4m3_of(fmaxf(q, 0.001953125f));
}
// scale byte of a block of 32: the least power of two s in [2^-127, 2^127] with m <= 6 s; 1 if m is 0
__device__ __forceinline__ uint32_t fp4_scale32(float m) {
  const uint32_t b = __float_as_uint(m), e = b >> 23;
  if (b == 0u) return 127u;
  // m = f 2^(e - 127), 1 <= f < 2: s = 2^(e - 129), or twice that above 1.5 (in subnormal m, the smallest s is far enough)
  const uint32_t up = (b & 0x7fffffu) > 0x400000u ? 1u : 0u;
  return e + up < 2u ? 0u : min(e + up - 2u, 254u);
}
// Codes of eight values: of a block of 16 over d = fmul(g, scale), of a block of 32 whose scale byte is b (exact products).  A zero of either sign has the code 0.
template <bool SAFE>
__device__ __forceinline__ uint32_t fp4_codes16(const float (&p)[8], const Fp4Row& r, float scale) {
  const float d = __fmul_rn(r.g, scale);
  float q[8];
  if (!SAFE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = __fdiv_rn(p[i], d) + 0.f;
    return e2m1_of8(q);
  }
  const float y = rcp_approx(d);
  const float2 yy = make_float2(y, y), nd = make_float2(-d, -d);
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const float2 v = make_float2(p[i], p[i + 1]), t = __fmul2_rn(v, yy);
    const float2 x = __ffma2_rn(__ffma2_rn(t, nd, v), yy, t);
    q[i] = x.x;
    q[i + 1] = x.y;
  }
  return e2m1_of8(q);
}
__device__ __forceinline__ uint32_t fp4_codes32(const float (&p)[8], uint32_t b) {
  const float y = power_of_two(254u - b);
  const float2 yy = make_float2(y, y), zero = make_float2(0.f, 0.f);
  float q[8];
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const float2 x = __ffma2_rn(make_float2(p[i], p[i + 1]), yy, zero);
    q[i] = x.x;
    q[i + 1] = x.y;
  }
  return e2m1_of8(q);
}

}  // namespace ssdi8
