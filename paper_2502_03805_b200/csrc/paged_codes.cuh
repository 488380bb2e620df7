// Rows of the paged cache on their way in: pieces of source rows as floats, and scales and codes (criticalkv.h states the rules).
#pragma once
#include <cuda_bf16.h>

#include "paged_common.cuh"

namespace ckv {

// (a, b) rounded to two e4m3 codes, a in the low byte.
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
  uint16_t v;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(v) : "f"(b), "f"(a));
  return v;
}

// 16 bytes of a source row as floats.
template <typename T> struct Piece;
template <> struct Piece<float> {
  static constexpr int V = 4;
  static __device__ __forceinline__ void get(const uint4& r, float (&x)[4]) {
    x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ uint4 put(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
__device__ __forceinline__ uint32_t bf16x2(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <> struct Piece<__nv_bfloat16> {
  static constexpr int V = 8;
  static __device__ __forceinline__ void get(const uint4& r, float (&x)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 put(const float (&x)[8]) {
    return make_uint4(bf16x2(x[0], x[1]), bf16x2(x[2], x[3]), bf16x2(x[4], x[5]), bf16x2(x[6], x[7]));
  }
};

// Largest magnitudes are found on the bit patterns, whose order puts NaN above infinity, so a row with a NaN gets a NaN scale.
template <int N> __device__ __forceinline__ uint32_t top_bits(const float (&x)[N]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  return top;
}

// Scale of a row whose largest magnitude has the bits `top`.
template <int FMT> __device__ __forceinline__ float row_scale(uint32_t top) {
  constexpr float kTop = FMT == CKV_CACHE_E2M1 ? 2688.f : FMT == CKV_CACHE_E4M3 ? 448.f : 127.f;
  float scale = __fdiv_rn(__uint_as_float(top), kTop);
  if (scale < kLeastScale) scale = kLeastScale;
  // a row that reaches the largest float must not read back as infinity because the quotient was rounded up
  if (top < 0x7f800000u && __fmul_rn(scale, kTop) == INFINITY) scale = __uint_as_float(__float_as_uint(scale) - 1);
  return scale;
}

// Codes of four elements; r: reciprocal of the row's scale.
template <int FMT> __device__ __forceinline__ uint32_t encode4(const float* x, float r) {
  float y[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = __fmul_rn(x[j], r);
  if (FMT == CKV_CACHE_E4M3) return e4m3x2(y[0], y[1]) | (e4m3x2(y[2], y[3]) << 16);
  uint32_t code = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    code |= ((uint32_t)min(max(__float2int_rn(y[j]), -127), 127) & 0xffu) << (8 * j);   // NaN becomes 0
  return code;
}

// Scale of a group of 16 elements of a 4-bit row as an e4m3 code: largest magnitude of the group, reciprocal r of the row's
// scale (of which `finite` says whether it is one), and the factor of the group's elements.
__device__ __forceinline__ uint32_t group_scale(float top, float r, bool finite, float& factor) {
  const uint32_t g = finite ? e4m3x2(__fmul_rn(__fmul_rn(top, r), 1.f / 6.f), 0.f) : 0u;
  const float s = e4m3_to_float(g);
  factor = s > 0.f ? __fdiv_rn(r, s) : 0.f;
  return g;
}

// Eight elements as e2m1 codes, the first in the lowest half byte; zeros where the factor is 0 (infinities and NaN, and the
// sign of zeros, included).
__device__ __forceinline__ uint32_t encode8_e2m1(const float* x, float factor) {
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = __fmul_rn(x[j], factor);
  uint32_t code;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(code)
      : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  return factor == 0.f ? 0u : code;
}

}  // namespace ckv
