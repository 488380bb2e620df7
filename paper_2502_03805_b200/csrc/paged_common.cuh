// The paged cache as its kernels see it, and the conversions of its formats.
#pragma once
#include <cuda_fp16.h>

#include <type_traits>

#include "ckv_internal.h"

namespace ckv {

constexpr float kLeastScale = 7.888609052210118e-31f;   // 2^-100: smallest scale of a quantised row

struct Pages {
  char* page[2];             // k_pages, v_pages
  float* scale[2];           // [num_pages << page_shift], null for the plain format
  uint8_t* group[2];         // [num_pages << page_shift, dh / 16] e4m3, e2m1 format only
  const int32_t* table;      // [nseq * Hkv, max_pages]
  long long page_stride;     // bytes from page to page
  long long capacity;        // max_pages << page_shift, at most 2^31 - 1
  int Hkv, max_pages, num_pages, page_shift;
};

inline Pages pages_of(const CacheDims& d) {
  Pages p;
  p.page[0] = (char*)d.k_pages; p.page[1] = (char*)d.v_pages;
  p.scale[0] = d.k_scale; p.scale[1] = d.v_scale;
  p.table = d.page_table;
  p.group[0] = d.k_group; p.group[1] = d.v_group;
  p.page_stride = stored_bytes(d.format, d.dtype, d.page_stride);
  p.capacity = d.capacity;
  p.Hkv = d.Hkv; p.max_pages = d.max_pages; p.num_pages = d.num_pages; p.page_shift = d.page_shift;
  return p;
}

// Two e4m3 codes (low byte first) as two halves: exact, every e4m3 value is a half.
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
  return h;
}

// Eight e2m1 codes (lowest half byte first) as pairs of halves: exact.  For words that are loaded as 32 bits or more, and for what
// is masked and mixed from such.  nvcc 12.9 keeps two 16-bit loads in one register and then converts bytes of the wrong half (a prmt
// in front, which makes a register of the word, prevents that at 4 % of a decode call).
__device__ __forceinline__ void e2m1x8_to_half2(uint32_t eight, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(eight));
}
// Four of them, which a 16-bit load may give, by shifts that place a code's exponent and fraction bits in a half that is 2^-14 times
// its value: exact.
__device__ __forceinline__ void e2m1x4_to_half2(uint32_t four, uint32_t (&h)[2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t two = ((four >> (8 * i)) & 0xfu) | (((four >> (8 * i)) & 0xf0u) << 12);
    const uint32_t bits = ((two & 0x00080008u) << 12) | ((two & 0x00070007u) << 9);
    const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&bits), __half2half2(__ushort_as_half(0x7400)));   // 2^14
    h[i] = *reinterpret_cast<const uint32_t*>(&x);
  }
}
__device__ __forceinline__ float e4m3_to_float(uint32_t one) {
  const uint32_t h = e4m3x2_to_half2(one);
  return __half2float(__ushort_as_half((unsigned short)h));
}

// Eight e2m1 codes of a group with the e4m3 scale `group` as floats: code times group scale, exact in a half.
__device__ __forceinline__ void decode8_e2m1(uint32_t eight, uint32_t group, float (&x)[8]) {
  uint32_t h[4];
  e2m1x8_to_half2(eight, h);
  const uint32_t two = e4m3x2_to_half2(group * 0x101u);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 y = __hmul2(*reinterpret_cast<const __half2*>(&h[i]), *reinterpret_cast<const __half2*>(&two));
    const float2 f = __half22float2(y);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}

// Four codes as floats, exact: bytes, or for e2m1 the low four half bytes.
template <int FMT> __device__ __forceinline__ void decode4(uint32_t code, float (&x)[4]) {
  if (FMT == CKV_CACHE_E2M1) {
    uint32_t h[2];
    e2m1x4_to_half2(code, h);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  } else if (FMT == CKV_CACHE_E4M3) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t h = e4m3x2_to_half2(code >> (16 * i));
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(code >> (8 * i));
  }
}

}  // namespace ckv
