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
  p.page_stride = d.page_stride * (d.format == CKV_CACHE_PLAIN ? (d.dtype == CKV_F32 ? 4 : 2) : 1);
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

// Four 8-bit codes as floats, exact.
template <int FMT> __device__ __forceinline__ void decode4(uint32_t code, float (&x)[4]) {
  if (FMT == CKV_CACHE_E4M3) {
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
