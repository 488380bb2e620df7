// A pair of a row turned by an angle, spelled out with its roundings: rope.cu and append.cu give the same bits because both take
// these, and not by what a compiler makes of a sum of products.
#pragma once

namespace ckv {

// (a, b) -> (a cos - b sin, b cos + a sin): a product is rounded, and the sum of it and the other one.  The second sum's rounded
// product is that of a where bf16 rows are turned in whole vectors (`vectors`), that of b elsewhere.
__device__ __forceinline__ float turned_first(float a, float b, float c, float s) { return __fmaf_rn(a, c, -__fmul_rn(b, s)); }
__device__ __forceinline__ float turned_second(float a, float b, float c, float s, bool vectors) {
  return vectors ? __fmaf_rn(b, c, __fmul_rn(a, s)) : __fmaf_rn(a, s, __fmul_rn(b, c));
}

}  // namespace ckv
