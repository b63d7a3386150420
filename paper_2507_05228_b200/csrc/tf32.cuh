// fp32 operands in two tf32 parts for warp-level products.
#pragma once

#include <stdint.h>

namespace cascade {

__device__ __forceinline__ void mma_tf32(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// x = hi + lo, hi the upper 11 bits of the mantissa, lo rounded to tf32 by the product's truncation: hi hi + hi lo + lo hi keeps what
// lies above 2^-21 of a product.  hi is cut off for keys and values, and rounded for queries and weights: the signs of the parts that
// hi leaves out are then not those of the operands on both sides, and the missing lo lo averages out.
__device__ __forceinline__ void cut(float x, uint32_t& hi, uint32_t& lo) {
  hi = __float_as_uint(x) & 0xffffe000u;
  lo = __float_as_uint(x - __uint_as_float(hi)) + 0x1000u;
}
__device__ __forceinline__ void cut_rounded(float x, uint32_t& hi, uint32_t& lo) {  // x: at most 1
  hi = (__float_as_uint(x) + 0x1000u) & 0xffffe000u;
  lo = __float_as_uint(x - __uint_as_float(hi)) + 0x1000u;
}
// The same for any x.  Added to all ones, a NaN of the GPU's own, the half step would wrap around to zero, and the largest finite values
// would become infinite: beyond what rounds to a finite value nothing is added.  NaN and infinities then have a lo that is NaN.
// (512 fp32 rows over 4000, 32 / 8 heads of 128: 718 us without, so 729; by cvt.rna.satfinite 736.)
__device__ __forceinline__ void cut_query(float x, uint32_t& hi, uint32_t& lo) {
  const uint32_t half = fabsf(x) < 0x1.ffep127f ? 0x1000u : 0u;
  hi = (__float_as_uint(x) + half) & 0xffffe000u;
  lo = __float_as_uint(x - __uint_as_float(hi)) + half;
}

}  // namespace cascade
