// The first X of an orthogonalised update: G as the sum of two fp16 numbers (see newton_schulz.cu).
#pragma once

#include <cmath>

#include "products.cuh"

namespace sf {
namespace {

template <bool kF32>
__device__ __forceinline__ float element(const void* G, int64_t i) {
  if constexpr (kF32) return __ldg(reinterpret_cast<const float*>(G) + i);
  else return bf16_bits_to_float(__ldg(reinterpret_cast<const uint16_t*>(G) + i));
}

// G 2^k in fp16 (two terms of a float32 G; a bf16 G fits one), k such that its norm lies in [2^13, 2^14); what is left of the norm, a factor of
// 1 to 2 that is no power of two, goes into the first step's float32 arithmetic (*first), so that a bf16 G is not rounded at all. A G
// of zeros stays zero; where G's norm is not finite the factor is NaN, and so is every result.
struct NsScale { float lo, hi; };      // two powers of two whose product is 2^k
__device__ __forceinline__ NsScale ns_scale_of(double squares, float* first) {
  const double norm = sqrt(squares);
  int k = 0;
  float f = 0.f;
  if (!(norm < INFINITY)) {
    f = __uint_as_float(0x7FC00000u);
  } else if (norm > 0) {
    k = 13 - ilogb(norm);
    f = (float)(16384.0 / scalbn(norm, k));
  }
  *first = f;
  const int h = k / 2;
  return NsScale{scalbnf(1.f, h), scalbnf(1.f, k - h)};
}
__device__ __forceinline__ void ns_terms(float x, const NsScale& z, uint16_t& hi, uint16_t& lo) {
  const float y = x * z.lo * z.hi;
  const __half h = __float2half_rn(y), l = __float2half_rn(y - __half2float(h));
  hi = __half_as_ushort(h);
  lo = __half_as_ushort(l);
}

}  // namespace
}  // namespace sf
