// Partial sums of a gradient that several CTAs have made, added up in an order that does not depend on the launch.
#pragma once

#include "sf_common.cuh"

namespace sf {
namespace {

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float lo32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi32(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// out[c] = bf16(sum over p of parts[p][c]), 32 columns to a CTA, 32 runs of p added up by 32 x 8 threads and then in their order.
__global__ void __launch_bounds__(256)
sum_parts_kernel(const float4* __restrict__ parts, int count, int vecs, uint2* __restrict__ out) {
  __shared__ float4 part[32][8];
  const int c = (int)blockIdx.x * 8 + ((int)threadIdx.x & 7), p0 = (int)threadIdx.x >> 3;
  pdl_wait();
  pdl_trigger();
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < vecs) {
#pragma unroll 4
    for (int p = p0; p < count; p += 32) {
      const float4 v = __ldcg(parts + (int64_t)p * vecs + c);
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
  }
  part[p0][threadIdx.x & 7] = s;
  __syncthreads();
  if (p0 != 0 || c >= vecs) return;
#pragma unroll
  for (int k = 1; k < 32; ++k) {
    const float4 v = part[k][threadIdx.x & 7];
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  }
  out[c] = make_uint2(pack2(s.x, s.y), pack2(s.z, s.w));
}

inline int launch_sum_parts(const float* parts, int count, int64_t cols, void* out, cudaStream_t s) {
  const int64_t vecs = cols / 4;
  return launch_pdl(sum_parts_kernel, dim3((unsigned)((vecs + 7) / 8)), 256, 0, s, (const float4*)parts, count, (int)vecs, (uint2*)out);
}

}  // namespace
}  // namespace sf
