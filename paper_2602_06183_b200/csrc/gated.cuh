// Internal interface of the gated feed-forward block and of the 4-bit products: the kernel on CTA pairs for long operands
// (pair_product.cuh), the weight-streaming kernel for few tokens (few_tokens.cuh), and what both compute in their epilogues.
#pragma once

#include <cuda.h>

#include <cstdint>
#include <initializer_list>

#include "gemm_tc.cuh"
#include "sf_common.cuh"
#include "tc_ptx.cuh"

namespace sf {

// Operand formats of a product.
enum OperandFmt { FMT_BF16 = 0, FMT_NV = 1, FMT_MX = 2 };

// ---- activations ----------------------------------------------------------------------------------------
// Value and derivative of the gate's activation in float32. The sigmoid is written with the exponential of -x, so that neither
// tail cancels: 1 / (1 + e^-x) is 0 or 1 to within rounding there, and x times it underflows as the function does (rcp.approx holds to an
// ulp for every denominator; the fast division gives 0 from 2^126 on, which x < -87 reaches).
__device__ __forceinline__ float rcp32(float x) {
  float r;
  asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// max(x, 0) that keeps a NaN, as the products and the other activations do (fmaxf answers 0).
__device__ __forceinline__ float relu32(float x) {
  float r;
  asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float sigmoid32(float x) { return rcp32(1.f + __expf(-x)); }

// The normal distribution from its tail, Phi(-x) = e^(-x^2 / 2) p(1 / (1 + 0.3 x)) for x >= 0: the tail over its exponential is smooth in that
// variable, and a polynomial of degree 8 (weighted least squares over 0 <= x <= 14, the weights raised where the relative error was
// largest until it was level) is within 1.2e-7 of it (1.7e-7 beyond the fit, up to 14.5, where the exponential vanishes), 4e-7 in float32
// arithmetic (the reciprocal rounded to nearest). The tail also has the exponential's error, whose argument is rounded: x^2 2^-24 of itself, 1e-5 near x = 13. A library call
// that is as exact took the epilogue of the 1999 x 5504 x 1408 product 9600 issue cycles a tile, next to 11 300 of its main loop.
// e: the exponential, which the density shares.
__device__ __forceinline__ float normal_cdf(float g, float& e) {
  const float x = fabsf(g), t = rcp32(fmaf(0.3f, x, 1.f));
  float p = 0.038378290832042694f;
  p = fmaf(p, t, -0.16916611790657043f);
  p = fmaf(p, t, 0.22866007685661316f);
  p = fmaf(p, t, -0.07650648057460785f);
  p = fmaf(p, t, 0.1425355225801468f);
  p = fmaf(p, t, 0.09468352049589157f);
  p = fmaf(p, t, 0.12192033976316452f);
  p = fmaf(p, t, 0.1194876879453659f);
  p = fmaf(p, t, 7.168875981733436e-06f);
  e = __expf(-0.5f * g * g);
  const float tail = e * p;
  return g < 0.f ? tail : 1.f - tail;
}

template <int kAct>
__device__ __forceinline__ void gate_act(float g, float& a, float& da) {
  if constexpr (kAct == SF_ACT_SILU) {
    const float s = sigmoid32(g);
    a = g * s;
    da = s * fmaf(g, 1.f - s, 1.f);
  } else if constexpr (kAct == SF_ACT_GELU) {
    float e;
    const float c = normal_cdf(g, e);
    a = g * c;
    da = fmaf(g, 0.3989422804014327f * e, c);
  } else if constexpr (kAct == SF_ACT_GELU_TANH) {
    // 0.5 (1 + tanh(z)) = sigmoid(2 z), z = sqrt(2 / pi) (g + 0.044715 g^3); the sigmoid is 0 or 1 long before the square is cut off, which
    // without that would be infinite from 2^64 on and meet a factor of 0 in the derivative
    constexpr float k = 1.5957691216057308f, c3 = 0.044715f;
    const float g2 = fminf(g * g, 1e30f), s = sigmoid32(k * g * fmaf(c3, g2, 1.f));
    a = g * s;
    da = fmaf(a * (1.f - s), k * fmaf(3.f * c3, g2, 1.f), s);
  } else {
    const float r = relu32(g);
    a = kAct == SF_ACT_RELU ? r : r * r;
    da = kAct == SF_ACT_RELU ? (r > 0.f ? 1.f : r) : 2.f * r;
  }
}

// Calls f with the run-time activation (uniform over the grid) as a constant.
template <int kAct> struct ActTag { static constexpr int value = kAct; };
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  switch (act) {
    case SF_ACT_SILU: f(ActTag<SF_ACT_SILU>{}); break;
    case SF_ACT_GELU: f(ActTag<SF_ACT_GELU>{}); break;
    case SF_ACT_GELU_TANH: f(ActTag<SF_ACT_GELU_TANH>{}); break;
    case SF_ACT_RELU: f(ActTag<SF_ACT_RELU>{}); break;
    default: f(ActTag<SF_ACT_SQRELU>{}); break;
  }
}

inline bool act_ok(int act) { return act >= SF_ACT_SILU && act <= SF_ACT_SQRELU; }

// True in one lane of the (converged) warp. A warp that issues tcgen05 or TMA instructions walks its loop whole and issues in this
// lane: control flow and addresses are then the same for every lane, and the descriptors stay in uniform registers, where the
// instructions want them. With the loop inside a branch of lane 0 a 4-bit product of 2048 x 2304 x 65536 took 194 us instead of 113.
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.b32 %0, 1, 0, p;\n\t}\n" : "=r"(r));
  return r != 0;
}
// Four floats of the shared memory of a CTA of the cluster, at this CTA's own address of the same place.
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t saddr, uint32_t rank) {
  float4 v;
  asm volatile(
      "{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n\t}\n"
      : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(saddr), "r"(rank) : "memory");
  return v;
}
// ptx::smem_desc at address 0, as a constant, and the address that is added to it: in units of 16 bytes, without the bits above that name the
// CTA of the cluster and would run into the descriptor's next field.
__host__ __device__ constexpr uint64_t desc_proto(uint32_t lbo, uint32_t sbo, uint32_t swizzle) {
  return (uint64_t)(lbo >> 4) << 16 | (uint64_t)(sbo >> 4) << 32 | 1ull << 46 | (uint64_t)swizzle << 61;
}
__device__ __forceinline__ uint32_t desc_address(const void* p) { return (ptx::smem_u32(p) >> 4) & 0x3FFFu; }

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) { return float_to_bf16_bits(lo) | (float_to_bf16_bits(hi) << 16); }

// Instruction descriptor of the block-scaled kinds with E2M1 operands: scale format in bit 23 (0 E4M3, 1 power of two), the byte of
// a row's scale word that an instruction starts with in bits 4-5 (B) and 29-30 (A).
__host__ __device__ constexpr uint32_t idesc_fp4(uint32_t M, uint32_t N, int fmt) {
  return (1u << 7) | (1u << 10) | ((N >> 3) << 17) | (fmt == FMT_MX ? 1u << 23 : 0u) | ((M >> 7) << 27);
}

// ---- tensor maps ------------------------------------------------------------------------------------------
int sm_count_now();
// [rows, cols] of 4-byte floats, box 32 x 32, 128-byte swizzle.
int make_tmap_f32(void* map, const void* base, int64_t rows, int64_t cols);
// Stores of bf16 [rows, cols], box 32 x 32, 64-byte swizzle.
int make_tmap_store(void* map, void* base, int64_t rows, int64_t cols);
// Scale tiles of a 4-bit operand: [row blocks][tiles along K][128 words], box {128, tiles, 1}.
int make_tmap_scales(void* map, const void* base, int64_t row_blocks, int64_t k_tiles, uint32_t box_tiles);

// ---- products -----------------------------------------------------------------------------------------------
// A matrix operand: bf16 [rows, K] or, for the 4-bit formats, codes [rows, K / 2] with their scale tiles.
struct Operand {
  const void* data;
  const void* scales;
};

// Whether nothing that a call writes lies in what it reads or in something else that it writes. (The launches of a call read their inputs
// while others store results, so a shared byte would give results that depend on the order.) Absent ones are NULL.
struct Span {
  const void* p;
  size_t n;
};
inline bool meet(const Span& a, const Span& b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  return x && y && x < y + b.n && y < x + a.n;
}
inline bool apart(std::initializer_list<Span> written, std::initializer_list<Span> read) {
  for (const Span* w = written.begin(); w != written.end(); ++w) {
    for (const Span& r : read)
      if (meet(*w, r)) return false;
    for (const Span* v = written.begin(); v != w; ++v)
      if (meet(*w, *v)) return false;
  }
  return true;
}

}  // namespace sf
