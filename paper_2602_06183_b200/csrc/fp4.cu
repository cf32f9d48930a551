// Microscaled 4-bit operands: E2M1 codes with a scale to every block of a row, the passes between bf16 and that form, and the products.
//
//   code of a value   e2m1(x scale / sf): 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign, to nearest, ties to the even code, clamped at 6
//   SF_FP4_NV         blocks of 16, sf = e4m3(amax / 6), amax the block's largest |x scale|
//   SF_FP4_MX         blocks of 32, sf = 2^(floor(log2 amax) - 2), the exponent at least -127
//
// Scales are stored as the products read them: tiles of 128 rows x 4 scales, 512 bytes, scale c of row r at 16 (r % 32) + 4 (r / 32) + c;
// tiles of a row block follow each other along the row.
#include <cuda_fp4.h>

#include "fp8_fmt.cuh"
#include "products.cuh"

namespace sf {
namespace {

constexpr size_t kStatus = 256;

__device__ __forceinline__ int64_t scale_word(int64_t row, int64_t word, int64_t k_tiles) {     // of 4 scales, in words
  return ((row >> 7) * k_tiles + word) * 128 + (row & 31) * 4 + ((row >> 5) & 3);
}

// Eight E2M1 codes of eight floats, the first in the lowest nibble.
__device__ __forceinline__ uint32_t e2m1x8(const float* y) {
  uint32_t w;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}\n"
      : "=r"(w) : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  return w;
}

// Both passes are bounded by the instructions of their elements (the first forms, with an address worked out for every unit and every
// step in float32, took 241 instructions for 16 elements quantised and 125 for 8 read back: 38 and 37 us at 16384 x 4096, blocks of 16, where
// the memory needs 27; now 28.5 and 28.9). So a warp takes 128 units of one row, four a lane, whose addresses differ by constants; rows of fewer
// than 64 units share a warp (kShort: 2^lg slots a row). A scale of the tensor that is a power of two multiplies without
// rounding, and then goes into the factor of the block.
constexpr int kUnits = 4, kQuantThreads = 256;
struct WarpPlace { int64_t row; uint32_t c; };                         // of slot 0
__device__ __forceinline__ WarpPlace warp_place(uint32_t segments, int lg) {
  const uint32_t w = blockIdx.x * (kQuantThreads / 32) + (threadIdx.x >> 5), group = w / segments;
  return WarpPlace{(int64_t)group << (7 - lg), (w - group * segments) * 128u};
}

__device__ __forceinline__ float scale_value(uint32_t byte, int fmt) {
  if (fmt == FMT_NV) return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)byte, __NV_E4M3)));
  return byte == 255u ? __uint_as_float(0x7FFFFFFFu) : byte == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
}

// A unit is 16 consecutive elements of a row: one block (NV) or half of one (MX, whose other half is the neighbouring lane's).
// The quotient x / sf is needed to its last bit, since a bf16 value is often exactly half way between two codes. With r the reciprocal of
// sf rounded down and e = (1 - r sf) r what it lacks, x r + x e has an error of 2^-46 of itself before its one rounding, and a quotient
// of a 24-bit and a 4-bit number is never that near to the middle of two floats without being a float: the result is the
// rounded quotient. Two instructions an element instead of a division. Since e is not negative, both terms have the sign of x: a zero
// and an infinity keep theirs.
template <int kFmt, bool kPow2, bool kShort>
__global__ void __launch_bounds__(kQuantThreads)
quantize_fp4_kernel(const uint4* __restrict__ X, int64_t rows, uint32_t chunks, int64_t ld, float scale, uint32_t k_tiles, uint32_t segments, int lg,
                    uint2* __restrict__ codes, uint32_t* __restrict__ scales) {
  // a row's units are rounded up to whole scale words (4 or 8 units): those beyond the row write its padding scales
  constexpr uint32_t kPerWord = kFmt == FMT_NV ? 4 : 8;
  const uint32_t lane = threadIdx.x & 31u, per_row = k_tiles * kPerWord;
  const WarpPlace at = warp_place(segments, lg);
  auto row_of = [&](int j) { return kShort ? at.row + ((32u * j + lane) >> lg) : at.row; };
  auto unit_of = [&](int j) { return kShort ? (32u * j + lane) & ((1u << lg) - 1u) : at.c + 32u * j + lane; };
  pdl_wait();
  pdl_trigger();
  uint4 x[kUnits][2];
  const uint4* src = X + ((at.row * ld) >> 3) + 2 * (at.c + lane);
#pragma unroll
  for (int j = 0; j < kUnits; ++j) {
    if (row_of(j) < rows && unit_of(j) < chunks) {
      const uint4* p = kShort ? X + ((row_of(j) * ld) >> 3) + 2 * unit_of(j) : src + 64 * j;
      x[j][0] = __ldg(p);
      x[j][1] = __ldg(p + 1);
    } else {
      x[j][0] = x[j][1] = make_uint4(0u, 0u, 0u, 0u);
    }
  }
  const int64_t code0 = at.row * chunks + at.c + lane, word0 = scale_word(at.row, (at.c + lane) / kPerWord, k_tiles);
#pragma unroll
  for (int j = 0; j < kUnits; ++j) {
    const uint32_t w[8] = {x[j][0].x, x[j][0].y, x[j][0].z, x[j][0].w, x[j][1].x, x[j][1].y, x[j][1].z, x[j][1].w};
    // the block's largest magnitude in bf16 (a NaN wins), then its product with the scale, which keeps the order
    __nv_bfloat162 m2 = __habs2(*reinterpret_cast<const __nv_bfloat162*>(&w[0]));
#pragma unroll
    for (int i = 1; i < 8; ++i) m2 = __hmax2_nan(m2, __habs2(*reinterpret_cast<const __nv_bfloat162*>(&w[i])));
    if (kFmt == FMT_MX) {
      const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, *reinterpret_cast<const uint32_t*>(&m2), 1);
      m2 = __hmax2_nan(m2, *reinterpret_cast<const __nv_bfloat162*>(&other));
    }
    const float amax = fabsf(__fmul_rn(__bfloat162float(__hmax_nan(__low2bfloat16(m2), __high2bfloat16(m2))), scale));
    uint32_t byte;
    float v[16], rc, rest = 0.f;
    if constexpr (kFmt == FMT_NV) {
      byte = (uint32_t)__nv_cvt_float_to_fp8(__fdiv_rn(amax, 6.f), __NV_SATFINITE, __NV_E4M3);
      const float sf = scale_value(byte, kFmt);
      rc = sf > 0.f ? __frcp_rd(sf) : 0.f;
      rest = sf > 0.f ? __fmul_rn(__fmaf_rn(-rc, sf, 1.f), rc) : 0.f;
    } else {
      // the biased exponent less 2; 255 with a mantissa is NaN, and so is that scale
      const uint32_t bits = __float_as_uint(amax);
      byte = bits > 0x7F800000u ? 255u : (uint32_t)max((int)(bits >> 23) - 2, 0);
      rc = __uint_as_float((254u - min(byte, 253u)) << 23);                               // a power of two: exact
    }
    auto quotients = [&](bool folded) {
      if (folded) { rc *= scale; rest *= scale; }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float f = __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
        if (!folded) f = __fmul_rn(f, scale);
        v[i] = kFmt == FMT_NV ? __fmaf_rn(f, rc, __fmul_rn(f, rest)) : __fmul_rn(f, rc);
      }
    };
    // (the factor of a block, between 2^-9 and 2^9 for NV, must stay normal with the tensor's, which is between 2^-60 and 2^60)
    if (kPow2 && (kFmt == FMT_NV || (byte >= 64u && byte <= 190u))) quotients(true);
    else quotients(false);
    const bool in_rows = row_of(j) < rows, live = in_rows && unit_of(j) < chunks;
    // four scales leave as one word
    uint32_t word = live ? byte & 0xFFu : 0u;
    constexpr int kStep = kPerWord / 4;
    word |= __shfl_down_sync(0xFFFFFFFFu, word, kStep) << 8;
    word |= __shfl_down_sync(0xFFFFFFFFu, word, 2 * kStep) << 16;
    if (in_rows && unit_of(j) < per_row && lane % kPerWord == 0)
      scales[kShort ? scale_word(row_of(j), unit_of(j) / kPerWord, k_tiles) : word0 + j * (32 / kPerWord) * 128] = word;
    if (live) codes[kShort ? row_of(j) * chunks + unit_of(j) : code0 + 32 * j] = make_uint2(e2m1x8(v), e2m1x8(v + 8));
  }
}

// Eight codes as bf16 pairs, exact: the two bytes of each magnitude are looked up for four codes at a time.
__device__ __forceinline__ void e2m1_to_bf16x8(uint32_t q, uint32_t (&o)[4]) {
  const uint32_t m = q & 0x77777777u;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t sel = m >> (16 * h), s = q >> (16 * h);
    const uint32_t lo = __byte_perm(0xC0800000u, 0xC0804000u, sel), hi = __byte_perm(0x3F3F3F00u, 0x40404040u, sel);
    o[2 * h] = __byte_perm(lo, hi, 0x5140u) | (s & 0x8u) << 12 | (s & 0x80u) << 24;
    o[2 * h + 1] = __byte_perm(lo, hi, 0x7362u) | (s & 0x800u) << 4 | (s & 0x8000u) << 16;
  }
}

// A unit is eight elements: a word of codes, 16 bytes of results. code * sf is exact (two bits times four) before the product with alpha. An
// alpha that is a power of two keeps it so, and then the product of code and sf alpha is taken in bf16, which holds its six bits.
template <int kFmt, bool kPow2, bool kShort>
__global__ void __launch_bounds__(kQuantThreads)
dequantize_fp4_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t rows, uint32_t units, uint32_t k_tiles,
                      float alpha, int alpha_exp, uint32_t segments, int lg, uint4* __restrict__ Y, int64_t ld) {
  constexpr uint32_t kPerScale = kFmt == FMT_NV ? 2 : 4;
  const uint32_t lane = threadIdx.x & 31u;
  const WarpPlace at = warp_place(segments, lg);
  auto row_of = [&](int j) { return kShort ? at.row + ((32u * j + lane) >> lg) : at.row; };
  auto unit_of = [&](int j) { return kShort ? (32u * j + lane) & ((1u << lg) - 1u) : at.c + 32u * j + lane; };
  pdl_wait();
  pdl_trigger();
  uint32_t q[kUnits], by[kUnits];
  const uint32_t* src = codes + at.row * units + at.c + lane;
  const uint32_t n0 = (at.c + lane) / kPerScale;
  const uint8_t* sc = scales + 4 * scale_word(at.row, n0 >> 2, k_tiles) + (n0 & 3);
#pragma unroll
  for (int j = 0; j < kUnits; ++j) {
    q[j] = by[j] = 0;
    if (row_of(j) < rows && unit_of(j) < units) {
      if (kShort) {
        const uint32_t n = unit_of(j) / kPerScale;
        q[j] = __ldg(codes + row_of(j) * units + unit_of(j));
        by[j] = __ldg(scales + 4 * scale_word(row_of(j), n >> 2, k_tiles) + (n & 3));
      } else {
        q[j] = __ldg(src + 32 * j);
        by[j] = __ldg(sc + j * (32 / kPerScale / 4) * 512);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < kUnits; ++j) {
    uint32_t o[4];
    // (in range: neither factor nor product leaves bf16's normal numbers)
    const int e = (int)by[j] - 127;
    if (kPow2 && (kFmt == FMT_NV || (e >= -100 && e <= 100 && e + alpha_exp >= -100 && e + alpha_exp <= 100))) {
      e2m1_to_bf16x8(q[j], o);
      const __nv_bfloat162 f = __float2bfloat162_rn(scale_value(by[j], kFmt) * alpha);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&o[i]), f);
        o[i] = *reinterpret_cast<const uint32_t*>(&r);
      }
    } else {
      // (up to 6 2^127 leaves float32 before the product with a small alpha brings it back: two powers of two change sides, exactly)
      const bool far = kFmt == FMT_MX && by[j] >= 250u && by[j] < 255u && fabsf(alpha) < 1.f;
      const float sf = scale_value(far ? by[j] - 2u : by[j], kFmt), al = far ? 4.f * alpha : alpha;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __half2 h = __half2(__nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)(q[j] >> (8 * i) & 0xFFu), __NV_E2M1));
        o[i] = bf16x2(__fmul_rn(__fmul_rn(__low2float(h), sf), al), __fmul_rn(__fmul_rn(__high2float(h), sf), al));
      }
    }
    if (row_of(j) < rows && unit_of(j) < units)
      Y[kShort ? ((row_of(j) * ld) >> 3) + unit_of(j) : ((at.row * ld) >> 3) + at.c + lane + 32 * j] = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// How the units of rows are dealt out to warps (see above).
struct QuantGrid { uint32_t segments; int lg; int64_t blocks; bool is_short; };
QuantGrid quant_grid(int64_t rows, int64_t per_row) {
  QuantGrid g{1, 0, 0, per_row < 64};
  while (((int64_t)1 << g.lg) < per_row && g.lg < 7) ++g.lg;
  if (!g.is_short) { g.lg = 7; g.segments = (uint32_t)ceil_div(per_row, 128); }
  g.blocks = ceil_div(ceil_div(rows, 128 >> g.lg) * g.segments, kQuantThreads / 32);
  return g;
}
// Whether a factor is a power of two whose products with a block's factors stay normal; its exponent.
bool plain_power(float f, int* e) {
  const float m = std::frexp(f, e);
  *e -= 1;
  return m == 0.5f && *e >= -60 && *e <= 60;
}

int fmt_of(int format) { return format == SF_FP4_NV ? FMT_NV : format == SF_FP4_MX ? FMT_MX : -1; }

Span codes_span(const void* p, int64_t rows, int64_t cols) { return {p, (size_t)rows * (size_t)cols / 2}; }
Span scales_span(const void* p, int64_t rows, int64_t cols, int format) {
  return {p, (size_t)ceil_div(rows, 128) * (size_t)scale_tiles(fmt_of(format), cols) * 512};
}
// bf16 rows, from the first element to the last
Span rows_span(const void* p, int64_t rows, int64_t cols, int64_t ld) { return {p, 2 * ((size_t)(rows - 1) * (size_t)ld + (size_t)cols)}; }

template <int kFmt>
int fp4_plan(int64_t M, int64_t N, int64_t K, bool gated, sf_fp4_plan* plan) {
  const int nkb = k_blocks(kFmt, K);
  PairPlan p;
  if (gated ? gated_by_few(kFmt, M, nkb) : M <= kFewTokens) {
    FewArgs a{};
    a.T = (int)M; a.N = (int)N; a.nkb = nkb; a.in_terms = 1;
    NoMaps none;
    SF_TRY(gated ? (run_few<kFmt, FK_GATED>(a, nullptr, none, &p)) : (run_few<kFmt, FK_NT>(a, nullptr, none, &p)));
    *plan = sf_fp4_plan{SF_GATED_FEW, p.bn, p.parts};
  } else if (gated) {
    *plan = sf_fp4_plan{SF_GATED_TILES, 256, 1};
  } else {
    SF_TRY(plan_fp4(M, N, nkb, &p));
    *plan = sf_fp4_plan{p.mode == PM_SPLIT ? SF_GATED_SPLIT : SF_GATED_TILES, p.bn, p.parts};
  }
  return SF_OK;
}

int fp4_shape(int64_t rows, int64_t cols, int format) {
  if (fmt_of(format) < 0) return SF_ERR_UNSUPPORTED;
  return rows < 0 || cols < 0 || cols % 32 || rows > kMaxSize || cols > kMaxSize ? SF_ERR_SHAPE : SF_OK;
}

}  // namespace
}  // namespace sf

using namespace sf;

extern "C" {

int sf_fp4_sizes(int64_t rows, int64_t cols, int format, size_t* codes_bytes, size_t* scales_bytes) {
  SF_TRY(fp4_shape(rows, cols, format));
  if (!codes_bytes || !scales_bytes) return SF_ERR_NULL;
  *codes_bytes = codes_span(nullptr, rows, cols).n;
  *scales_bytes = scales_span(nullptr, rows, cols, format).n;
  return SF_OK;
}

int sf_fp4_quantize(const void* X, int64_t rows, int64_t cols, int64_t ld, int format, float scale, void* codes, void* scales, void* stream) {
  SF_TRY(fp4_shape(rows, cols, format));
  if (rows == 0 || cols == 0) return SF_OK;
  if (!X || !codes || !scales) return SF_ERR_NULL;
  if (ld < cols || ld % 8 || !aligned16(X) || !aligned16(codes) || !aligned16(scales)) return SF_ERR_ALIGN;
  if (std::isinf(scale)) return SF_ERR_UNSUPPORTED;         // (0 times it is NaN, which a block's largest magnitude does not show)
  if (!apart({codes_span(codes, rows, cols), scales_span(scales, rows, cols, format)}, {rows_span(X, rows, cols, ld)})) return SF_ERR_UNSUPPORTED;
  const int fmt = fmt_of(format);
  const int64_t k_tiles = scale_tiles(fmt, cols);
  const QuantGrid g = quant_grid(rows, k_tiles * (fmt == FMT_NV ? 4 : 8));
  if (g.blocks > 0x0FFFFFFF) return SF_ERR_SHAPE;
  SF_TRY(check_arch());
  int e;
  const bool p2 = plain_power(scale, &e);
  auto kern = fmt == FMT_NV ? (p2 ? (g.is_short ? quantize_fp4_kernel<FMT_NV, true, true> : quantize_fp4_kernel<FMT_NV, true, false>)
                                  : (g.is_short ? quantize_fp4_kernel<FMT_NV, false, true> : quantize_fp4_kernel<FMT_NV, false, false>))
                            : (p2 ? (g.is_short ? quantize_fp4_kernel<FMT_MX, true, true> : quantize_fp4_kernel<FMT_MX, true, false>)
                                  : (g.is_short ? quantize_fp4_kernel<FMT_MX, false, true> : quantize_fp4_kernel<FMT_MX, false, false>));
  return launch_pdl(kern, dim3((unsigned)g.blocks), kQuantThreads, 0, (cudaStream_t)stream, (const uint4*)X, rows, (uint32_t)(cols / 16), ld,
                    scale, (uint32_t)k_tiles, g.segments, g.lg, (uint2*)codes, (uint32_t*)scales);
}

int sf_fp4_dequantize(const void* codes, const void* scales, int64_t rows, int64_t cols, int format, float alpha, void* Y, int64_t ld,
                      void* stream) {
  SF_TRY(fp4_shape(rows, cols, format));
  if (rows == 0 || cols == 0) return SF_OK;
  if (!Y || !codes || !scales) return SF_ERR_NULL;
  if (ld < cols || ld % 8 || !aligned16(Y) || !aligned16(codes) || !aligned16(scales)) return SF_ERR_ALIGN;
  if (!apart({rows_span(Y, rows, cols, ld)}, {codes_span(codes, rows, cols), scales_span(scales, rows, cols, format)})) return SF_ERR_UNSUPPORTED;
  const int fmt = fmt_of(format);
  const QuantGrid g = quant_grid(rows, cols / 8);
  if (g.blocks > 0x0FFFFFFF) return SF_ERR_SHAPE;
  SF_TRY(check_arch());
  int e;
  const bool p2 = plain_power(alpha, &e);
  auto kern = fmt == FMT_NV ? (p2 ? (g.is_short ? dequantize_fp4_kernel<FMT_NV, true, true> : dequantize_fp4_kernel<FMT_NV, true, false>)
                                  : (g.is_short ? dequantize_fp4_kernel<FMT_NV, false, true> : dequantize_fp4_kernel<FMT_NV, false, false>))
                            : (p2 ? (g.is_short ? dequantize_fp4_kernel<FMT_MX, true, true> : dequantize_fp4_kernel<FMT_MX, true, false>)
                                  : (g.is_short ? dequantize_fp4_kernel<FMT_MX, false, true> : dequantize_fp4_kernel<FMT_MX, false, false>));
  return launch_pdl(kern, dim3((unsigned)g.blocks), kQuantThreads, 0, (cudaStream_t)stream, (const uint32_t*)codes, (const uint8_t*)scales, rows,
                    (uint32_t)(cols / 8), (uint32_t)scale_tiles(fmt, cols), alpha, e, g.segments, g.lg, (uint4*)Y, ld);
}

int sf_gemm_fp4_workspace_size(int64_t Mr, int64_t Nc, int64_t K, size_t* bytes) {
  if (!bytes) return SF_ERR_NULL;
  if (Mr < 0 || Nc < 0 || K <= 0 || Nc % 8 || K % 32 || Mr > kMaxSize || Nc > kMaxSize || K > kMaxSize) return SF_ERR_SHAPE;
  *bytes = kStatus;
  return SF_OK;
}

int sf_gemm_fp4_plan(int64_t Mr, int64_t Nc, int64_t K, int format, int gated, sf_fp4_plan* plan) {
  size_t need;
  if (fmt_of(format) < 0) return SF_ERR_UNSUPPORTED;
  SF_TRY(sf_gemm_fp4_workspace_size(Mr, Nc, K, &need));
  if (!plan) return SF_ERR_NULL;
  *plan = sf_fp4_plan{SF_GATED_NONE, 0, 0};
  if (Mr == 0 || Nc == 0) return SF_OK;
  return format == SF_FP4_NV ? fp4_plan<FMT_NV>(Mr, Nc, K, gated != 0, plan) : fp4_plan<FMT_MX>(Mr, Nc, K, gated != 0, plan);
}

int sf_gemm_fp4(const void* A, const void* a_scales, const void* B, const void* b_scales, int format, void* C, int64_t Mr, int64_t Nc,
                int64_t K, float alpha, void* workspace, size_t workspace_bytes, void* stream) {
  size_t need;
  if (fmt_of(format) < 0) return SF_ERR_UNSUPPORTED;
  SF_TRY(sf_gemm_fp4_workspace_size(Mr, Nc, K, &need));
  if (Mr == 0 || Nc == 0) return SF_OK;
  if (!A || !a_scales || !B || !b_scales || !C || !workspace) return SF_ERR_NULL;
  if (!aligned16(A) || !aligned16(a_scales) || !aligned16(B) || !aligned16(b_scales) || !aligned16(C) || !aligned16(workspace)) return SF_ERR_ALIGN;
  if (workspace_bytes < need) return SF_ERR_WORKSPACE;
  if (!apart({rows_span(C, Mr, Nc, Nc), {workspace, need}}, {codes_span(A, Mr, K), scales_span(a_scales, Mr, K, format), codes_span(B, Nc, K),
                                                            scales_span(b_scales, Nc, K, format)}))
    return SF_ERR_UNSUPPORTED;
  SF_TRY(check_arch());
  const Operand a{A, a_scales}, b{B, b_scales};
  return format == SF_FP4_NV ? run_nt<FMT_NV>(a, b, Mr, Nc, K, alpha, C, (int*)workspace, (cudaStream_t)stream)
                             : run_nt<FMT_MX>(a, b, Mr, Nc, K, alpha, C, (int*)workspace, (cudaStream_t)stream);
}

int sf_gemm_fp4_gated(const void* A, const void* a_scales, const void* Bg, const void* bg_scales, const void* Bu, const void* bu_scales,
                      int format, int act, void* H, int64_t Mr, int64_t Nc, int64_t K, float alpha_g, float alpha_u, void* workspace,
                      size_t workspace_bytes, void* stream) {
  size_t need;
  if (fmt_of(format) < 0 || !act_ok(act)) return SF_ERR_UNSUPPORTED;
  SF_TRY(sf_gemm_fp4_workspace_size(Mr, Nc, K, &need));
  if (Mr == 0 || Nc == 0) return SF_OK;
  if (!A || !a_scales || !Bg || !bg_scales || !Bu || !bu_scales || !H || !workspace) return SF_ERR_NULL;
  if (!aligned16(A) || !aligned16(a_scales) || !aligned16(Bg) || !aligned16(bg_scales) || !aligned16(Bu) || !aligned16(bu_scales) ||
      !aligned16(H) || !aligned16(workspace))
    return SF_ERR_ALIGN;
  if (workspace_bytes < need) return SF_ERR_WORKSPACE;
  if (!apart({rows_span(H, Mr, Nc, Nc), {workspace, need}},
             {codes_span(A, Mr, K), scales_span(a_scales, Mr, K, format), codes_span(Bg, Nc, K), scales_span(bg_scales, Nc, K, format),
              codes_span(Bu, Nc, K), scales_span(bu_scales, Nc, K, format)}))
    return SF_ERR_UNSUPPORTED;
  SF_TRY(check_arch());
  const Operand a{A, a_scales}, g{Bg, bg_scales}, u{Bu, bu_scales};
  return format == SF_FP4_NV
             ? run_gated<FMT_NV>(a, g, u, Mr, Nc, K, act, alpha_g, alpha_u, H, nullptr, nullptr, (int*)workspace, (cudaStream_t)stream)
             : run_gated<FMT_MX>(a, g, u, Mr, Nc, K, act, alpha_g, alpha_u, H, nullptr, nullptr, (int*)workspace, (cudaStream_t)stream);
}

}  // extern "C"
