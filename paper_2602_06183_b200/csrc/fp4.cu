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
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w |= (uint32_t)__nv_cvt_float2_to_fp4x2(make_float2(y[2 * i], y[2 * i + 1]), __NV_E2M1, cudaRoundNearest) << (8 * i);
  return w;
}

// A thread takes 16 consecutive elements of a row: one block (NV) or half of one (MX, whose other half is the neighbouring lane's).
// The quotient x / sf is needed to its last bit, since a bf16 value is often exactly half way between two codes. With r the reciprocal of
// sf rounded down and e = (1 - r sf) r what it lacks, x r + x e has an error of 2^-46 of itself before its one rounding, and a quotient
// of a 24-bit and a 4-bit number is never that near to the middle of two floats without being a float: the result is the
// rounded quotient. Two instructions an element instead of a division. Since e is not negative, both terms have the sign of x: a zero
// and an infinity keep theirs.
template <int kFmt>
__global__ void __launch_bounds__(256)
quantize_fp4_kernel(const uint4* __restrict__ X, int64_t rows, int chunks, int64_t ld, float scale, int k_tiles, uint2* __restrict__ codes,
                    uint32_t* __restrict__ scales) {
  pdl_wait();
  pdl_trigger();
  // a row's threads are rounded up to whole scale words (4 or 8 threads): those beyond the row write its padding scales
  constexpr int kPerWord = kFmt == FMT_NV ? 4 : 8;
  const int per_row = k_tiles * kPerWord;
  const int64_t idx = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int64_t r = idx / per_row;
  const int c = (int)(idx - r * per_row);
  const bool live = r < rows && c < chunks;
  uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (live) {
    const uint4* src = X + ((r * ld) >> 3) + 2 * c;
    const uint4 a = __ldg(src), b = __ldg(src + 1);
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
  }
  float v[16];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[2 * i] = __fmul_rn(bf16_bits_to_float(w[i] & 0xFFFFu), scale);
    v[2 * i + 1] = __fmul_rn(bf16_bits_to_float(w[i] >> 16), scale);
  }
  // as integers, magnitudes are ordered like the values, infinity and NaN above all of them
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) amax = max(amax, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  if (kFmt == FMT_MX) amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
  uint32_t byte;
  float sf;
  if constexpr (kFmt == FMT_NV) {
    byte = (uint32_t)__nv_cvt_float_to_fp8(__fdiv_rn(__uint_as_float(amax), 6.f), __NV_SATFINITE, __NV_E4M3);
    sf = __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)byte, __NV_E4M3)));
  } else {
    const int e = (int)(amax >> 23);                       // biased exponent; 255 with a mantissa is NaN, and so is that scale
    byte = amax > 0x7F800000u ? 255u : (uint32_t)max(e - 2, 0);
    sf = byte == 255u ? __uint_as_float(0x7FFFFFFFu) : byte == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
  }
  float y[16];
  if constexpr (kFmt == FMT_NV) {
    const float rc = sf > 0.f ? __frcp_rd(sf) : 0.f, rest = sf > 0.f ? __fmul_rn(__fmaf_rn(-rc, sf, 1.f), rc) : 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = __fmaf_rn(v[i], rc, __fmul_rn(v[i], rest));
  } else {
    const float rc = __uint_as_float((254u - min(byte, 253u)) << 23);                     // a power of two: exact
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = __fmul_rn(v[i], rc);
  }
  // four scales leave as one word
  uint32_t word = byte & 0xFFu;
  if (!live) word = 0;
  constexpr int kStep = kPerWord / 4;
  word |= __shfl_down_sync(0xFFFFFFFFu, word, kStep) << 8;
  word |= __shfl_down_sync(0xFFFFFFFFu, word, 2 * kStep) << 16;
  if (r < rows && c % kPerWord == 0) scales[scale_word(r, c / kPerWord, k_tiles)] = word;
  if (live) codes[r * chunks + c] = make_uint2(e2m1x8(y), e2m1x8(y + 8));
}

// Four codes to two words of bf16 values times sf.
__device__ __forceinline__ float e2m1_value(uint32_t code) {
  // magnitudes in units of a half: 0 1 2 3 4 6 8 12, a nibble each
  const float m = (float)((0xC8643210u >> (4 * (code & 7u))) & 15u) * 0.5f;
  return code & 8u ? -m : m;
}

template <int kFmt>
__global__ void __launch_bounds__(256)
dequantize_fp4_kernel(const uint2* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t rows, int chunks, int k_tiles, float alpha,
                      uint4* __restrict__ Y, int64_t ld) {
  pdl_wait();
  pdl_trigger();
  const int64_t idx = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int64_t r = idx / chunks;
  if (r >= rows) return;
  const int c = (int)(idx - r * chunks);
  const int n = kFmt == FMT_NV ? c : c >> 1;
  const uint32_t byte = __ldg(scales + 4 * scale_word(r, n >> 2, k_tiles) + (n & 3));
  float sf;
  if constexpr (kFmt == FMT_NV) sf = __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)byte, __NV_E4M3)));
  else sf = byte == 255u ? __uint_as_float(0x7FFFFFFFu) : byte == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
  const uint2 q = __ldg(codes + idx);
  uint32_t o[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = (i < 4 ? q.x >> (8 * i) : q.y >> (8 * (i - 4))) & 0xFFu;
    o[i] = bf16x2(__fmul_rn(__fmul_rn(e2m1_value(b & 15u), sf), alpha), __fmul_rn(__fmul_rn(e2m1_value(b >> 4), sf), alpha));
  }
  uint4* dst = Y + ((r * ld) >> 3) + 2 * c;
  dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
  dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
}

int fmt_of(int format) { return format == SF_FP4_NV ? FMT_NV : format == SF_FP4_MX ? FMT_MX : -1; }

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
  *codes_bytes = (size_t)rows * (size_t)cols / 2;
  *scales_bytes = (size_t)ceil_div(rows, 128) * (size_t)scale_tiles(fmt_of(format), cols) * 512;
  return SF_OK;
}

int sf_fp4_quantize(const void* X, int64_t rows, int64_t cols, int64_t ld, int format, float scale, void* codes, void* scales, void* stream) {
  SF_TRY(fp4_shape(rows, cols, format));
  if (rows == 0 || cols == 0) return SF_OK;
  if (!X || !codes || !scales) return SF_ERR_NULL;
  if (ld < cols || ld % 8 || !aligned16(X) || !aligned16(codes) || !aligned16(scales)) return SF_ERR_ALIGN;
  const int fmt = fmt_of(format);
  const int64_t k_tiles = scale_tiles(fmt, cols), threads = rows * k_tiles * (fmt == FMT_NV ? 4 : 8), blocks = ceil_div(threads, 256);
  if (blocks > 0x7FFFFFFF) return SF_ERR_SHAPE;
  SF_TRY(check_arch());
  return launch_pdl(fmt == FMT_NV ? quantize_fp4_kernel<FMT_NV> : quantize_fp4_kernel<FMT_MX>, dim3((unsigned)blocks), 256, 0,
                    (cudaStream_t)stream, (const uint4*)X, rows, (int)(cols / 16), ld, scale, (int)k_tiles, (uint2*)codes, (uint32_t*)scales);
}

int sf_fp4_dequantize(const void* codes, const void* scales, int64_t rows, int64_t cols, int format, float alpha, void* Y, int64_t ld,
                      void* stream) {
  SF_TRY(fp4_shape(rows, cols, format));
  if (rows == 0 || cols == 0) return SF_OK;
  if (!Y || !codes || !scales) return SF_ERR_NULL;
  if (ld < cols || ld % 8 || !aligned16(Y) || !aligned16(codes) || !aligned16(scales)) return SF_ERR_ALIGN;
  const int fmt = fmt_of(format);
  const int64_t blocks = ceil_div(rows * (cols / 16), 256);
  if (blocks > 0x7FFFFFFF) return SF_ERR_SHAPE;
  SF_TRY(check_arch());
  return launch_pdl(fmt == FMT_NV ? dequantize_fp4_kernel<FMT_NV> : dequantize_fp4_kernel<FMT_MX>, dim3((unsigned)blocks), 256, 0,
                    (cudaStream_t)stream, (const uint2*)codes, (const uint8_t*)scales, rows, (int)(cols / 16),
                    (int)scale_tiles(fmt, cols), alpha, (uint4*)Y, ld);
}

int sf_gemm_fp4_workspace_size(int64_t Mr, int64_t Nc, int64_t K, size_t* bytes) {
  if (!bytes) return SF_ERR_NULL;
  if (Mr < 0 || Nc < 0 || K <= 0 || Nc % 8 || K % 32 || Mr > kMaxSize || Nc > kMaxSize || K > kMaxSize) return SF_ERR_SHAPE;
  *bytes = kStatus;
  return SF_OK;
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
  SF_TRY(check_arch());
  const Operand a{A, a_scales}, g{Bg, bg_scales}, u{Bu, bu_scales};
  return format == SF_FP4_NV
             ? run_gated<FMT_NV>(a, g, u, Mr, Nc, K, act, alpha_g, alpha_u, H, nullptr, nullptr, (int*)workspace, (cudaStream_t)stream)
             : run_gated<FMT_MX>(a, g, u, Mr, Nc, K, act, alpha_g, alpha_u, H, nullptr, nullptr, (int*)workspace, (cudaStream_t)stream);
}

}  // extern "C"
