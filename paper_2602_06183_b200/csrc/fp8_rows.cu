// C = bf16(alpha a_scales[row] A B^T) of E4M3 operands, for any number of rows of A: what the norm's 8-bit output, a scale to every token, is
// made for. The kernels are those of the gated block and of the 4-bit products (few tokens: the weights are streamed past them; more: tiles
// on CTA pairs) with tcgen05.mma.kind::f8f6f4; the scales are factors of the epilogue. 1 x 16384 x 4096: 13.0 us (67 MB, 5.2 TB/s, weights from
// HBM); 8192 x 16384 x 4096: 378 (2.9 PFLOP/s) in short runs, 435 (2.5) under the power cap, the tensor pipe active in 92 % of the cycles.
#include "products.cuh"

namespace sf {
namespace {

constexpr size_t kStatus = 256;

}  // namespace
}  // namespace sf

using namespace sf;

extern "C" {

int sf_gemm_fp8_rows_workspace_size(int64_t Mr, int64_t Nc, int64_t K, size_t* bytes) {
  if (!bytes) return SF_ERR_NULL;
  if (Mr < 0 || Nc < 0 || K <= 0 || Nc % 8 || K % 16 || Mr > kMaxSize || Nc > kMaxSize || K > kMaxSize) return SF_ERR_SHAPE;
  *bytes = kStatus;
  return SF_OK;
}

int sf_gemm_fp8_rows(const void* A, const void* a_scales, const void* B, void* C, int64_t Mr, int64_t Nc, int64_t K, float alpha, void* workspace,
                     size_t workspace_bytes, void* stream) {
  size_t need;
  SF_TRY(sf_gemm_fp8_rows_workspace_size(Mr, Nc, K, &need));
  if (Mr == 0 || Nc == 0) return SF_OK;
  if (!A || !a_scales || !B || !C || !workspace) return SF_ERR_NULL;
  if (!aligned16(A) || !aligned16(a_scales) || !aligned16(B) || !aligned16(C) || !aligned16(workspace)) return SF_ERR_ALIGN;
  if (workspace_bytes < need) return SF_ERR_WORKSPACE;
  const size_t m = (size_t)Mr, n = (size_t)Nc, k = (size_t)K;
  if (!apart({{C, 2 * m * n}, {workspace, need}}, {{A, m * k}, {a_scales, 4 * m}, {B, n * k}})) return SF_ERR_UNSUPPORTED;
  SF_TRY(check_arch());
  const Operand a{A, a_scales}, b{B, nullptr};
  return run_nt<FMT_E4M3>(a, b, Mr, Nc, K, alpha, C, (int*)workspace, (cudaStream_t)stream);
}

}  // extern "C"
