// Orthogonalising an update by Newton-Schulz products: X_0 = G / |G| (Frobenius), and a number of times
//     A = X X^T,   X <- (a I + b A + c A^2) X            with X as wide as it is high at least (G, or its transpose)
// which takes every singular value of X through the quintic a s + b s^3 + c s^5 and leaves the singular vectors.
//
// A quintic that brings small singular values up quickly (a = 3.4) also brings up what rounding puts in their place, 3.4 times with every
// step, and the values near 1 it moves about rather than to 1. So the operands' roundings decide what comes out. With X in bf16 the error
// against 64 bits is 1 to 2 percent for a random matrix and 10 to 30 for one of low rank. Here:
//   - operands are fp16 (11 bits to bf16's 8, the same rate), kept in range by powers of two: |X| <= 1.25 in every norm that matters, so X
//     is held as 2^14 X, A as 2^14 A, B as 2^12 B;
//   - X is kept as a sum of two fp16 numbers. The products see the first; a X, the larger part for small singular values, is added in
//     float32 from both. This alone takes the error at rank 8 from 2.6 % to 0.03 %, and costs no product;
//   - the diagonals of A and B, which are far larger than the rest, are held apart in float32 and multiplied in the epilogues:
//     A = D + A', A^2 = D^2 + D A' + A' D + A'^2, B X = diag(B) X + B' X. A matrix of 512 x 2048: 0.3 % to 0.05 %.
// What the roundings leave with five steps of the usual quintic: 0.02 to 0.15 % where G is of full rank, 0.3 % usually and 1 % at most where it is of low
// rank or has rows that are copies, whose roundings are alike. The final rounding to bf16 is 0.17 %.
//
// A wide matrix could take g steps at once by products of the small side: X becomes Q X, Q a product of polynomials of the first A, and the next A
// is A B^2. Five steps of 4096 x 16384 took 2400 us so (single steps: 3980). It is not done: where G has components, a^g X is cancelled by what is held
// in fp16, and errors were 3 to 20 times those of single steps for matrices far from full rank (equal rows 1.8 %, ten steps of copied rows
// 5 %). Second terms of Q and of all matrices in the products mend that and cost what is saved; two steps at once in the first group only save a tenth, and
// leave 4 % after ten steps.
//
// Launches: norm (partial sums in double), conversion (with the transposition of a high G), then PK_GRAM, PK_SYMM and PK_APPLY of
// pair_product.cuh for every step. Half of the tiles of the symmetric ones are computed. Small sides of up to 128 are one launch
// (newton_small.cuh). Five steps, back to back: 1021 x 253 97 us (17 launches, each its latency), 2048 x 2048 243 (0.71 PFLOP/s: products of 11
// to 19 us whose tiles take 7 to 9), 4096 x 16384 3980 (1.12 PFLOP/s of 4.5 TFLOP; power cap).
#include "newton_small.cuh"

namespace sf {
namespace {

constexpr size_t kStatus = 256, kScalars = 256;       // status word; the first step's factor
constexpr int kNormCtas = 512;
constexpr int64_t kMostSide = 1 << 24, kMostSmall = 1 << 16;

struct NsShape {
  int64_t m, n, ldm, ldn, mp;          // small and large side, leading dimensions, m in whole tiles
  bool high;                           // G has more rows than columns
  size_t sums, sym[2], diag[2], x[4], total;              // A and B; X and the next one, two terms each
};

int ns_shape(int64_t rows, int64_t cols, NsShape* z) {
  if (rows < 0 || cols < 0 || rows > kMostSide || cols > kMostSide) return SF_ERR_SHAPE;
  z->high = rows > cols;
  z->m = z->high ? cols : rows;
  z->n = z->high ? rows : cols;
  if (z->m > kMostSmall) return SF_ERR_SHAPE;
  auto up8 = [](int64_t v) { return (v + 7) / 8 * 8; };
  z->ldm = up8(z->m);
  z->ldn = up8(z->n);
  z->mp = ceil_div(z->m, 256) * 256;
  size_t o = kStatus + kScalars;
  auto take = [&](size_t bytes) { const size_t r = o; o += (bytes + 255) & ~(size_t)255; return r; };
  z->sums = take(8 * kNormCtas);
  for (int i = 0; i < 2; ++i) {
    z->sym[i] = take(2 * (size_t)z->m * (size_t)z->ldm);
    z->diag[i] = take(4 * (size_t)z->mp);
  }
  for (int i = 0; i < 4; ++i) z->x[i] = take(2 * (size_t)z->m * (size_t)z->ldn);
  z->total = o;
  return SF_OK;
}

// ---- the norm ---------------------------------------------------------------------------------------------
// Squares are summed in double: neither the largest nor the smallest float32 has one that leaves its range, and the sum does not depend on
// how the rows lie. wide: rows of whole pieces of 16 bytes on their boundaries, four of which are under way at once.
template <bool kF32>
__device__ __forceinline__ double sum_squares(const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  double s = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kF32) {
      const double x = __uint_as_float(w[i]);
      s = fma(x, x, s);
    } else {
      const double x = bf16_bits_to_float(w[i] & 0xFFFFu), y = bf16_bits_to_float(w[i] >> 16);
      s = fma(x, x, s);
      s = fma(y, y, s);
    }
  }
  return s;
}
template <bool kF32>
__global__ void __launch_bounds__(256)
ns_norm_kernel(const void* __restrict__ G, int64_t rows, int64_t cols, int64_t ld, int wide, double* __restrict__ sums) {
  __shared__ double part[8];
  pdl_wait();
  pdl_trigger();
  constexpr int kPiece = kF32 ? 4 : 8;
  const int64_t per_row = wide ? cols / kPiece : cols, first = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  const int64_t dr = step / per_row, dc = step - dr * per_row;
  int64_t r = first / per_row, c = first - r * per_row;
  auto next = [&] {
    r += dr;
    c += dc;
    if (c >= per_row) { c -= per_row; ++r; }
  };
  double s = 0;
  if (wide) {
    while (r < rows) {
      uint4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = make_uint4(0u, 0u, 0u, 0u);
        if (r < rows) v[i] = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(G) + (r * ld + c * kPiece) * (kF32 ? 4 : 2)));
        next();
      }
      s += (sum_squares<kF32>(v[0]) + sum_squares<kF32>(v[1])) + (sum_squares<kF32>(v[2]) + sum_squares<kF32>(v[3]));
    }
  } else {
    for (; r < rows; next()) {
      const double x = element<kF32>(G, r * ld + c);
      s = fma(x, x, s);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < 8; ++w) s += part[w];
    sums[blockIdx.x] = s;
  }
}

// ---- the first X -------------------------------------------------------------------------------------------
__device__ __forceinline__ NsScale ns_scale(const double* __restrict__ sums, int count, float* first, double* shared) {
  double s = 0;
  for (int i = threadIdx.x; i < count; i += 256) s += __ldcg(sums + i);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = s;
  __syncthreads();
  s = shared[0];
#pragma unroll
  for (int w = 1; w < 8; ++w) s += shared[w];
  float f;
  const NsScale z = ns_scale_of(s, &f);
  if (blockIdx.x == 0 && threadIdx.x == 0) *first = f;
  return z;
}
// As it lies: pieces of eight elements of a row (the last one of a row may be short; the padding behind it is written as 0).
template <bool kF32>
__global__ void __launch_bounds__(256)
ns_convert_kernel(const void* __restrict__ G, int64_t rows, int64_t cols, int64_t ld, int wide, const double* __restrict__ sums, int count,
                  float* __restrict__ first, uint4* __restrict__ hi, uint4* __restrict__ lo) {
  __shared__ double shared[8];
  pdl_wait();
  pdl_trigger();
  const NsScale z = ns_scale(sums, count, first, shared);
  const int64_t per_row = (cols + 7) / 8, total = rows * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per_row, c = (i - r * per_row) * 8;
    float x[8];
    if (wide) {                                            // whole pieces on 16-byte boundaries
      if constexpr (kF32) {
        const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(G) + r * ld + c);
        const float4 u = __ldg(p), v = __ldg(p + 1);
        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = v.x; x[5] = v.y; x[6] = v.z; x[7] = v.w;
      } else {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(G) + r * ld + c));
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) { x[2 * j] = bf16_bits_to_float(w[j] & 0xFFFFu); x[2 * j + 1] = bf16_bits_to_float(w[j] >> 16); }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = c + j < cols ? element<kF32>(G, r * ld + c + j) : 0.f;
    }
    uint32_t h[4], l[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint16_t h0, l0, h1, l1;
      ns_terms(x[2 * j], z, h0, l0);
      ns_terms(x[2 * j + 1], z, h1, l1);
      h[j] = h0 | (uint32_t)h1 << 16;
      l[j] = l0 | (uint32_t)l1 << 16;
    }
    hi[i] = make_uint4(h[0], h[1], h[2], h[3]);
    if (kF32) lo[i] = make_uint4(l[0], l[1], l[2], l[3]);
  }
}

// Transposed: X [cols, ldn] from G [rows, cols], 64 x 64 elements to a CTA at a time.
template <bool kF32>
__global__ void __launch_bounds__(256)
ns_convert_transposed_kernel(const void* __restrict__ G, int64_t rows, int64_t cols, int64_t ld, const double* __restrict__ sums, int count,
                             float* __restrict__ first, int64_t ldn, uint16_t* __restrict__ hi, uint16_t* __restrict__ lo) {
  __shared__ double shared[8];
  __shared__ float tile[64][65];
  pdl_wait();
  pdl_trigger();
  const NsScale z = ns_scale(sums, count, first, shared);
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
  const int64_t tiles_c = (cols + 63) / 64, tiles = (rows + 63) / 64 * tiles_c;
  for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    const int64_t r0 = t / tiles_c * 64, c0 = (t - t / tiles_c * tiles_c) * 64;
    __syncthreads();
#pragma unroll
    for (int j = y; j < 64; j += 4)
      if (r0 + j < rows && c0 + x < cols) tile[j][x] = element<kF32>(G, (r0 + j) * ld + c0 + x);
    __syncthreads();
#pragma unroll
    for (int j = y; j < 64; j += 4)
      if (c0 + j < cols && r0 + x < rows) {
        uint16_t h, l;
        ns_terms(tile[x][j], z, h, l);
        hi[(c0 + j) * ldn + r0 + x] = h;
        if (kF32) lo[(c0 + j) * ldn + r0 + x] = l;
      }
  }
}

// Whether the quintic keeps the singular values in the range that the fp16 operands are scaled for: from [0, 1.25] into itself, and its
// factors within theirs. p: the largest |a + b l + c l^2| of an eigenvalue l of A, which is at most 1.25^2.
bool ns_bounded(double a, double b, double c, double* p) {
  if (!(std::fabs(a) <= 8 && std::fabs(b) <= 8 && std::fabs(c) <= 8)) return false;
  constexpr double top = 1.5625;
  auto f = [&](double s) { return std::fabs(s * (a + s * s * (b + s * s * c))); };
  auto q = [&](double l) { return l * (b + l * c); };
  double most = f(1.25), most_b = std::fabs(q(top));
  *p = std::fmax(std::fabs(a), std::fabs(a + q(top)));
  const double disc = 9 * b * b - 20 * a * c;                              // a + 3 b l + 5 c l^2 = 0, l = s^2
  for (int i = 0; i < 2; ++i) {
    const double l = c != 0 ? (disc < 0 ? -1 : (-3 * b + (i ? 1 : -1) * std::sqrt(disc)) / (10 * c)) : b != 0 ? -a / (3 * b) : -1;
    if (l > 0 && l < top) most = std::fmax(most, f(std::sqrt(l)));
  }
  const double l = c != 0 ? -b / (2 * c) : -1;
  if (l > 0 && l < top) {
    most_b = std::fmax(most_b, std::fabs(q(l)));
    *p = std::fmax(*p, std::fabs(a + q(l)));
  }
  return most <= 1.25 && most_b <= 7.5;
}

// The whole update in one launch, where it fits: *taken says whether it was made. (A cluster of 16 CTAs is more than every device has to offer.)
template <bool kF32, int kTiles>
int launch_small(const SmallShape& z, const SmallArgs& a, cudaStream_t s, bool* taken) {
  auto kern = ns_small_kernel<kF32, kTiles>;
  static std::atomic<int> most[64]{};  // CTAs of a cluster that the device takes, found once: 1 to 16, or -1
  int dev = 0;
  SF_CUDA_TRY(cudaGetDevice(&dev));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)z.ctas);
  cfg.blockDim = dim3(kSmallThreads);
  cfg.dynamicSmemBytes = z.smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)z.ctas;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  int have = dev >= 0 && dev < 64 ? most[dev].load() : 0;
  if (have == 0) {
    SF_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallSmem));
    SF_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    have = -1;
    for (int n = kSmallCtas; n >= 1 && have < 0; n /= 2) {
      cudaLaunchConfig_t q = cfg;
      cudaLaunchAttribute at = attr[0];
      at.val.clusterDim.x = (unsigned)n;
      q.gridDim = dim3((unsigned)n);
      q.dynamicSmemBytes = kSmallSmem;
      q.stream = nullptr;
      q.attrs = &at;
      q.numAttrs = 1;
      int fit = 0;
      SF_CUDA_TRY(cudaOccupancyMaxActiveClusters(&fit, kern, &q));
      if (fit > 0) have = n;
    }
    if (dev >= 0 && dev < 64) most[dev] = have;
  }
  *taken = z.ctas <= have;
  if (!*taken) return SF_OK;
  SF_CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, a));
  return SF_OK;
}

size_t matrix_bytes(int64_t rows, int64_t cols, int64_t ld, int size) {
  return rows > 0 && cols > 0 ? (size_t)size * ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) : 0;
}

}  // namespace
}  // namespace sf

using namespace sf;

extern "C" {

int sf_orthogonalize_workspace_size(int64_t rows, int64_t cols, size_t* bytes) {
  NsShape z;
  SF_TRY(ns_shape(rows, cols, &z));
  if (!bytes) return SF_ERR_NULL;
  *bytes = z.total;
  return SF_OK;
}

int sf_orthogonalize(const void* G, int type, int64_t rows, int64_t cols, int64_t ldg, int steps, float a, float b, float c, float scale, void* O,
                     int64_t ldo, void* workspace, size_t workspace_bytes, void* stream) {
  NsShape z;
  if (type != SF_BF16 && type != SF_F32) return SF_ERR_UNSUPPORTED;
  SF_TRY(ns_shape(rows, cols, &z));
  double p_most;
  if (steps < 1 || steps > 64 || !ns_bounded(a, b, c, &p_most)) return SF_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return SF_OK;
  if (!G || !O || !workspace) return SF_ERR_NULL;
  const int size = type == SF_F32 ? 4 : 2;
  if (ldg < cols || ldo < cols || (uintptr_t)G % size || (uintptr_t)O % 2 || !aligned16(workspace)) return SF_ERR_ALIGN;
  if (workspace_bytes < z.total) return SF_ERR_WORKSPACE;
  if (!apart({{O, matrix_bytes(rows, cols, ldo, 2)}, {workspace, z.total}}, {{G, matrix_bytes(rows, cols, ldg, size)}})) return SF_ERR_UNSUPPORTED;
  SF_TRY(check_arch());
  cudaStream_t s = (cudaStream_t)stream;
  uint8_t* w = (uint8_t*)workspace;
  float* first = (float*)(w + kStatus);
  double* sums = (double*)(w + z.sums);
  const bool f32 = type == SF_F32;
  SmallShape small;
  if (small_shape(z.m, z.n, &small)) {
    SmallArgs q{};
    q.G = G; q.O = (uint16_t*)O; q.ldg = ldg; q.ldo = ldo;
    q.m = (int)z.m; q.n = (int)z.n; q.high = z.high; q.steps = steps;
    q.a = a; q.b = b; q.c = c; q.scale = scale / 16384.f;
    q.mp = small.mp; q.w = small.w; q.ldx = small.ldx; q.ldm = small.ldm;
    bool taken = false;
    SF_TRY(small.tiles == 1 ? (f32 ? launch_small<true, 1>(small, q, s, &taken) : launch_small<false, 1>(small, q, s, &taken))
                            : (f32 ? launch_small<true, 2>(small, q, s, &taken) : launch_small<false, 2>(small, q, s, &taken)));
    if (taken) return SF_OK;
  }
  const int piece = 16 / size;
  const bool wide = aligned16(G) && ldg % piece == 0 && cols % 8 == 0;
  const int64_t pieces = rows * (wide ? cols / piece : cols);
  const int norm_ctas = (int)(ceil_div(pieces, 512) < kNormCtas ? ceil_div(pieces, 512) : kNormCtas);
  SF_TRY(launch_pdl(f32 ? ns_norm_kernel<true> : ns_norm_kernel<false>, dim3(norm_ctas), 256, 0, s, G, rows, cols, ldg, (int)wide, sums));
  if (z.high) {
    const int64_t tiles = ceil_div(rows, 64) * ceil_div(cols, 64), most = 8 * sm_count_now();
    SF_TRY(launch_pdl(f32 ? ns_convert_transposed_kernel<true> : ns_convert_transposed_kernel<false>, dim3((unsigned)(tiles < most ? tiles : most)), 256, 0,
                      s, G, rows, cols, ldg, (const double*)sums, norm_ctas, first, z.ldn, (uint16_t*)(w + z.x[0]), (uint16_t*)(w + z.x[1])));
  } else {
    const int64_t ctas = ceil_div(rows * ceil_div(cols, 8), 256), most = 8 * sm_count_now();
    SF_TRY(launch_pdl(f32 ? ns_convert_kernel<true> : ns_convert_kernel<false>, dim3((unsigned)(ctas < most ? ctas : most)), 256, 0, s, G, rows, cols, ldg,
                      (int)wide, (const double*)sums, norm_ctas, first, (uint4*)(w + z.x[0]), (uint4*)(w + z.x[1])));
  }
  NsPairArgs p{};
  p.jobs = 1;
  p.status = (int*)workspace;
  p.M[0] = p.N[0] = (int)z.m;
  p.ns.scale = scale / 16384.f;
  p.ns.transposed = z.high;
  const bool direct = aligned16(O) && ldo % 8 == 0;
  // exponents: of A 14, of B so that it stays below 2^15
  const int e_b = 14 - (int)std::ceil(std::log2(std::fmax(p_most, 1.0)));
  uint8_t *const A = w + z.sym[0], *const B = w + z.sym[1];
  float *const diag_a = (float*)(w + z.diag[0]), *const diag_b = (float*)(w + z.diag[1]);
  for (int step = 0; step < steps; ++step) {
    const uint8_t *xh = w + z.x[2 * (step & 1)], *xl = w + z.x[2 * (step & 1) + 1];
    uint8_t *yh = w + z.x[2 * (~step & 1)], *yl = w + z.x[2 * (~step & 1) + 1];
    NsPairArgs q = p;
    q.ns.first = step == 0 ? first : nullptr;
    q.ns.diag_out = diag_a;
    q.ns.up = 0x1p14f;
    q.ns.down = 0x1p-28f;
    q.nkb = q.nkb0 = k_blocks(FMT_F16, z.n);
    SF_TRY((launch_best<PK_GRAM, FMT_F16>(q, s, [&](CUtensorMap* m, int bn) {
      SF_TRY(make_tmap_2d(&m[0], xh, z.m, z.n, z.ldn, 64, 128, true));
      SF_TRY(make_tmap_2d(&m[1], xh, z.m, z.n, z.ldn, 64, bn / 2, true));
      return make_tmap_store(&m[2], A, z.m, z.m, z.ldm);
    })));
    q = p;
    q.ns.a = a; q.ns.b = b; q.ns.c = c;
    q.ns.diag_in = diag_a;
    q.ns.diag_out = diag_b;
    q.ns.up = std::ldexp(1.f, e_b);
    q.ns.down = 0x1p-28f;
    q.ns.down1 = 0x1p-14f;
    q.nkb = q.nkb0 = k_blocks(FMT_F16, z.m);
    SF_TRY((launch_best<PK_SYMM, FMT_F16>(q, s, [&](CUtensorMap* m, int bn) {
      SF_TRY(make_tmap_2d(&m[0], A, z.m, z.m, z.ldm, 64, 128, true));
      SF_TRY(make_tmap_2d(&m[1], A, z.m, z.m, z.ldm, 64, bn / 2, true));
      SF_TRY(make_tmap_store(&m[2], B, z.m, z.m, z.ldm));
      return make_tmap_store(&m[3], A, z.m, z.m, z.ldm);
    })));
    q = p;
    q.ns.first = step == 0 ? first : nullptr;
    q.ns.last = step == steps - 1;
    q.ns.out = direct ? nullptr : (uint16_t*)O;
    q.ns.ldo = ldo;
    q.ns.two_terms = step > 0 || f32;
    q.ns.diag_in = diag_b;
    q.ns.down = std::ldexp(1.f, -e_b);
    q.N[0] = (int)z.n;
    q.nkb = q.nkb0 = k_blocks(FMT_F16, z.m);
    SF_TRY((launch_best<PK_APPLY, FMT_F16>(q, s, [&](CUtensorMap* m, int) {
      SF_TRY(make_tmap_2d(&m[0], B, z.m, z.m, z.ldm, 64, 128, true));
      SF_TRY(make_tmap_2d(&m[1], xh, z.m, z.n, z.ldn, 64, 64, true));
      SF_TRY(make_tmap_store(&m[2], xh, z.m, z.n, z.ldn));
      SF_TRY(make_tmap_store(&m[3], xl, z.m, z.n, z.ldn));
      SF_TRY(make_tmap_store(&m[5], yl, z.m, z.n, z.ldn));
      if (!q.ns.last) return make_tmap_store(&m[4], yh, z.m, z.n, z.ldn);
      return direct ? make_tmap_store(&m[4], O, rows, cols, ldo) : make_tmap_store(&m[4], yh, z.m, z.n, z.ldn);
    })));
  }
  return SF_OK;
}

}  // extern "C"
