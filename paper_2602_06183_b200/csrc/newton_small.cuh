// All steps of a small orthogonalised update in one launch (see newton_schulz.cu for the iteration, its roundings and its scales).
//
// A product of small matrices on CTA pairs is latency: 64 x 512 took 17 launches, 62 us, and 27.5 in one (16 x 16 53 / 16, 64 x 4000 78 / 42,
// 128 x 512 69 / 52, 128 x 2000 78 / 68; graph replay, four calls to a graph). Here one cluster of up to 16 CTAs keeps X from the
// first step to the last, every CTA some of its columns: in float32 in the registers of the warps that make them, as fp16 operand in
// shared memory. What has to cross goes through distributed shared memory, with two cluster barriers a step: the partial sums of A = X X^T
// over a CTA's columns are sent to the CTAs that add them up, a part each, in the order of the senders; these send the sums to all, and every CTA
// has A whole, makes all of B = a I + b A + c A^2 (128 rows at most: less work than an exchange) and multiplies its columns. The products are mma.sync of
// 16 x 8 x 16; instructions issued, not products, are what a step takes. (With A and B exchanged through the L2 a step of 128 x 512 took 10 us, with the sums
// fetched where they lie, latencies one behind the other, 20.)
#pragma once

#include "newton_first.cuh"

namespace sf {
namespace {

constexpr int kSmallThreads = 512, kSmallWarps = kSmallThreads / 32, kSmallMost = 128, kSmallCtas = 16, kSmallTiles = 2;
constexpr int kSmallSmem = 196608;     // the most that a problem takes
constexpr int kSmallCols = 64;         // of a CTA, before more CTAs are taken

struct SmallShape {
  int mp, w, ctas;                     // small side in whole 32s; columns of a CTA, a multiple of 32; CTAs
  int tiles;                           // of 32 x 32 of X, to a warp
  int ldx, ldm;                        // halves to a row in shared memory: an odd number of 16-byte pieces, for ldmatrix
  size_t smem;
};
__host__ __device__ constexpr int small_blocks(int mp) { return (mp / 16) * (mp / 16 + 1) / 2; }     // of 16 x 16 of the lower half of A

// Whether a problem fits, and how it is laid out.
inline bool small_shape(int64_t m, int64_t n, SmallShape* z) {
  if (m > kSmallMost || m < 1 || n < 1 || n > (1 << 18)) return false;
  z->mp = (int)ceil_div(m, 32) * 32;
  z->ctas = 1;
  while (z->ctas < kSmallCtas && z->ctas * kSmallCols < n) z->ctas *= 2;
  z->w = (int)ceil_div(n, z->ctas * 32) * 32;
  z->tiles = (int)ceil_div(z->w, 32 * (kSmallWarps / (z->mp / 32)));
  z->ldx = z->w + 8;
  z->ldm = z->mp + 8;
  z->smem = (size_t)z->mp * (2 * (size_t)z->ldx + 4 * z->ldm + 8) + 1024 * (size_t)(small_blocks(z->mp) + ceil_div(small_blocks(z->mp), z->ctas) * z->ctas);
  return z->tiles <= kSmallTiles && z->smem <= kSmallSmem;
}

struct SmallArgs {
  const void* G;
  uint16_t* O;
  int64_t ldg, ldo;
  int m, n, high, steps;               // high: G and O are n x m
  float a, b, c, scale;
  int mp, w, ldx, ldm;
};

__device__ __forceinline__ void mma_f16_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix4(uint32_t at, uint32_t (&v)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t at, uint32_t (&v)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at) : "memory");
}
// This lane's address in 16 rows x 16 columns of a row-major matrix of halves: as a first factor (and, transposed, as a second one whose k
// are the rows), or as a second one whose columns are the rows.
__device__ __forceinline__ uint32_t as_first(int ld, int lane) { return (uint32_t)((lane & 15) * ld + (lane >> 4) * 8) * 2u; }
__device__ __forceinline__ uint32_t as_second(int ld, int lane) { return (uint32_t)(((lane & 7) + (lane >> 4) * 8) * ld + (lane >> 3 & 1) * 8) * 2u; }

// Two neighbouring elements of a row of a symmetric matrix, and of its mirror image.
__device__ __forceinline__ void put_pair(uint16_t* mat, int ld, int row, int col, uint32_t w, bool mirrored) {
  *reinterpret_cast<uint32_t*>(mat + row * ld + col) = w;
  if (mirrored) {
    mat[col * ld + row] = (uint16_t)w;
    mat[(col + 1) * ld + row] = (uint16_t)(w >> 16);
  }
}
// M M^T of rows bi and bj of 16 each, `k` columns: the sums of a block as two fragments.
__device__ __forceinline__ void small_block(uint32_t first, uint32_t second, int k, float (&d)[2][4]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) d[h][0] = d[h][1] = d[h][2] = d[h][3] = 0.f;
#pragma unroll 2
  for (int i = 0; i < k; i += 16, first += 32, second += 32) {
    uint32_t x[4], y[4];
    ldmatrix4(first, x);
    ldmatrix4(second, y);
    mma_f16_16816(d[0], x, y[0], y[1]);
    mma_f16_16816(d[1], x, y[2], y[3]);
  }
}
__device__ __forceinline__ double ld_cluster_f64(uint32_t saddr, uint32_t rank) {
  double v;
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.f64 %0, [a];\n\t}\n" : "=d"(v) : "r"(saddr), "r"(rank) : "memory");
  return v;
}

__device__ __forceinline__ void st_cluster_f4(uint32_t saddr, uint32_t rank, const float4& v) {
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tst.shared::cluster.v4.f32 [a], {%2, %3, %4, %5};\n\t}\n"
               ::"r"(saddr), "r"(rank), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

template <bool kF32, int kTiles>
__global__ void __launch_bounds__(kSmallThreads, 1)
ns_small_kernel(const SmallArgs a) {
  extern __shared__ uint4 small_smem[];
  __shared__ double squares[kSmallWarps], square;
  __shared__ uint8_t block_at[2][small_blocks(kSmallMost)];
  const int blocks = small_blocks(a.mp), nb = a.mp / 16;
  uint16_t *xh = reinterpret_cast<uint16_t*>(small_smem), *mat_a = xh + a.mp * a.ldx, *mat_b = mat_a + a.mp * a.ldm;
  float *diag_a = reinterpret_cast<float*>(mat_b + a.mp * a.ldm), *diag_b = diag_a + a.mp;
  // [block][fragment][lane] of all sums; [block of this CTA][sender][fragment][lane] of the partial ones (block u belongs to CTA u % ctas)
  float4 *sums = reinterpret_cast<float4*>(diag_b + a.mp), *parts = sums + blocks * 64;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, cta = (int)cluster_ctarank(), ctas = (int)gridDim.x;
  const int c0 = cta * a.w;
  // this warp's tiles of X: rows r0 on, columns from t 32 beside + c of the CTA's on
  const int row_blocks = a.mp / 32, beside = kSmallWarps / row_blocks, r0 = warp % row_blocks * 32, c = warp / row_blocks * 32;
  const bool works = warp < row_blocks * beside;
  const int fr = lane >> 2, fc = (lane & 3) * 2;           // of a fragment: row (and eight further), first of two columns

  for (int u = threadIdx.x; u < blocks; u += kSmallThreads) {
    int bi = 0, bj = u;
    while (bj > bi) bj -= ++bi;
    block_at[0][u] = (uint8_t)bi;
    block_at[1][u] = (uint8_t)bj;
  }
  pdl_wait();
  pdl_trigger();
  // X's element (row, column) lies at G[row][c0 + column], or, where G is high, at G[c0 + column][row]
  float x[kTiles][2][4][4];
  double s = 0;
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = r0 + i * 16 + (e >> 1) * 8 + fr, in = t * 32 * beside + c + j * 8 + fc + (e & 1), col = c0 + in;
          x[t][i][j][e] = works && in < a.w && row < a.m && col < a.n ? element<kF32>(a.G, a.high ? col * a.ldg + row : row * a.ldg + col) : 0.f;
        }
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) s = fma((double)x[t][i][j][e], (double)x[t][i][j][e], s);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if (lane == 0) squares[warp] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kSmallWarps; ++w) s += squares[w];
    square = s;
  }
  cluster_sync_all();
  s = 0;
  for (int k = 0; k < ctas; ++k) s += ld_cluster_f64(smem_u32(&square), (uint32_t)k);
  float first;
  const NsScale z = ns_scale_of(s, &first);
  // X, rounded, as the products' operand
  auto operand = [&] {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      if (!works || t * 32 * beside + c >= a.w) continue;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t* p = reinterpret_cast<uint32_t*>(xh + (r0 + i * 16 + fr) * a.ldx + t * 32 * beside + c + j * 8 + fc);
          p[0] = f16x2(x[t][i][j][0], x[t][i][j][1]);
          p[4 * a.ldx] = f16x2(x[t][i][j][2], x[t][i][j][3]);
        }
    }
  };
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[t][i][j][e] = x[t][i][j][e] * z.lo * z.hi;
  operand();
  __syncthreads();
  const uint32_t x_first = smem_u32(xh) + as_first(a.ldx, lane), x_second = smem_u32(xh) + as_second(a.ldx, lane);
  const uint32_t a_first = smem_u32(mat_a) + as_first(a.ldm, lane), a_second = smem_u32(mat_a) + as_second(a.ldm, lane);
  const uint32_t b_first = smem_u32(mat_b) + as_first(a.ldm, lane);
  const uint32_t x_row = 32u * a.ldx, m_row = 32u * a.ldm; // bytes of 16 rows
  constexpr float k14 = 1.f / 16384.f;
#pragma unroll 1
  for (int step = 0; step < a.steps; ++step) {
    // partial sums of A, a block to a warp
#pragma unroll 1
    for (int u = warp; u < blocks; u += kSmallWarps) {
      float d[2][4];
      small_block(x_first + block_at[0][u] * x_row, x_second + block_at[1][u] * x_row, a.w, d);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        st_cluster_f4(smem_u32(parts + ((u / ctas * ctas + cta) * 2 + h) * 32 + lane), (uint32_t)(u % ctas), make_float4(d[h][0], d[h][1], d[h][2], d[h][3]));
    }
    cluster_sync_all();
    // their sums over the CTAs, to all of them
    const float f = first * first * (k14 * k14);
#pragma unroll 1
    for (int i = threadIdx.x; i < (blocks + ctas - 1 - cta) / ctas * 64; i += kSmallThreads) {
      const float4* in = parts + (i >> 6) * ctas * 64 + (i & 63);
      float4 v = in[0];
#pragma unroll 4
      for (int k = 1; k < ctas; ++k) {
        const float4 w = in[k * 64];
        v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
      }
      v = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
      const uint32_t to = smem_u32(sums + ((i >> 6) * ctas + cta) * 64 + (i & 63));
#pragma unroll 4
      for (int k = 0; k < ctas; ++k) st_cluster_f4(to, (uint32_t)k, v);
    }
    cluster_sync_all();
    // all of A: off the diagonal in fp16, on both sides of it, and the diagonal
#pragma unroll 1
    for (int u = warp; u < blocks; u += kSmallWarps) {
      const int bi = block_at[0][u], bj = block_at[1][u];
      const float4 v[2] = {sums[u * 64 + lane], sums[u * 64 + 32 + lane]};
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int i = bi * 16 + r * 8 + fr, j = bj * 16 + h * 8 + fc;
          float p = r ? v[h].z : v[h].x, q = r ? v[h].w : v[h].y;
          if (i == j) { diag_a[i] = p; p = 0.f; }
          if (i == j + 1) { diag_a[i] = q; q = 0.f; }
          put_pair(mat_a, a.ldm, i, j, f16x2(p * 16384.f, q * 16384.f), bi != bj);
        }
    }
    __syncthreads();
    // all of B
#pragma unroll 1
    for (int u = warp; u < blocks; u += kSmallWarps) {
      const int bi = block_at[0][u], bj = block_at[1][u];
      float d[2][4];
      small_block(a_first + bi * m_row, a_second + bj * m_row, a.mp, d);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int i = bi * 16 + r * 8 + fr, j = bj * 16 + h * 8 + fc;
          const float2 held = from_f16x2(*reinterpret_cast<const uint32_t*>(mat_a + i * a.ldm + j)), dj = *reinterpret_cast<const float2*>(diag_a + j);
          const float di = diag_a[i], xs[2] = {held.x * k14, held.y * k14}, ds[2] = {dj.x, dj.y};
          float o[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float p = d[h][2 * r + e] * (k14 * k14);
            o[e] = 4096.f * fmaf(a.c, fmaf(di + ds[e], xs[e], p), a.b * xs[e]);
            if (i == j + e) {
              diag_b[i] = fmaf(a.c, fmaf(di, di, p), fmaf(a.b, di, a.a));
              o[e] = 0.f;
            }
          }
          put_pair(mat_b, a.ldm, i, j, f16x2(o[0], o[1]), bi != bj);
        }
    }
    __syncthreads();
    // X: the diagonal's part in float32, the rest from the operands
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int at = t * 32 * beside + c;
      if (!works || at >= a.w) continue;
      float d[2][4][4] = {};
#pragma unroll 1
      for (int k = 0; k < nb; ++k) {
        uint32_t p[2][4], q[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          ldmatrix4(b_first + (uint32_t)((r0 >> 4) + i) * m_row + k * 32, p[i]);
          ldmatrix4_trans(x_first + k * x_row + (uint32_t)(at + 16 * i) * 2u, q[i]);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) mma_f16_16816(d[i][j], p[i], q[j >> 1][2 * (j & 1)], q[j >> 1][2 * (j & 1) + 1]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float dg = first * diag_b[r0 + i * 16 + r * 8 + fr], f12 = first * (1.f / 4096.f);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) x[t][i][j][2 * r + e] = fmaf(dg, x[t][i][j][2 * r + e], d[i][j][2 * r + e] * f12);
        }
    }
    __syncthreads();                   // every warp has read the operand
    operand();
    __syncthreads();
    first = 1.f;
  }
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = r0 + i * 16 + (e >> 1) * 8 + fr, in = t * 32 * beside + c + j * 8 + fc + (e & 1), col = c0 + in;
          if (works && in < a.w && row < a.m && col < a.n)
            a.O[a.high ? col * a.ldo + row : row * a.ldo + col] = (uint16_t)float_to_bf16_bits(x[t][i][j][e] * a.scale);
        }
  cluster_sync_all();                  // no CTA leaves while another may still send to it
}

}  // namespace
}  // namespace sf
