// Products of long operands on CTA pairs, for any sizes whose rows are multiples of 16 bytes: tcgen05.mma.cta_group::2 on 256 x kBN
// tiles, operands by TMA, accumulators in TMEM, epilogues that read and write whole chunks by TMA. Everything ragged is left to
// TMA: loads beyond an edge bring zeros, stores beyond it are not made.
//
//   PK_NT    C = alpha A B^T                                both K-major
//   PK_DX    C = A0 B0 + A1 B1                              A K-major, B stored [K, N]; one accumulation over both pairs
//   PK_DW    C_j = A_j^T B_j, up to three products          both stored [K, .]; one launch, tiles of one after those of the other
//   PK_FWD   H = act(A Bg^T) (A Bu^T)                       the even CTA of a pair holds rows of Bg, the odd one the same rows of Bu:
//            the first half of a tile's columns is the gate, the second half the other factor of the same features, so that the
//            product of the two is taken in registers and neither projection is written.
//   PK_FWD_SAVE  the same, and P = act(g), Q = u act'(g) in float32 for the backward pass
//   PK_BWD   dU = (A B) P, dG = (A B) Q                     A = dY, B = Wd [K, N]; dH is never written
//
// CTA = 10 warps: TMA producer, MMA issuer, two sets of four epilogue warps that share a tile's columns. Every wait is bounded
// (see gemm_tc.cu): on expiry the CTA raises the status word and leaves.
//
// 256 columns for two CTAs because a k-block of 64 then brings in 64 bytes a clock and SM next to 512 clocks of products, about what
// the L2 delivers; narrower tiles are fed worse and are taken only where they fill the pairs better (pair_plan).
// What bounds them, T 2048, D 4096, F 8192, each from cold caches: dW 255 us (1.62 PFLOP/s, tensor pipe 94 % of its active cycles), dX 187
// (1.47, 95 %), H with P and Q 180 (1.53, 86 %: 173 MB of stores beside it), Y 97 (1.41, 91 %: one round and a part), dH 110 (1.25,
// 77 %: reads 134 MB of P and Q in its epilogue). Repeated back to back they draw the power limit and the clock falls to 1.2-1.5 GHz.
// Products of 4 bits, 4096 x 4096 x 8192, blocks of 16: 56 us (4.9 PFLOP/s, 78 %).
#pragma once

#include "gated.cuh"

namespace sf {
namespace {

using namespace ptx;

enum PairKind { PK_NT, PK_DX, PK_DW, PK_FWD, PK_FWD_SAVE, PK_BWD };

constexpr int kPairThreads = 320;
constexpr int kPairSmemMax = 232448;

// Full-width tiles; tiles of a width that the launch says (a multiple of 32; PK_FWD, whose two halves are, of 64), for products that
// fill the pairs better with it; and such tiles with the reduction split over the pairs of a cluster, one tile to a cluster, for
// long reductions of few tiles.
enum PairMode { PM_FULL, PM_WIDTH, PM_SPLIT };

template <int kKind, int kBN, int kFmt, int kMode>
struct PairCfg {
  static constexpr bool kFp4 = kFmt != FMT_BF16;
  static constexpr bool kAMN = kKind == PK_DW;
  static constexpr bool kBMN = kKind == PK_DX || kKind == PK_DW || kKind == PK_BWD;
  static constexpr bool kGated = kKind == PK_FWD || kKind == PK_FWD_SAVE;
  static constexpr bool kWide = kKind == PK_FWD_SAVE || kKind == PK_BWD;         // float32 chunks in the epilogue
  static constexpr int kHalf = kBN / 2;                                          // columns of B that a CTA holds
  static constexpr int kBChunks = (kHalf + 63) / 64;                             // MN-major B: chunks of 64 columns
  static constexpr int kABytes = 16384;
  static constexpr int kBBytes = kBMN ? kBChunks * 8192 : kHalf * 128;
  // 4-bit operands: a stage is 256 K; scale tiles of 512 bytes hold 128 rows x 4 scales = 64 (NV) or 128 (MX) K
  static constexpr int kTiles = kFmt == FMT_NV ? 4 : kFmt == FMT_MX ? 2 : 0;      // scale tiles of a row block and stage
  static constexpr int kBBlocks = kBN / 128;                                     // row blocks of B's scales
  static constexpr int kScaleBytes = kTiles * 512 * (1 + kBBlocks);
  static constexpr int kStageBytes = kABytes + kBBytes + kScaleBytes;
  static constexpr int kEpiWarpBytes = kWide ? 8192 : 4096;
  static constexpr int kRoom = (kPairSmemMax - 2048 - 8 * kEpiWarpBytes) / kStageBytes;
  static constexpr int kStages = kRoom < 8 ? kRoom : 8;
  static constexpr int kSmem = 1024 + kStages * kStageBytes + 8 * kEpiWarpBytes + 1024;
  // two accumulators; 4-bit tiles of 256 columns leave room for one next to the scales
  static constexpr int kAccs = kFp4 && kBN == 256 ? 1 : 2;
  static constexpr uint32_t kScaleCol = kAccs * kBN;
  static constexpr uint32_t kScaleACols = kTiles * 4, kScaleCols = kScaleACols * (1 + kBBlocks);    // of one stage
  static constexpr int kMaps = kKind == PK_DW ? 9 : kKind == PK_DX ? 5 : kKind == PK_NT ? (kFp4 ? 5 : 3)
                             : kKind == PK_FWD ? (kFp4 ? 7 : 4) : 6;
  static_assert(kBN == 256 || (kFp4 && kBN == 128), "tile width");
  static_assert(kMode == PM_FULL || !kFp4 || (kMode == PM_SPLIT && kBN == 128), "4-bit operands: widths of whole row blocks of scales");
  static_assert(!kFp4 || kKind == PK_NT || (kKind == PK_FWD && kBN == 256), "4-bit operands: K-major, whole row blocks of scales");
  static_assert(kStages >= 3 && kSmem <= kPairSmemMax && kSmem > 228 * 1024 / 2, "one CTA per SM");
  static_assert(kScaleCol + 2 * kScaleCols <= 512, "TMEM columns");
};

struct PairArgs {
  int jobs;
  int num_m[3], num_n[3];            // tiles of each job
  int M[3], N[3];                    // its output (PK_FWD: N features)
  int nkb, nkb0;                     // k-blocks in all, and of the first pair of operands (PK_DX)
  int act;
  int bn;                            // tile width (PM_WIDTH, PM_SPLIT)
  int parts;                         // pairs of a cluster (PM_SPLIT)
  // PK_DW of up to 16 tokens, whose sums of two (A's in the jobs of the mask, else B's) have their second terms from this row on: 0 otherwise
  int term_rows, sums_in_a;
  float alpha, alpha2;
  int early_next;                    // the next launch is let in at the start: several rounds of tiles (see long_dense in gemm_tc.cu), or it runs beside
  // Beside the launch before it, which let it in behind its own wait and whose results it does not read (its end is waited for at the end, so that the
  // order of the stream is kept; that launch does not wait for this one): that one holds the pairs from `first_late` on for about
  // `late_rounds` tiles of this one, which those pairs leave to the others.
  int beside, first_late, late_rounds;
  int* status;
};
template <int N> struct PairMaps { CUtensorMap m[N]; };

struct PairCtl {
  uint64_t full[8], empty[8], tmem_full[2], tmem_empty[2], epi_full[8];
  uint32_t tmem_base;
  int abort_flag;
};

struct PairTile { int job, m0, n0; };     // first row of the pair's tile, first column (PK_FWD: first feature)

// The n-th tile of a pair: every num_pairs-th one; the first late_rounds rounds are shared by the pairs that are not late.
__device__ __forceinline__ int nth_tile(const PairArgs& a, int n, int pair, int num_pairs) {
  const int r = a.late_rounds, e = a.first_late;
  if (r == 0) return pair + n * num_pairs;
  return pair >= e ? r * e + n * num_pairs + pair : n < r ? n * e + pair : r * e + (n - r) * num_pairs + pair;
}

// The raster of the other products: bands of eight tile rows, rows fastest inside a band, so that the tiles which run at
// the same time share few operand panels.
template <int kKind>
__device__ __forceinline__ PairTile pair_tile(const PairArgs& a, int tile, int cols) {
  int j = 0;
  if (kKind == PK_DW) {
    while (j < a.jobs - 1 && tile >= a.num_m[j] * a.num_n[j]) { tile -= a.num_m[j] * a.num_n[j]; ++j; }
  }
  const int num_m = a.num_m[j], num_n = a.num_n[j];
  const int per_band = 8 * num_n, band = tile / per_band, rem = tile - band * per_band;
  const int gm = min(8, num_m - band * 8), nt = rem / gm;
  return PairTile{j, (band * 8 + rem - nt * gm) * 256, nt * cols};
}

__device__ __forceinline__ void tma_load_3d_2cta(void* dst, const CUtensorMap* m, uint64_t* bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(bar) & kPeerBitMask), "r"(x), "r"(y), "r"(z)
      : "memory");
}

// One chunk of 32 x 32 results as this lane's row, through a 4 KB buffer (two to a warp, taken in turn) to the map's matrix.
// 64 (bf16) or 128 (float32) bytes a row, swizzled as the map has it.
__device__ __forceinline__ void put_chunk_begin(int lane) {
  if (lane == 0) bulk_wait_read<1>();                      // the store before the last has been read out of its buffer
  __syncwarp();
}
__device__ __forceinline__ void put_chunk_end(const CUtensorMap* m, const uint8_t* b, int col, int row, int lane) {
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) {
    tma_store_2d(m, b, col, row);
    bulk_commit();
  }
}
__device__ __forceinline__ void row_bf16(uint8_t* b, int lane, const uint32_t (&w)[16]) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    *reinterpret_cast<uint4*>(b + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)) = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
}
__device__ __forceinline__ void row_f32(uint8_t* b, int lane, const uint32_t (&w)[32]) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    *reinterpret_cast<uint4*>(b + lane * 128 + ((j ^ (lane & 7)) << 4)) = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
}
// Block-scaled 4-bit products: E2M1 operands, one scale per 16 (E4M3) or 32 (power of two) K; K = 64 per instruction.
template <int kFmt>
__device__ __forceinline__ void mma_fp4_2cta(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t acc) {
  if constexpr (kFmt == FMT_NV)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}\n"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc) : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}\n"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc) : "memory");
}
__device__ __forceinline__ void tmem_cp_scales_2cta(uint32_t taddr, uint64_t sdesc) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(sdesc) : "memory");
}
// 32 columns of this lane's row, added up over the parts of a cluster in their order; four parts' loads are under way at once.
__device__ __forceinline__ void sum_parts(uint32_t (&v)[32], uint32_t from, int rank, int parts) {
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    float4 x[4][2];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (s < parts) x[s][j] = ld_cluster_f4(from + (uint32_t)(2 * h + j) * 2048u, (uint32_t)(2 * s + rank));
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float4 a = x[0][j];
#pragma unroll
      for (int s = 1; s < 4; ++s)
        if (s < parts) { a.x += x[s][j].x; a.y += x[s][j].y; a.z += x[s][j].z; a.w += x[s][j].w; }
      v[8 * h + 4 * j] = __float_as_uint(a.x); v[8 * h + 4 * j + 1] = __float_as_uint(a.y);
      v[8 * h + 4 * j + 2] = __float_as_uint(a.z); v[8 * h + 4 * j + 3] = __float_as_uint(a.w);
    }
  }
}
// mma_commit_2cta for any pair of a cluster: `pair` its number.
__device__ __forceinline__ void commit_pair(uint64_t* bar, int pair) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
      ::"r"(smem_u32(bar)), "h"((uint16_t)(3 << (2 * pair)))
      : "memory");
}

template <int kKind, int kBN, int kFmt, int kMode>
__global__ void __launch_bounds__(kPairThreads, 1)
pair_product_kernel(const __grid_constant__ PairMaps<PairCfg<kKind, kBN, kFmt, kMode>::kMaps> maps, const PairArgs args) {
  using Cfg = PairCfg<kKind, kBN, kFmt, kMode>;
  constexpr bool kFp4 = Cfg::kFp4, kGated = Cfg::kGated, kVar = kMode != PM_FULL, kSplit = kMode == PM_SPLIT;
  constexpr int kStages = Cfg::kStages, kAccs = Cfg::kAccs;
  const int bn = kVar ? args.bn : kBN, half = bn / 2;      // this CTA's columns of B
  const int tile_cols = kGated ? half : bn;                // output columns of a tile
  extern __shared__ uint8_t smem_dyn[];
  uint8_t* smem = smem_dyn + align_pad(smem_dyn, 1024);
  uint8_t* epi = smem + kStages * Cfg::kStageBytes;
  PairCtl* ctl = reinterpret_cast<PairCtl*>(epi + 8 * Cfg::kEpiWarpBytes);
  volatile int* abort_flag = &ctl->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cta = (int)cluster_ctarank(), rank = cta & 1, part = kSplit ? cta >> 1 : 0;
  // the tiles of this pair (of this cluster, where pairs share one), and its k-blocks
  const int parts = kSplit ? args.parts : 1;
  const int pair = kSplit ? (int)blockIdx.x / (2 * parts) : blockIdx.x >> 1, num_pairs = kSplit ? 0x3FFFFFFF : gridDim.x >> 1;
  const int kb0 = kSplit ? args.nkb * part / parts : 0, kb1 = kSplit ? args.nkb * (part + 1) / parts : args.nkb;
  const int b_chunks = (half + 63) >> 6;                   // MN-major B: chunks of 64 columns
  const bool sums = kKind == PK_DW && kMode != PM_SPLIT && args.term_rows > 0;
  const uint32_t stage_tx = sums   ? 2u * (uint32_t)(8192 + b_chunks * 4096)
                            : kVar ? 2u * (uint32_t)(Cfg::kABytes + (Cfg::kBMN ? b_chunks * 8192 : half * 128) + Cfg::kScaleBytes)
                                   : 2u * Cfg::kStageBytes;
  int num_tiles = args.num_m[0] * args.num_n[0];
  if (kKind == PK_DW)
    for (int j = 1; j < args.jobs; ++j) num_tiles += args.num_m[j] * args.num_n[j];

  if (threadIdx.x == 0) {
    for (int i = 0; i < (kKind == PK_DW ? 2 : 3); ++i) prefetch_tmap(&maps.m[i * (kKind == PK_DW ? 3 : 1)]);
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&ctl->full[s], 1);
      mbar_init(&ctl->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&ctl->tmem_full[b], 1);
      mbar_init(&ctl->tmem_empty[b], 16);                  // eight epilogue warps of either CTA
    }
    for (int w = 0; w < 8; ++w) mbar_init(&ctl->epi_full[w], 1);
    ctl->abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc_2cta(&ctl->tmem_base, 512);
    tmem_relinquish_2cta();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  if (!args.beside) pdl_wait();
  if (args.early_next) pdl_trigger();
  const uint32_t tmem_base = ctl->tmem_base;

  if (warp == 0) {
    // =========================== TMA producer (both CTAs) ===========================
    const bool issues = elect_one();
    uint32_t stage = 0, phase = 0;
    bool ok = true;
    for (int n = 0, tile; ok && (tile = nth_tile(args, n, pair, num_pairs)) < num_tiles; ++n) {
      const PairTile t = pair_tile<kKind>(args, tile, tile_cols);
      const int m0 = t.m0 + rank * 128;
      const int n0 = kGated ? t.n0 : t.n0 + rank * half;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait_warp(&ctl->empty[stage], phase ^ 1, abort_flag)) { ok = false; break; }
        if (issues) {
          uint8_t* sA = smem + stage * Cfg::kStageBytes;
          uint8_t* sB = sA + Cfg::kABytes;
          uint64_t* bar = &ctl->full[stage];
          if (rank == 0) mbar_arrive_expect_tx(bar, stage_tx);                            // the bytes of both CTAs
          const bool second = kKind == PK_DX && kb >= args.nkb0;
          const int k = (second ? kb - args.nkb0 : kb) * 64;
          if (sums) {
            // 16 rows of the first terms, then 16 of the second ones, each with the other operand's rows: two products instead of four (rows
            // of second terms that meet the other operand's zeros are finite)
            const bool in_a = args.sums_in_a >> t.job & 1;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int kA = in_a ? h * args.term_rows : 0, kB = in_a ? 0 : h * args.term_rows;
              tma_load_2d_2cta(sA + h * 2048, &maps.m[t.job], bar, m0, kA);
              tma_load_2d_2cta(sA + 8192 + h * 2048, &maps.m[t.job], bar, m0 + 64, kA);
#pragma unroll
              for (int c = 0; c < Cfg::kBChunks; ++c)
                if (!kVar || c < b_chunks) tma_load_2d_2cta(sB + c * 8192 + h * 2048, &maps.m[3 + t.job], bar, n0 + c * 64, kB);
            }
          } else {
            if constexpr (kKind == PK_DW) {
              tma_load_2d_2cta(sA, &maps.m[t.job], bar, m0, k);
              tma_load_2d_2cta(sA + 8192, &maps.m[t.job], bar, m0 + 64, k);
            } else {
              tma_load_2d_2cta(sA, &maps.m[second ? 1 : 0], bar, k, m0);
            }
            const CUtensorMap* mb = kKind == PK_DW ? &maps.m[3 + t.job] : kKind == PK_DX ? &maps.m[second ? 3 : 2]
                                  : kGated ? &maps.m[1 + rank] : &maps.m[1];
            if constexpr (Cfg::kBMN) {
#pragma unroll
              for (int c = 0; c < Cfg::kBChunks; ++c)
                if (!kVar || c < b_chunks) tma_load_2d_2cta(sB + c * 8192, mb, bar, n0 + c * 64, k);
            } else {
              tma_load_2d_2cta(sB, mb, bar, k, n0);
            }
            if constexpr (kFp4) {
              uint8_t* sS = sB + Cfg::kBBytes;
              tma_load_3d_2cta(sS, &maps.m[kGated ? 4 : 3], bar, 0, kb * Cfg::kTiles, m0 >> 7);
#pragma unroll
              for (int b = 0; b < Cfg::kBBlocks; ++b)        // the scales of all of the tile's columns, in both CTAs
                tma_load_3d_2cta(sS + (1 + b) * Cfg::kTiles * 512, &maps.m[kGated ? 5 + b : 4], bar, 0, kb * Cfg::kTiles,
                                 kGated ? t.n0 >> 7 : (t.n0 >> 7) + b);
            }
          }
        }
        if (++stage == kStages) { stage = 0; phase ^= 1; }
      }
    }
    pdl_trigger();
  } else if (warp == 1) {
    // =========================== MMA issuer (leader CTA only) ===========================
    if (rank == 0) {
      constexpr uint32_t idesc_full = kFp4 ? idesc_fp4(256, kBN, kFmt) : idesc_bf16(256, kBN, Cfg::kAMN, Cfg::kBMN, false);
      const uint32_t idesc = kVar ? idesc_full - ((uint32_t)(kBN - bn) >> 3 << 17) : idesc_full;
      constexpr uint64_t a_proto = desc_proto(Cfg::kAMN ? 8192 : 16, 1024, kSwizzle128B);
      constexpr uint64_t b_proto = desc_proto(Cfg::kBMN ? 8192 : 16, 1024, kSwizzle128B);
      constexpr uint64_t s_proto = desc_proto(128, 128, kSwizzleNone);
      const uint32_t smem16 = desc_address(smem), tmem = __shfl_sync(0xFFFFFFFFu, tmem_base, 0);
      constexpr uint32_t a_step = (Cfg::kAMN ? 2048 : 32) >> 4, b_step = (Cfg::kBMN ? 2048 : 32) >> 4;
      const bool issues = elect_one();
      uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0, blocks = 0;
      bool ok = true;
      for (int n = 0, tile; ok && (tile = nth_tile(args, n, pair, num_pairs)) < num_tiles; ++n) {
        if (!mbar_wait_warp(&ctl->tmem_empty[acc], acc_phase ^ 1, abort_flag)) break;
        tc_fence_after();
        const uint32_t d = tmem + acc * kBN;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!mbar_wait_warp(&ctl->full[stage], phase, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint32_t s16 = smem16 + stage * (uint32_t)(Cfg::kStageBytes >> 4);
          const uint64_t a = a_proto + s16, b = b_proto + (s16 + (Cfg::kABytes >> 4));
          const uint32_t more = kb > kb0 ? 1u : 0u;
          if constexpr (kFp4) {
            // The stage's scales go to TMEM, into one of two buffers in turn, ahead of the products that read them. The products that read
            // this buffer last are those of two blocks ago: their end has been signalled with their stage.
            if (blocks >= 2) {
              const uint32_t back = stage >= 2 ? stage - 2 : stage + kStages - 2;
              if (!mbar_wait_warp(&ctl->empty[back], stage >= 2 ? phase : phase ^ 1u, abort_flag)) { ok = false; break; }
            }
            const uint32_t sa = tmem + Cfg::kScaleCol + (blocks & 1u) * Cfg::kScaleCols, sb = sa + Cfg::kScaleACols;
            const uint64_t sd = s_proto + (s16 + ((Cfg::kABytes + Cfg::kBBytes) >> 4));
            if (issues) {
#pragma unroll
              for (int i = 0; i < Cfg::kTiles; ++i) {
                tmem_cp_scales_2cta(sa + 4 * i, sd + 32 * i);
#pragma unroll
                for (int j = 0; j < Cfg::kBBlocks; ++j)
                  tmem_cp_scales_2cta(sb + 4 * (i * Cfg::kBBlocks + j), sd + 32 * ((1 + j) * Cfg::kTiles + i));
              }
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const int i = kFmt == FMT_NV ? k : k >> 1;                                 // tile, and first scale in its words
                const uint32_t id = kFmt == FMT_NV ? 0u : (uint32_t)(k & 1) * 2u;
                mma_fp4_2cta<kFmt>(d, a + k * a_step, b + k * b_step, idesc | id << 4 | id << 29, sa + 4 * i, sb + 4 * i * Cfg::kBBlocks,
                                   k > 0 ? 1u : more);
              }
              commit_pair(&ctl->empty[stage], part);
            }
          } else if (issues) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (kKind != PK_DW || k < 2 || !sums) mma_f16_2cta(d, a + k * a_step, b + k * b_step, idesc, k > 0 ? 1u : more);
            commit_pair(&ctl->empty[stage], part);
          }
          __syncwarp();
          ++blocks;
          if (++stage == kStages) { stage = 0; phase ^= 1; }
        }
        if (!ok) break;
        if (issues) commit_pair(&ctl->tmem_full[acc], part);
        __syncwarp();
        if (++acc == (uint32_t)kAccs) { acc = 0; acc_phase ^= 1; }
      }
    }
  } else {
    // =========================== epilogue (warps 2..9, both CTAs) ===========================
    const int q = warp & 3, set = (warp - 2) >> 2;
    uint8_t* bufs = epi + (warp - 2) * Cfg::kEpiWarpBytes;
    uint64_t* loaded = &ctl->epi_full[warp - 2];
    constexpr int kBufBytes = Cfg::kEpiWarpBytes / 2;
    uint32_t acc = 0, acc_phase = 0, buf = 0, load_phase = 0;
    auto put16 = [&](const CUtensorMap* m, const uint32_t (&w)[16], int col, int row) {
      put_chunk_begin(lane);
      row_bf16(bufs + buf * kBufBytes, lane, w);
      put_chunk_end(m, bufs + buf * kBufBytes, col, row, lane);
      buf ^= 1u;
    };
    auto put32 = [&](const CUtensorMap* m, const uint32_t (&w)[32], int col, int row) {
      put_chunk_begin(lane);
      row_f32(bufs + buf * kBufBytes, lane, w);
      put_chunk_end(m, bufs + buf * kBufBytes, col, row, lane);
      buf ^= 1u;
    };
    for (int n = 0, tile; (tile = nth_tile(args, n, pair, num_pairs)) < num_tiles; ++n) {
      const PairTile t = pair_tile<kKind>(args, tile, tile_cols);
      const int row = t.m0 + rank * 128 + q * 32;
      const int M = kKind == PK_DW ? args.M[t.job] : args.M[0], N = kKind == PK_DW ? args.N[t.job] : args.N[0];
      // chunks of 32 output columns that are there; the two sets take them in turn
      const int chunks = row < M ? min(tile_cols >> 5, (N - t.n0 + 31) >> 5) : 0;
      auto fetch = [&](int ch) {                           // PK_BWD: P and Q of a chunk
        if (lane == 0) {
          bulk_wait_read<0>();
          mbar_arrive_expect_tx(loaded, 8192u);
          tma_load_2d(bufs, &maps.m[2], loaded, t.n0 + ch * 32, row);
          tma_load_2d(bufs + 4096, &maps.m[3], loaded, t.n0 + ch * 32, row);
        }
      };
      if (kKind == PK_BWD && part * 2 + set < chunks) fetch(part * 2 + set);
      if (!mbar_wait_warp(&ctl->tmem_full[acc], acc_phase, abort_flag)) {
        if constexpr (!kSplit) break;
      }
      tc_fence_after();
      const uint32_t taddr = tmem_base + acc * kBN + ((uint32_t)(q * 32) << 16);
      bool ok = true;
      auto release = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_leader(&ctl->tmem_empty[acc]);
      };
      // gate (v) and other factor (u) of a chunk to H and, where they are kept, P and Q
      auto gated_chunk = [&](uint32_t (&v)[32], uint32_t (&u)[32], int col) {
        uint32_t h[16];
        with_act(args.act, [&](auto tag) {
          constexpr int kAct = decltype(tag)::value;
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            float a[2], da[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float g = __uint_as_float(v[i + e]), uu = __uint_as_float(u[i + e]);
              if (kFp4) { g *= args.alpha; uu *= args.alpha2; }
              gate_act<kAct>(g, a[e], da[e]);
              v[i + e] = __float_as_uint(a[e]);
              u[i + e] = __float_as_uint(uu * da[e]);
              a[e] *= uu;
            }
            h[i >> 1] = bf16x2(a[0], a[1]);
          }
        });
        put16(&maps.m[3], h, col, row);
        if constexpr (kKind == PK_FWD_SAVE) {
          put32(&maps.m[4], v, col, row);
          put32(&maps.m[5], u, col, row);
        }
      };
      auto plain_chunk = [&](const uint32_t (&v)[32], uint32_t (&w)[16]) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float lo = __uint_as_float(v[2 * i]), hi = __uint_as_float(v[2 * i + 1]);
          if (kFp4) { lo *= args.alpha; hi *= args.alpha; }
          w[i] = bf16x2(lo, hi);
        }
      };
      // a chunk's accumulator columns to its outputs
      auto chunk = [&](uint32_t (&v)[32], uint32_t (&u)[32], int ch) {
        const int col = t.n0 + ch * 32;
        if constexpr (kGated) {
          gated_chunk(v, u, col);
        } else if constexpr (kKind == PK_BWD) {
          uint32_t du[16], dg[16];
          if (!mbar_wait_warp(loaded, load_phase, abort_flag)) return false;
          load_phase ^= 1u;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float4 p = *reinterpret_cast<const float4*>(bufs + lane * 128 + ((j ^ (lane & 7)) << 4));
            const float4 r = *reinterpret_cast<const float4*>(bufs + 4096 + lane * 128 + ((j ^ (lane & 7)) << 4));
            const float d0 = __uint_as_float(v[4 * j]), d1 = __uint_as_float(v[4 * j + 1]), d2 = __uint_as_float(v[4 * j + 2]),
                        d3 = __uint_as_float(v[4 * j + 3]);
            du[2 * j] = bf16x2(d0 * p.x, d1 * p.y); du[2 * j + 1] = bf16x2(d2 * p.z, d3 * p.w);
            dg[2 * j] = bf16x2(d0 * r.x, d1 * r.y); dg[2 * j + 1] = bf16x2(d2 * r.z, d3 * r.w);
          }
          __syncwarp();                                    // every row has been read: the results take its place
          row_bf16(bufs, lane, du);
          row_bf16(bufs + 4096, lane, dg);
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            tma_store_2d(&maps.m[5], bufs, col, row);
            tma_store_2d(&maps.m[4], bufs + 4096, col, row);
            bulk_commit();
          }
        } else {
          uint32_t w[16];
          plain_chunk(v, w);
          put16(&maps.m[kKind == PK_DW ? 6 + t.job : kKind == PK_DX ? 4 : 2], w, col, row);
        }
        return true;
      };
      if constexpr (kAccs == 1) {
        // One accumulator: the next main loop waits for it, so all of it is read into registers and handed back before anything
        // is made of it (4099 x 8192 x 2048 gated, blocks of 16: 133 -> 112 us; 16384 x 4096 x 4096, blocks of 32: 122 -> 98).
        if constexpr (kGated) {
          uint32_t v[2][32], u[2][32];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            tmem_ld_32x32b_x32(taddr + (set + 2 * i) * 32, v[i]);
            tmem_ld_32x32b_x32(taddr + kBN / 2 + (set + 2 * i) * 32, u[i]);
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) { tmem_ld_wait_on(v[i]); tmem_ld_wait_on(u[i]); }
          release();
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (set + 2 * i < chunks) gated_chunk(v[i], u[i], t.n0 + (set + 2 * i) * 32);
        } else {
          constexpr int kMine = kBN / 64;
          uint32_t v[kMine][32];
#pragma unroll
          for (int i = 0; i < kMine; ++i) tmem_ld_32x32b_x32(taddr + (set + 2 * i) * 32, v[i]);
#pragma unroll
          for (int i = 0; i < kMine; ++i) tmem_ld_wait_on(v[i]);
          release();
#pragma unroll
          for (int i = 0; i < kMine; ++i)
            if (set + 2 * i < chunks) {
              uint32_t w[16];
              plain_chunk(v[i], w);
              put16(&maps.m[2], w, t.n0 + (set + 2 * i) * 32, row);
            }
        }
      } else if constexpr (kSplit) {
        // this pair's sum over its part of K, [four columns][row][4], where the ring was: every product has been made
        if (chunks > 0) {
          float4* mine = reinterpret_cast<float4*>(smem) + q * 32 + lane;
#pragma unroll 1
          for (int ch = set; ch < bn >> 5; ch += 2) {
            uint32_t v[32];
            tmem_ld_32x32b_x32(taddr + ch * 32, v);
            tmem_ld_wait_on(v);
#pragma unroll
            for (int j = 0; j < 8; ++j)
              mine[(ch * 8 + j) * 128] = make_float4(__uint_as_float(v[4 * j]), __uint_as_float(v[4 * j + 1]), __uint_as_float(v[4 * j + 2]),
                                                     __uint_as_float(v[4 * j + 3]));
          }
        }
      } else {
#pragma unroll 1
        for (int ch = set; ch < chunks; ch += 2) {
          uint32_t v[32], u[32];
          tmem_ld_32x32b_x32(taddr + ch * 32, v);
          if constexpr (kGated) tmem_ld_32x32b_x32(taddr + half + ch * 32, u);
          tmem_ld_wait_on(v);
          if constexpr (kGated) tmem_ld_wait_on(u);
          if (!(ok = chunk(v, u, ch))) break;
          if (kKind == PK_BWD && ch + 2 < chunks) fetch(ch + 2);
        }
        if (!ok) break;
        release();
      }
      if (++acc == (uint32_t)kAccs) { acc = 0; acc_phase ^= 1; }
      if constexpr (kSplit) {
        __syncwarp();
        tc_fence_before();
        cluster_sync_all();                                // every pair's sum is there
        // the pairs share the tile's chunks, two to a pair at a time, and add them up in the order of the parts
        const uint32_t from = smem_u32(smem) + (uint32_t)(q * 32 + lane) * 16u;
#pragma unroll 1
        for (int ch = part * 2 + set; ch < chunks; ch += 2 * parts) {
          uint32_t v[32], u[32];
          if (kKind == PK_BWD && ch != part * 2 + set) fetch(ch);
          sum_parts(v, from + (uint32_t)ch * 16384u, rank, parts);
          if constexpr (kGated) sum_parts(u, from + (uint32_t)(ch + (half >> 5)) * 16384u, rank, parts);
          if (!chunk(v, u, ch)) break;
        }
      }
    }
    if (lane == 0) bulk_wait_all();
  }

  if (kSplit && warp < 2) {
    __syncwarp();
    cluster_sync_all();                                    // with the epilogue warps, see there
  }
  // =========================== teardown ===========================
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && ctl->abort_flag) {
    atomicExch(args.status, 1);
    drain_after_expiry();
  }
  if (args.beside) pdl_wait();                             // this launch ends after the one before it
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_2cta(tmem_base, 512);
  }
}

template <int kKind, int kBN, int kFmt, int kMode>
int launch_pair(const PairMaps<PairCfg<kKind, kBN, kFmt, kMode>::kMaps>& maps, PairArgs a, cudaStream_t s) {
  using Cfg = PairCfg<kKind, kBN, kFmt, kMode>;
  auto kern = pair_product_kernel<kKind, kBN, kFmt, kMode>;
  static std::atomic<bool> attr_done[64]{};
  int dev = 0;
  SF_CUDA_TRY(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64 || !attr_done[dev]) {
    SF_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmem));
    if (dev >= 0 && dev < 64) attr_done[dev] = true;
  }
  const int bn = kMode == PM_FULL ? kBN : a.bn, cols = Cfg::kGated ? bn / 2 : bn, parts = kMode == PM_SPLIT ? a.parts : 1;
  int64_t tiles = 0;
  for (int j = 0; j < a.jobs; ++j) {
    a.num_m[j] = (a.M[j] + 255) / 256;
    a.num_n[j] = (a.N[j] + cols - 1) / cols;
    tiles += (int64_t)a.num_m[j] * a.num_n[j];
  }
  if (tiles > 0x3FFFFFFF / (2 * parts)) return SF_ERR_SHAPE;
  const int64_t most = sm_count_now() / 2, pairs = kMode == PM_SPLIT ? tiles * parts : tiles < most ? tiles : most;
  a.early_next |= kMode != PM_SPLIT && tiles > most && (tiles / most + 1) * a.nkb >= 128;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * pairs));
  cfg.blockDim = dim3(kPairThreads);
  cfg.dynamicSmemBytes = Cfg::kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)(2 * parts);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  SF_CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, maps, a));
  return SF_OK;
}

}  // namespace
}  // namespace sf
