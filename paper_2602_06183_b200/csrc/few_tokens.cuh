// Products of few tokens with whole weight matrices, T at most kN:
//   FK_NT     C[T, N] = alpha X[T, K] W[N, K]^T
//   FK_GATED  H = act(alpha_g X Wg^T) (alpha_u X Wu^T), optionally P and Q
//   FK_DX     C = X0 W0 + X1 W1, the weights stored [K, N]; one accumulation over both pairs
//   FK_BWD    dU = (X W) P, dG = (X W) Q, the weights stored [K, N]
// What bounds them is reading the weights once, so the weights are the instruction's 128 rows and the tokens its
// few columns, and the reduction is split over the CTAs of a cluster until every SM has weights to read: each computes
// a partial sum of its own K range in TMEM, leaves it in its shared memory, and the cluster adds the partial sums up in the order
// of the ranges (the same every time) through distributed shared memory.
// One token, D 4096, F 16384, cold: both projections 48.5 us (268 MB, 5.5 TB/s), the down projection 28.6 (134 MB, 4.7 TB/s); 16384 x 4096 of
// 4 bits 13.4 alone (38 MB), 9.0 behind other launches. What is left is the start of the stream and the sums at its end.
//
// CTA = 10 warps: TMA producer, MMA issuer, four warps that read the accumulator out; all of them add up (with six, whose loads
// are few at a time, 100 tokens through both projections of 8192 x 2048 took 15.7 us, with ten 12.1). Every wait is bounded (see gemm_tc.cu); the
// cluster barriers are reached by every warp because their own waits are.
#pragma once

#include "gated.cuh"

namespace sf {
namespace {

using namespace ptx;

constexpr int kFewThreads = 320;
constexpr int kFewStages = 10;       // of the ring, at most

constexpr uint32_t pow2_cols(uint32_t n) { return n <= 32 ? 32 : n <= 64 ? 64 : n <= 128 ? 128 : n <= 256 ? 256 : 512; }

enum FewKind { FK_NT, FK_GATED, FK_DX, FK_BWD };

template <int kFmt, int kKind, int kN>
struct FewCfg {
  static constexpr bool kFp4 = kFmt != FMT_BF16, kGated = kKind == FK_GATED, kWMN = kKind == FK_DX || kKind == FK_BWD;
  static constexpr int kMats = kGated ? 2 : 1;
  static constexpr int kTiles = kFmt == FMT_NV ? 4 : kFmt == FMT_MX ? 2 : 0;
  static constexpr int kWBytes = 16384, kXBytes = kN * 128;
  static constexpr int kScaleBytes = kTiles * 512 * (kMats + 1);
  static constexpr int kStageBytes = kMats * kWBytes + kXBytes + kScaleBytes;
  static constexpr int kPartBytes = kMats * kN * 128 * 4;
  static constexpr uint32_t kScaleCol = kMats * kN, kScaleCols = kTiles * 4 * (kMats + 1);
  static constexpr uint32_t kTmem = pow2_cols(kScaleCol + 2 * kScaleCols);
  // one CTA to an SM, or two (one sets up and adds up while the other streams) while their columns and partial sums fit
  static constexpr int stages(int per_sm) {
    const int n = ((per_sm == 2 ? 115712 : 232448) - 2048) / kStageBytes;
    return n < kFewStages ? n : kFewStages;
  }
  static constexpr int smem(int per_sm) { return 2048 + stages(per_sm) * kStageBytes; }
  static constexpr int kMostPerSm = kTmem <= 256 && stages(2) >= 2 && kPartBytes <= stages(2) * kStageBytes ? 2 : 1;
  static_assert(stages(1) >= 2 && kPartBytes <= stages(1) * kStageBytes, "shared memory");
};

struct FewArgs {
  int T, N, nkb;                     // tokens, output columns, k-blocks (64 K of bf16, 256 K of 4 bits)
  int in_terms, out_terms;           // 2: the tokens' operand, or the results, are sums of two bf16: rows t and T + t (see kTwoTerms)
  int nkb0;                          // FK_DX: those of the first pair
  int act;
  int stages;                        // of the ring
  int early_weights;                 // the launch before this one does not write the weights, and waited for those that may have
  int early_next;                    // the next launch runs beside this one
  float alpha, alpha2;
  void* C;                           // [T, N] bf16 (FK_BWD: dU)
  void* C2;                          // FK_BWD: dG
  float *P, *Q;                      // FK_GATED: written, optional; FK_BWD: read
  int* status;
};
struct FewMaps { CUtensorMap x, w0, w1, sx, s0, s1; };      // (FK_DX: the second pair is w1 and sx)

struct FewCtl {
  uint64_t full[kFewStages], empty[kFewStages], done;
  uint32_t tmem_base;
  int abort_flag;
};

__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* m, uint64_t* bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
// This warp's 32 lanes x 16 columns, complete when it returns.
__device__ __forceinline__ void tmem_ld_32x32b_x16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
        "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr) : "memory");
}
template <int kFmt>
__device__ __forceinline__ void mma_fp4_1cta(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t acc) {
  if constexpr (kFmt == FMT_NV)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}\n"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc) : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}\n"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc) : "memory");
}
__device__ __forceinline__ void tmem_cp_scales(uint32_t taddr, uint64_t sdesc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(sdesc) : "memory");
}

// The weights' part of a stage, and the tokens'.
template <int kFmt, int kKind, int kN>
__device__ __forceinline__ void load_weights(const FewMaps& maps, uint8_t* sw, uint64_t* bar, int kb, int f0, int nkb0) {
  using Cfg = FewCfg<kFmt, kKind, kN>;
  mbar_arrive_expect_tx(bar, (uint32_t)Cfg::kStageBytes);
  if constexpr (Cfg::kWMN) {
    const bool second = kKind == FK_DX && kb >= nkb0;
    const CUtensorMap* w = second ? &maps.w1 : &maps.w0;
    const int k = (second ? kb - nkb0 : kb) * 64;
    tma_load_2d(sw, w, bar, f0, k);
    tma_load_2d(sw + 8192, w, bar, f0 + 64, k);
    return;
  }
  tma_load_2d(sw, &maps.w0, bar, kb * 64, f0);
  if (Cfg::kGated) tma_load_2d(sw + Cfg::kWBytes, &maps.w1, bar, kb * 64, f0);
  if constexpr (Cfg::kFp4) {
    uint8_t* ss = sw + Cfg::kMats * Cfg::kWBytes + Cfg::kXBytes;
    tma_load_3d(ss, &maps.s0, bar, 0, kb * Cfg::kTiles, f0 >> 7);
    if (Cfg::kGated) tma_load_3d(ss + Cfg::kTiles * 512, &maps.s1, bar, 0, kb * Cfg::kTiles, f0 >> 7);
  }
}
template <int kFmt, int kKind, int kN>
__device__ __forceinline__ void load_tokens(const FewMaps& maps, uint8_t* sw, uint64_t* bar, int kb, int nkb0) {
  using Cfg = FewCfg<kFmt, kKind, kN>;
  uint8_t* sx = sw + Cfg::kMats * Cfg::kWBytes;
  const bool second = kKind == FK_DX && kb >= nkb0;
  tma_load_2d(sx, second ? &maps.sx : &maps.x, bar, (second ? kb - nkb0 : kb) * 64, 0);
  if constexpr (Cfg::kFp4) tma_load_3d(sx + Cfg::kXBytes + Cfg::kMats * Cfg::kTiles * 512, &maps.sx, bar, 0, kb * Cfg::kTiles, 0);
}

template <int kFmt, int kKind, int kN>
__global__ void __launch_bounds__(kFewThreads, FewCfg<kFmt, kKind, kN>::kMostPerSm)
few_tokens_kernel(const __grid_constant__ FewMaps maps, const FewArgs args) {
  using Cfg = FewCfg<kFmt, kKind, kN>;
  constexpr bool kFp4 = Cfg::kFp4, kGated = Cfg::kGated;
  constexpr int kMats = Cfg::kMats, kTiles = Cfg::kTiles;
  const uint32_t stages = (uint32_t)args.stages;
  extern __shared__ uint8_t smem_dyn[];
  uint8_t* smem = smem_dyn + align_pad(smem_dyn, 1024);
  FewCtl* ctl = reinterpret_cast<FewCtl*>(smem + stages * Cfg::kStageBytes);
  volatile int* abort_flag = &ctl->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int S = (int)cluster_size(), rank = (int)cluster_ctarank();
  const int f0 = (int)(blockIdx.x / S) * 128;               // first of this cluster's 128 weight rows
  const int kb0 = (int)((int64_t)args.nkb * rank / S), kb1 = (int)((int64_t)args.nkb * (rank + 1) / S);

  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < stages; ++s) {
      mbar_init(&ctl->full[s], 1);
      mbar_init(&ctl->empty[s], 1);
    }
    mbar_init(&ctl->done, 1);
    ctl->abort_flag = 0;
    fence_mbar_init();
  }
  if (threadIdx.x >= 64 && threadIdx.x < 70) prefetch_tmap(&maps.x + (threadIdx.x - 64));
  if (warp == 1) {
    tmem_alloc(&ctl->tmem_base, Cfg::kTmem);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = ctl->tmem_base;

  // The launch before this one writes the tokens, and may read what this one writes. Waiting here also keeps that launch's time out of the
  // budgets of the roles' own waits, which the first tokens end.
  if (warp != 0) pdl_wait();
  if (warp == 0) {
    const bool issues = elect_one();
    // what fits the ring of weights that are known to be there is fetched while the launch before this one ends
    const int early = args.early_weights ? min((int)stages, kb1 - kb0) : 0;
    if (issues)
      for (int i = 0; i < early; ++i) load_weights<kFmt, kKind, kN>(maps, smem + i * Cfg::kStageBytes, &ctl->full[i], kb0 + i, f0, args.nkb0);
    __syncwarp();
    pdl_wait();
    if (args.early_next) pdl_trigger();
    uint32_t stage = 0, phase = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!mbar_wait_warp(&ctl->empty[stage], phase ^ 1, abort_flag)) break;
      if (issues) {
        uint8_t* sw = smem + stage * Cfg::kStageBytes;
        if (kb - kb0 >= early) load_weights<kFmt, kKind, kN>(maps, sw, &ctl->full[stage], kb, f0, args.nkb0);
        load_tokens<kFmt, kKind, kN>(maps, sw, &ctl->full[stage], kb, args.nkb0);
      }
      if (++stage == stages) { stage = 0; phase ^= 1; }
    }
    pdl_trigger();
  } else if (warp == 1) {
    constexpr uint32_t idesc = kFp4 ? idesc_fp4(128, kN, kFmt) : idesc_bf16(128, kN, Cfg::kWMN, false, false);
    constexpr uint64_t proto = desc_proto(16, 1024, kSwizzle128B), w_proto = desc_proto(Cfg::kWMN ? 8192 : 16, 1024, kSwizzle128B);
    constexpr uint32_t w_step = (Cfg::kWMN ? 2048 : 32) >> 4;
    constexpr uint64_t s_proto = desc_proto(128, 128, kSwizzleNone);
    const uint32_t smem16 = desc_address(smem), tmem = __shfl_sync(0xFFFFFFFFu, tmem_base, 0);
    const bool issues = elect_one();
    uint32_t stage = 0, phase = 0;
    bool ok = true;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!mbar_wait_warp(&ctl->full[stage], phase, abort_flag)) { ok = false; break; }
      tc_fence_after();
      const uint32_t s16 = smem16 + stage * (uint32_t)(Cfg::kStageBytes >> 4);
      const uint64_t w = w_proto + s16, x = proto + (s16 + (kMats * Cfg::kWBytes >> 4));
      const uint32_t scol = tmem + Cfg::kScaleCol + ((uint32_t)(kb - kb0) & 1u) * Cfg::kScaleCols;
      const uint32_t more = kb > kb0 ? 1u : 0u;
      // scales: one of two buffers in turn; the products of two blocks ago, which read this one, have signalled their end with their stage
      if (kFp4 && kb - kb0 >= 2) {
        const uint32_t back = stage >= 2 ? stage - 2 : stage + stages - 2;
        if (!mbar_wait_warp(&ctl->empty[back], stage >= 2 ? phase : phase ^ 1u, abort_flag)) { ok = false; break; }
      }
      if (issues) {
        if constexpr (kFp4) {
          const uint64_t sd = s_proto + (s16 + ((kMats * Cfg::kWBytes + Cfg::kXBytes) >> 4));
#pragma unroll
          for (int i = 0; i < kTiles * (kMats + 1); ++i) tmem_cp_scales(scol + 4 * i, sd + 32 * i);
        }
#pragma unroll
        for (int m = 0; m < kMats; ++m)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint64_t wd = w + (m * (Cfg::kWBytes >> 4) + k * w_step), xd = x + 2 * k;
            if constexpr (kFp4) {
              const int i = kFmt == FMT_NV ? k : k >> 1;
              const uint32_t id = kFmt == FMT_NV ? 0u : (uint32_t)(k & 1) * 2u;
              mma_fp4_1cta<kFmt>(tmem + m * kN, wd, xd, idesc | id << 4 | id << 29, scol + 4 * (m * kTiles + i),
                                 scol + 4 * (kMats * kTiles + i), k > 0 ? 1u : more);
            } else {
              mma_f16(tmem + m * kN, wd, xd, idesc, k > 0 ? 1u : more);
            }
          }
        mma_commit(&ctl->empty[stage]);
      }
      __syncwarp();
      if (++stage == stages) { stage = 0; phase ^= 1; }
    }
    if (ok && issues) mma_commit(&ctl->done);
  } else if (warp < 6) {
    // every product has been made, so every load has landed and the ring is free: the partial sums go there, [matrix][token][row]
    if (mbar_wait_warp(&ctl->done, 0, abort_flag)) {
      tc_fence_after();
      const int q = warp & 3;
      float* part = reinterpret_cast<float*>(smem) + q * 32 + lane;
#pragma unroll 1
      for (int m = 0; m < kMats; ++m)
#pragma unroll 1
        for (int c = m * kN; c < m * kN + args.in_terms * args.T; c += 16) {
          uint32_t v[16];
          tmem_ld_32x32b_x16(tmem_base + c + ((uint32_t)(q * 32) << 16), v);
#pragma unroll
          for (int i = 0; i < 16; ++i) part[(c + i) * 128] = __uint_as_float(v[i]);
        }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && ctl->abort_flag) {
    atomicExch(args.status, 1);
    drain_after_expiry();
  }
  if (S > 1) cluster_sync_all();                           // every partial sum of the cluster is there (0.6 us, alone too)
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, Cfg::kTmem);
  }
  // the cluster's threads share the sums, four neighbouring output columns to a thread; all partial sums of a value are fetched at once
  const uint32_t part = smem_u32(smem);
  for (int i = rank * kFewThreads + threadIdx.x; i < args.T * 32; i += S * kFewThreads) {
    const int t = i >> 5, p = (i & 31) * 4, f = f0 + p;
    if (f >= args.N) continue;
    float4 x[kMats][4], sum[kMats];
    for (int term = 0; term < args.in_terms; ++term)
#pragma unroll
      for (int s0 = 0; s0 < 8; s0 += 4) {
        if (s0 >= S) break;
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int m = 0; m < kMats; ++m) {
            const uint32_t at = part + (uint32_t)((m * kN + term * args.T + t) * 128 + p) * 4u;
            if (s0 + s < S) x[m][s] = ld_cluster_f4(at, s0 + s);
          }
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int m = 0; m < kMats; ++m) {
            if (s0 + s == 0 && term == 0) sum[m] = x[m][0];
            else if (s0 + s < S) { sum[m].x += x[m][s].x; sum[m].y += x[m][s].y; sum[m].z += x[m][s].z; sum[m].w += x[m][s].w; }
          }
      }
    float a[4] = {sum[0].x, sum[0].y, sum[0].z, sum[0].w};
    if (kFp4)
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] *= args.alpha;
    const int64_t at = (int64_t)t * args.N + f;
    if constexpr (kGated) {
      const float4 y = sum[kMats - 1];
      float b[4] = {y.x, y.y, y.z, y.w}, d[4];
      if (kFp4)
#pragma unroll
        for (int e = 0; e < 4; ++e) b[e] *= args.alpha2;
      with_act(args.act, [&](auto tag) {
#pragma unroll
        for (int e = 0; e < 4; ++e) gate_act<decltype(tag)::value>(a[e], a[e], d[e]);
      });
      if (args.P) {
        *reinterpret_cast<float4*>(args.P + at) = make_float4(a[0], a[1], a[2], a[3]);
        *reinterpret_cast<float4*>(args.Q + at) = make_float4(b[0] * d[0], b[1] * d[1], b[2] * d[2], b[3] * d[3]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] *= b[e];
    }
    // four results of a row: rounded, and where the row has a second term, what the rounding left
    auto put = [&](void* C, const float (&v)[4]) {
      uint16_t* c = reinterpret_cast<uint16_t*>(C) + at;
      const uint32_t lo = bf16x2(v[0], v[1]), hi = bf16x2(v[2], v[3]);
      *reinterpret_cast<uint2*>(c) = make_uint2(lo, hi);
      if ((kKind == FK_GATED || kKind == FK_BWD) && args.out_terms == 2) {
        const uint32_t w[2] = {lo, hi};
        float rest[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float r = __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
          rest[e] = isfinite(r) ? v[e] - r : 0.f;
        }
        *reinterpret_cast<uint2*>(c + (int64_t)args.T * args.N) = make_uint2(bf16x2(rest[0], rest[1]), bf16x2(rest[2], rest[3]));
      }
    };
    if constexpr (kKind == FK_BWD) {
      const float4 p = __ldg(reinterpret_cast<const float4*>(args.P + at)), r = __ldg(reinterpret_cast<const float4*>(args.Q + at));
      const float dg[4] = {a[0] * r.x, a[1] * r.y, a[2] * r.z, a[3] * r.w};
      put(args.C2, dg);
      a[0] *= p.x; a[1] *= p.y; a[2] *= p.z; a[3] *= p.w;
    }
    put(args.C, a);
  }
  if (S > 1) cluster_sync_all();                           // no CTA leaves while another reads its shared memory
}

template <int kFmt, int kKind, int kN>
void few_config(cudaLaunchConfig_t& cfg, cudaLaunchAttribute (&attr)[2], int64_t N, int S, int per_sm, cudaStream_t s) {
  cfg = {};
  cfg.gridDim = dim3((unsigned)((N + 127) / 128 * S));
  cfg.blockDim = dim3(kFewThreads);
  cfg.dynamicSmemBytes = FewCfg<kFmt, kKind, kN>::smem(per_sm);
  cfg.stream = s;
  attr[0] = {};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)S;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1] = {};
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
}

// How many clusters of 1 to 8 CTAs a device holds at once with one CTA to an SM (a cluster stays within one of the chip's groups of
// SMs, whose size is no multiple of most numbers); with two it is taken for twice as many. Asked once; every thread that asks
// gets the same answer.
struct FewRoom {
  int clusters[8];
  std::atomic<int> set;
};
template <int kFmt, int kKind, int kN>
int few_room(const FewRoom** room) {
  using Cfg = FewCfg<kFmt, kKind, kN>;
  static FewRoom rooms[64];
  static FewRoom other;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) {                // no device: what the chip that this is written for answers
    static const FewRoom usual{{148, 74, 45, 33, 26, 22, 15, 15}, {1}};
    cudaGetLastError();
    *room = &usual;
    return SF_OK;
  }
  FewRoom& r = dev >= 0 && dev < 64 ? rooms[dev] : other;
  *room = &r;
  if (r.set.load(std::memory_order_acquire) && &r != &other) return SF_OK;
  auto kern = few_tokens_kernel<kFmt, kKind, kN>;
  SF_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::smem(1)));
  SF_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
  for (int S = 1; S <= 8; ++S) {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    few_config<kFmt, kKind, kN>(cfg, attr, 128 * 1024, S, 1, nullptr);
    cfg.numAttrs = 1;
    int n = 0;
    SF_CUDA_TRY(cudaOccupancyMaxActiveClusters(&n, kern, &cfg));
    r.clusters[S - 1] = n;
  }
  r.set.store(1, std::memory_order_release);
  return SF_OK;
}

template <int kFmt, int kKind, int kN>
int launch_few(const FewMaps& maps, FewArgs a, int S, int per_sm, cudaStream_t s) {
  a.stages = FewCfg<kFmt, kKind, kN>::stages(per_sm);
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attr[2];
  few_config<kFmt, kKind, kN>(cfg, attr, a.N, S, per_sm, s);
  SF_CUDA_TRY(cudaLaunchKernelEx(&cfg, few_tokens_kernel<kFmt, kKind, kN>, maps, a));
  return SF_OK;
}

}  // namespace
}  // namespace sf
