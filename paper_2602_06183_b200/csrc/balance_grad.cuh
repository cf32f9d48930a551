// The balance loss's gradients on warp-level tensor instructions (see router_balance.cu for the formulas and what bounds them).
#pragma once

#include "gated.cuh"
#include "sums.cuh"

namespace sf {
namespace {

using namespace ptx;

constexpr int kMostExperts = 16;

struct Softmax { float p[kMostExperts], lse; };
// Of E logits; entries from E on are 0.
__device__ __forceinline__ Softmax softmax_of(const float* __restrict__ l, int E) {
  Softmax s;
  float top = -INFINITY;
  if ((E & 3) == 0) {                  // rows on 16-byte boundaries
#pragma unroll
    for (int e = 0; e < kMostExperts; e += 4) {
      const float4 v = e < E ? __ldg(reinterpret_cast<const float4*>(l + e)) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      s.p[e] = v.x; s.p[e + 1] = v.y; s.p[e + 2] = v.z; s.p[e + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < kMostExperts; ++e) s.p[e] = e < E ? __ldg(l + e) : -INFINITY;
  }
#pragma unroll
  for (int e = 0; e < kMostExperts; ++e) top = fmaxf(top, s.p[e]);
  const float from = top == -INFINITY ? 0.f : top;         // (a row of -infinities is NaN: 0 / 0)
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < kMostExperts; ++e) {
    s.p[e] = e < E ? expf(s.p[e] - from) : 0.f;
    sum += s.p[e];
  }
  const float inv = 1.f / sum;
#pragma unroll
  for (int e = 0; e < kMostExperts; ++e) s.p[e] *= inv;
  s.lse = from + logf(sum);
  return s;
}

struct BalanceArgs {
  const float* logits;
  const int *expert, *counts;
  const float* dloss;
  const uint16_t* means;
  float* parts;                        // [gridDim.y][E][D]
  uint16_t* dmeans;                    // instead of parts: the runs of a slab are a cluster, which adds them up itself
  int* status;
  int64_t T, rows;                     // rows: tokens of a CTA, a multiple of kTile
  int D, E;
  float cb, cz;
  int adds, writes;                    // there is a dX_in, a dX
};
struct BalanceMaps { CUtensorMap x, in, out; };

// A warp owns 64 columns and walks its CTA's tokens in tiles of 32, with a ring of its own: X and dX_in by TMA (rows of 128 bytes, swizzled), dX
// written over dX_in and stored from there. The eight warps share dl only, which 256 threads compute for 256 tokens at a time.
constexpr int kTile = 32, kWarps = 8, kSlab = 64 * kWarps, kChunk = 32 * kWarps, kRing = 3;
constexpr int kTileBytes = kTile * 128, kDlBytes = kChunk * 32;         // of one operand; of one term of a chunk's dl (16 bf16 a token)
constexpr int kGradSmem = 1024 + kWarps * kRing * 2 * kTileBytes + 2 * 2 * kDlBytes + 512;
static_assert(kGradSmem <= 232448, "shared memory");

struct BalanceCtl {
  uint64_t full[kWarps][kRing];
  uint32_t out[2][kWarps];             // tokens of a tile that are left out
  int abort_flag;
};
static_assert(sizeof(BalanceCtl) <= 512, "control block");

__device__ __forceinline__ void ldmatrix_x4(uint32_t saddr, uint32_t (&v)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(saddr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t saddr, uint32_t (&v)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(saddr) : "memory");
}
// (not volatile: the compiler may move it among the others)
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Four floats of shared memory of the cluster's CTA `rank`, at this CTA's address `saddr`.
__device__ __forceinline__ float4 ld_cluster(uint32_t saddr, uint32_t rank) {
  float4 v;
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n\t}\n"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(saddr), "r"(rank) : "memory");
  return v;
}
// Where the half `h` (8 experts) of a token's dl lies: neighbouring rows of 32 bytes, halves exchanged in every other four rows, so that eight
// rows of a half touch all banks once.
__device__ __forceinline__ uint32_t dl_at(int token, int h) { return (uint32_t)(token * 32 + ((h ^ (token >> 2 & 1)) << 4)); }

__global__ void __launch_bounds__(32 * kWarps, 1)
balance_grad_kernel(const __grid_constant__ BalanceMaps maps, const BalanceArgs a) {
  extern __shared__ uint8_t smem_dyn[];
  uint8_t* smem = smem_dyn + align_pad(smem_dyn, 1024);
  uint8_t* dls = smem + kWarps * kRing * 2 * kTileBytes;
  BalanceCtl* ctl = reinterpret_cast<BalanceCtl*>(dls + 2 * 2 * kDlBytes);
  volatile int* abort_flag = &ctl->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int col = (int)blockIdx.x * kSlab + warp * 64;
  const bool works = col < a.D;
  const int64_t t0 = (int64_t)blockIdx.y * a.rows, t1 = t0 + a.rows < a.T ? t0 + a.rows : a.T;
  const int tiles = (int)((t1 - t0 + kTile - 1) / kTile);
  uint8_t* ring = smem + warp * (kRing * 2 * kTileBytes);

  if (lane == 0) {
    for (int s = 0; s < kRing; ++s) mbar_init(&ctl->full[warp][s], 1);
    if (warp == 0) ctl->abort_flag = 0;
    fence_mbar_init();
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();

  const bool loads = works && lane == 0;
  auto fetch = [&](int tile) {
    uint64_t* bar = &ctl->full[warp][tile % kRing];
    uint8_t* at = ring + (tile % kRing) * 2 * kTileBytes;
    const int row = (int)(t0 + (int64_t)tile * kTile);
    mbar_arrive_expect_tx(bar, (uint32_t)(a.adds ? 2 * kTileBytes : kTileBytes));
    tma_load_2d(at, &maps.x, bar, col, row);
    if (a.adds) tma_load_2d(at + kTileBytes, &maps.in, bar, col, row);
  };
  if (loads)
    for (int i = 0; i < kRing - 1 && i < tiles; ++i) fetch(i);

  float count[kMostExperts];
  long long all = 0;
#pragma unroll
  for (int e = 0; e < kMostExperts; ++e) {
    const int n = e < a.E ? __ldg(a.counts + e) : 0;
    count[e] = (float)n;
    all += n;
  }
  const float inv = all > 0 ? 1.f / (float)all : 0.f, g = a.dloss ? __ldg(a.dloss) : 1.f;
  const float k1 = g * a.cb * (float)a.E * inv * inv, k2 = g * 2.f * a.cz * inv;

  // the means as the second operand: 16 experts x 8 columns, eight times
  uint32_t mean[8][2];
  float dm[8][4];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int c = col + j * 8 + (lane >> 2);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int e = (lane & 3) * 2 + h * 8;
      uint32_t w = 0;
      if (c < a.D && e < a.E) w = __ldg(a.means + (int64_t)e * a.D + c);
      if (c < a.D && e + 1 < a.E) w |= (uint32_t)__ldg(a.means + (int64_t)(e + 1) * a.D + c) << 16;
      mean[j][h] = w;
    }
    dm[j][0] = dm[j][1] = dm[j][2] = dm[j][3] = 0.f;
  }

  bool ok = true;
  uint32_t phases = 0;                                     // of the ring's barriers
  for (int tile = 0; tile < tiles; ++tile) {
    const int chunk = tile / kWarps & 1;
    uint8_t* hi = dls + chunk * 2 * kDlBytes;
    if (tile % kWarps == 0) {
      // dl of the next 256 tokens, one to a thread
      const int64_t t = t0 + (int64_t)tile * kTile + threadIdx.x;
      bool counts = false;
      uint32_t h[8], l[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = l[i] = 0u;
      if (t < t1) counts = (unsigned)__ldg(a.expert + t) < (unsigned)a.E;
      if (counts) {
        const Softmax s = softmax_of(a.logits + t * a.E, a.E);
        float mean_n = 0.f;
#pragma unroll
        for (int e = 0; e < kMostExperts; ++e) mean_n = fmaf(count[e], s.p[e], mean_n);
#pragma unroll
        for (int e = 0; e < kMostExperts; e += 2) {
          const float x = s.p[e] * fmaf(k1, count[e] - mean_n, k2 * s.lse), y = s.p[e + 1] * fmaf(k1, count[e + 1] - mean_n, k2 * s.lse);
          h[e >> 1] = pack2(x, y);
          l[e >> 1] = pack2(x - lo32(h[e >> 1]), y - hi32(h[e >> 1]));
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t at = dl_at(threadIdx.x, i);
        *reinterpret_cast<uint4*>(hi + at) = make_uint4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]);
        *reinterpret_cast<uint4*>(hi + kDlBytes + at) = make_uint4(l[4 * i], l[4 * i + 1], l[4 * i + 2], l[4 * i + 3]);
      }
      const uint32_t left_out = __ballot_sync(0xFFFFFFFFu, t < t1 && !counts);
      if (lane == 0) ctl->out[chunk][warp] = left_out;
      __syncthreads();                 // (this buffer's last readers have passed the barrier of the chunk in between)
    }
    if (!works || !ok) continue;
    uint8_t* sx = ring + (tile % kRing) * 2 * kTileBytes;
    uint8_t* sd = sx + kTileBytes;
    if (!mbar_wait_warp(&ctl->full[warp][tile % kRing], phases >> (tile % kRing) & 1u, abort_flag)) { ok = false; continue; }
    phases ^= 1u << (tile % kRing);
    // a token that is left out may hold anything: 0 times it is to be 0
    for (uint32_t left = ctl->out[chunk][tile % kWarps]; left; left &= left - 1)
      *reinterpret_cast<uint32_t*>(sx + (__ffs(left) - 1) * 128 + lane * 4) = 0u;
    __syncwarp();
#pragma unroll
    for (int half = 0; half < 2; ++half) {                 // 16 tokens
      const int tok = (tile % kWarps) * kTile + half * 16;
      uint32_t ah[4], al[4], th[4], tl[4];                 // dl as 16 tokens x 16 experts, and transposed
      const uint32_t base = smem_u32(hi);
      const uint32_t n_at = dl_at(tok + (lane & 15), lane >> 4), t_at = dl_at(tok + (lane & 7) + (lane >> 4) * 8, lane >> 3 & 1);
      ldmatrix_x4(base + n_at, ah);
      ldmatrix_x4(base + kDlBytes + n_at, al);
      ldmatrix_x4_trans(base + t_at, th);
      ldmatrix_x4_trans(base + kDlBytes + t_at, tl);
      // eight products at a time, none of which waits for the one before it
      uint32_t b[8][2];                                    // X, 16 tokens x 8 columns, as the second operand
      float d[8][4];
      const int r = half * 16 + (lane >> 2);
      uint8_t* const p = sd + r * 128 + (lane & 3) * 4;     // of chunk j: 16 (j ^ (r & 7)) on; eight rows on, the same
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        uint32_t x[4];
        const int row = half * 16 + (lane & 15);
        ldmatrix_x4_trans(smem_u32(sx) + (uint32_t)(row * 128 + (((j + (lane >> 4)) ^ (row & 7)) << 4)), x);
        b[j][0] = x[0]; b[j][1] = x[1]; b[j + 1][0] = x[2]; b[j + 1][1] = x[3];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        d[j][0] = d[j][1] = d[j][2] = d[j][3] = 0.f;
        if (a.adds) {
          const uint32_t u = *reinterpret_cast<const uint32_t*>(p + ((j ^ (r & 7)) << 4)), v = *reinterpret_cast<const uint32_t*>(p + 1024 + ((j ^ (r & 7)) << 4));
          d[j][0] = lo32(u); d[j][1] = hi32(u); d[j][2] = lo32(v); d[j][3] = hi32(v);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) mma_16816(dm[j], th, b[j][0], b[j][1]);
#pragma unroll
      for (int j = 0; j < 8; ++j) mma_16816(d[j], ah, mean[j][0], mean[j][1]);
#pragma unroll
      for (int j = 0; j < 8; ++j) mma_16816(dm[j], tl, b[j][0], b[j][1]);
#pragma unroll
      for (int j = 0; j < 8; ++j) mma_16816(d[j], al, mean[j][0], mean[j][1]);
      if (a.writes) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          *reinterpret_cast<uint32_t*>(p + ((j ^ (r & 7)) << 4)) = pack2(d[j][0], d[j][1]);
          *reinterpret_cast<uint32_t*>(p + 1024 + ((j ^ (r & 7)) << 4)) = pack2(d[j][2], d[j][3]);
        }
      }
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      if (a.writes) {
        tma_store_2d(&maps.out, sd, col, (int)(t0 + (int64_t)tile * kTile));
        bulk_commit();
      }
      // the stage of the tile before this one, whose store has been read out of it by now
      if (tile + kRing - 1 < tiles) {
        bulk_wait_read<1>();
        fetch(tile + kRing - 1);
      }
    }
    __syncwarp();
  }
  if (a.dmeans) {
    if (lane == 0) bulk_wait_all();
    __syncwarp();
    // [16 experts][64 columns] of the warp, in its ring's place
    if (works) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          *reinterpret_cast<float2*>(ring + ((lane >> 2) + h * 8) * 256 + (j * 8 + (lane & 3) * 2) * 4) = make_float2(dm[j][2 * h], dm[j][2 * h + 1]);
    }
    cluster_sync_all();
    const int runs = (int)gridDim.y;
    for (int i = (int)blockIdx.y * 32 * kWarps + (int)threadIdx.x; i < a.E * (kSlab / 4); i += runs * 32 * kWarps) {
      const int e = i / (kSlab / 4), c = i % (kSlab / 4) * 4, to = (int)blockIdx.x * kSlab + c;
      if (to >= a.D) continue;
      const uint32_t from = smem_u32(smem) + (uint32_t)((c >> 6) * kRing * 2 * kTileBytes + e * 256 + (c & 63) * 4);
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k = 0; k < runs; ++k) {
        const float4 v = ld_cluster(from, (uint32_t)k);
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
      *reinterpret_cast<uint2*>(a.dmeans + (int64_t)e * a.D + to) = make_uint2(pack2(s.x, s.y), pack2(s.z, s.w));
    }
    cluster_sync_all();                // (the others have read this CTA's sums)
  }
  if (a.parts && works && ok) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = col + j * 8 + (lane & 3) * 2;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int e = (lane >> 2) + h * 8;
        if (c < a.D && e < a.E)
          *reinterpret_cast<float2*>(a.parts + ((int64_t)blockIdx.y * a.E + e) * a.D + c) = make_float2(dm[j][2 * h], dm[j][2 * h + 1]);
      }
    }
  }
  if (lane == 0) bulk_wait_all();
  __syncthreads();
  if (threadIdx.x == 0 && ctl->abort_flag) {
    atomicExch(a.status, 1);
    drain_after_expiry();
  }
  __syncthreads();
}

}  // namespace
}  // namespace sf
