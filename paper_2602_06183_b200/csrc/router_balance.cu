// The router's balance loss. With p = softmax(l) of a token's logits, n_e the tokens that went to expert e and n all that went to one:
//   balance = E sum_e (n_e / n) (sum_t p_te / n)          1 where the experts are used evenly, up to E
//   z       = sum_t lse_t^2 / n                           lse = log sum_e exp(l_te)
//   loss    = cb balance + cz z
//   dl_te   = dloss p_te (cb E / n^2 (n_e - sum_j n_j p_tj) + 2 cz lse_t / n)
//   dX      = dX_in + dl means,   dmeans = dl^T X          (l = X means^T)
// A token whose expert lies outside [0, E) (padding) is left out of all sums and has dl = 0. n_e is counted, not differentiated.
//
// Forward: 4 E + 4 bytes a token, one launch; the CTA that finishes last adds up what the others left. Backward: 6 bytes an element of X
// (X and dX_in in, dX out) and 4 T D E flops, one launch and one that adds up the CTAs' partial sums of dmeans.
//
// Memory bounds the backward pass only if the products stay out of its way: as float32 multiply-adds they took 417 us where the bytes take 62 (16384
// tokens, D 4096, E 16). Sixteen experts are one side of a warp's m16n8k16 product, so both run there: dX = dl means with the means'
// fragments of a warp's 64 columns in 16 registers, dmeans = dl^T X with its sums in 32. dl is a sum of two bf16 numbers (16 bits), X and
// the means are bf16 as they come, sums are in float32.
#include "gated.cuh"
#include "sums.cuh"

#define SF_TRY(expr)              \
  do {                            \
    int _st = (expr);             \
    if (_st != SF_OK) return _st; \
  } while (0)

namespace sf {
namespace {

using namespace ptx;

constexpr int kMostExperts = 16;
constexpr int64_t kMostTokens = (int64_t)1 << 28, kMostCols = (int64_t)1 << 20;
constexpr int kLossCtas = 148, kLossThreads = 256;
constexpr size_t kHead = 256, kDone = 128;                 // status word; the word that counts the CTAs that have finished

// (z in double: a masked row's log-sum-exp may be the lowest float32, whose square is none)
struct LossPart { float p[kMostExperts]; double z; int n[kMostExperts]; };

struct Softmax { float p[kMostExperts], lse; };
// Of E logits; entries from E on are 0.
__device__ __forceinline__ Softmax softmax_of(const float* __restrict__ l, int E) {
  Softmax s;
  float top = -INFINITY;
#pragma unroll
  for (int e = 0; e < kMostExperts; ++e) {
    s.p[e] = e < E ? __ldg(l + e) : -INFINITY;
    top = fmaxf(top, s.p[e]);
  }
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

__global__ void __launch_bounds__(kLossThreads)
balance_loss_kernel(const float* __restrict__ logits, const int* __restrict__ expert, int64_t T, int E, float cb, float cz, float* __restrict__ loss,
                    int* __restrict__ counts, LossPart* __restrict__ parts, unsigned* __restrict__ done) {
  __shared__ LossPart warps[kLossThreads / 32];
  __shared__ int last;
  pdl_wait();
  pdl_trigger();
  LossPart a{};
  for (int64_t t = (int64_t)blockIdx.x * kLossThreads + threadIdx.x; t < T; t += (int64_t)gridDim.x * kLossThreads) {
    const int ex = __ldg(expert + t);
    if ((unsigned)ex >= (unsigned)E) continue;
    const Softmax s = softmax_of(logits + t * E, E);
    a.z = fma((double)s.lse, (double)s.lse, a.z);
#pragma unroll
    for (int e = 0; e < kMostExperts; ++e) {
      a.p[e] += s.p[e];
      a.n[e] += ex == e;
    }
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a.z += __shfl_xor_sync(0xFFFFFFFFu, a.z, o);
#pragma unroll
    for (int e = 0; e < kMostExperts; ++e) {
      a.p[e] += __shfl_xor_sync(0xFFFFFFFFu, a.p[e], o);
      a.n[e] += __shfl_xor_sync(0xFFFFFFFFu, a.n[e], o);
    }
  }
  if (lane == 0) warps[warp] = a;
  __syncthreads();
  // the warps' sums, in their order: a value to a lane
  if (warp == 0) {
    LossPart& out = parts[blockIdx.x];
    double z = 0;
    float p = 0.f;
    int n = 0;
#pragma unroll
    for (int w = 0; w < kLossThreads / 32; ++w) {
      if (lane == 16) z += warps[w].z;
      if (lane < 16) { p += warps[w].p[lane]; n += warps[w].n[lane]; }
    }
    if (lane == 16) out.z = z;
    if (lane < 16) { out.p[lane] = p; out.n[lane] = n; }
    __threadfence();
    __syncwarp();
    if (lane == 0) last = atomicInc(done, gridDim.x - 1) == gridDim.x - 1;      // (and back to 0 with the last one)
  }
  __syncthreads();
  if (!last) return;                   // (the whole CTA)
  __threadfence();
  // one expert to a lane, z in lane 16; every eighth part to a warp, then the warps' sums in their order
  __shared__ double sums[kLossThreads / 32][17];
  __shared__ int nums[kLossThreads / 32][16];
  double p = 0;
  int n = 0;
  if (lane < 17) {
#pragma unroll 4
    for (int i = warp; i < (int)gridDim.x; i += kLossThreads / 32) {
      p += lane < 16 ? (double)__ldcg(&parts[i].p[lane]) : __ldcg(&parts[i].z);
      if (lane < 16) n += __ldcg(&parts[i].n[lane]);
    }
    sums[warp][lane] = p;
    if (lane < 16) nums[warp][lane] = n;
  }
  __syncthreads();
  if (warp != 0) return;
  if (lane < 17)
    for (int w = 1; w < kLossThreads / 32; ++w) {
      p += sums[w][lane];
      if (lane < 16) n += nums[w][lane];
    }
  long long all = n;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, o, 16);
  all = __shfl_sync(0xFFFFFFFFu, all, 0);
  const double inv = all > 0 ? 1.0 / (double)all : 0.0;
  double b = lane < 16 ? ((double)n * inv) * (p * inv) * E : 0.0;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) b += __shfl_xor_sync(0xFFFFFFFFu, b, o, 16);
  const double z = __shfl_sync(0xFFFFFFFFu, p, 16) * inv;
  if (lane < E) counts[lane] = n;
  if (lane == 0) {
    loss[0] = (float)((double)cb * b + (double)cz * z);
    loss[1] = (float)b;
    loss[2] = (float)z;
  }
}

struct BalanceArgs {
  const float* logits;
  const int *expert, *counts;
  const float* dloss;
  const uint16_t* means;
  float* parts;                        // [gridDim.y][E][D]
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

// Into how many runs the tokens are cut: one CTA to an SM with the slabs, tiles of tokens at least.
constexpr int kGradCtas = 148;
int64_t balance_runs(int64_t T, int64_t D) {
  const int64_t slabs = (D + kSlab - 1) / kSlab, tiles = (T + kTile - 1) / kTile;
  int64_t runs = kGradCtas / slabs;
  if (runs < 1) runs = 1;
  return runs < tiles ? runs : tiles;
}

int balance_shape(int64_t T, int64_t D, int E) {
  return T < 0 || T > kMostTokens || D <= 0 || D % 8 || D > kMostCols || E < 1 || E > kMostExperts ? SF_ERR_SHAPE : SF_OK;
}

}  // namespace
}  // namespace sf

using namespace sf;

extern "C" {

int sf_router_balance_workspace_size(int64_t T, int64_t D, int E, size_t* bytes) {
  SF_TRY(balance_shape(T, D, E));
  if (!bytes) return SF_ERR_NULL;
  const size_t fwd = sizeof(LossPart) * kLossCtas, bwd = 4 * (size_t)balance_runs(T, D) * (size_t)E * (size_t)D;
  *bytes = kHead + (fwd > bwd ? fwd : bwd);
  return SF_OK;
}

int sf_router_balance_fwd(const void* logits, const void* expert, int64_t T, int E, float balance_coef, float z_coef, void* loss, void* counts,
                          void* workspace, size_t workspace_bytes, void* stream) {
  SF_TRY(balance_shape(T, 8, E));
  if (!loss || !counts || !workspace || (T > 0 && (!logits || !expert))) return SF_ERR_NULL;
  if (!aligned16(logits) || !aligned16(expert) || !aligned16(loss) || !aligned16(counts) || !aligned16(workspace)) return SF_ERR_ALIGN;
  const size_t need = kHead + sizeof(LossPart) * kLossCtas, t4 = 4 * (size_t)T;
  if (workspace_bytes < need) return SF_ERR_WORKSPACE;
  if (!apart({{loss, 12}, {counts, 4 * (size_t)E}, {workspace, need}}, {{logits, t4 * (size_t)E}, {expert, t4}})) return SF_ERR_UNSUPPORTED;
  SF_TRY(check_arch());
  const int64_t ctas = (T + kLossThreads - 1) / kLossThreads;
  return launch_pdl(balance_loss_kernel, dim3((unsigned)(ctas < 1 ? 1 : ctas < kLossCtas ? ctas : kLossCtas)), kLossThreads, 0, (cudaStream_t)stream,
                    (const float*)logits, (const int*)expert, T, E, balance_coef, z_coef, (float*)loss, (int*)counts,
                    (LossPart*)((uint8_t*)workspace + kHead), (unsigned*)((uint8_t*)workspace + kDone));
}

int sf_router_balance_bwd(const void* logits, const void* expert, const void* counts, const void* dloss, const void* X, const void* means, int64_t T,
                          int64_t D, int E, float balance_coef, float z_coef, const void* dX_in, void* dX, void* dmeans, void* workspace,
                          size_t workspace_bytes, void* stream) {
  size_t need;
  SF_TRY(sf_router_balance_workspace_size(T, D, E, &need));
  if (!aligned16(dX) || !aligned16(dmeans)) return SF_ERR_ALIGN;
  cudaStream_t s = (cudaStream_t)stream;
  const size_t ed = 2 * (size_t)E * (size_t)D;
  if (T == 0) {                                            // no token: an empty sum
    SF_TRY(check_arch());
    if (dmeans) SF_CUDA_TRY(cudaMemsetAsync(dmeans, 0, ed, s));
    return SF_OK;
  }
  if (!dX && !dmeans) return SF_OK;
  if (!logits || !expert || !counts || !X || !means || !workspace) return SF_ERR_NULL;
  if (!aligned16(logits) || !aligned16(expert) || !aligned16(counts) || (uintptr_t)dloss % 4 || !aligned16(X) || !aligned16(means) || !aligned16(dX_in) ||
      !aligned16(workspace))
    return SF_ERR_ALIGN;
  if (workspace_bytes < need) return SF_ERR_WORKSPACE;
  const size_t td = 2 * (size_t)T * (size_t)D, t4 = 4 * (size_t)T;
  const Span rest[] = {{logits, t4 * (size_t)E}, {expert, t4}, {counts, 4 * (size_t)E}, {dloss, 4}, {X, td}, {means, ed}};
  const Span work{workspace, need};
  // dX may take the place of dX_in
  if (!apart({{dX, td}, {dmeans, ed}, work}, {rest[0], rest[1], rest[2], rest[3], rest[4], rest[5], {dX && dX == dX_in ? nullptr : dX_in, td}}) ||
      !apart({{dmeans, ed}, work}, {{dX_in, td}}))
    return SF_ERR_UNSUPPORTED;
  SF_TRY(check_arch());
  BalanceArgs a{};
  a.logits = (const float*)logits; a.expert = (const int*)expert; a.counts = (const int*)counts; a.dloss = (const float*)dloss;
  a.means = (const uint16_t*)means;
  a.parts = dmeans ? (float*)((uint8_t*)workspace + kHead) : nullptr;
  a.status = (int*)workspace;
  a.adds = dX && dX_in; a.writes = dX != nullptr;
  a.T = T; a.D = (int)D; a.E = E; a.cb = balance_coef; a.cz = z_coef;
  int64_t runs = balance_runs(T, D);
  a.rows = ((T + runs - 1) / runs + kTile - 1) / kTile * kTile;
  runs = (T + a.rows - 1) / a.rows;
  BalanceMaps maps;
  SF_TRY(make_tmap_2d(&maps.x, X, T, D, D, 64, kTile, true));
  SF_TRY(make_tmap_2d(&maps.in, dX_in ? dX_in : X, T, D, D, 64, kTile, true));
  SF_TRY(make_tmap_2d(&maps.out, dX ? dX : X, T, D, D, 64, kTile, true));
  static std::atomic<bool> attr_done[64]{};
  int dev = 0;
  SF_CUDA_TRY(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64 || !attr_done[dev]) {
    SF_CUDA_TRY(cudaFuncSetAttribute(balance_grad_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kGradSmem));
    if (dev >= 0 && dev < 64) attr_done[dev] = true;
  }
  SF_TRY(launch_pdl(balance_grad_kernel, dim3((unsigned)((D + kSlab - 1) / kSlab), (unsigned)runs), 32 * kWarps, (size_t)kGradSmem, s, maps, a));
  if (!dmeans) return SF_OK;
  return launch_sum_parts(a.parts, (int)runs, (int64_t)E * D, dmeans, s);
}

}  // extern "C"
