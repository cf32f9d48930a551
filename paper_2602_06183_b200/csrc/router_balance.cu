// The router's balance loss. With p = softmax(l) of a token's logits, n_e the tokens that went to expert e and n all that went to one:
//   balance = E sum_e (n_e / n) (sum_t p_te / n)          1 where the experts are used evenly, up to E
//   z       = sum_t lse_t^2 / n                           lse = log sum_e exp(l_te)
//   loss    = cb balance + cz z
//   dl_te   = dloss p_te (cb E / n^2 (n_e - sum_j n_j p_tj) + 2 cz lse_t / n)
//   dX      = dX_in + dl means,   dmeans = dl^T X          (l = X means^T)
// A token whose expert lies outside [0, E) (padding) is left out of all sums and has dl = 0. n_e is counted, not differentiated.
//
// Forward: 4 E + 4 bytes a token, one launch; the CTA that finishes last adds up what the others left (one token
// 2.6 us, 16384 of 16 experts 5.7, a million 27.9 in graph replay, here and below four calls to a graph). Backward: 6 bytes an element of X
// (X and dX_in in, dX out) and 4 T D E flops, one launch and one that adds up the CTAs' partial sums of dmeans (short batches: one).
//
// Memory bounds the backward pass only if the products stay out of its way: as float32 multiply-adds they took 417 us where the bytes take 62 (16384
// tokens, D 4096, E 16; now 72 alone, 5.6 TB/s, both calls 85). Sixteen experts are one side of a warp's m16n8k16 product, so both run there: dX = dl means with the means'
// fragments of a warp's 64 columns in 16 registers, dmeans = dl^T X with its sums in 32. dl is a sum of two bf16 numbers (16 bits), X and
// the means are bf16 as they come, sums are in float32.
#include "balance_grad.cuh"

#define SF_TRY(expr)              \
  do {                            \
    int _st = (expr);             \
    if (_st != SF_OK) return _st; \
  } while (0)

namespace sf {
namespace {

using namespace ptx;

constexpr int64_t kMostTokens = (int64_t)1 << 28, kMostCols = (int64_t)1 << 20;
constexpr int kLossCtas = 296, kLossThreads = 256, kLossWarps = kLossThreads / 32;
constexpr size_t kHead = 256, kDone = 128;                 // status word; the word that counts the CTAs that have finished

// What a CTA adds up. (z in double: a masked row's log-sum-exp may be the lowest float32, whose square is none)
struct LossPart { float p[kMostExperts]; int n[kMostExperts]; double z; };

// Sixteen sums over a warp's lanes in sixteen shuffles: half of them change hands at every step. The sum of value e is in lanes 2 e and 2 e + 1.
__device__ __forceinline__ float sixteen_sums(float (&v)[kMostExperts], int lane) {
#pragma unroll
  for (int h = 8; h > 0; h >>= 1) {
    const bool up = lane & 2 * h;
#pragma unroll
    for (int i = 0; i < h; ++i) {
      const float give = up ? v[i] : v[i + h], keep = up ? v[i + h] : v[i];
      v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, 2 * h);
    }
  }
  return v[0] + __shfl_xor_sync(0xFFFFFFFFu, v[0], 1);
}

// One launch: a CTA's sums go to memory, and the one that finishes last adds them up in their order. (A single CTA keeps them.)
__global__ void __launch_bounds__(kLossThreads)
balance_loss_kernel(const float* __restrict__ logits, const int* __restrict__ expert, int64_t T, int E, float cb, float cz, float* __restrict__ loss,
                    int* __restrict__ counts, LossPart* __restrict__ parts, unsigned* __restrict__ done) {
  __shared__ LossPart warps[kLossWarps];
  __shared__ double sums[kLossWarps][kMostExperts + 1];
  __shared__ int nums[kLossWarps][kMostExperts], last;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  pdl_trigger();
  float p[kMostExperts];
#pragma unroll
  for (int e = 0; e < kMostExperts; ++e) p[e] = 0.f;
  double z = 0;
  int n = 0;                           // of expert `lane`
  for (int64_t t0 = (int64_t)blockIdx.x * kLossThreads; t0 < T; t0 += (int64_t)gridDim.x * kLossThreads) {
    const int64_t t = t0 + threadIdx.x;
    const int ex = t < T ? __ldg(expert + t) : -1;
    const bool counts_here = (unsigned)ex < (unsigned)E;
#pragma unroll
    for (int e = 0; e < kMostExperts; ++e) {
      const unsigned all = __ballot_sync(0xFFFFFFFFu, counts_here && ex == e);
      if (lane == e) n += __popc(all);
    }
    if (!counts_here) continue;
    const Softmax s = softmax_of(logits + t * E, E);
    z = fma((double)s.lse, (double)s.lse, z);
#pragma unroll
    for (int e = 0; e < kMostExperts; ++e) p[e] += s.p[e];
  }
  const float mine = sixteen_sums(p, lane);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xFFFFFFFFu, z, o);
  if ((lane & 1) == 0) warps[warp].p[lane >> 1] = mine;
  if (lane < kMostExperts) warps[warp].n[lane] = n;
  if (lane == 0) warps[warp].z = z;
  __syncthreads();
  // the warps' sums, in their order: p and z a value to a lane (z in the sixteenth), n beside
  double a = 0;
  n = 0;
  if (warp == 0 && lane <= kMostExperts) {
    float f = 0.f;
#pragma unroll
    for (int w = 0; w < kLossWarps; ++w) {
      if (lane < kMostExperts) { f += warps[w].p[lane]; n += warps[w].n[lane]; }
      else a += warps[w].z;
    }
    if (lane < kMostExperts) a = f;
    if (gridDim.x > 1) {
      LossPart& out = parts[blockIdx.x];
      if (lane < kMostExperts) { out.p[lane] = f; out.n[lane] = n; }
      else out.z = a;
    }
  }
  if (gridDim.x > 1) {
    if (warp == 0) {
      __threadfence();
      __syncwarp();
      if (lane == 0) last = atomicInc(done, gridDim.x - 1) == gridDim.x - 1;      // (and back to 0 with the last one)
    }
    __syncthreads();
    if (!last) return;                 // (the whole CTA)
    __threadfence();
    // every eighth part to a warp, then the warps' sums in their order
    a = 0;
    n = 0;
    if (lane <= kMostExperts) {
#pragma unroll 8
      for (int i = warp; i < (int)gridDim.x; i += kLossWarps) {
        a += lane < kMostExperts ? (double)__ldcg(&parts[i].p[lane]) : __ldcg(&parts[i].z);
        if (lane < kMostExperts) n += __ldcg(&parts[i].n[lane]);
      }
      sums[warp][lane] = a;
      if (lane < kMostExperts) nums[warp][lane] = n;
    }
    __syncthreads();
    if (warp == 0 && lane <= kMostExperts) {
#pragma unroll
      for (int w = 1; w < kLossWarps; ++w) {
        a += sums[w][lane];
        if (lane < kMostExperts) n += nums[w][lane];
      }
    }
  }
  if (warp != 0) return;
  int all = lane < kMostExperts ? n : 0;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, o, 16);
  all = __shfl_sync(0xFFFFFFFFu, all, 0);
  const double inv = all > 0 ? 1.0 / (double)all : 0.0;
  double b = lane < kMostExperts ? ((double)n * inv) * (a * inv) * E : 0.0;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) b += __shfl_xor_sync(0xFFFFFFFFu, b, o, 16);
  const double zm = __shfl_sync(0xFFFFFFFFu, a, kMostExperts) * inv;
  if (lane < E) counts[lane] = n;
  if (lane == 0) {
    loss[0] = (float)((double)cb * b + (double)cz * zm);
    loss[1] = (float)b;
    loss[2] = (float)zm;
  }
}

// Into how many runs the tokens are cut: one CTA to an SM with the slabs, tiles of tokens at least.
constexpr int kGradCtas = 148;
int64_t balance_runs(int64_t T, int64_t D) {
  const int64_t slabs = (D + kSlab - 1) / kSlab, tiles = (T + kTile - 1) / kTile;
  int64_t runs = kGradCtas / slabs;
  if (runs < 1) runs = 1;
  return runs < tiles ? runs : tiles;
}

// Short batches, of a tile to a run: the runs of a slab are a cluster, which adds up its sums itself, and one launch is all. Two launches / one, us, from the
// host (in graph replay), E 5: 33 x 1408 11.5 / 9.6 (7.2 / 7.2), 256 x 4096 11.4 / 9.3 (7.7 / 7.7), 100 x 8192 11.5 / 9.5 (8.2 / 7.7). Two tiles to a run cost
// more than the launch: 400 x 4096 7.7 / 9.2 in graph replay; and so do clusters that do not all fit at once (256 x 8192, sixteen of eight CTAs: 8.7 / 14.4).
bool balance_joins(int64_t T, int64_t D) {
  const int64_t tiles = (T + kTile - 1) / kTile, slabs = (D + kSlab - 1) / kSlab;
  return tiles == 1 || (tiles <= 8 && tiles * slabs <= 64);
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
  a.status = (int*)workspace;
  a.adds = dX && dX_in; a.writes = dX != nullptr;
  a.T = T; a.D = (int)D; a.E = E; a.cb = balance_coef; a.cz = z_coef;
  const bool joins = dmeans && balance_joins(T, D);
  a.parts = dmeans && !joins ? (float*)((uint8_t*)workspace + kHead) : nullptr;
  a.dmeans = joins ? (uint16_t*)dmeans : nullptr;
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
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((D + kSlab - 1) / kSlab), (unsigned)runs);
  cfg.blockDim = dim3(32 * kWarps);
  cfg.dynamicSmemBytes = kGradSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = attr[1].val.clusterDim.z = 1;
  attr[1].val.clusterDim.y = joins ? (unsigned)runs : 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  SF_CUDA_TRY(cudaLaunchKernelEx(&cfg, balance_grad_kernel, maps, a));
  if (!dmeans || joins) return SF_OK;
  return launch_sum_parts(a.parts, (int)runs, (int64_t)E * D, dmeans, s);
}

}  // extern "C"
