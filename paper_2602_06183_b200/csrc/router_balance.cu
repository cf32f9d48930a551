// The router's balance loss. With p = softmax(l) of a token's logits, n_e the tokens that went to expert e and n all that went to one:
//   balance = E sum_e (n_e / n) (sum_t p_te / n)          1 where the experts are used evenly, up to E
//   z       = sum_t lse_t^2 / n                           lse = log sum_e exp(l_te)
//   loss    = cb balance + cz z
//   dl_te   = dloss p_te (cb E / n^2 (n_e - sum_j n_j p_tj) + 2 cz lse_t / n)
//   dX      = dX_in + dl means,   dmeans = dl^T X          (l = X means^T)
// A token whose expert lies outside [0, E) (padding) is left out of all sums and has dl = 0. n_e is counted, not differentiated.
//
// Forward: 4 E + 4 bytes a token, one launch; the CTA that finishes last adds up what the others left. Backward: 6 bytes an element of X
// (X and dX_in in, dX out) and 4 T D E flops; a CTA recomputes dl of its tokens from the logits, each thread holds four columns of the
// means and of their gradient in registers, and the CTAs' partial sums are added up by a second launch.
#include "gated.cuh"
#include "sums.cuh"

#define SF_TRY(expr)              \
  do {                            \
    int _st = (expr);             \
    if (_st != SF_OK) return _st; \
  } while (0)

namespace sf {
namespace {

constexpr int kMostExperts = 16;
constexpr int64_t kMostTokens = (int64_t)1 << 28, kMostCols = (int64_t)1 << 20;
constexpr int kLossCtas = 148, kLossThreads = 256;
constexpr size_t kHead = 256;                              // the first word counts the CTAs that have finished

struct LossPart { float p[kMostExperts]; float z; int n[kMostExperts]; };

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
    a.z = fmaf(s.lse, s.lse, a.z);
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
  if (threadIdx.x == 0) {
    for (int w = 1; w < kLossThreads / 32; ++w) {
      a.z += warps[w].z;
#pragma unroll
      for (int e = 0; e < kMostExperts; ++e) { a.p[e] += warps[w].p[e]; a.n[e] += warps[w].n[e]; }
    }
    parts[blockIdx.x] = a;
    __threadfence();
    last = atomicInc(done, gridDim.x - 1) == gridDim.x - 1;      // (and back to 0 with the last one)
  }
  __syncthreads();
  if (!last || warp != 0) return;
  __threadfence();
  // one expert to a lane, the parts in their order; z in lane 16
  double p = 0;
  long long n = 0;
  if (lane < 17)
    for (int i = 0; i < (int)gridDim.x; ++i) {
      p += lane < 16 ? __ldcg(&parts[i].p[lane]) : __ldcg(&parts[i].z);
      if (lane < 16) n += __ldcg(&parts[i].n[lane]);
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
  if (lane < E) counts[lane] = (int)n;
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
  const uint16_t *X, *means, *dX_in;
  uint16_t* dX;
  float* parts;                        // [gridDim.y][E][D]
  int64_t T, rows;                     // rows: tokens of a CTA
  int D, E;
  float cb, cz;
};
constexpr int kTile = 64;              // tokens whose dl a CTA holds at a time
constexpr int kSlab = 512;             // columns of a CTA, four to a thread

template <int kE>
__global__ void __launch_bounds__(kSlab / 4)
balance_grad_kernel(const BalanceArgs a) {
  __shared__ float dl[kTile][kE];
  const int col = (int)blockIdx.x * kSlab + (int)threadIdx.x * 4;
  const bool in = col < a.D;           // (D is a multiple of 8)
  pdl_wait();
  pdl_trigger();
  float m[kE][4], dm[kE][4], count[kE];
  long long all = 0;
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    const uint2 w = in && e < a.E ? __ldg(reinterpret_cast<const uint2*>(a.means + (int64_t)e * a.D + col)) : make_uint2(0u, 0u);
    m[e][0] = lo32(w.x); m[e][1] = hi32(w.x); m[e][2] = lo32(w.y); m[e][3] = hi32(w.y);
    dm[e][0] = dm[e][1] = dm[e][2] = dm[e][3] = 0.f;
    const int n = e < a.E ? __ldg(a.counts + e) : 0;
    count[e] = (float)n;
    all += n;
  }
  const float inv = all > 0 ? 1.f / (float)all : 0.f, g = a.dloss ? __ldg(a.dloss) : 1.f;
  const float k1 = g * a.cb * (float)a.E * inv * inv, k2 = g * 2.f * a.cz * inv;
  const int64_t t0 = (int64_t)blockIdx.y * a.rows, t1 = t0 + a.rows < a.T ? t0 + a.rows : a.T;
  for (int64_t t = t0; t < t1; t += kTile) {
    const int n = (int)(t1 - t < kTile ? t1 - t : kTile);
    __syncthreads();
    if ((int)threadIdx.x < n) {
      const int64_t at = t + threadIdx.x;
      const bool counts = (unsigned)__ldg(a.expert + at) < (unsigned)a.E;
      const Softmax s = softmax_of(a.logits + at * a.E, a.E);
      float mean = 0.f;
#pragma unroll
      for (int e = 0; e < kE; ++e) mean = fmaf(count[e], s.p[e], mean);
#pragma unroll
      for (int e = 0; e < kE; ++e) dl[threadIdx.x][e] = counts ? s.p[e] * fmaf(k1, count[e] - mean, k2 * s.lse) : 0.f;
    }
    __syncthreads();
    if (!in) continue;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const int64_t at = (t + i) * a.D + col;
      const uint2 xw = __ldg(reinterpret_cast<const uint2*>(a.X + at));
      const uint2 dw = a.dX_in ? *reinterpret_cast<const uint2*>(a.dX_in + at) : make_uint2(0u, 0u);
      const float x[4] = {lo32(xw.x), hi32(xw.x), lo32(xw.y), hi32(xw.y)};
      float d[4] = {lo32(dw.x), hi32(dw.x), lo32(dw.y), hi32(dw.y)};
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const float l = dl[i][e];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          d[k] = fmaf(l, m[e][k], d[k]);
          dm[e][k] = fmaf(l, x[k], dm[e][k]);
        }
      }
      if (a.dX) *reinterpret_cast<uint2*>(a.dX + at) = make_uint2(pack2(d[0], d[1]), pack2(d[2], d[3]));
    }
  }
  if (!a.parts || !in) return;
#pragma unroll
  for (int e = 0; e < kE; ++e)
    if (e < a.E) *reinterpret_cast<float4*>(a.parts + ((int64_t)blockIdx.y * a.E + e) * a.D + col) = make_float4(dm[e][0], dm[e][1], dm[e][2], dm[e][3]);
}

// Into how many runs the tokens are cut: about three CTAs to an SM with the slabs, of a tile of tokens at least.
constexpr int kGradCtas = 444;
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
                    (LossPart*)((uint8_t*)workspace + kHead), (unsigned*)workspace);
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
  if (!logits || !expert || !counts || !X || !means || (dmeans && !workspace)) return SF_ERR_NULL;
  if (!aligned16(logits) || !aligned16(expert) || !aligned16(counts) || (uintptr_t)dloss % 4 || !aligned16(X) || !aligned16(means) || !aligned16(dX_in) ||
      !aligned16(workspace))
    return SF_ERR_ALIGN;
  if (dmeans && workspace_bytes < need) return SF_ERR_WORKSPACE;
  const size_t td = 2 * (size_t)T * (size_t)D, t4 = 4 * (size_t)T;
  const Span rest[] = {{logits, t4 * (size_t)E}, {expert, t4}, {counts, 4 * (size_t)E}, {dloss, 4}, {X, td}, {means, ed}};
  const Span work{dmeans ? workspace : nullptr, need};
  // dX may take the place of dX_in
  if (!apart({{dX, td}, {dmeans, ed}, work}, {rest[0], rest[1], rest[2], rest[3], rest[4], rest[5], {dX && dX == dX_in ? nullptr : dX_in, td}}) ||
      !apart({{dmeans, ed}, work}, {{dX_in, td}}))
    return SF_ERR_UNSUPPORTED;
  SF_TRY(check_arch());
  BalanceArgs a{};
  a.logits = (const float*)logits; a.expert = (const int*)expert; a.counts = (const int*)counts; a.dloss = (const float*)dloss;
  a.X = (const uint16_t*)X; a.means = (const uint16_t*)means; a.dX_in = (const uint16_t*)dX_in; a.dX = (uint16_t*)dX;
  a.parts = dmeans ? (float*)((uint8_t*)workspace + kHead) : nullptr;
  a.T = T; a.D = (int)D; a.E = E; a.cb = balance_coef; a.cz = z_coef;
  int64_t runs = balance_runs(T, D);
  a.rows = ((T + runs - 1) / runs + kTile - 1) / kTile * kTile;
  runs = (T + a.rows - 1) / a.rows;
  auto kern = E <= 4 ? balance_grad_kernel<4> : E <= 8 ? balance_grad_kernel<8> : balance_grad_kernel<16>;
  SF_TRY(launch_pdl(kern, dim3((unsigned)((D + kSlab - 1) / kSlab), (unsigned)runs), kSlab / 4, 0, s, a));
  if (!dmeans) return SF_OK;
  return launch_sum_parts(a.parts, (int)runs, (int64_t)E * D, dmeans, s);
}

}  // extern "C"
