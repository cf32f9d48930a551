// Root-mean-square norm of a residual stream, in front of the layer:
//   forward   S = bf16(X + R),  r = 1 / sqrt(mean_row(S^2) + eps),  y = S r gamma  ->  bf16, or E4M3 codes with a scale to every row
//   backward  n = S r,  q = dY gamma,  dX = dS + r (q - n mean_row(q n)),  dgamma = sum over rows of dY n
// The norm is that of the sum as it is stored, so that the backward pass, which has only the stored one, differentiates what was computed.
// Sums are in float32; S, y, dX and dgamma are rounded once each.
//
// Memory bounds them: 8 bytes an element forward (7 with codes) and 8 backward. A row stays in the registers of one group of threads from
// its load to its store; the only thing that crosses warps is a row's sum. In graph replay (here and below four calls to a graph): 16384 x 4096 forward
// 82 us (6.6 TB/s), backward 84 (6.4 TB/s) with the sum of dgamma's parts; 8192 x 4096 to E4M3 rows 40.4 (5.8 TB/s); one row of 4096 2.6, a launch. 4096 x
// 32768 backward 277 (3.9 TB/s): a row's vectors are too many for a second stage of the ring.
#include "fp8_fmt.cuh"
#include "gated.cuh"
#include "sums.cuh"

#define SF_TRY(expr)              \
  do {                            \
    int _st = (expr);             \
    if (_st != SF_OK) return _st; \
  } while (0)

namespace sf {
namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 28;
constexpr int64_t kMaxWidth = 32768;
constexpr size_t kHead = 256;           // of a workspace: the status word of other calls and what they count there, left alone
constexpr int kBwdCtas = 148;          // of the backward pass, at most: each leaves one row of partial sums of dgamma

// Past the L1: every element is read once. (Not the read-only path: the sum may be written where an input lies.)
__device__ __forceinline__ uint4 load_once(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// A row's group of threads: 8, 16 or 32 lanes of a warp, or several warps that meet at a barrier of their own (the group's number + 1). Every
// lane of a warp comes to a reduction, whether its row is there or not.
struct Group {
  int index, lane, size;
  float* slots;                        // 2 x 64 of shared memory, taken in turn: one barrier to a reduction
  int turn;
  // The group's sum of v and, with kMax, its largest m (a magnitude).
  template <bool kMax>
  __device__ __forceinline__ void reduce(float& v, float& m) {
    for (int o = size < 32 ? size >> 1 : 16; o > 0; o >>= 1) {
      v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
      if (kMax) m = max_nan(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    }
    if (size > 32) {
      float* at = slots + turn * 64;
      turn ^= 1;
      const int warps = size >> 5, l = lane & 31;
      if (l == 0) {
        at[lane >> 5] = v;
        if (kMax) at[32 + (lane >> 5)] = m;
      }
      asm volatile("bar.sync %0, %1;" ::"r"(index + 1), "r"(size) : "memory");
      v = l < warps ? at[l] : 0.f;
      if (kMax) m = l < warps ? at[32 + l] : 0.f;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
        if (kMax) m = max_nan(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
      }
    }
  }
};

// The nearest number of 22 bits (Veltkamp's splitting).
__device__ __forceinline__ float to_22_bits(float q) {
  const float c = __fmul_rn(q, 5.f);
  return __fsub_rn(c, __fsub_rn(c, q));
}

struct NormArgs {
  const uint16_t *X, *R, *gamma;
  int64_t ldx, T;
  uint16_t *sum, *Y;
  uint8_t* codes;
  float *scales, *rstd;
  float scale, eps;
  int D, tpr;                          // tpr: threads to a row
};

// Smallest magnitude that a row's scale is made for: a row of zeros has codes of 0 and a scale that is not 0.
constexpr float kLeastAmax = 1.2621774483536189e-29f;      // 2^-96
// A row's largest |S gamma|, down to which it is exact in float32, and so are those of 2^-10 of it, which have the last codes.
constexpr float kLeastProduct = 7.888609052210118e-31f;    // 2^-100

// A row's own scale takes its largest |y| to 448, and a code is that of 448 S gamma / max |S gamma|: r falls out. S gamma has 16 bits, 448 times it 19, so
// a quotient that is not half-way between two codes (five bits) is 2^-21 of it away at least. As S gamma times the rounded inverse it is off by 2^-23 of
// it; rounded to 22 bits, what is half-way is exactly that again, and goes to the even code. (7 in 100 000 of normal rows are. As y * (448 / top), rounded
// three times, the last bit decided. 8192 x 4096 back to back: 41.2 us so, 42.2 in 22 bits, 51.4 with a division.) top: the largest |S gamma|. Returns the inverse.
__device__ __forceinline__ float row_scale(float r, float top, float* to) {
  const float y_top = max_nan(top * r, kLeastAmax), scale = __fdiv_rn(y_top, 448.f);
  if (to) *to = scale;
  return y_top > kLeastAmax ? __fdiv_rn(448.f, top) : __fdiv_rn(r, scale);        // (or NaN)
}
__device__ __forceinline__ uint2 row_codes(const uint4& s, const uint4& w, float inv) {
  uint32_t b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    b[i] = e4m3x2(to_22_bits(lo32(word(s, i)) * lo32(word(w, i)) * inv), to_22_bits(hi32(word(s, i)) * hi32(word(w, i)) * inv));
  return make_uint2(b[0] | b[1] << 16, b[2] | b[3] << 16);
}
__device__ __forceinline__ uint4 sum_of(const uint4& s, const uint4& t) {
  return make_uint4(pack2(lo32(s.x) + lo32(t.x), hi32(s.x) + hi32(t.x)), pack2(lo32(s.y) + lo32(t.y), hi32(s.y) + hi32(t.y)),
                    pack2(lo32(s.z) + lo32(t.z), hi32(s.z) + hi32(t.z)), pack2(lo32(s.w) + lo32(t.w), hi32(s.w) + hi32(t.w)));
}
// The same once more for the rows of a warp, or of a group of several, of which one (far) has a |S gamma| that leaves float32's range or comes near its
// lower end: S is taken times a power of two near r. It is rare, so it reads S again, and is not inlined: 8192 x 4096 took 45.3 us back to back with S kept
// for it, 42.8 so, 42.2 with nothing of it.
__device__ __noinline__ void far_row(const NormArgs* a, Group g, int64_t row, int vecs, float r, bool far) {
  const uint4 *x = reinterpret_cast<const uint4*>(a->sum ? a->sum + row * a->D : a->X + row * a->ldx),
              *t = reinterpret_cast<const uint4*>(a->R + row * a->D), *gamma = reinterpret_cast<const uint4*>(a->gamma);
  const bool adds = !a->sum && a->R;
  const float p = far && r > 0.f && r < INFINITY ? __uint_as_float(__float_as_uint(r) & 0x7F800000u) : 1.f;
  auto scaled = [&](int c) {
    uint4 s = load_once(x + c);
    if (adds) s = sum_of(s, load_once(t + c));
    return make_uint4(pack2(lo32(s.x) * p, hi32(s.x) * p), pack2(lo32(s.y) * p, hi32(s.y) * p), pack2(lo32(s.z) * p, hi32(s.z) * p),
                      pack2(lo32(s.w) * p, hi32(s.w) * p));
  };
  float top = 0.f, none = 0.f;
  for (int c = g.lane; c < vecs; c += g.size) {
    const uint4 s = scaled(c), w = __ldg(gamma + c);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      top = max_nan(top, max_nan(fabsf(lo32(word(s, i)) * lo32(word(w, i))), fabsf(hi32(word(s, i)) * hi32(word(w, i)))));
  }
  g.reduce<true>(none, top);
  const float inv = row_scale(r / p, top, vecs && g.lane == 0 ? a->scales + row : nullptr);
  for (int c = g.lane; c < vecs; c += g.size) reinterpret_cast<uint2*>(a->codes + row * a->D)[c] = row_codes(scaled(c), __ldg(gamma + c), inv);
}

// kRows: codes with a scale to every row.
template <int V, bool kRows>
__global__ void __launch_bounds__(1024)
rmsnorm_kernel(const __grid_constant__ NormArgs a) {
  __shared__ float slots[4][128];       // (of groups of more than a warp)
  Group g;
  g.index = (int)threadIdx.x / a.tpr;
  g.lane = (int)threadIdx.x - g.index * a.tpr;
  g.size = a.tpr;
  g.slots = slots[a.tpr > 32 ? g.index : 0];
  g.turn = 0;
  const int64_t row = (int64_t)blockIdx.x * (blockDim.x / a.tpr) + g.index;
  const bool here = row < a.T;
  const int vecs = here ? a.D >> 3 : 0;                    // of this row
  const uint4* gamma = reinterpret_cast<const uint4*>(a.gamma);
  pdl_wait();
  pdl_trigger();
  uint4 s[V];
  {
    const uint4* x = reinterpret_cast<const uint4*>(a.X + row * a.ldx);
    const uint4* r = reinterpret_cast<const uint4*>(a.R + row * a.D);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = g.lane + j * a.tpr;
      s[j] = c < vecs ? load_once(x + c) : make_uint4(0u, 0u, 0u, 0u);
    }
    if (a.R) {
      uint4 t[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int c = g.lane + j * a.tpr;
        t[j] = c < vecs ? load_once(r + c) : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) s[j] = sum_of(s[j], t[j]);
    }
  }
  if (a.sum) {
    uint4* out = reinterpret_cast<uint4*>(a.sum + row * a.D);
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (g.lane + j * a.tpr < vecs) out[g.lane + j * a.tpr] = s[j];
  }
  // the largest |y| of a row is r times the largest |S gamma|: found beside the sum of squares, it costs no pass and no barrier of its own
  float ss = 0.f, top = 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    uint4 w = make_uint4(0u, 0u, 0u, 0u);
    if (kRows && g.lane + j * a.tpr < vecs) w = __ldg(gamma + g.lane + j * a.tpr);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float l = lo32(word(s[j], i)), h = hi32(word(s[j], i));
      ss = fmaf(l, l, ss);
      ss = fmaf(h, h, ss);
      if (kRows) top = max_nan(top, max_nan(fabsf(l * lo32(word(w, i))), fabsf(h * hi32(word(w, i)))));
    }
  }
  g.reduce<kRows>(ss, top);
  const float rstd = __frsqrt_rn(ss / (float)a.D + a.eps);
  if (a.rstd && here && g.lane == 0) a.rstd[row] = rstd;
  auto normed = [&](const uint4& v, const uint4& w, int i, float& l, float& h) {
    l = lo32(word(v, i)) * rstd * lo32(word(w, i));
    h = hi32(word(v, i)) * rstd * hi32(word(w, i));
  };
  if (a.Y) {
    uint4* y = reinterpret_cast<uint4*>(a.Y + row * a.D);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = g.lane + j * a.tpr;
      if (c >= vecs) continue;
      const uint4 w = __ldg(gamma + c);
      uint32_t o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float l, h;
        normed(s[j], w, i, l, h);
        o[i] = pack2(l, h);
      }
      y[c] = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
  uint2* q = reinterpret_cast<uint2*>(a.codes + row * a.D);
  if (kRows) {
    const float inv = row_scale(rstd, top, here && g.lane == 0 ? a.scales + row : nullptr);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = g.lane + j * a.tpr;
      if (c < vecs) q[c] = row_codes(s[j], __ldg(gamma + c), inv);
    }
    const bool far = here && !(top >= kLeastProduct && top < INFINITY);
    if (__any_sync(0xFFFFFFFFu, far)) far_row(&a, g, row, vecs, rstd, far);
  } else if (a.codes) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = g.lane + j * a.tpr;
      if (c >= vecs) continue;
      const uint4 w = __ldg(gamma + c);
      uint32_t b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float l, h;
        normed(s[j], w, i, l, h);
        b[i] = e4m3x2(__fmul_rn(l, a.scale), __fmul_rn(h, a.scale));
      }
      q[c] = make_uint2(b[0] | b[1] << 16, b[2] | b[3] << 16);
    }
  }
}

constexpr int kBwdSmem = 196608;       // of the ring, at most

struct NormBwdArgs {
  const uint16_t *dY, *S, *gamma, *dS;
  const float* rstd;
  int64_t T;
  uint16_t *dX, *dgamma;
  float* parts;                        // [gridDim.x, D]
  int D, tpr;
};

// Eight elements of dX: of dY, S, gamma and dS, with the row's r and its mean of q n.
__device__ __forceinline__ uint4 row_gradient(const uint4& d, const uint4& x, const uint4& w, const uint4& e, float r, float m) {
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t dw = word(d, i), xw = word(x, i), ww = word(w, i), ew = word(e, i);
    o[i] = pack2(fmaf(r, fmaf(-lo32(xw) * r, m, lo32(dw) * lo32(ww)), lo32(ew)), fmaf(r, fmaf(-hi32(xw) * r, m, hi32(dw) * hi32(ww)), hi32(ew)));
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

__device__ __forceinline__ void copy_async(uint32_t saddr, const uint4* p) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(saddr), "l"(p) : "memory");
}
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A group takes every so many rows; the vectors of the next kStages - 1 rows are on their way to shared memory while one is worked on. Each
// thread fetches what it will read itself, so nothing but a row's mean crosses threads. With the rows loaded into registers when their turn
// came (two groups of 256 threads to an SM) 16384 x 4096 took 112 us, DRAM waiting for the reductions.
template <int V, int kStages>
__global__ void __launch_bounds__(kStages == 1 ? 1024 : 512)
rmsnorm_bwd_kernel(const NormBwdArgs a) {
  __shared__ float slots[8][128];       // (of groups of more than a warp)
  extern __shared__ uint4 ring[];      // [stage][dY, S, dS][V][threads]; at the end the groups' sums
  const int groups = (int)blockDim.x / a.tpr;
  Group g;
  g.index = (int)threadIdx.x / a.tpr;
  g.lane = (int)threadIdx.x - g.index * a.tpr;
  g.size = a.tpr;
  g.slots = slots[a.tpr > 32 ? g.index : 0];
  g.turn = 0;
  const int vecs = a.D >> 3;
  const int64_t step = (int64_t)gridDim.x * groups, first = (int64_t)blockIdx.x * groups;
  const bool adds = a.dS && a.dX;
  pdl_wait();
  pdl_trigger();
  const uint32_t at = ptx::smem_u32(ring + threadIdx.x), piece = blockDim.x * 16u;
  auto fetch = [&](int64_t base, int stage) {
    const int64_t row = base + g.index;
    if (row < a.T) {
      const uint4 *dy = reinterpret_cast<const uint4*>(a.dY + row * a.D), *s = reinterpret_cast<const uint4*>(a.S + row * a.D),
                  *ds = reinterpret_cast<const uint4*>(a.dS + row * a.D);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int c = g.lane + j * a.tpr;
        if (c >= vecs) continue;
        const uint32_t to = at + (uint32_t)(stage * 3 * V + j) * piece;
        copy_async(to, dy + c);
        copy_async(to + V * piece, s + c);
        if (adds) copy_async(to + 2 * V * piece, ds + c);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) fetch(first + i * step, i);
  float dg[V][8];
  uint4 w[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int c = g.lane + j * a.tpr;
    w[j] = c < vecs ? __ldg(reinterpret_cast<const uint4*>(a.gamma) + c) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[j][i] = 0.f;
  }
  const float inv_d = 1.f / (float)a.D;
  int stage = 0;
  float r = first + g.index < a.T ? __ldg(a.rstd + first + g.index) : 0.f;
  for (int64_t base = first; base < a.T; base += step) {
    const int64_t row = base + g.index;
    const bool here = row < a.T;
    fetch(base + (kStages - 1) * step, stage == 0 ? kStages - 1 : stage - 1);
    const float r_next = row + step < a.T ? __ldg(a.rstd + row + step) : 0.f;
    copy_wait<kStages - 1>();
    const uint4* mine = ring + threadIdx.x + (size_t)stage * 3 * V * blockDim.x;
    float c1 = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (!here || g.lane + j * a.tpr >= vecs) continue;
      const uint4 d = mine[j * blockDim.x], x = mine[(V + j) * blockDim.x];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t dw = word(d, i), xw = word(x, i), ww = word(w[j], i);
        const float tl = lo32(dw) * (lo32(xw) * r), th = hi32(dw) * (hi32(xw) * r);
        dg[j][2 * i] += tl;
        dg[j][2 * i + 1] += th;
        c1 = fmaf(tl, lo32(ww), c1);
        c1 = fmaf(th, hi32(ww), c1);
      }
    }
    if (a.dX) {
      float none = 0.f;
      g.reduce<false>(c1, none);
      const float m = c1 * inv_d;
      uint4* out = reinterpret_cast<uint4*>(a.dX + row * a.D);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int c = g.lane + j * a.tpr;
        if (!here || c >= vecs) continue;
        const uint4 d = mine[j * blockDim.x], x = mine[(V + j) * blockDim.x],
                    e = adds ? mine[(2 * V + j) * blockDim.x] : make_uint4(0u, 0u, 0u, 0u);
        out[c] = row_gradient(d, x, w[j], e, r, m);
      }
    }
    r = r_next;
    if (++stage == kStages) stage = 0;
  }
  copy_wait<0>();                      // (what was fetched for rows that are not there: nothing, but the groups are counted)
  float* sums = reinterpret_cast<float*>(ring);            // [groups - 1][D]
  __syncthreads();                     // every thread has read what it fetched
  if (!a.dgamma) return;
  // the groups' sums, in their order
  if (g.index > 0)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = g.lane + j * a.tpr;
      float4* at = reinterpret_cast<float4*>(sums + (int64_t)(g.index - 1) * a.D + c * 8);
      if (c < vecs) {
        at[0] = make_float4(dg[j][0], dg[j][1], dg[j][2], dg[j][3]);
        at[1] = make_float4(dg[j][4], dg[j][5], dg[j][6], dg[j][7]);
      }
    }
  if (groups > 1) __syncthreads();
  if (g.index > 0) return;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int c = g.lane + j * a.tpr;
    if (c >= vecs) continue;
    for (int k = 0; k < groups - 1; ++k) {
      const float4* at = reinterpret_cast<const float4*>(sums + (int64_t)k * a.D + c * 8);
      const float4 p = at[0], q = at[1];
      dg[j][0] += p.x; dg[j][1] += p.y; dg[j][2] += p.z; dg[j][3] += p.w;
      dg[j][4] += q.x; dg[j][5] += q.y; dg[j][6] += q.z; dg[j][7] += q.w;
    }
    if (gridDim.x == 1) {              // one CTA had every row: its sums are the result
      reinterpret_cast<uint4*>(a.dgamma)[c] =
          make_uint4(pack2(dg[j][0], dg[j][1]), pack2(dg[j][2], dg[j][3]), pack2(dg[j][4], dg[j][5]), pack2(dg[j][6], dg[j][7]));
    } else {
      float4* at = reinterpret_cast<float4*>(a.parts + (int64_t)blockIdx.x * a.D + c * 8);
      at[0] = make_float4(dg[j][0], dg[j][1], dg[j][2], dg[j][3]);
      at[1] = make_float4(dg[j][4], dg[j][5], dg[j][6], dg[j][7]);
    }
  }
}

// Both gradients of a short batch in one launch. dgamma needs no sum along a row, only r, so the first CTAs take 32 columns of all rows each and the
// others the rows; dY and S are read twice, the second time from the L2. 8 x 4096: 2.6 us; 1999 x 1408: 6.7, 3.4 TB/s of what HBM would have to
// move. (Two CTAs of 512 threads to an SM: with the registers for one 2000 x 4096 took 17.5 us instead of 14.4.)
constexpr int kOnceCols = 32, kOnceRows = 2;
template <int V>
__global__ void __launch_bounds__(512, 2)
rmsnorm_bwd_once_kernel(const NormBwdArgs a, int col_ctas) {
  __shared__ float shared[8 * 128];    // columns: 32 of up to 16 warps; rows: as in the other kernels
  const int threads = (int)blockDim.x;
  pdl_wait();
  pdl_trigger();
  if ((int)blockIdx.x < col_ctas) {
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31, c = (int)blockIdx.x * (kOnceCols / 8) + (lane & 3);
    float dg[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[i] = 0.f;
    if (c < a.D >> 3) {
      const int64_t step = threads >> 2;
      for (int64_t t = threadIdx.x >> 2; t < a.T; t += kOnceRows * step) {
        uint4 d[kOnceRows], x[kOnceRows];
        float r[kOnceRows];
#pragma unroll
        for (int k = 0; k < kOnceRows; ++k) {
          const int64_t u = t + k * step;
          d[k] = x[k] = make_uint4(0u, 0u, 0u, 0u);
          r[k] = 0.f;
          if (u < a.T) {
            d[k] = __ldg(reinterpret_cast<const uint4*>(a.dY + u * a.D) + c);
            x[k] = __ldg(reinterpret_cast<const uint4*>(a.S + u * a.D) + c);
            r[k] = __ldg(a.rstd + u);
          }
        }
#pragma unroll
        for (int k = 0; k < kOnceRows; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            dg[2 * i] = fmaf(lo32(word(d[k], i)), lo32(word(x[k], i)) * r[k], dg[2 * i]);
            dg[2 * i + 1] = fmaf(hi32(word(d[k], i)), hi32(word(x[k], i)) * r[k], dg[2 * i + 1]);
          }
      }
    }
    // eight rows of a warp, then the warps in their order
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int o = 16; o >= 4; o >>= 1) dg[i] += __shfl_xor_sync(0xFFFFFFFFu, dg[i], o);
      if (lane < 4) shared[warp * kOnceCols + lane * 8 + i] = dg[i];
    }
    __syncthreads();
    const int col = (int)blockIdx.x * kOnceCols + (int)threadIdx.x;
    if (threadIdx.x >= kOnceCols || col >= a.D) return;
    float s = 0.f;
#pragma unroll 8
    for (int w = 0; w < threads >> 5; ++w) s += shared[w * kOnceCols + threadIdx.x];
    a.dgamma[col] = float_to_bf16_bits(s);
    return;
  }
  Group g;
  g.index = (int)threadIdx.x / a.tpr;
  g.lane = (int)threadIdx.x - g.index * a.tpr;
  g.size = a.tpr;
  g.slots = shared + (a.tpr > 32 ? g.index : 0) * 128;
  g.turn = 0;
  const int64_t row = (int64_t)((int)blockIdx.x - col_ctas) * (threads / a.tpr) + g.index;
  const bool here = row < a.T;
  const int vecs = here ? a.D >> 3 : 0;
  const uint4 *dy = reinterpret_cast<const uint4*>(a.dY + row * a.D), *s = reinterpret_cast<const uint4*>(a.S + row * a.D),
              *ds = reinterpret_cast<const uint4*>(a.dS + row * a.D), *gamma = reinterpret_cast<const uint4*>(a.gamma);
  const float r = here ? __ldg(a.rstd + row) : 0.f;
  uint4 d[V], x[V], e[V], w[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int c = g.lane + j * a.tpr;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    d[j] = c < vecs ? load_once(dy + c) : zero;            // (dX may take its place, or dS's)
    x[j] = c < vecs ? __ldg(s + c) : zero;
    w[j] = c < vecs ? __ldg(gamma + c) : zero;
    e[j] = c < vecs && a.dS ? load_once(ds + c) : zero;
  }
  float c1 = 0.f, none = 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      c1 = fmaf(lo32(word(d[j], i)) * (lo32(word(x[j], i)) * r), lo32(word(w[j], i)), c1);
      c1 = fmaf(hi32(word(d[j], i)) * (hi32(word(x[j], i)) * r), hi32(word(w[j], i)), c1);
    }
  g.reduce<false>(c1, none);
  const float m = c1 * (1.f / (float)a.D);
  uint4* out = reinterpret_cast<uint4*>(a.dX + row * a.D);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int c = g.lane + j * a.tpr;
    if (c < vecs) out[c] = row_gradient(d[j], x[j], w[j], e[j], r, m);
  }
}

// Vectors of a row to a thread, and threads to a row. Few rows: as many threads as there are vectors, for latency. Many: several vectors,
// whose loads are under way at once, and as many rows to an SM. Rows of less than a warp's 32 vectors share it.
struct RowPlan { int v, tpr; };
int whole_warps(int threads) { return (threads + 31) / 32 * 32; }
RowPlan fwd_plan(int64_t T, int64_t D) {
  const int vecs = (int)(D / 8);
  if (vecs <= 32) return RowPlan{1, vecs <= 8 ? 8 : vecs <= 16 ? 16 : 32};
  const int v = T <= sm_count_now() && vecs <= 1024 ? 1 : T <= sm_count_now() && vecs <= 2048 ? 2 : vecs <= 64 ? 2 : 4;
  return RowPlan{v, whole_warps((vecs + v - 1) / v)};
}
// Backward: up to 512 threads to a row, of one, two or four vectors each; a row of more than 16384 elements takes up to 1024. Four vectors make
// more rows of a CTA and fewer barriers a byte, two start and end sooner: 2 / 4 vectors, us: 16384 x 4096 91.4 / 84.3, 4096 x 8192 51.6 / 46.9, 8192 x 4096
// 49.3 / 47.1; 8192 x 2048 27.8 / 28.5.
RowPlan bwd_plan(int64_t T, int64_t D) {
  const int vecs = (int)(D / 8);
  if (vecs <= 32) return RowPlan{1, vecs <= 8 ? 8 : vecs <= 16 ? 16 : 32};
  const int v = vecs > 1024 || (vecs >= 512 && T >= 4096) ? 4 : 2;
  return RowPlan{v, whole_warps((vecs + v - 1) / v)};
}

// Up to where one launch does: as long as what its two kinds of CTAs read twice comes from the L2 the second time and a column's rows are not
// many. Two launches / one, us in graph replay: 8 x 4096 4.6 / 2.6, 300 x 8192 10.3 / 6.7, 1999 x 1408 9.2 / 6.7, 4096 x 1408 13.4 / 11.3, 2000 x 4096
// 15.4 / 14.4, 2000 x 64 4.6 / 4.6; 4096 x 4096 28.5 / 29.2, 2000 x 8192 30.0 / 30.0, 4096 x 512 7.7 / 9.8, 128 x 16384 10.8 / 10.8.
bool bwd_once(int64_t T, int64_t D) { return D <= 8192 && T * D <= (int64_t)1 << 23 && (T <= 2048 || T <= 3 * D); }
RowPlan once_plan(int64_t T, int64_t D) {
  const int vecs = (int)(D / 8);
  if (vecs <= 32) return RowPlan{1, vecs <= 8 ? 8 : vecs <= 16 ? 16 : 32};
  const int v = vecs <= 64 || (T <= sm_count_now() && vecs <= 512) ? 1 : 2;
  return RowPlan{v, whole_warps((vecs + v - 1) / v)};
}

int bwd_ctas(int64_t T) { return (int)(T < kBwdCtas ? T : kBwdCtas); }

int norm_shape(int64_t T, int64_t D) { return T < 0 || T > kMaxRows || D <= 0 || D % 8 || D > kMaxWidth ? SF_ERR_SHAPE : SF_OK; }

}  // namespace
}  // namespace sf

using namespace sf;

extern "C" {

int sf_rmsnorm_fwd(const void* X, int64_t ldx, const void* residual, const void* gamma, int64_t T, int64_t D, float eps, void* sum, void* Y,
                   void* codes, void* scales, float scale, void* rstd, void* stream) {
  SF_TRY(norm_shape(T, D));
  if (!(eps >= 0.f)) return SF_ERR_UNSUPPORTED;
  if (T == 0) return SF_OK;
  if (!X || !gamma || (!Y && !codes) || (scales && !codes)) return SF_ERR_NULL;
  if (ldx < D || ldx % 8 || !aligned16(X) || !aligned16(residual) || !aligned16(gamma) || !aligned16(sum) || !aligned16(Y) || !aligned16(codes) ||
      !aligned16(scales) || !aligned16(rstd))
    return SF_ERR_ALIGN;
  const size_t td = 2 * (size_t)T * (size_t)D, t4 = 4 * (size_t)T;
  const Span x{X, 2 * ((size_t)(T - 1) * (size_t)ldx + (size_t)D)}, r{residual, td};
  // the sum may take the place of one of the two that it is made of, and of nothing else
  const bool in_x = sum && sum == X && ldx == D, in_r = sum && sum == residual;
  if (!apart({{sum, td}, {Y, td}, {codes, td / 2}, {scales, t4}, {rstd, t4}},
             {in_x ? Span{nullptr, 0} : x, in_r ? Span{nullptr, 0} : r, {gamma, 2 * (size_t)D}}) ||
      ((in_x || in_r) && !apart({{Y, td}, {codes, td / 2}, {scales, t4}, {rstd, t4}}, {x, r})))
    return SF_ERR_UNSUPPORTED;
  SF_TRY(check_arch());
  const RowPlan p = fwd_plan(T, D);
  // CTAs of 256 threads: with 128 the rate at which CTAs start was in the way (8192 x 4096 46.3 us instead of 42.6, to E4M3 46.1 instead of 39.5)
  const int groups = p.tpr >= 256 ? 1 : 256 / p.tpr;
  NormArgs a{};
  a.X = (const uint16_t*)X; a.R = (const uint16_t*)residual; a.gamma = (const uint16_t*)gamma; a.ldx = ldx; a.T = T;
  a.sum = (uint16_t*)sum; a.Y = (uint16_t*)Y; a.codes = (uint8_t*)codes; a.scales = (float*)scales; a.rstd = (float*)rstd;
  a.scale = scale; a.eps = eps; a.D = (int)D; a.tpr = p.tpr;
  auto kern = scales ? (p.v == 1 ? rmsnorm_kernel<1, true> : p.v == 2 ? rmsnorm_kernel<2, true> : rmsnorm_kernel<4, true>)
                     : (p.v == 1 ? rmsnorm_kernel<1, false> : p.v == 2 ? rmsnorm_kernel<2, false> : rmsnorm_kernel<4, false>);
  return launch_pdl(kern, dim3((unsigned)((T + groups - 1) / groups)), (unsigned)(groups * p.tpr), 0, (cudaStream_t)stream, a);
}

int sf_rmsnorm_bwd_workspace_size(int64_t T, int64_t D, size_t* bytes) {
  SF_TRY(norm_shape(T, D));
  if (!bytes) return SF_ERR_NULL;
  *bytes = kHead + 4 * (size_t)bwd_ctas(T) * (size_t)D;
  return SF_OK;
}

int sf_rmsnorm_bwd(const void* dY, const void* sum, const void* gamma, const void* rstd, const void* dS, int64_t T, int64_t D, void* dX,
                   void* dgamma, void* workspace, size_t workspace_bytes, void* stream) {
  size_t need;
  SF_TRY(sf_rmsnorm_bwd_workspace_size(T, D, &need));
  if (!aligned16(dX) || !aligned16(dgamma)) return SF_ERR_ALIGN;
  cudaStream_t s = (cudaStream_t)stream;
  if (T == 0) {                                            // no row: an empty sum
    SF_TRY(check_arch());
    if (dgamma) SF_CUDA_TRY(cudaMemsetAsync(dgamma, 0, 2 * (size_t)D, s));
    return SF_OK;
  }
  if (!dX && !dgamma) return SF_OK;
  if (!dY || !sum || !gamma || !rstd || (dgamma && !workspace)) return SF_ERR_NULL;
  if (!aligned16(dY) || !aligned16(sum) || !aligned16(gamma) || !aligned16(rstd) || !aligned16(dS) || !aligned16(workspace)) return SF_ERR_ALIGN;
  if (dgamma && workspace_bytes < need) return SF_ERR_WORKSPACE;
  const size_t td = 2 * (size_t)T * (size_t)D, d2 = 2 * (size_t)D;
  const Span parts{dgamma ? workspace : nullptr, need};
  // dX may take the place of dY or of dS
  if (!apart({{dX, td}, {dgamma, d2}, parts}, {{dX && dX == dY ? nullptr : dY, td}, {sum, td}, {gamma, d2}, {rstd, 4 * (size_t)T}, {dX && dX == dS ? nullptr : dS, td}}) ||
      !apart({{dgamma, d2}, parts}, {{dY, td}, {dS, td}}))
    return SF_ERR_UNSUPPORTED;
  SF_TRY(check_arch());
  NormBwdArgs a{};
  a.dY = (const uint16_t*)dY; a.S = (const uint16_t*)sum; a.gamma = (const uint16_t*)gamma; a.dS = (const uint16_t*)dS; a.rstd = (const float*)rstd;
  a.T = T; a.dX = (uint16_t*)dX; a.dgamma = (uint16_t*)dgamma; a.D = (int)D;
  a.parts = dgamma ? (float*)((uint8_t*)workspace + kHead) : nullptr;
  if (bwd_once(T, D)) {
    const RowPlan p = once_plan(T, D);
    const int most = T > kBwdCtas ? 512 : 256, groups = p.tpr >= most ? 1 : most / p.tpr;
    const int64_t cols = dgamma ? (D + kOnceCols - 1) / kOnceCols : 0, rows = dX ? (T + groups - 1) / groups : 0;      // CTAs
    a.tpr = p.tpr;
    auto launch = [&](int64_t c, int64_t r) {
      return launch_pdl(p.v == 1 ? rmsnorm_bwd_once_kernel<1> : rmsnorm_bwd_once_kernel<2>, dim3((unsigned)(c + r)), (unsigned)(groups * p.tpr), 0, s, a, (int)c);
    };
    if (dX != dY || !cols) return launch(cols, rows);
    SF_TRY(launch(cols, 0));                               // the columns' sums first: dX takes dY's place
    return launch(0, rows);
  }
  const RowPlan p = bwd_plan(T, D);
  const int ctas = bwd_ctas(T);
  const int64_t rows = (T + ctas - 1) / ctas;              // of a CTA
  int groups = p.tpr > 512 ? 1 : 512 / p.tpr;
  if (groups > rows) groups = (int)rows;
  while (groups * p.tpr % 32) ++groups;                    // whole warps
  a.tpr = p.tpr;
  const int threads = groups * p.tpr, stages = p.v == 1 ? 4 : p.v == 2 ? 3 : threads > 512 ? 1 : 2;
  const size_t smem = (size_t)stages * 3 * p.v * threads * 16;
  auto kern = p.v == 1 ? rmsnorm_bwd_kernel<1, 4> : p.v == 2 ? rmsnorm_bwd_kernel<2, 3> : stages == 2 ? rmsnorm_bwd_kernel<4, 2> : rmsnorm_bwd_kernel<4, 1>;
  static std::atomic<bool> attr_done[64]{};
  int dev = 0;
  SF_CUDA_TRY(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64 || !attr_done[dev]) {
    for (auto k : {rmsnorm_bwd_kernel<1, 4>, rmsnorm_bwd_kernel<2, 3>, rmsnorm_bwd_kernel<4, 2>, rmsnorm_bwd_kernel<4, 1>})
      SF_CUDA_TRY(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kBwdSmem));
    if (dev >= 0 && dev < 64) attr_done[dev] = true;
  }
  SF_TRY(launch_pdl(kern, dim3((unsigned)ctas), (unsigned)threads, smem, s, a));
  if (!dgamma || ctas == 1) return SF_OK;
  return launch_sum_parts(a.parts, ctas, D, dgamma, s);
}

}  // extern "C"
