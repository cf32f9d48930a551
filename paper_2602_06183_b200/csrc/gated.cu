// The gated feed-forward block (the three-matrix FFN that the paper's FLOP count of 18 B T D F stands for, Section 5.1):
//   forward   H = act(X Wg^T) * (X Wu^T),  Y = H Wd^T                                   two launches
//   backward  dH = dY Wd,  dU = dH P,  dG = dH Q   with P = act(G), Q = U act'(G)       one launch, dH stays in TMEM
//             dX = dG Wg + dU Wu                                                        one launch, one accumulation
//             dWd = dY^T H,  dWg = dG^T X,  dWu = dU^T X                                one launch, tiles of all three
//
// Roundings: G, U and dH stay in float32. H, dG and dU are rounded to bf16 once, because they are operands of the next product (with up to 16
// tokens they are sums of two bf16 numbers, see kTwoTerms); P and
// Q are kept in float32 (8 bytes a hidden value where bf16 would take 4), because dG and dU would otherwise be rounded two or three times: the
// error of dWu against 64 bits is then 1.8 times that of a result that is rounded once at its end, with them it is 1.4 times.
#include "products.cuh"

namespace sf {

int sm_count_now() {
  static std::atomic<int> n[64]{};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) { cudaGetLastError(); return 148; }
  if (n[dev] == 0) {
    int v = 0;
    if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || v <= 0) v = 148;
    n[dev] = v;
  }
  return n[dev];
}

namespace {

int encode_2d(void* map, CUtensorMapDataType type, int bytes, const void* base, int64_t rows, int64_t cols, int64_t ld, CUtensorMapSwizzle swizzle) {
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * bytes};
  const cuuint32_t box[2] = {32, 32};
  return encode_map(map, type, 2, base, dims, strides, box, swizzle);
}

}  // namespace

int make_tmap_f32(void* map, const void* base, int64_t rows, int64_t cols) {
  return encode_2d(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, base, rows, cols, cols, CU_TENSOR_MAP_SWIZZLE_128B);
}
int make_tmap_store(void* map, const void* base, int64_t rows, int64_t cols, int64_t ld) {
  return encode_2d(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, rows, cols, ld ? ld : cols, CU_TENSOR_MAP_SWIZZLE_64B);
}
int make_tmap_scales(void* map, const void* base, int64_t row_blocks, int64_t k_tiles, uint32_t box_tiles) {
  const cuuint64_t dims[3] = {128, (cuuint64_t)k_tiles, (cuuint64_t)row_blocks}, strides[2] = {512, 512 * (cuuint64_t)k_tiles};
  const cuuint32_t box[3] = {128, box_tiles, 1};
  return encode_map(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_NONE);
}

namespace {

constexpr size_t kStatus = 256;
size_t padded(size_t n) { return (n + 255) & ~(size_t)255; }

struct GatedSizes {
  size_t h, f;          // bytes of an operand in between (one or two bf16 [T, F]) and of a float32 [T, F]
};
int gated_sizes(const sf_gated_ffn_desc* d, GatedSizes* z) {
  if (!d) return SF_ERR_NULL;
  if (!act_ok(d->act)) return SF_ERR_UNSUPPORTED;
  if (d->T < 0 || d->D <= 0 || d->F <= 0 || d->D % 8 || d->F % 8 || d->T > kMaxSize || d->D > kMaxSize || d->F > kMaxSize) return SF_ERR_SHAPE;
  const size_t n = (size_t)d->T * (size_t)d->F;
  z->h = padded(2 * n * terms_of(d->T));
  z->f = padded(4 * n);
  return SF_OK;
}

struct GradJob { const void *A, *B; int64_t M, N; void* C; int a_terms, b_terms; };     // C[M, N] = A[T, M]^T B[T, N]

}  // namespace

}  // namespace sf

using namespace sf;

extern "C" {

int sf_gated_ffn_workspace_size(const sf_gated_ffn_desc* desc, size_t* fwd_ctx_bytes, size_t* workspace_bytes) {
  GatedSizes z;
  SF_TRY(gated_sizes(desc, &z));
  if (!fwd_ctx_bytes || !workspace_bytes) return SF_ERR_NULL;
  *fwd_ctx_bytes = z.h + 2 * z.f;
  *workspace_bytes = kStatus + 2 * z.h;
  return SF_OK;
}

int sf_gated_ffn_step_plan(const sf_gated_ffn_desc* desc, sf_gated_ffn_plan* plan) {
  GatedSizes z;
  SF_TRY(gated_sizes(desc, &z));
  if (!plan) return SF_ERR_NULL;
  *plan = sf_gated_ffn_plan{};
  if (desc->T == 0) return SF_OK;
  const int T = (int)desc->T, D = (int)desc->D, F = (int)desc->F;
  const int kd = k_blocks(FMT_BF16, D), kf = k_blocks(FMT_BF16, F), kt = (int)ceil_div(T, 64);
  auto few = [&](auto kind, int i, int N, int nkb, int terms) {
    FewArgs a{};
    a.T = T; a.N = N; a.nkb = nkb; a.in_terms = terms;
    PairPlan p;
    NoMaps none;
    SF_TRY((run_few<FMT_BF16, decltype(kind)::value>(a, nullptr, none, &p)));
    plan->form[i] = SF_GATED_FEW; plan->cols[i] = p.bn; plan->parts[i] = p.parts;
    return (int)SF_OK;
  };
  auto pairs = [&](int kind, int i, std::initializer_list<PairJob> jobs, int nkb) {
    PairArgs a{};
    for (const PairJob& j : jobs) { a.M[a.jobs] = (int)j.M; a.N[a.jobs++] = (int)j.N; }
    a.nkb = nkb;
    PairPlan p;
    SF_TRY(plan_pairs(kind, a, &p));
    plan->form[i] = p.mode == PM_SPLIT ? SF_GATED_SPLIT : SF_GATED_TILES; plan->cols[i] = p.bn; plan->parts[i] = p.parts;
    return (int)SF_OK;
  };
  if (gated_by_few(FMT_BF16, T, kd)) {
    SF_TRY(few(ActTag<FK_GATED>{}, SF_GATED_H, F, kd, 1));
    plan->form[SF_GATED_H_KEPT] = plan->form[SF_GATED_H]; plan->cols[SF_GATED_H_KEPT] = plan->cols[SF_GATED_H];
    plan->parts[SF_GATED_H_KEPT] = plan->parts[SF_GATED_H];
  } else {
    SF_TRY(pairs(PK_FWD, SF_GATED_H, {{T, F}}, kd));
    SF_TRY(pairs(PK_FWD_SAVE, SF_GATED_H_KEPT, {{T, F}}, kd));
  }
  if (T <= kFewTokens) {
    SF_TRY(few(ActTag<FK_NT>{}, SF_GATED_Y, D, kf, terms_of(T)));
    SF_TRY(few(ActTag<FK_BWD>{}, SF_GATED_DH, F, kd, 1));
    SF_TRY(few(ActTag<FK_DX>{}, SF_GATED_DX, D, 2 * kf, terms_of(T)));
  } else {
    SF_TRY(pairs(PK_NT, SF_GATED_Y, {{T, D}}, kf));
    SF_TRY(pairs(PK_BWD, SF_GATED_DH, {{T, F}}, kd));
    SF_TRY(pairs(PK_DX, SF_GATED_DX, {{T, D}}, 2 * kf));
  }
  return pairs(PK_DW, SF_GATED_DW, {{D, F}, {F, D}, {F, D}}, kt);
}

int sf_gated_ffn_fwd(const sf_gated_ffn_desc* desc, const void* X, const void* Wg, const void* Wu, const void* Wd, void* Y,
                     void* fwd_ctx, size_t fwd_ctx_bytes, void* workspace, size_t workspace_bytes, void* stream) {
  GatedSizes z;
  SF_TRY(gated_sizes(desc, &z));
  if (desc->T == 0) return SF_OK;
  if (!X || !Wg || !Wu || !Wd || !Y || !workspace) return SF_ERR_NULL;
  if (!aligned16(X) || !aligned16(Wg) || !aligned16(Wu) || !aligned16(Wd) || !aligned16(Y) || !aligned16(workspace) ||
      (fwd_ctx && !aligned16(fwd_ctx)))
    return SF_ERR_ALIGN;
  if ((fwd_ctx && fwd_ctx_bytes < z.h + 2 * z.f) || workspace_bytes < kStatus + (fwd_ctx ? 0 : z.h)) return SF_ERR_WORKSPACE;
  const size_t td = 2 * (size_t)desc->T * (size_t)desc->D, df = 2 * (size_t)desc->D * (size_t)desc->F;
  if (!apart({{Y, td}, {fwd_ctx, z.h + 2 * z.f}, {workspace, kStatus + (fwd_ctx ? 0 : z.h)}}, {{X, td}, {Wg, df}, {Wu, df}, {Wd, df}}))
    return SF_ERR_UNSUPPORTED;
  SF_TRY(check_arch());
  cudaStream_t s = (cudaStream_t)stream;
  uint8_t* h = fwd_ctx ? (uint8_t*)fwd_ctx : (uint8_t*)workspace + kStatus;
  float* p = fwd_ctx ? (float*)(h + z.h) : nullptr;
  float* q = fwd_ctx ? (float*)(h + z.h + z.f) : nullptr;
  int* status = (int*)workspace;
  trace_mark(s);
  SF_TRY(run_gated<FMT_BF16>({X, nullptr}, {Wg, nullptr}, {Wu, nullptr}, desc->T, desc->F, desc->D, desc->act, 1.f, 1.f, h, p, q, status, s,
                             terms_of(desc->T)));
  trace_mark(s);
  SF_TRY(run_nt<FMT_BF16>({h, nullptr}, {Wd, nullptr}, desc->T, desc->D, desc->F, 1.f, Y, status, s, true,
                          terms_of(desc->T)));
  trace_mark(s);
  return SF_OK;
}

int sf_gated_ffn_bwd(const sf_gated_ffn_desc* desc, const void* dY, const void* X, const void* Wg, const void* Wu, const void* Wd,
                     const void* fwd_ctx, size_t fwd_ctx_bytes, void* dX, void* dWg, void* dWu, void* dWd, void* workspace,
                     size_t workspace_bytes, void* stream) {
  GatedSizes z;
  SF_TRY(gated_sizes(desc, &z));
  const int64_t T = desc->T, D = desc->D, F = desc->F;
  cudaStream_t s = (cudaStream_t)stream;
  if (!aligned16(dX) || !aligned16(dWg) || !aligned16(dWu) || !aligned16(dWd)) return SF_ERR_ALIGN;
  if (T == 0) {                                            // no token: the weights' gradients are empty sums
    SF_TRY(check_arch());
    for (void* w : {dWg, dWu, dWd})
      if (w) SF_CUDA_TRY(cudaMemsetAsync(w, 0, 2 * (size_t)D * (size_t)F, s));
    return SF_OK;
  }
  if (!dX && !dWg && !dWu && !dWd) return SF_OK;
  if (!dY || !X || !Wg || !Wu || !Wd || !fwd_ctx || !workspace) return SF_ERR_NULL;
  if (!aligned16(dY) || !aligned16(X) || !aligned16(Wg) || !aligned16(Wu) || !aligned16(Wd) || !aligned16(fwd_ctx) || !aligned16(workspace))
    return SF_ERR_ALIGN;
  if (fwd_ctx_bytes < z.h + 2 * z.f || workspace_bytes < kStatus + 2 * z.h) return SF_ERR_WORKSPACE;
  const size_t td = 2 * (size_t)T * (size_t)D, df = 2 * (size_t)D * (size_t)F;
  if (!apart({{dX, td}, {dWg, df}, {dWu, df}, {dWd, df}, {workspace, kStatus + 2 * z.h}},
             {{dY, td}, {X, td}, {Wg, df}, {Wu, df}, {Wd, df}, {fwd_ctx, z.h + 2 * z.f}}))
    return SF_ERR_UNSUPPORTED;
  SF_TRY(check_arch());
  const uint8_t* h = (const uint8_t*)fwd_ctx;
  uint8_t* dg = (uint8_t*)workspace + kStatus;
  uint8_t* du = dg + z.h;
  PairArgs a{};
  a.status = (int*)workspace;
  a.jobs = 1;
  const bool few = T <= kFewTokens;
  const int terms = terms_of(T);
  FewArgs f{};
  f.T = (int)T; f.status = (int*)workspace;
  trace_mark(s);
  if (dX || dWg || dWu) {
    const int nkb = k_blocks(FMT_BF16, D);
    const float *p = (const float*)(h + z.h), *q = (const float*)(h + z.h + z.f);
    if (few) {
      f.N = (int)F; f.nkb = f.nkb0 = nkb; f.in_terms = 1; f.out_terms = terms; f.C = du; f.C2 = dg; f.P = const_cast<float*>(p); f.Q = const_cast<float*>(q);
      SF_TRY((run_few<FMT_BF16, FK_BWD>(f, s, [&](FewMaps& m, int n) {
        SF_TRY(kmajor_map(&m.x, FMT_BF16, dY, T, D, n));
        SF_TRY(mn_map(&m.w0, Wd, D, F));
        m.w1 = m.w0;
        m.sx = m.s0 = m.s1 = m.x;
        return (int)SF_OK;
      })));
    } else {
      a.M[0] = (int)T; a.N[0] = (int)F; a.nkb = a.nkb0 = nkb;
      SF_TRY(launch_best<PK_BWD>(a, s, [&](CUtensorMap* m, int) {
        SF_TRY(kmajor_map(&m[0], FMT_BF16, dY, T, D, 128));
        SF_TRY(mn_map(&m[1], Wd, D, F));
        SF_TRY(make_tmap_f32(&m[2], p, T, F));
        SF_TRY(make_tmap_f32(&m[3], q, T, F));
        SF_TRY(make_tmap_store(&m[4], dg, T, F));
        return make_tmap_store(&m[5], du, T, F);
      }));
    }
  }
  trace_mark(s);
  const bool beside = dX && (dWg || dWu || dWd) && !trace_on();      // the weights' gradients run beside dX
  PairPlan dx_plan;
  if (dX) {
    const int nkb = k_blocks(FMT_BF16, F);
    if (few) {
      f.N = (int)D; f.nkb0 = nkb; f.nkb = 2 * nkb; f.C = dX; f.early_weights = 1; f.early_next = beside;
      f.in_terms = terms; f.out_terms = 1;
      SF_TRY((run_few<FMT_BF16, FK_DX>(f, s, [&](FewMaps& m, int n) {
        SF_TRY(kmajor_map(&m.x, FMT_BF16, dg, T * terms, F, n));
        SF_TRY(kmajor_map(&m.sx, FMT_BF16, du, T * terms, F, n));
        SF_TRY(mn_map(&m.w0, Wg, F, D));
        SF_TRY(mn_map(&m.w1, Wu, F, D));
        m.s0 = m.s1 = m.x;
        return (int)SF_OK;
      }, &dx_plan)));
    } else {
      a.early_next = beside;
      a.M[0] = (int)T; a.N[0] = (int)D; a.nkb0 = nkb; a.nkb = 2 * nkb;
      SF_TRY(launch_best<PK_DX>(a, s, [&](CUtensorMap* m, int) {
        SF_TRY(kmajor_map(&m[0], FMT_BF16, dg, T, F, 128));
        SF_TRY(kmajor_map(&m[1], FMT_BF16, du, T, F, 128));
        SF_TRY(mn_map(&m[2], Wg, F, D));
        SF_TRY(mn_map(&m[3], Wu, F, D));
        return make_tmap_store(&m[4], dX, T, D);
      }, &dx_plan));
      a.early_next = 0;
    }
  }
  trace_mark(s);
  GradJob jobs[3];
  a.jobs = 0;
  if (dWd) jobs[a.jobs++] = {dY, h, D, F, dWd, 1, terms};
  if (dWg) jobs[a.jobs++] = {dg, X, F, D, dWg, terms, 1};
  if (dWu) jobs[a.jobs++] = {du, X, F, D, dWu, terms, 1};
  if (a.jobs == 0) {
    trace_mark(s);
    return SF_OK;
  }
  for (int j = 0; j < a.jobs; ++j) {
    a.M[j] = (int)jobs[j].M; a.N[j] = (int)jobs[j].N;
    a.sums_in_a |= (jobs[j].a_terms == 2) << j;
  }
  a.nkb = a.nkb0 = (int)ceil_div(T, 64);
  a.term_rows = terms == 2 ? (int)T : 0;
  SF_TRY(launch_best<PK_DW>(a, s, [&](CUtensorMap* m, int) {
    for (int j = 0; j < a.jobs; ++j) {
      SF_TRY(mn_map(&m[j], jobs[j].A, T * jobs[j].a_terms, jobs[j].M, terms == 2 ? 16 : 64));
      SF_TRY(mn_map(&m[3 + j], jobs[j].B, T * jobs[j].b_terms, jobs[j].N, terms == 2 ? 16 : 64));
      SF_TRY(make_tmap_store(&m[6 + j], jobs[j].C, jobs[j].M, jobs[j].N));
    }
    for (int j = a.jobs; j < 3; ++j)
      for (int i = 0; i < 9; i += 3) m[i + j] = m[i];
    return (int)SF_OK;
  }, nullptr, beside ? &dx_plan : nullptr));
  trace_mark(s);
  return SF_OK;
}

}  // extern "C"
