// Host side of the products of the gated block and of 4-bit operands: tensor maps, choice of kernel and tile, launches.
#pragma once

#include <cmath>
#include <type_traits>

#include "few_tokens.cuh"
#include "pair_product.cuh"

#define SF_TRY(expr)              \
  do {                            \
    int _st = (expr);             \
    if (_st != SF_OK) return _st; \
  } while (0)

namespace sf {
namespace {

// Up to this many tokens the weights are streamed past them (few_tokens.cuh), which is the better side where the weights are large.
// Few tokens against pairs, us: forward of 77 x 1408 x 5504 20 / 28, of 128 x 2048 x 2048 17.8 / 21.3, 100 x 8192 x 1024 of 4 bits
// 7.3 / 11.7; the other way at the upper end (step of 128 x 2048 x 8192 128 / 116).
constexpr int64_t kFewTokens = 128;

// Two projections are an exception beyond 64 tokens where the reduction is short: there is little of it to split, and the sums of twice the
// columns through shared memory are most of the time. Forward of the block, both projections by few tokens / on pairs, us back to back:
// 123 x 360 x 264 19.1 / 11.9, 100 x 512 x 512 14.4 / 11.2, 128 x 1024 x 1024 16.0 / 13.2; but 128 x 2048 x 2048 18.1 / 20.0. The projections of
// 4 bits alone, 128 x 512 x 512 7.9 / 6.1, 128 x 4096 x 2048 10.5 / 9.1; but 70 x 2048 x 4096 8.3 / 10.8, 96 x 1024 x 8192 11.5 / 15.5.
inline bool gated_by_few(int fmt, int64_t T, int nkb) { return T <= 64 || (T <= kFewTokens && nkb > (fmt == FMT_BF16 ? 16 : 8)); }

// Up to this many tokens the operands in between (H, dG, dU) are held as sums of two bf16 numbers, which the few-token products take as
// twice the tokens: there is room for them in the instruction's columns, and the products wait for the weights. With so few tokens
// a result rests on a handful of large hidden values, and rounding those once showed: the error of Y against 64 bits was 1.3 to 1.6 times
// that of a result that is rounded at its end only (1 x 1480 x 600), now it is the same.
constexpr int64_t kTwoTerms = 16;
inline int terms_of(int64_t T) { return T <= kTwoTerms ? 2 : 1; }

constexpr int64_t kMaxSize = (int64_t)1 << 28;      // of a dimension: coordinates and counts stay within 32 bits

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// K in 2-byte units of a row, and k-blocks (64 units each)
inline int64_t row_units(int fmt, int64_t K) { return fmt == FMT_BF16 ? K : K / 4; }
inline int k_blocks(int fmt, int64_t K) { return (int)ceil_div(row_units(fmt, K), 64); }
// scale tiles along K of a 4-bit operand
inline int64_t scale_tiles(int fmt, int64_t K) { return ceil_div(K, fmt == FMT_NV ? 64 : 128); }

inline int kmajor_map(void* m, int fmt, const void* p, int64_t rows, int64_t K, uint32_t box_rows) {
  return make_tmap_2d(m, p, rows, row_units(fmt, K), row_units(fmt, K), 64, box_rows, true);
}
inline int mn_map(void* m, const void* p, int64_t K, int64_t cols, uint32_t box_rows = 64) {
  return make_tmap_2d(m, p, K, cols, cols, 64, box_rows, true);
}
inline int scale_map(void* m, int fmt, const void* p, int64_t rows, int64_t K) {
  return make_tmap_scales(m, p, ceil_div(rows, 128), scale_tiles(fmt, K), fmt == FMT_NV ? 4 : 2);
}

inline int64_t tiles_of(int64_t M, int64_t N, int64_t cols) { return ceil_div(M, 256) * ceil_div(N, cols); }

// How a product on CTA pairs is cut, by its estimated clocks. Persistent tiles: rounds of nkb stages. Split: rounds of clusters, each with
// its part of the stages, and with the sums through distributed shared memory and an epilogue that nothing runs beside.
//   A stage of bn columns takes the tensor pipe 2 bn clocks, and shared memory the bytes that are written and read, 128 a clock
//   (A 16 KB; B 64 bytes a column, MN-major B written in chunks of 64 columns).
// Beside them: what a tile's epilogue takes on eight warps, which counts where it is longer than the main loop and after the last tile. Its
// part that does not depend on the width: three gradients of 2528 x 14128 from 4 tokens took 100 us in tiles of 64 columns, 78 of 128, 72 of
// 192 and 68 of 256, that is 1900, 2970, 4070 and 4980 clocks a tile.
struct PairPlan { int mode, bn, parts; int64_t pairs; double clocks, per_tile; };      // pairs that it holds; estimates
struct PairJob { int64_t M, N; };
inline PairPlan pair_plan(int kind, const PairJob* jobs, int njobs, int64_t nkb, const FewRoom& room) {
  const bool gated = kind == PK_FWD || kind == PK_FWD_SAVE, bmn = kind == PK_DX || kind == PK_DW || kind == PK_BWD;
  const double chunk = kind == PK_FWD ? 1200 : kind == PK_FWD_SAVE ? 2400 : kind == PK_BWD ? 2200 : 1000;   // 32 output columns of a warp
  PairPlan best{PM_FULL, 256, 1, 0, 0, 0};
  double least = 0;
  const int64_t pairs = sm_count_now() / 2;
  for (int bn = 256; bn >= 64; bn -= gated ? 64 : 32) {
    const int cols = gated ? bn / 2 : bn;
    int64_t tiles = 0;
    for (int j = 0; j < njobs; ++j) tiles += tiles_of(jobs[j].M, jobs[j].N, cols);
    const double smem = bmn ? 256 + 64 * ceil_div(bn, 128) + bn / 2 : 256 + bn, stage = smem > 2 * bn ? smem : 2 * bn;
    const double epilogue = 900 + chunk * (double)ceil_div(cols, 64);
    for (int S = 1; S <= 4 && S <= nkb; ++S) {
      const int64_t at_once = S == 1 ? pairs : room.clusters[2 * S - 1];
      if (at_once <= 0) continue;
      const double rounds = (double)ceil_div(tiles, at_once), loop = (double)ceil_div(nkb, S) * stage;
      double c;
      if (S == 1) c = rounds * (loop + 200 > epilogue ? loop + 200 : epilogue) + epilogue;
      else c = rounds * (loop + 2500 + bn * 3 + ((double)ceil_div(cols, 64 * S)) * (chunk + 250 * S * (gated ? 2 : 1)));
      if (least == 0 || c < 0.97 * least) {
        best = PairPlan{S > 1 ? PM_SPLIT : bn == 256 ? PM_FULL : PM_WIDTH, bn, S, (tiles < at_once ? tiles : at_once) * S, c,
                        loop + 200 > epilogue ? loop + 200 : epilogue};
        least = c;
      }
    }
  }
  return best;
}

// Over how many CTAs of a cluster the reduction of a few-token product is split and how many CTAs share an SM, by the estimated time:
// rounds of clusters; the time of a stage at its share of the memory's rate (which a part of the SMs does not reach: the 134 MB of the
// 4096 x 16384 down projection took 3 us more on 128 of them than on all), at what one SM takes in, or at what its ring holds in
// flight; what a round costs beside; and the sums, which grow with the CTAs that a value comes from (128 tokens, 2048 x 8192 of 4
// bits: 8.2 us over 4, 9.9 over 8).
struct FewPlan { int S, per_sm; double us; };
template <typename Cfg>
FewPlan few_plan(int64_t N, int nkb, const FewRoom& room) {
  const int64_t units = ceil_div(N, 128);
  FewPlan best{1, 1, 0};
  double least = 0;
  const double sms = sm_count_now();
  for (int per_sm = 1; per_sm <= Cfg::kMostPerSm; ++per_sm)
    for (int S = 1; S <= 8 && S <= nkb; ++S) {
      const int64_t slots = (int64_t)room.clusters[S - 1] * per_sm;
      if (slots <= 0) continue;
      const double at_once = (double)((units < slots ? units : slots) * S), rounds = (double)ceil_div(units, slots);
      const int ring = Cfg::stages(per_sm) < nkb / S + 1 ? Cfg::stages(per_sm) : nkb / S + 1;
      const double part = at_once / sms;
      double us = Cfg::kStageBytes * at_once / (6.5e6 * (part < 1 ? std::sqrt(part) : 1.0));
      const double sm = Cfg::kStageBytes * (part <= 1 ? 1 : per_sm) / 0.075e6, flight = 1.8 / ring;
      us = us > sm ? us : sm;
      us = us > flight ? us : flight;
      us = rounds * (us * (double)ceil_div(nkb, S) + (per_sm == 2 ? 1.0 : 1.5)) + (S > 1 ? 0.6 + 0.05 * S * Cfg::kPartBytes / 8192 : 0.0);
      if (least == 0 || us < 0.98 * least) { best = FewPlan{S, per_sm, us}; least = us; }
    }
  return best;
}

// Of a few-token product: its operands by their maps (see FewMaps; the tokens' box is kN rows), then the launch; without `make` the plan only.
struct NoMaps {};
template <int kFmt, int kKind, int kN, typename F>
int run_few_n(const FewArgs& a, cudaStream_t s, F& make, PairPlan* taken) {
  using Cfg = FewCfg<kFmt, kKind, kN>;
  const FewRoom* room;
  SF_TRY((few_room<kFmt, kKind, kN>(&room)));
  const FewPlan plan = few_plan<Cfg>(a.N, a.nkb, *room);
  if (taken) *taken = PairPlan{PM_SPLIT, kN, plan.S, ceil_div(ceil_div(a.N, 128) * plan.S, 2 * plan.per_sm), plan.us * 1900, 0};
  if constexpr (!std::is_same_v<F, NoMaps>) {
    FewMaps m;
    SF_TRY(make(m, kN));
    return launch_few<kFmt, kKind, kN>(m, a, plan.S, plan.per_sm, s);
  }
  return SF_OK;
}
template <int kFmt, int kKind, typename F>
int run_few(const FewArgs& a, cudaStream_t s, F&& make, PairPlan* taken = nullptr) {
  const int columns = a.T * a.in_terms;
  if (columns <= 16) return run_few_n<kFmt, kKind, 16>(a, s, make, taken);
  if (columns <= 32) return run_few_n<kFmt, kKind, 32>(a, s, make, taken);
  if (columns <= 64) return run_few_n<kFmt, kKind, 64>(a, s, make, taken);
  if (columns <= 96) return run_few_n<kFmt, kKind, 96>(a, s, make, taken);
  return run_few_n<kFmt, kKind, 128>(a, s, make, taken);
}
// X W^T with one matrix, or two of one shape.
template <int kFmt, int kKind>
int run_few_rows(const Operand& X, const Operand& W0, const Operand& W1, int64_t N, int64_t K, const FewArgs& a, cudaStream_t s) {
  return run_few<kFmt, kKind>(a, s, [&](FewMaps& m, int n) {
    SF_TRY(kmajor_map(&m.x, kFmt, X.data, (int64_t)a.T * a.in_terms, K, n));
    SF_TRY(kmajor_map(&m.w0, kFmt, W0.data, N, K, 128));
    m.w1 = m.w0;
    if (kKind == FK_GATED) SF_TRY(kmajor_map(&m.w1, kFmt, W1.data, N, K, 128));
    m.sx = m.s0 = m.s1 = m.x;
    if (kFmt != FMT_BF16) {
      SF_TRY(scale_map(&m.sx, kFmt, X.scales, a.T, K));
      SF_TRY(scale_map(&m.s0, kFmt, W0.scales, N, K));
      if (kKind == FK_GATED) SF_TRY(scale_map(&m.s1, kFmt, W1.scales, N, K));
    }
    return (int)SF_OK;
  });
}

// Launches the kernel of a plan: make(maps, bn) fills the tensor maps for tiles of that width.
template <int kKind, typename F>
int launch_plan(const PairPlan& plan, PairArgs a, cudaStream_t s, F&& make) {
  PairMaps<PairCfg<kKind, 256, FMT_BF16, PM_FULL>::kMaps> maps;
  SF_TRY(make(maps.m, plan.bn));
  a.bn = plan.bn;
  a.parts = plan.parts;
  return plan.mode == PM_FULL    ? launch_pair<kKind, 256, FMT_BF16, PM_FULL>(maps, a, s)
         : plan.mode == PM_WIDTH ? launch_pair<kKind, 256, FMT_BF16, PM_WIDTH>(maps, a, s)
                                 : launch_pair<kKind, 256, FMT_BF16, PM_SPLIT>(maps, a, s);
}
// The same from the sizes.
inline int plan_pairs(int kind, const PairArgs& a, PairPlan* plan) {
  const FewRoom* room;
  SF_TRY((few_room<FMT_BF16, FK_NT, 16>(&room)));          // (one CTA to an SM, like the pairs')
  PairJob jobs[3];
  for (int j = 0; j < a.jobs; ++j) jobs[j] = PairJob{a.M[j], a.N[j]};
  *plan = pair_plan(kind, jobs, a.jobs, a.nkb, *room);
  return SF_OK;
}
template <int kKind, typename F>
int launch_best(const PairArgs& a, cudaStream_t s, F&& make, PairPlan* taken = nullptr, const PairPlan* beside = nullptr) {
  PairPlan plan;
  SF_TRY(plan_pairs(kKind, a, &plan));
  if (taken) *taken = plan;
  if (!beside) return launch_plan<kKind>(plan, a, s, make);
  PairArgs b = a;
  b.beside = 1;
  const int64_t pairs = sm_count_now() / 2;
  if (beside->pairs < pairs && plan.mode != PM_SPLIT) {
    b.first_late = (int)(pairs - beside->pairs);
    b.late_rounds = (int)(beside->clocks / plan.per_tile);
    // (fewer tiles than pairs, or all of them made before the late ones come: the plain order)
    int64_t tiles = 0;
    for (int j = 0; j < a.jobs; ++j) tiles += tiles_of(a.M[j], a.N[j], plan.bn);
    if (tiles <= b.first_late) b.late_rounds = 0;
  }
  return launch_plan<kKind>(plan, b, s, make);
}

// A 4-bit product, by the same estimate: rounds of tiles of 256 or of 128 columns, a stage of either (bounded by what the L2 delivers), what a
// tile costs beside; or tiles of 128 columns with the reduction split over two to four pairs of a cluster (300 x 1024 x 8192 12.0 us
// unsplit, 8.9 over three; 513 x 1032 x 4096 8.3 and 7.8 over two; gated ones, whose sums are twice as many, gained nothing: 11.0 and 11.1
// at 513 x 1032 x 4096).
inline int plan_fp4(int64_t M, int64_t N, int64_t nkb, PairPlan* plan) {
  const FewRoom* room;
  SF_TRY((few_room<FMT_BF16, FK_NT, 16>(&room)));
  const int64_t pairs = sm_count_now() / 2, tiles = tiles_of(M, N, 128);
  const double wide = (double)ceil_div(tiles_of(M, N, 256), pairs) * (nkb * 600 + 900) + 4900;
  const double narrow = (double)ceil_div(tiles, pairs) * (nkb * 450 + 200) + 2900;
  *plan = wide <= narrow ? PairPlan{PM_FULL, 256, 1, 0, wide, 0} : PairPlan{PM_FULL, 128, 1, 0, narrow, 0};
  for (int S = 2; S <= 4 && S <= nkb; ++S) {
    const int64_t at_once = room->clusters[2 * S - 1];
    if (at_once <= 0) continue;
    const double c = (double)ceil_div(tiles, at_once) * ((double)ceil_div(nkb, S) * 450 + 4600 + (double)ceil_div(128, 64 * S) * (1000 + 250 * S));
    if (c < 0.97 * plan->clocks) *plan = PairPlan{PM_SPLIT, 128, S, 0, c, 0};
  }
  return SF_OK;
}

template <int kFmt, int kBN, int kMode>
int run_nt_fp4(const Operand& A, const Operand& B, int64_t K, void* C, const PairArgs& a, cudaStream_t s) {
  PairMaps<5> m;
  SF_TRY(kmajor_map(&m.m[0], kFmt, A.data, a.M[0], K, 128));
  SF_TRY(kmajor_map(&m.m[1], kFmt, B.data, a.N[0], K, kBN / 2));
  SF_TRY(make_tmap_store(&m.m[2], C, a.M[0], a.N[0]));
  SF_TRY(scale_map(&m.m[3], kFmt, A.scales, a.M[0], K));
  SF_TRY(scale_map(&m.m[4], kFmt, B.scales, a.N[0], K));
  return launch_pair<PK_NT, kBN, kFmt, kMode>(m, a, s);
}

// C[M, N] = alpha A B^T; M, N, K > 0. early_weights: the launch before this one is another product of the same call, which does not
// write B. terms: 2 where A is a sum (few tokens).
template <int kFmt>
int run_nt(const Operand& A, const Operand& B, int64_t M, int64_t N, int64_t K, float alpha, void* C, int* status, cudaStream_t s,
           bool early_weights = false, int terms = 1) {
  const int nkb = k_blocks(kFmt, K);
  if (M <= kFewTokens) {
    FewArgs a{};
    a.T = (int)M; a.N = (int)N; a.nkb = nkb; a.alpha = a.alpha2 = alpha; a.C = C; a.status = status;
    a.early_weights = early_weights; a.in_terms = terms; a.out_terms = 1;
    return run_few_rows<kFmt, FK_NT>(A, B, B, N, K, a, s);
  }
  PairArgs a{};
  a.jobs = 1; a.M[0] = (int)M; a.N[0] = (int)N; a.nkb = a.nkb0 = nkb; a.alpha = alpha; a.status = status;
  if constexpr (kFmt == FMT_BF16) {
    return launch_best<PK_NT>(a, s, [&](CUtensorMap* m, int bn) {
      SF_TRY(kmajor_map(&m[0], kFmt, A.data, M, K, 128));
      SF_TRY(kmajor_map(&m[1], kFmt, B.data, N, K, bn / 2));
      return make_tmap_store(&m[2], C, M, N);
    });
  } else {
    PairPlan plan;
    SF_TRY(plan_fp4(M, N, nkb, &plan));
    a.bn = plan.bn; a.parts = plan.parts;
    return plan.mode == PM_SPLIT ? run_nt_fp4<kFmt, 128, PM_SPLIT>(A, B, K, C, a, s)
         : plan.bn == 256        ? run_nt_fp4<kFmt, 256, PM_FULL>(A, B, K, C, a, s)
                                 : run_nt_fp4<kFmt, 128, PM_FULL>(A, B, K, C, a, s);
  }
}

// H = act(alpha_g A Bg^T) (alpha_u A Bu^T); P, Q (bf16 operands; both or neither): act(g) and u act'(g) in float32. M, N, K > 0. terms: 2
// where H is a sum (few tokens).
template <int kFmt>
int run_gated(const Operand& A, const Operand& Bg, const Operand& Bu, int64_t M, int64_t N, int64_t K, int act, float alpha_g,
              float alpha_u, void* H, float* P, float* Q, int* status, cudaStream_t s, int terms = 1) {
  const int nkb = k_blocks(kFmt, K);
  if (gated_by_few(kFmt, M, nkb)) {
    FewArgs a{};
    a.T = (int)M; a.N = (int)N; a.nkb = nkb; a.act = act; a.alpha = alpha_g; a.alpha2 = alpha_u; a.C = H; a.P = P; a.Q = Q;
    a.status = status; a.in_terms = 1; a.out_terms = terms;
    return run_few_rows<kFmt, FK_GATED>(A, Bg, Bu, N, K, a, s);
  }
  PairArgs a{};
  a.jobs = 1; a.M[0] = (int)M; a.N[0] = (int)N; a.nkb = a.nkb0 = nkb; a.act = act; a.alpha = alpha_g; a.alpha2 = alpha_u;
  a.status = status;
  auto operands = [&](CUtensorMap* m, int bn) {
    SF_TRY(kmajor_map(&m[0], kFmt, A.data, M, K, 128));
    SF_TRY(kmajor_map(&m[1], kFmt, Bg.data, N, K, bn / 2));
    SF_TRY(kmajor_map(&m[2], kFmt, Bu.data, N, K, bn / 2));
    return make_tmap_store(&m[3], H, M, N);
  };
  if constexpr (kFmt != FMT_BF16) {
    PairMaps<7> m;
    SF_TRY(operands(m.m, 256));
    SF_TRY(scale_map(&m.m[4], kFmt, A.scales, M, K));
    SF_TRY(scale_map(&m.m[5], kFmt, Bg.scales, N, K));
    SF_TRY(scale_map(&m.m[6], kFmt, Bu.scales, N, K));
    return launch_pair<PK_FWD, 256, kFmt, PM_FULL>(m, a, s);
  } else if (P) {
    return launch_best<PK_FWD_SAVE>(a, s, [&](CUtensorMap* m, int bn) {
      SF_TRY(operands(m, bn));
      SF_TRY(make_tmap_f32(&m[4], P, M, N));
      return make_tmap_f32(&m[5], Q, M, N);
    });
  } else {
    return launch_best<PK_FWD>(a, s, operands);
  }
}

}  // namespace
}  // namespace sf
