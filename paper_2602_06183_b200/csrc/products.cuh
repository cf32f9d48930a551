// Host side of the products of the gated block and of 4-bit operands: tensor maps, choice of kernel and tile, launches.
#pragma once

#include <cmath>

#include "few_tokens.cuh"
#include "pair_product.cuh"

#define SF_TRY(expr)              \
  do {                            \
    int _st = (expr);             \
    if (_st != SF_OK) return _st; \
  } while (0)

namespace sf {
namespace {

// Up to this many tokens the weights are streamed past them (few_tokens.cuh).
#ifndef SF_FEW_TOKENS
#define SF_FEW_TOKENS 128
#endif
constexpr int64_t kFewTokens = SF_FEW_TOKENS;

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
inline int mn_map(void* m, const void* p, int64_t K, int64_t cols) { return make_tmap_2d(m, p, K, cols, cols, 64, 64, true); }
inline int scale_map(void* m, int fmt, const void* p, int64_t rows, int64_t K) {
  return make_tmap_scales(m, p, ceil_div(rows, 128), scale_tiles(fmt, K), fmt == FMT_NV ? 4 : 2);
}

// Tile width of a product on CTA pairs by its estimated clocks: rounds of tiles, each of nkb stages and what a tile costs beside them. A
// stage of 256 columns takes the tensor pipe 512 clocks; narrower ones are bounded by shared memory (operands written once, read
// once, 128 bytes a clock).
inline int pair_width(int64_t tiles256, int64_t tiles128, int64_t tiles64, int64_t nkb) {
  const int64_t pairs = sm_count_now() / 2, tiles[3] = {tiles256, tiles128, tiles64};
  const int width[3] = {256, 128, 64}, stage[3] = {512, 384, 320}, beside[3] = {900, 700, 600};
  int best = 0;
  double least = 0;
  for (int i = 0; i < 3; ++i) {
    const double c = (double)ceil_div(tiles[i], pairs) * (double)(nkb * stage[i] + beside[i]) + 4.0 * width[i];
    if (i == 0 || c < 0.97 * least) { best = i; least = c; }
  }
  return width[best];
}
inline int64_t tiles_of(int64_t M, int64_t N, int64_t cols) { return ceil_div(M, 256) * ceil_div(N, cols); }

// Over how many CTAs of a cluster the reduction of a few-token product is split and how many CTAs share an SM, by the estimated time:
// rounds of clusters; the time of a stage at its share of the memory's rate (which a part of the SMs does not reach: the 134 MB of the
// 4096 x 16384 down projection took 3 us more on 128 of them than on all), at what one SM takes in, or at what its ring holds in
// flight; what a round costs beside; and the sums, which grow with the CTAs that a value comes from (128 tokens, 2048 x 8192 of 4
// bits: 8.2 us over 4, 9.9 over 8).
struct FewPlan { int S, per_sm; };
template <typename Cfg>
FewPlan few_plan(int64_t N, int nkb, const FewRoom& room) {
  const int64_t units = ceil_div(N, 128);
  FewPlan best{1, 1};
  double least = 0;
  for (int per_sm = 1; per_sm <= Cfg::kMostPerSm; ++per_sm)
    for (int S = 1; S <= 8 && S <= nkb; ++S) {
      const int64_t slots = (int64_t)room.clusters[S - 1] * per_sm;
      if (slots <= 0) continue;
      const double at_once = (double)((units < slots ? units : slots) * S), rounds = (double)ceil_div(units, slots);
      const int ring = Cfg::stages(per_sm) < nkb / S + 1 ? Cfg::stages(per_sm) : nkb / S + 1;
      const double part = at_once / sm_count_now();
      double us = Cfg::kStageBytes * at_once / (6.5e6 * (part < 1 ? std::sqrt(part) : 1.0));
      const double sm = Cfg::kStageBytes * (part <= 1 ? 1 : per_sm) / 0.075e6, flight = 1.8 / ring;
      us = us > sm ? us : sm;
      us = us > flight ? us : flight;
      us = rounds * (us * (double)ceil_div(nkb, S) + (per_sm == 2 ? 1.0 : 1.5)) + (S > 1 ? 0.3 + 0.05 * S * Cfg::kPartBytes / 8192 : 0.0);
      if (least == 0 || us < 0.98 * least) { best = FewPlan{S, per_sm}; least = us; }
    }
  return best;
}

template <int kFmt, bool kGated, int kN>
int run_few_n(const Operand& X, const Operand& W0, const Operand& W1, int64_t N, int64_t K, FewArgs a, cudaStream_t s) {
  using Cfg = FewCfg<kFmt, kGated, kN>;
  FewMaps m;
  SF_TRY(kmajor_map(&m.x, kFmt, X.data, a.T, K, kN));
  SF_TRY(kmajor_map(&m.w0, kFmt, W0.data, N, K, 128));
  m.w1 = m.w0;
  if (kGated) SF_TRY(kmajor_map(&m.w1, kFmt, W1.data, N, K, 128));
  m.sx = m.s0 = m.s1 = m.x;
  if (Cfg::kFp4) {
    SF_TRY(scale_map(&m.sx, kFmt, X.scales, a.T, K));
    SF_TRY(scale_map(&m.s0, kFmt, W0.scales, N, K));
    if (kGated) SF_TRY(scale_map(&m.s1, kFmt, W1.scales, N, K));
  }
  const FewRoom* room;
  SF_TRY((few_room<kFmt, kGated, kN>(&room)));
  const FewPlan plan = few_plan<Cfg>(N, a.nkb, *room);
  return launch_few<kFmt, kGated, kN>(m, a, plan.S, plan.per_sm, s);
}
template <int kFmt, bool kGated>
int run_few(const Operand& X, const Operand& W0, const Operand& W1, int64_t N, int64_t K, const FewArgs& a, cudaStream_t s) {
  if (a.T <= 16) return run_few_n<kFmt, kGated, 16>(X, W0, W1, N, K, a, s);
  if (a.T <= 32) return run_few_n<kFmt, kGated, 32>(X, W0, W1, N, K, a, s);
  if (a.T <= 64) return run_few_n<kFmt, kGated, 64>(X, W0, W1, N, K, a, s);
  if (a.T <= 96) return run_few_n<kFmt, kGated, 96>(X, W0, W1, N, K, a, s);
  return run_few_n<kFmt, kGated, 128>(X, W0, W1, N, K, a, s);
}

template <int kFmt, int kBN>
int run_nt_pair(const Operand& A, const Operand& B, int64_t K, void* C, const PairArgs& a, cudaStream_t s) {
  PairMaps<PairCfg<PK_NT, kBN, kFmt>::kMaps> m;
  SF_TRY(kmajor_map(&m.m[0], kFmt, A.data, a.M[0], K, 128));
  SF_TRY(kmajor_map(&m.m[1], kFmt, B.data, a.N[0], K, kBN / 2));
  SF_TRY(make_tmap_store(&m.m[2], C, a.M[0], a.N[0]));
  if constexpr (kFmt != FMT_BF16) {
    SF_TRY(scale_map(&m.m[3], kFmt, A.scales, a.M[0], K));
    SF_TRY(scale_map(&m.m[4], kFmt, B.scales, a.N[0], K));
  }
  return launch_pair<PK_NT, kBN, kFmt>(m, a, s);
}

// C[M, N] = alpha A B^T; M, N, K > 0. early_weights: the launch before this one is another product of the same call, which does not
// write B.
template <int kFmt>
int run_nt(const Operand& A, const Operand& B, int64_t M, int64_t N, int64_t K, float alpha, void* C, int* status, cudaStream_t s,
           bool early_weights = false) {
  const int nkb = k_blocks(kFmt, K);
  if (M <= kFewTokens) {
    FewArgs a{};
    a.T = (int)M; a.N = (int)N; a.nkb = nkb; a.alpha = a.alpha2 = alpha; a.C = C; a.status = status;
    a.early_weights = early_weights;
    return run_few<kFmt, false>(A, B, B, N, K, a, s);
  }
  PairArgs a{};
  a.jobs = 1; a.M[0] = (int)M; a.N[0] = (int)N; a.nkb = a.nkb0 = nkb; a.alpha = alpha; a.status = status;
  const int w = pair_width(tiles_of(M, N, 256), tiles_of(M, N, 128), kFmt == FMT_BF16 ? tiles_of(M, N, 64) : (int64_t)1 << 40, nkb);
  if (w == 256) return run_nt_pair<kFmt, 256>(A, B, K, C, a, s);
  if constexpr (kFmt == FMT_BF16)
    if (w == 64) return run_nt_pair<kFmt, 64>(A, B, K, C, a, s);
  return run_nt_pair<kFmt, 128>(A, B, K, C, a, s);
}

template <int kKind, int kFmt, int kBN>
int run_gated_pair(const Operand& A, const Operand& Bg, const Operand& Bu, int64_t K, void* H, float* P, float* Q, const PairArgs& a,
                   cudaStream_t s) {
  PairMaps<PairCfg<kKind, kBN, kFmt>::kMaps> m;
  SF_TRY(kmajor_map(&m.m[0], kFmt, A.data, a.M[0], K, 128));
  SF_TRY(kmajor_map(&m.m[1], kFmt, Bg.data, a.N[0], K, kBN / 2));
  SF_TRY(kmajor_map(&m.m[2], kFmt, Bu.data, a.N[0], K, kBN / 2));
  SF_TRY(make_tmap_store(&m.m[3], H, a.M[0], a.N[0]));
  if constexpr (kKind == PK_FWD_SAVE) {
    SF_TRY(make_tmap_f32(&m.m[4], P, a.M[0], a.N[0]));
    SF_TRY(make_tmap_f32(&m.m[5], Q, a.M[0], a.N[0]));
  }
  if constexpr (kFmt != FMT_BF16) {
    SF_TRY(scale_map(&m.m[4], kFmt, A.scales, a.M[0], K));
    SF_TRY(scale_map(&m.m[5], kFmt, Bg.scales, a.N[0], K));
    SF_TRY(scale_map(&m.m[6], kFmt, Bu.scales, a.N[0], K));
  }
  return launch_pair<kKind, kBN, kFmt>(m, a, s);
}

// H = act(alpha_g A Bg^T) (alpha_u A Bu^T); P, Q (bf16 operands; both or neither): act(g) and u act'(g) in float32. M, N, K > 0.
template <int kFmt>
int run_gated(const Operand& A, const Operand& Bg, const Operand& Bu, int64_t M, int64_t N, int64_t K, int act, float alpha_g,
              float alpha_u, void* H, float* P, float* Q, int* status, cudaStream_t s) {
  const int nkb = k_blocks(kFmt, K);
  if (M <= kFewTokens) {
    FewArgs a{};
    a.T = (int)M; a.N = (int)N; a.nkb = nkb; a.act = act; a.alpha = alpha_g; a.alpha2 = alpha_u; a.C = H; a.P = P; a.Q = Q;
    a.status = status;
    return run_few<kFmt, true>(A, Bg, Bu, N, K, a, s);
  }
  PairArgs a{};
  a.jobs = 1; a.M[0] = (int)M; a.N[0] = (int)N; a.nkb = a.nkb0 = nkb; a.act = act; a.alpha = alpha_g; a.alpha2 = alpha_u;
  a.status = status;
  if constexpr (kFmt != FMT_BF16) {
    return run_gated_pair<PK_FWD, kFmt, 256>(A, Bg, Bu, K, H, nullptr, nullptr, a, s);
  } else {
    const int w = pair_width(tiles_of(M, N, 128), tiles_of(M, N, 64), tiles_of(M, N, 32), nkb);
    if (P) {
      if (w == 256) return run_gated_pair<PK_FWD_SAVE, kFmt, 256>(A, Bg, Bu, K, H, P, Q, a, s);
      if (w == 128) return run_gated_pair<PK_FWD_SAVE, kFmt, 128>(A, Bg, Bu, K, H, P, Q, a, s);
      return run_gated_pair<PK_FWD_SAVE, kFmt, 64>(A, Bg, Bu, K, H, P, Q, a, s);
    }
    if (w == 256) return run_gated_pair<PK_FWD, kFmt, 256>(A, Bg, Bu, K, H, P, Q, a, s);
    if (w == 128) return run_gated_pair<PK_FWD, kFmt, 128>(A, Bg, Bu, K, H, P, Q, a, s);
    return run_gated_pair<PK_FWD, kFmt, 64>(A, Bg, Bu, K, H, P, Q, a, s);
  }
}

}  // namespace
}  // namespace sf
