// How the element-wise layer operators are launched: host code only, so that a host program can
// ask it.
#pragma once

#include <cstdint>

namespace pspo {

// Calls that move this much go past the caches, which would not hold their outputs until the
// next call reads them; smaller ones leave them there.
constexpr int64_t kPastBytes = int64_t(160) << 20;

// Rows of the grid along its second axis: until some 2,048 work-groups are there, at most `most`.
inline int64_t parts_for(int64_t gx, int64_t most) {
  const int64_t parts = gx >= 2048 ? 1 : (2048 + gx - 1) / gx;
  return parts < most ? parts : most;
}

// ---- head norms -------------------------------------------------------------------
constexpr int kQkWaves = 4;   // of a work-group; each takes a token at a time

// Lanes of a head of D entries, eight on each.
inline int lanes_of(int D) {
  int L = 1;
  while (L * 8 < D) L <<= 1;
  return L;
}
inline int64_t token_groups(int64_t N) { return (N + kQkWaves - 1) / kQkWaves; }

// The forward: a token's passes (64 / lanes heads each, queries and then keys) over `parts` rows of
// the grid, `per_part` of them each.  Few tokens: several waves, each with its own angles.
struct QkForward {
  int64_t gx;
  int passes_q, passes_k, parts, per_part;
};
inline QkForward qk_forward(int64_t N, int Hq, int Hk, int D) {
  const int heads = 64 / lanes_of(D);
  QkForward p{};
  p.gx = token_groups(N);
  p.passes_q = (Hq + heads - 1) / heads;
  p.passes_k = (Hk + heads - 1) / heads;
  const int passes = p.passes_q + p.passes_k;
  const int parts = (int)parts_for(p.gx, passes);
  p.per_part = (passes + parts - 1) / parts;
  p.parts = (passes + p.per_part - 1) / p.per_part;
  return p;
}

// Work-groups of the backward and side: four to a CU keep some 16 waves with their loads in
// flight; with more tokens than waves each takes several.
constexpr int kBwdGroups = 1024;
inline int bwd_groups(int64_t N) {
  const int64_t g = token_groups(N);
  return (int)(g < kBwdGroups ? g : kBwdGroups);
}

// The forward stores past the caches, the backward loads and stores (28,481 tokens of 32 heads of
// 128: 89 -> 73 us, 171 -> 162 us, before the later steps; the forward's loads too 84).
inline bool qk_past(int64_t N, int64_t heads, int D, int bytes, bool backward) {
  return N * heads * D * bytes * (backward ? 3 : 2) >= kPastBytes;
}

// ---- dropout ----------------------------------------------------------------------
// Work-groups of 256 threads as (256 / lanes) rows x lanes: rows shorter than a wave share one;
// long rows of few tokens are split over the grid's second axis, `per_part` groups of eight each.
struct DropPlan {
  int lanes;
  int64_t gx, parts;
  int32_t per_part;
  bool past;   // past the caches: 113,926 x 3584 with the residual (2.45 GB) 451 -> 418 us
};
// vecs: groups of eight in a row; moved: bytes of an entry's loads and store.
inline DropPlan drop_plan(int64_t N, int64_t vecs, int moved) {
  DropPlan p{};
  p.lanes = 64;
  while (p.lanes > 1 && p.lanes / 2 >= vecs) p.lanes /= 2;
  const int rows_per = 256 / p.lanes;
  p.gx = (N + rows_per - 1) / rows_per;
  // one step of one row's lanes at least per part
  const int64_t steps = (vecs + p.lanes - 1) / p.lanes;
  p.parts = parts_for(p.gx, steps);
  p.per_part = (int32_t)((steps + p.parts - 1) / p.parts * p.lanes);
  p.parts = (vecs + p.per_part - 1) / p.per_part;
  p.past = N * vecs * 8 * moved >= kPastBytes && p.lanes == 64;
  return p;
}

}  // namespace pspo
