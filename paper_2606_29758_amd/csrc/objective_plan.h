// How the calls of the objectives are covered by launches, and the workspace that takes: host code only,
// so that a host program can ask it.
#pragma once

#include "row_plan.h"
#include "skinny.h"

namespace pspo {

constexpr int kGroup = 64;         // vocabulary entries of one (reference, sum)
constexpr int kPassRows = 16;      // rows of a work-group in one pass over W
constexpr int kFewGroup = 2048;    // ... where the logits are kept in float32
constexpr int kOnePassGroup = 16;  // ... in one pass over W
// Ways of a call, by its size (way_of): tiles; up to 64 rows, logits and d_hidden in one pass over W, or,
// where d is too wide for that or no gradient is wanted, the logits in float32 first.
enum { kTiles, kFew, kOnePass };

constexpr int kPassWaves = 4;
constexpr int kMostPassWidth = 28 * 32 * kPassWaves;   // what the registers of a work-group to a CU hold
constexpr int pass_per_cu(int parts) { return parts <= 4 ? 4 : (parts <= 12 ? 2 : 1); }

constexpr int kMostVocab = 1 << 21, kMostWidth = 1 << 20;   // a tile's rows stay below 2^31 bytes
constexpr int kMostRows = 1 << 23;   // 256 threads to each: a launch holds fewer than 2^32
constexpr int64_t kMostEntries = int64_t(1) << 36;            // of a matrix: fewer tiles than a launch holds

// One pass over W for each 16 rows against the tiles: 40 rows, d = 3584, V = 152064 927 us a call, 65
// rows by tiles 966; 64 of them in one pass 1,097; 64 rows, 1536, 151936 456, 65 by tiles 455; 160, 46996
// 55, by tiles 63.  Few: without gradients, or wider than one pass is built for.
inline int way_of(int64_t N, int64_t d, bool grads) {
  if (N > kSkinnyTokens) return kTiles;
  if (!grads || d > kMostPassWidth) return kFew;
  return N <= 3 * kPassRows || d <= 12 * 32 * kPassWaves ? kOnePass : kTiles;
}
// Work-groups of one pass for each 16 rows: as many as run at once, but with four blocks of the
// vocabulary to each beyond one a CU (their sums are read again: 5 rows, d = 376, V = 22700 47 us with
// 1,024 of them, 39 with 354).  From d = 520 on one to a CU is better for up to 32 rows (17, d = 1536,
// V = 151936 357 / 383 us a call), two for more (40: 458 / 416).
inline int64_t pass_groups(int64_t N, int64_t d, int64_t V) {
  const int64_t parts = (d + 32 * kPassWaves - 1) / (32 * kPassWaves);
  const int64_t per_cu = parts > 4 && N <= 32 ? 1 : pass_per_cu((int)parts);
  const int64_t blocks = (V + kPassRows - 1) / kPassRows;
  const int64_t one = 256 / ((std::max<int64_t>(N, 1) + kPassRows - 1) / kPassRows);
  const int64_t most = std::min(one * per_cu, std::max(one, blocks / 4)) / kNumXcd * kNumXcd;
  return std::min(blocks, most);
}

// The forward product: rows in tiles of 160 to 224 where 256 would be too many of the last (against 256
// alone, whole calls: 777 rows, d = 1536, V = 151936 1,300 -> 1,261 us, 1,301 rows 1,861 -> 1,822).
constexpr int kForwardColumns[3] = {160, 192, 224};
inline Plan plan_forward(int64_t V, int64_t N, int64_t d) {
  const int nk = (int)((d + kRowK - 1) / kRowK);
  Plan best = plan_of(V, N, nk, false);
  for (const int columns : kForwardColumns) {
    const Plan p = plan_tile(V, N, nk, 256, columns, false);
    if (p.us < best.us) best = p;
  }
  return best;
}
// What the K parts of any plan of up to N rows take (the tiles of 160 and more columns are narrower than
// the 256 that slab_reserve counts, but there may be more of them).
inline int64_t forward_reserve(int64_t V, int64_t N, int64_t d) {
  int64_t bytes = slab_reserve(V, N, (int)d);
  const int64_t most = std::min<int64_t>((d + kRowK - 1) / kRowK / 4, 32);   // parts, plan_tile's limits
  if (most < 2) return bytes;
  for (const int64_t columns : kForwardColumns) {
    const int64_t tiles = ((V + 255) / 256) * ((N + columns - 1) / columns);
    bytes = std::max(bytes, std::min<int64_t>(tiles, 256) * most * 256 * columns * 4);
  }
  return std::min(bytes, kSlabBytes);
}

struct Layout {
  int64_t ld, groups;
  int group;
  int64_t use, zs, c, part, f, ids, g, terms, copy, e, z, slab, seqs, pairs, total;
};
// R, P: sequences and pairs of the preference loss.
inline Layout layout_of(int64_t N, int64_t d, int64_t V, int64_t k, int64_t R, int64_t P, bool grads) {
  Layout s{};
  s.ld = round_up(V, kGroup);
  const int way = way_of(N, d, grads);
  s.group = way == kFew ? kFewGroup : way == kOnePass ? kOnePassGroup : kGroup;
  s.groups = (V + s.group - 1) / s.group;
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t x = at;
    at = round_up(at + bytes, 256);
    return x;
  };
  s.use = take(N * 4);
  s.zs = take(N * k * 8);
  s.c = take(N * 4);
  s.part = take(N * s.groups * 8);
  s.f = take(N * 4);
  s.ids = take(N * k * 4);
  s.g = take(N * k * 4);
  s.terms = take(N * 4 * 8);
  s.copy = take(N * d * 2);
  s.z = take(way == kFew ? N * s.ld * 4 : 0);
  s.e = take(way == kFew && !grads ? 0 : N * s.ld * 2);
  int64_t slab = way == kOnePass ? pass_groups(N, d, V) * N * d * 4 : way == kTiles ? forward_reserve(V, N, d) : 0;
  if (grads && way != kOnePass) {
    const int64_t M[3] = {d, d, 0}, C[3] = {N, V, 0}, nk[3] = {(V + kRowK - 1) / kRowK, (N + kRowK - 1) / kRowK, 0};
    slab = std::max({slab, jobs_reserve(M, C, nk), slab_reserve(d, N, (int)V), slab_reserve(d, V, (int)N)});
  }
  s.slab = take(slab);
  s.seqs = take(R * 3 * 8);
  s.pairs = take(P * 2 * 8);
  s.total = at;
  return s;
}
inline bool sizes_fit(int64_t N, int64_t d, int64_t V) {
  return N >= 0 && d > 0 && V > 0 && d % 8 == 0 && d <= kMostWidth && V <= kMostVocab && N <= kMostRows &&
         N * d <= kMostEntries && N * V <= kMostEntries && V * d <= kMostEntries;
}
// Sequences (256 threads to each) and pairs; every sequence looks at every pair.
inline bool pairs_fit(int64_t R, int64_t P) { return R <= 1 << 23 && R * P <= kMostEntries; }
// Enough for any call of up to N rows (16, 32, 48 and 64 may take more than a few rows more do), with
// gradients for the calls without them too.
inline size_t workspace_size(int64_t N, int64_t d, int64_t V, int64_t k, int64_t R, int64_t P, bool grads) {
  if (!sizes_fit(N, d, V)) return 0;
  int64_t most = 0;
  for (const bool with : {false, grads}) {
    most = std::max(most, layout_of(N, d, V, k, R, P, with).total);
    for (int64_t few = kPassRows; few <= kSkinnyTokens; few += kPassRows)
      if (few < N) most = std::max(most, layout_of(few, d, V, k, R, P, with).total);
  }
  return (size_t)most;
}

// One gradient product, in 256 or 128 square tiles.
inline Plan plan_square(int64_t M, int64_t N, int K) {
  const int nk = (K + kRowK - 1) / kRowK;
  const Plan small = plan_tile(M, N, nk, 128, 128, false), big = plan_tile(M, N, nk, 256, 256, false);
  return big.us <= small.us ? big : small;
}
// Both as one launch (against two, us a call: 1 row, d = 1536, V = 151936 411 / 472; 1,301, 1000, 50257 492 /
// 528; 4,096, 3584, 152064 10,602 / 10,818; 4,999 of the same 13,024 / 12,871).  One alone goes as a product,
// whose last round is split along K (8,192 rows, d = 3584: 13,536 against 14,105).
inline JobPlan plan_gradients(int64_t N, int64_t d, int64_t V) {
  const int64_t M[3] = {d, d, 0}, C[3] = {N, V, 0};
  const int nk[3] = {(int)((V + kRowK - 1) / kRowK), (int)((N + kRowK - 1) / kRowK), 0};
  const JobPlan big = plan_jobs(M, C, nk, 256), small = plan_jobs(M, C, nk, 128);
  return big.us <= small.us ? big : small;
}

}  // namespace pspo
