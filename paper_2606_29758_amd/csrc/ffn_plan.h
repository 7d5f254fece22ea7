// How the gated feed-forward block's products are covered by launches, and the workspace that
// takes: host code only, so that a host program can ask it.
#pragma once

#include "row_plan.h"
#include "skinny.h"

namespace pspo {

// The three products behind dh, as one launch: dx, the two upper weights' gradients, the
// lower one's.
inline JobPlan plan_backward(int64_t N, int64_t d, int64_t f) {
  const int64_t M[3] = {N > 0 ? d : 0, d, f}, C[3] = {N, 2 * f, d};
  const int kd = (int)((f + kRowK - 1) / kRowK * 2), kn = (int)((N + kRowK - 1) / kRowK);
  const int nk[3] = {kd, kn, kn};
  const JobPlan big = plan_jobs(M, C, nk, 256), small = plan_jobs(M, C, nk, 128);
  return big.us <= small.us ? big : small;
}

// Whether a forward of N tokens goes by the kernels of skinny.h.  They read every token's rows again for
// each 16 rows of the weights, the 128 x 64 tiles write and join slabs instead: us a call, this
// way / tiles, on 6 d f bytes of weights: d = 3584, f = 14336 (308 MB) N = 1 65 / 77, 16 90 / 82;
// 1536, 6144 (57 MB) N = 16 26 / 28, 32 33 / 30; 2048, 800 (10 MB) N = 48 17 / 26; 512, 1344
// (4 MB) N = 64 15 / 19.
inline bool few_tokens(int64_t N, int64_t d, int64_t f) {
  return N <= kSkinnyTokens && (N - 12) * (6 * d * f) <= int64_t(300) << 20;
}

inline int64_t jobs_reserve(int64_t N, int64_t d, int64_t f) {
  const int64_t M[3] = {N > 0 ? d : 0, d, f}, C[3] = {N, 2 * f, d};
  const int64_t nk[3] = {(f + kRowK - 1) / kRowK * 2, (N + kRowK - 1) / kRowK, (N + kRowK - 1) / kRowK};
  return jobs_reserve(M, C, nk);
}

// Workspace layout of one call; no part of it shrinks with more tokens.
struct Space {
  int64_t h, dgu, pre, slab, total;
};
inline Space space_of(int64_t N, int64_t d, int64_t f, bool backward, bool kept) {
  Space s{};
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t a = at;
    at = round_up(at + bytes, 256);
    return a;
  };
  s.h = take(N * f * 2);
  int64_t slab = 0;
  if ((!backward || !kept) && !few_tokens(N, d, f)) slab = slab_reserve(2 * f, N, (int)d);
  if (backward) {
    s.dgu = take(N * 2 * f * 2);
    if (!kept) s.pre = take(N * 2 * f * 4);
    slab = std::max({slab, slab_reserve(f, N, (int)d), jobs_reserve(N, d, f)});
  } else if (!few_tokens(N, d, f)) {
    slab = std::max(slab, slab_reserve(d, N, (int)f));
  }
  s.slab = take(slab);
  s.total = at;
  return s;
}

}  // namespace pspo
