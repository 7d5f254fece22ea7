// How the gated feed-forward block's products are covered by launches, and the workspace that
// takes: host code only, so that a host program can ask it.
#pragma once

#include <algorithm>

#include "rowgemm.h"
#include "skinny.h"

namespace pspo {

// ---- plan ---------------------------------------------------------------------------
// How a product of M x N entries over nk stages is covered: tiles of 256 x 256 (one
// work-group to a CU), 128 x 128 (two) or 128 x 64 (three), the first `whole` of them launched
// as they are and the rest in `parts` parts of K (parts = 1: all are whole).
struct Plan {
  int tile, tile_n, tiles_m, tiles_n, whole, parts;
  double us;
};
constexpr int64_t kSlabBytes = int64_t(256) << 20;   // most that the parts of one product take

// The cover of least estimated time: a stage of a full round takes 1.45, 1.1 or 0.9 us, one
// with a work-group to a CU 0.7 us (128 x 128) or 0.5 us, each tile 20, 10 or 6 us beyond its
// stages (dh, whose epilogue moves 14 bytes an entry: 55 or 16); the slabs of the parts are written
// and read at 4.5 TB/s, and a further launch with its join takes 8 us.
inline Plan plan_tile(int64_t M, int64_t N, int nk, int tile, int tile_n, bool dh) {
  Plan p{};
  p.tile = tile;
  p.tile_n = tile_n;
  p.tiles_m = (int)((M + tile - 1) / tile);
  p.tiles_n = (int)((N + tile_n - 1) / tile_n);
  const int64_t total = (int64_t)p.tiles_m * p.tiles_n, slots = tile == 256 ? 256 : tile_n == 128 ? 512 : 768;
  const double extra = tile == 256 ? (dh ? 55 : 20) : tile_n == 128 ? (dh ? 16 : 10) : 6;
  const double stage = tile == 256 ? 1.45 : tile_n == 128 ? 1.1 : 0.9;
  const double single = tile == 256 ? 1.45 : tile_n == 128 ? 0.7 : 0.5;
  auto time = [&](int64_t groups, int stages, double per_tile) {
    const int64_t turns = (groups + slots - 1) / slots, rest = groups - (turns - 1) * slots;
    const double last = rest <= 256 ? single : stage;
    return (double)(turns - 1) * (stages * stage + per_tile) + stages * last + per_tile;
  };
  const int64_t before = (total - 1) / slots * slots, rest = total - before;   // the last round's tiles
  p.whole = (int)total;
  p.parts = 1;
  p.us = time(total, nk, extra);
  const double start = before ? time(before, nk, extra) : 0.0;
  const int64_t bytes = (int64_t)tile * tile_n * 4;
  // what a part writes: the columns that exist
  const double written = (double)tile * (double)std::min<int64_t>(N, tile_n) * 4;
  for (int s = 2; s <= 32 && s * 4 <= nk && rest * s * bytes <= kSlabBytes; ++s) {
    const double us = start + time(rest * s, (nk + s - 1) / s, tile == 256 ? 10 : 5) + 8 + (double)(rest * s) * written * 2 / 4.5e6;
    if (us < p.us) {
      p.us = us;
      p.whole = (int)before;
      p.parts = s;
    }
  }
  return p;
}
// dh: the product with that epilogue; the others may use 128 x 64, for few columns.
inline Plan plan_of(int64_t M, int64_t N, int nk, bool dh) {
  Plan best = plan_tile(M, N, nk, 128, 128, dh);
  const Plan big = plan_tile(M, N, nk, 256, 256, dh);
  if (big.us <= best.us) best = big;
  if (!dh && N <= 64) {
    const Plan thin = plan_tile(M, N, nk, 128, 64, dh);
    if (thin.us < best.us) best = thin;
  }
  return best;
}
// A work-group alone on its CU has its stages' loads wait for memory, with one stage in flight:
// launches of no more work-groups than CUs take a ring of four stages instead of two.
constexpr int kDeep = 4;
inline bool deep_ring(int64_t groups) { return groups <= 256; }

// The three products behind dh, as one launch: dx, the two upper weights' gradients, the
// lower one's.  All tiles of a size; a product whose tiles have more K stages than a
// work-group's share of the whole is split along K.
struct JobPlan {
  int tile;
  int tiles_m[3], tiles_n[3], parts[3];
  int64_t slab[3], slab_bytes;   // bytes from the slabs' start; all of them
  double us;
};
inline JobPlan plan_jobs(const int64_t (&M)[3], const int64_t (&N)[3], const int (&nk)[3], int tile) {
  JobPlan p{};
  p.tile = tile;
  const int64_t slots = tile == 256 ? 256 : 512, bytes = (int64_t)tile * tile * 4;
  int64_t units = 0, groups = 0;
  for (int i = 0; i < 3; ++i) {
    p.tiles_m[i] = (int)((M[i] + tile - 1) / tile);
    p.tiles_n[i] = (int)((N[i] + tile - 1) / tile);
    units += (int64_t)p.tiles_m[i] * p.tiles_n[i] * nk[i];
  }
  const int64_t share = std::max<int64_t>(units / slots, 4);
  int longest = 0;
  for (int i = 0; i < 3; ++i) {
    const int64_t tiles = (int64_t)p.tiles_m[i] * p.tiles_n[i];
    int64_t s = std::min<int64_t>((nk[i] + share - 1) / share, 32);
    s = std::max<int64_t>(std::min<int64_t>(s, tiles ? kSlabBytes / 3 / (tiles * bytes) : 1), 1);
    p.parts[i] = (int)s;
    p.slab[i] = p.slab_bytes;
    if (s > 1) p.slab_bytes += tiles * s * bytes;
    groups += tiles * s;
    if (tiles) longest = std::max(longest, (int)((nk[i] + s - 1) / s));
  }
  // A round's stages, half of the longest part idle at the end, the slabs out and in.  A stage of
  // the small tiles takes 0.85 us here (stages of different products meet on a CU; with 1.1 as for
  // one product, 777 tokens, d = 1000, f = 4104 would take the large tiles: 72 us with its join
  // against 61; 300 tokens, d = 2048, f = 8192: 116 against 98).
  const bool alone = tile == 128 && groups <= 256;
  const double stage = tile == 256 ? 1.45 : alone ? 0.7 : 0.85;
  const double rounds = (double)groups / (double)slots;
  p.us = std::max((double)units / (double)slots + longest * 0.5, (double)longest) * stage +
         std::max(rounds, 1.0) * (tile == 256 ? 10 : 5) + (double)p.slab_bytes * 2 / 4.5e6 + (p.slab_bytes ? 8 : 0);
  return p;
}
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

// Most that the parts of any N' <= N take: the plans' own need goes up and down with N (a last
// round of few tiles is cut finer than one of many), and a workspace asked for N has to serve
// fewer tokens too.  Tiles of 128 x 64 take no more than the 128 x 128 ones stand for here; up to
// 128 columns those have as many rounds as the 256 x 256 ones, shorter, and are taken.
inline int64_t slab_reserve(int64_t M, int64_t N, int K) {
  const int64_t most = std::min<int64_t>((K + kRowK - 1) / kRowK / 4, 32);   // parts, plan_tile's limits
  if (most < 2) return 0;
  int64_t bytes = 0;
  for (const int64_t tile : {128, 256}) {
    if (tile == 256 && N <= 128) break;
    const int64_t tiles = ((M + tile - 1) / tile) * ((N + tile - 1) / tile), slots = tile == 256 ? 256 : 512;
    bytes = std::max(bytes, std::min(tiles, slots) * most * tile * tile * 4);
  }
  return std::min(bytes, kSlabBytes);
}
inline int64_t jobs_reserve(int64_t N, int64_t d, int64_t f) {
  const int64_t M[3] = {N > 0 ? d : 0, d, f}, C[3] = {N, 2 * f, d};
  const int64_t nk[3] = {(f + kRowK - 1) / kRowK * 2, (N + kRowK - 1) / kRowK, (N + kRowK - 1) / kRowK};
  int64_t bytes = 0;
  for (const int64_t tile : {128, 256}) {
    int64_t sum = 0;
    for (int i = 0; i < 3; ++i) {
      const int64_t most = std::min<int64_t>((nk[i] + 3) / 4, 32);   // plan_jobs: a share is 4 stages at least
      // a product of as many tiles as there are slots has more stages in its share than a tile holds
      const int64_t tiles = std::min<int64_t>(((M[i] + tile - 1) / tile) * ((C[i] + tile - 1) / tile),
                                              tile == 256 ? 256 : 512);
      if (most >= 2) sum += std::min(tiles * most * tile * tile * 4, kSlabBytes / 3);
    }
    bytes = std::max(bytes, sum);
  }
  return bytes;
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
