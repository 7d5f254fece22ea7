// Host build of the objectives' plans (objective_plan.h): over many sizes, what the launches take of the workspace
// lies within their part of it, a size asked for N rows holds every call of fewer, and no product has more tiles than a
// launch holds, up to the largest sizes.  Prints "ok", or names the first failing size and exits 1.
#include <cstdio>
#include <vector>

#include "objective_plan.h"

using namespace pspo;

static int64_t parts_of(const Plan& p) {
  return p.parts == 1 ? 0 : ((int64_t)p.tiles_m * p.tiles_n - p.whole) * p.parts * p.tile * p.tile_n * 4;
}

// The limits that a call would find only after its first launches.
static bool launches(const Plan& p) { return (int64_t)p.tiles_m * p.tiles_n < int64_t(1) << 23; }
static bool launches(const JobPlan& p) {
  int64_t blocks = 0;
  for (int i = 0; i < 3; ++i) {
    const int64_t tiles = (int64_t)p.tiles_m[i] * p.tiles_n[i];
    if (tiles >= int64_t(1) << 23) return false;
    blocks += (tiles + 7) / 8 * 8 * p.parts[i];
  }
  return blocks < int64_t(1) << 24;
}

static int check(int64_t N, int64_t d, int64_t V, int64_t& most) {
  for (const bool grads : {false, true}) {
    const Layout s = layout_of(N, d, V, 1, 0, 0, grads);
    const int64_t room = s.seqs - s.slab;
    int64_t need = 0;
    const int way = way_of(N, d, grads);
    if (way == kTiles) need = parts_of(plan_forward(V, N, d));
    if (way == kOnePass) need = pass_groups(N, d, V) * N * d * 4;
    if (grads && way != kOnePass) {
      need = std::max(need, parts_of(plan_square(d, N, (int)V)));
      need = std::max(need, parts_of(plan_square(d, V, (int)N)));
      need = std::max(need, plan_gradients(N, d, V).slab_bytes);
    }
    const int64_t entries = way == kFew && !grads ? 0 : N * s.ld * 2;
    const bool apart = s.groups * s.group >= V && s.ld % 64 == 0 && s.ld >= V && s.slab - s.e >= entries;
    most = std::max(most, s.total);
    const bool held = N == 0 || (launches(plan_forward(V, N, d)) && launches(plan_square(d, N, (int)V)) &&
                                 launches(plan_square(d, V, (int)N)) && launches(plan_gradients(N, d, V)));
    const bool fine = held && need <= room && apart && (int64_t)workspace_size(N, d, V, 1, 0, 0, true) >= most &&
                      (way != kOnePass || pass_groups(N, d, V) >= 1);
    if (!fine) {
      std::printf("FAIL N %lld d %lld V %lld grads %d way %d: need %lld room %lld\n", (long long)N, (long long)d,
                  (long long)V, (int)grads, way, (long long)need, (long long)room);
      return 1;
    }
  }
  return 0;
}

int main() {
  const int64_t sizes[][2] = {{3584, 152064}, {1536, 151936}, {1000, 50257}, {520, 32003}, {128, 2048},  {8, 1},
                              {8, 65},        {64, 300},      {2048, 300},   {4096, 1000}, {8192, 777},  {3592, 40},
                              {8, 2097152},   {72, 131399},   {16384, 5000}, {264, 8},     {1544, 45},   {3584, 1}};
  for (const auto& w : sizes) {
    int64_t most = 0;
    for (int64_t N = 0; N < 1500; ++N)
      if (check(N, w[0], w[1], most)) return 1;
    for (int64_t N = 1501; N < 12000; N += 7)
      if (check(N, w[0], w[1], most)) return 1;
  }
  unsigned long long x = 1;
  auto next = [&](int64_t n) {
    x = x * 6364136223846793005ull + 1442695040888963407ull;
    return (int64_t)((x >> 33) % (unsigned long long)n);
  };
  for (int i = 0; i < 60000; ++i) {
    int64_t most = 0;
    const int64_t d = 8 * (1 + next(i % 2 ? 64 : 1200)), V = 1 + next(i % 3 ? 3000 : 200000);
    if (check(next(i % 5 ? 600 : 20000), d, V, most)) return 1;
  }
  const int64_t large[][3] = {{1 << 23, 8, 8}, {1 << 23, 1 << 13, 8}, {1 << 23, 8, 1 << 13}, {1 << 18, 1 << 18, 1 << 18},
                              {1 << 15, 1 << 15, 1 << 21}, {1 << 16, 1 << 20, 1 << 16}, {1, 1 << 20, 1 << 16},
                              {65, 1 << 15, 1 << 21}, {(1 << 23) - 1, 8184, 8191}, {520193, 132096, 130049}};
  for (const auto& s : large) {
    int64_t most = 0;
    if (!sizes_fit(s[0], s[1], s[2])) {
      std::printf("FAIL %lld %lld %lld does not fit\n", (long long)s[0], (long long)s[1], (long long)s[2]);
      return 1;
    }
    if (check(s[0], s[1], s[2], most)) return 1;
  }
  std::printf("ok\n");
  return 0;
}
