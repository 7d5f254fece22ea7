// Host build of the gated feed-forward block's plans (ffn_plan.h).
//   ffn_plan_check need          : over many sizes, the slabs that the plans take lie within the workspace;
//                                  prints "ok", or names the first failing size and exits 1
//   ffn_plan_check cover N d f.. : the kernels that each call launches, one a line:
//                                  N d f product tile tile_n ring parts
// (tile 0: the kernels of few tokens; ring and parts as ffn.hip's product() and run_jobs() choose them).
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "ffn_plan.h"

using namespace pspo;

static int stages(int64_t K) { return (int)((K + kRowK - 1) / kRowK); }

static int64_t slab_of(int64_t M, int64_t N, int64_t K, bool dh) {
  if (M == 0 || N == 0) return 0;
  const Plan p = plan_of(M, N, stages(K), dh);
  return p.parts == 1 ? 0 : ((int64_t)p.tiles_m * p.tiles_n - p.whole) * p.parts * p.tile * p.tile_n * 4;
}

static int check(int64_t N, int64_t d, int64_t f) {
  const bool few = few_tokens(N, d, f);
  const int64_t gu = few ? 0 : slab_of(2 * f, N, d, false), down = few ? 0 : slab_of(d, N, f, false);
  const int64_t dh = slab_of(f, N, d, true), jobs = plan_backward(N, d, f).slab_bytes;
  const Space fwd = space_of(N, d, f, false, false), kept = space_of(N, d, f, true, true),
              own = space_of(N, d, f, true, false);
  const bool ok = gu <= fwd.total - fwd.slab && down <= fwd.total - fwd.slab && dh <= kept.total - kept.slab &&
                  jobs <= kept.total - kept.slab && gu <= own.total - own.slab && dh <= own.total - own.slab &&
                  jobs <= own.total - own.slab;
  if (!ok) std::printf("FAIL N %lld d %lld f %lld\n", (long long)N, (long long)d, (long long)f);
  return ok ? 0 : 1;
}

static void product(int64_t N, int64_t d, int64_t f, const char* name, int64_t M, int64_t K, bool dh) {
  const Plan p = plan_of(M, N, stages(K), dh);
  auto line = [&](int64_t groups, int parts) {
    std::printf("%lld %lld %lld %s %d %d %d %d\n", (long long)N, (long long)d, (long long)f, name, p.tile, p.tile_n,
                p.tile == 128 && deep_ring(groups) ? kDeep : 2, parts);
  };
  if (p.whole > 0) line(p.whole, 1);
  const int64_t rest = (int64_t)p.tiles_m * p.tiles_n - p.whole;
  if (rest > 0) line(rest * p.parts, p.parts);
}

static void cover(int64_t N, int64_t d, int64_t f) {
  if (few_tokens(N, d, f)) {
    std::printf("%lld %lld %lld gate_up 0 %d 0 1\n", (long long)N, (long long)d, (long long)f, (int)(N + 15) / 16 * 16);
    std::printf("%lld %lld %lld down 0 %d 0 1\n", (long long)N, (long long)d, (long long)f, (int)(N + 15) / 16 * 16);
  } else {
    product(N, d, f, "gate_up", 2 * f, d, false);
    product(N, d, f, "down", d, f, false);
  }
  product(N, d, f, "dh", f, d, true);
  const JobPlan p = plan_backward(N, d, f);
  int64_t blocks = 0;
  for (int i = 0; i < 3; ++i) blocks += round_up((int64_t)p.tiles_m[i] * p.tiles_n[i], kNumXcd) * p.parts[i];
  const char* names[3] = {"dx", "dw_up", "dw_down"};
  for (int i = 0; i < 3; ++i)
    std::printf("%lld %lld %lld %s %d %d %d %d\n", (long long)N, (long long)d, (long long)f, names[i], p.tile, p.tile,
                p.tile == 128 && deep_ring(blocks) ? kDeep : 2, p.parts[i]);
}

int main(int argc, char** argv) {
  if (argc >= 2 && !std::strcmp(argv[1], "need")) {
    const int64_t widths[][2] = {{3584, 14336}, {1536, 6144}, {1000, 4104}, {64, 72},     {8, 8},     {8, 4096},
                                 {4096, 8},     {2048, 800},  {512, 1344},  {568, 7952},  {136, 200}, {8192, 28672},
                                 {1536, 8960},  {3584, 18944}, {72, 120000}, {120000, 72}, {88, 3768}};
    for (const auto& w : widths) {
      for (int64_t N = 0; N < 1500; ++N)
        if (check(N, w[0], w[1])) return 1;
      for (int64_t N = 1501; N < 20000; N += 3)
        if (check(N, w[0], w[1])) return 1;
      for (int64_t N = 20000; N < 400000; N += 117)
        if (check(N, w[0], w[1])) return 1;
    }
    unsigned long long x = 1;
    auto next = [&](int64_t n) {
      x = x * 6364136223846793005ull + 1442695040888963407ull;
      return (int64_t)((x >> 33) % (unsigned long long)n);
    };
    for (int i = 0; i < 200000; ++i)
      if (check(1 + next(int64_t(1) << (4 + next(16))), 8 * (1 + next(int64_t(1) << (1 + next(12)))),
                8 * (1 + next(int64_t(1) << (1 + next(12))))))
        return 1;
    std::printf("ok\n");
    return 0;
  }
  if (argc >= 2 && !std::strcmp(argv[1], "cover") && (argc - 2) % 3 == 0) {
    for (int i = 2; i < argc; i += 3) cover(std::atoll(argv[i]), std::atoll(argv[i + 1]), std::atoll(argv[i + 2]));
    return 0;
  }
  return 2;
}
