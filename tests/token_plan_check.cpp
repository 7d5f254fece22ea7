// Host build of the element-wise layer operators' launch shapes (token_plan.h), one line an argument:
//   qk:N,Hq,Hk,D,bytes    -> lanes, passes a wave takes in the forward, whether a step of four passes holds both
//                            queries and keys, past the caches (forward), tokens a wave takes in the backward,
//                            past the caches (backward)
//   drop:N,d,moved        -> lanes, past the caches, rows of the grid's second axis
#include <cstdio>

#include "token_plan.h"

using namespace pspo;

int main(int argc, char** argv) {
  for (int i = 1; i < argc; ++i) {
    int N, Hq, Hk, D, b;
    if (std::sscanf(argv[i], "qk:%d,%d,%d,%d,%d", &N, &Hq, &Hk, &D, &b) == 5) {
      const QkForward p = qk_forward(N, Hq, Hk, D);
      bool both = false;
      for (int r = 0; r < p.parts; ++r)
        for (int s = r * p.per_part; s < (r + 1) * p.per_part; s += 4) {
          const int last = s + 3 < (r + 1) * p.per_part - 1 ? s + 3 : (r + 1) * p.per_part - 1;
          both = both || (s < p.passes_q && last >= p.passes_q && p.passes_q < p.passes_q + p.passes_k);
        }
      std::printf("%d %d %d %d %d %d\n", lanes_of(D), p.per_part, both, qk_past(N, Hq + Hk, D, b, false),
                  (int)((token_groups(N) + bwd_groups(N) - 1) / bwd_groups(N)), qk_past(N, Hq + Hk, D, b, true));
    } else if (std::sscanf(argv[i], "drop:%d,%d,%d", &N, &D, &b) == 3) {
      const DropPlan p = drop_plan(N, D / 8, b);
      std::printf("%d %d %d\n", p.lanes, p.past, (int)p.parts);
    } else {
      return 2;
    }
  }
  return 0;
}
