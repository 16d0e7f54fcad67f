// Says how the library cuts products (test infrastructure, host only): for each line "M F K parts" of the input "few", or
// tile, parts of K, whether K ends inside a step, and whether a workgroup has several units of work.
#include <cstdio>

#include "../../paper_2609_32628_amd/csrc/plan.hpp"

int main() {
  long long M, F, K;
  int parts;
  while (std::scanf("%lld %lld %lld %d", &M, &F, &K, &parts) == 4) {
    if (da2::few_rows(M, F, K, parts)) {
      std::printf("few 1 0 0 %lld\n", (long long)da2::partial_bytes(M, F, K, parts));
      continue;
    }
    const da2::Plan p = da2::plan_of(M, F * parts, K);
    const long long side = p.big ? 256 : 128, units = (F * parts + side - 1) / side * ((M + side - 1) / side) * p.splits;
    std::printf("%s %d %d %d %lld\n", p.big ? "big" : "small", p.splits, K % da2::kStep != 0, units > (p.big ? 256 : 512),
                (long long)da2::partial_bytes(M, F, K, parts));
  }
  return 0;
}
