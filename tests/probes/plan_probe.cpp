// Says how the library cuts products (test infrastructure, host only): for each line "M F K parts lo" of the input "few", or the
// tile; then parts of K, whether K ends inside a step, whether a workgroup has several units of work, and the partial sums' bytes.
#include <cstdio>

#include "../../paper_2609_32628_amd/csrc/plan.hpp"

int main() {
  long long M, F, K;
  int parts, lo;
  while (std::scanf("%lld %lld %lld %d %d", &M, &F, &K, &parts, &lo) == 5) {
    if (da2::few_rows(M, F, K, parts, lo)) {
      std::printf("few 1 0 0 %lld\n", (long long)da2::partial_bytes(M, F, K, parts, lo));
      continue;
    }
    const da2::Plan p = da2::plan_of(M, F * parts, lo ? 2 * K : K);
    const long long side = p.big ? 256 : 128, units = (F * parts + side - 1) / side * ((M + side - 1) / side) * p.splits;
    std::printf("%s %d %d %d %lld\n", p.big ? "big" : "small", p.splits, (lo ? 2 * K : K) % da2::kStep != 0, units > (p.big ? 256 : 512),
                (long long)da2::partial_bytes(M, F, K, parts, lo));
  }
  return 0;
}
