// Which kernel a product takes and how it is cut. Plain C++: the launcher, the workspaces' sizes and a test on the CPU share it.
#pragma once

#include <stdint.h>

namespace da2 {

constexpr int kStep = 64;             // elements of K a step of the tiles
constexpr int kFewTokens = 16;  // rows of a product by one launch that reads the weights once

// Whether a product of M rows with (parts) F weight rows of K elements takes the kernel for few rows (lo: with rows in two numbers).
// It does not cut K: a workgroup of 16 features sums over all of it, and reads all M rows for them, which takes as long as 26 of
// theirs would (52 gated) and the M rows; on tiles a long sum is cut into parts, but rows in two numbers read the weights
// twice. So long sums go there only with the fewest rows and where the features give every CU a workgroup. Measured, few rows' kernel
// against tiles, us, with 1 and 16 rows: K = 2,048, 64 to 4,096 features 11.4 and 11.8 against 14.1 and 14.2; 5,120 x 5,120 15 and 21
// against 19 and 20; gated 2,048 x 2 x 5,504 12 and 14 against 17 and 17; 8,192 x 1,024 12 and 17 against 14 and 15; 8,960 x 1,536 13 and
// 19 against 17 and 17; 32,768 x 1,024 38 and 58 against 25 and 26; 131,072 x 64 140 and 223 against 27 and 28; gated 8,192 x 2 x 64 19
// and 24 against 14 and 15; of many features 13,824 x 5,120 34 and 50 against 33 and 34, 32,768 x 4,096 45 and 61 against 50 and 52,
// gated 5,120 x 2 x 5,120 27 and 32 against 28 and 29. Gradients of 16 x 64 weights over 4,096, 16,384 and 200,000 tokens, the
// whole call: 18, 39 and 363 against 21, 22 and 69. Two numbers, both passes of 2,048 to 2 x 5,504 features: 94 and 123 against 103 and
// 119, of 1,536 to 8,960: 66 and 88 against 71 and 83.
constexpr int64_t kFewSum = 320'000, kFewSumLo = 480'000;
constexpr int kFewestRows = 4;
constexpr int64_t kManyFeatures = 4096;
inline bool few_rows(int64_t M, int64_t F, int64_t K, int parts, bool lo = false) {
  if (M > kFewTokens) return false;
  if (M <= kFewestRows && F >= kManyFeatures) return true;
  return lo ? (26 + 2 * M) * K <= kFewSumLo : (26 * parts + M) * K <= kFewSum;
}

// How a product is cut otherwise: tiles of 256x256 or 128x128, and parts of K that are joined. The least by these times in us, fitted to
// 16 products of 100 to 8,192 rows: a round of workgroups takes 9 and 1.4 a step (big tiles, one workgroup a CU) or 8 and 0.95 (small,
// two a CU; 0.7 with one); a join takes 2.5, 0.1 a part, and the partial sums' bytes, written and read, at 4 TB/s. (5,120 x 1,280 x 8,192: 110
// with big tiles and two parts, 165 whole, 119 and 130 with small ones; 2,331 x 1,280 x 1,024: 20 with small tiles, 26 in two
// parts, 34 with big ones. Up to 64 parts: gradients of 48 x 144 weights over 257,570 tokens 582 us with at most 8, 233 with 64.)
// Of the long forward products it takes the faster tile, too, though it underrates what their epilogues cost: 32,760 x 1,536 x 4,608 with
// bias 448 to 475 with big tiles, 542 with small ones; 32,760 x 1,536 x 1,536 with gate and residual 181 to 184 and 203; 8,190 x 5,120 x
// 2 x 13,824 gated 1,780 and 2,249.
struct Plan {
  bool big;
  int splits;
};
inline Plan plan_of(int64_t M, int64_t R, int64_t K) {
  const int64_t big = ((M + 255) / 256) * ((R + 255) / 256), small = ((M + 127) / 128) * ((R + 127) / 128);
  const int64_t steps = (K + kStep - 1) / kStep;
  Plan best{false, 1};
  double least = 1e300;
  for (int64_t splits = 1; splits <= 64 && (splits == 1 || steps >= 4 * splits); splits *= 2) {
    const int64_t per = (steps + splits - 1) / splits, parts = (steps + per - 1) / per;
    const double join = parts > 1 ? 2.5 + 0.1 * parts + 8e-6 / 4 * static_cast<double>(parts) * static_cast<double>(M) * static_cast<double>(R) : 0.0;
    const double b = static_cast<double>((big * parts + 255) / 256) * (1.4 * per + 9) + join;
    const int64_t rest = small * parts % 512;
    const double s = static_cast<double>(small * parts / 512) * (0.95 * per + 8) + (rest > 256 ? 0.95 * per + 8 : rest ? 0.7 * per + 8 : 0.0) + join;
    if (b < least) {
      least = b;
      best = {true, static_cast<int>(parts)};
    }
    if (s < least) {
      least = s;
      best = {false, static_cast<int>(parts)};
    }
  }
  return best;
}

// Bytes of the partial sums of a product of M rows (lo: on tiles the two numbers are a sum twice as long).
inline int64_t partial_bytes(int64_t M, int64_t F, int64_t K, int parts, bool lo = false) {
  if (few_rows(M, F, K, parts, lo)) return 0;
  const Plan p = plan_of(M, F * parts, lo ? 2 * K : K);
  return p.splits > 1 ? 4 * p.splits * M * ((F * parts + 7) / 8 * 8) : 0;
}

}  // namespace da2
