// Host-side exercise of the projections, gated blocks and the norm and rotation of Q and K under AddressSanitizer and
// UndefinedBehaviorSanitizer (test infrastructure, CPU only): workspace sizes over the whole range of extents, and argument errors
// with extreme values. Compute calls are made only with arguments that validation rejects, so no kernel is ever launched.
#include <climits>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <cstdio>

#include "../../include/da2.h"

static int failures = 0;
#define EXPECT(cond)                                                  \
  do {                                                                \
    if (!(cond)) {                                                    \
      std::fprintf(stderr, "%s:%d: failed: %s\n", __FILE__, __LINE__, #cond); \
      ++failures;                                                     \
    }                                                                 \
  } while (0)

int main() {
  const int32_t E = DA2_ERR_INVALID_ARG, U = DA2_ERR_UNSUPPORTED, W = DA2_ERR_WORKSPACE;
  void* f1 = reinterpret_cast<void*>(0x1000);
  void* f2 = reinterpret_cast<void*>(0x2000);
  void* f3 = reinterpret_cast<void*>(0x3000);
  void* f4 = reinterpret_cast<void*>(0x4000);

  int64_t bytes = -1;
  for (int32_t B : {1, 3, 65535, 65536})
    for (int32_t N : {1, 16, 17, 777, 1 << 20, INT32_MAX})
      for (int32_t K : {1, 8, 1283, 1 << 20, INT32_MAX})
        for (int32_t F : {1, 64, 13824, 1 << 20, INT32_MAX})
          for (int32_t train = 0; train < 2; ++train) {
            const da2_proj p{B, N, 1, K, 1, F, DA2_ACT_SILU, DA2_BF16};
            bytes = -1;
            const int32_t a = da2_linear_ws_bytes(&p, train, &bytes);
            EXPECT(a == E || (a == DA2_OK && bytes >= 0));
            bytes = -1;
            const int32_t b = da2_glu_ws_bytes(&p, train, &bytes);
            EXPECT(b == E || (b == DA2_OK && bytes >= 0));
          }
  const da2_proj bad{INT32_MIN, INT32_MIN, INT32_MIN, INT32_MIN, INT32_MIN, INT32_MIN, INT32_MIN, INT32_MIN};
  EXPECT(da2_linear_ws_bytes(&bad, 0, &bytes) == E && da2_glu_ws_bytes(&bad, 1, &bytes) == E);

  const da2_proj p{2, 100, 1, 8192, 1, 128, DA2_ACT_NONE, DA2_BF16};
  const da2_tensor x{100 * 8192, 100 * 8192, 8192, DA2_BF16, 0}, y{100 * 128, 100 * 128, 128, DA2_BF16, 0};
  const da2_tensor wide{INT64_MAX, INT64_MAX, INT64_MAX, DA2_BF16, 0}, low{INT64_MIN, INT64_MIN, INT64_MIN, DA2_BF16, 0};
  const auto linear = [&](const da2_tensor* a, int64_t stride, const da2_tensor* b, int64_t gate, int64_t ws) {
    return da2_linear(&p, f1, a, f2, stride, nullptr, f1, gate, nullptr, nullptr, f3, b, nullptr, f4, ws, nullptr);
  };
  EXPECT(linear(&x, 8192, &y, 0, 0) == W);
  EXPECT(linear(&wide, 8192, &y, 0, 0) == E && linear(&low, 8192, &y, 0, 0) == E);
  EXPECT(linear(&x, 8192, &wide, 0, 0) == E && linear(&x, 8192, &low, 0, 0) == E);
  EXPECT(linear(&x, INT64_MAX, &y, 0, 0) == E && linear(&x, INT64_MIN, &y, 0, 0) == E);
  EXPECT(linear(&x, 8192, &y, INT64_MAX, 0) == E && linear(&x, 8192, &y, INT64_MIN, 0) == E);
  EXPECT(linear(&x, 8192, &y, 0, INT64_MIN) == W);
  const da2_proj wide_p{1, 100, 1, 64, 1, 1 << 20, DA2_ACT_NONE, DA2_BF16};
  EXPECT(da2_glu(&wide_p, f1, &x, f2, 1 << 22, nullptr, f3, &y, nullptr, f4, 0, nullptr) == E);
  EXPECT(da2_linear_bwd(&p, f1, &y, f2, &x, f3, 8192, nullptr, 0, nullptr, nullptr, nullptr, nullptr, INT64_MAX, nullptr, nullptr, f4, 0, nullptr) == E);
  EXPECT(da2_linear_bwd(&p, f1, &y, f2, &x, f3, 8192, nullptr, 0, nullptr, nullptr, nullptr, f4, INT64_MAX, nullptr, nullptr, f4, 0, nullptr) == E);

  da2_rope_desc r{DA2_ROPE_HALF, 64, 1, {64, 0, 0}};
  da2_norm_desc n{DA2_NORM_RMS, DA2_FP32, 0, 0, 0, 1e-6};
  const da2_tensor q{15 * 64, 5 * 64, 64, DA2_BF16, 0};
  const double turns[32] = {};
  for (int32_t d : {1, 64, 512, 513, int32_t(INT32_MAX), int32_t(INT32_MIN)})
    for (int32_t v : {1, 40, 65535, int32_t(INT32_MAX), int32_t(INT32_MIN)}) {
      const da2_rope_rows s{v, 3, 3, v, d, 0, 0, 0};
      bytes = -1;
      const int32_t st = da2_qk_norm_rope_ws_bytes(&s, &bytes);
      EXPECT(st == E || st == U || (st == DA2_OK && bytes > 0));
    }
  const da2_rope_rows s{2, 3, 3, 5, 64, 0, 0, 0};
  const auto qk = [&](const da2_tensor* a, const da2_tensor* b, double scale, int64_t pos) {
    return da2_qk_norm_rope(&r, turns, scale, (const int32_t*)f1, pos, &s, &n, nullptr, nullptr, f1, a, f2, b, f3, a, f4, b, nullptr);
  };
  EXPECT(qk(&wide, &q, 1.0, 5) == E && qk(&q, &wide, 1.0, 5) == E && qk(&q, &low, 1.0, 5) == E);
  EXPECT(qk(&q, &q, NAN, 5) == E && qk(&q, &q, 1.0, INT64_MIN) == E && qk(&q, &q, 1.0, INT64_MAX) == E);
  if (failures == 0) std::puts("layer ABI checks passed");
  return failures != 0;
}
