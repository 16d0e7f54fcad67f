// Host-side exercise of the token operators under AddressSanitizer and Undefined-
// BehaviorSanitizer (test infrastructure, CPU only): workspace sizes, rotary plans
// and every argument error of the compute entry points. Compute calls are made only
// with arguments that validation rejects, so no kernel is ever launched.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "../../include/da2.h"

static int failures = 0;
#define EXPECT(cond)                                                  \
  do {                                                                \
    if (!(cond)) {                                                    \
      std::fprintf(stderr, "%s:%d: failed: %s\n", __FILE__, __LINE__, #cond); \
      ++failures;                                                     \
    }                                                                 \
  } while (0)

static da2_tensor T(int64_t B, int64_t H, int64_t N, int64_t C, int dtype) {
  (void)B;
  return da2_tensor{H * N * C, N * C, C, dtype, 0};
}

int main() {
  const int32_t E = DA2_ERR_INVALID_ARG, U = DA2_ERR_UNSUPPORTED, W = DA2_ERR_WORKSPACE;
  void* f1 = reinterpret_cast<void*>(0x1000);
  void* f2 = reinterpret_cast<void*>(0x2000);
  void* f3 = reinterpret_cast<void*>(0x3000);
  void* f4 = reinterpret_cast<void*>(0x4000);

  // row norms: sizes over the range of widths and types, extremes included
  int64_t bytes = -1;
  for (int32_t C : {1, 3, 8, 64, 1283, 5120, 12288, 12289, 20001, 1 << 24})
    for (int32_t rows : {1, 7, 70001, INT32_MAX})
      for (int dtype = 0; dtype < 3; ++dtype) {
        const da2_rows r{1, 1, rows, C};
        EXPECT(da2_norm_ws_bytes(&r, dtype, 0, &bytes) == DA2_OK && bytes >= 8ll * C);
      }
  const da2_rows many{65535, 1, 1, 64};
  EXPECT(da2_norm_ws_bytes(&many, 0, 1, &bytes) == DA2_OK && bytes >= 65535ll * 8 * 64);
  for (const da2_rows& r : {da2_rows{0, 1, 1, 1}, da2_rows{1, -1, 1, 1}, da2_rows{1, 1, 0, 1}, da2_rows{1, 1, 1, 0},
                            da2_rows{65536, 1, 1, 1}, da2_rows{1, 65536, 65536, 1}, da2_rows{1, 1, 1, (1 << 24) + 1},
                            da2_rows{65535, 65535, 1, 1}, da2_rows{INT32_MAX, INT32_MAX, INT32_MAX, INT32_MAX}})
    EXPECT(da2_norm_ws_bytes(&r, 0, 0, &bytes) == E);
  const da2_rows r{2, 3, 5, 64};
  const da2_norm_desc n{DA2_NORM_LAYER, DA2_FP32, 0, 0, 0, 1e-6};
  const da2_tensor t = T(2, 3, 5, 64, DA2_BF16);
  const da2_tensor over{15 * 64, 5 * 64, 63, DA2_BF16, 0}, far{int64_t(1) << 41, 5 * 64, 64, DA2_BF16, 0};
  const da2_tensor wide{INT64_MAX, INT64_MAX, INT64_MAX, DA2_BF16, 0};
  EXPECT(da2_norm(f1, &t, &r, &n, nullptr, nullptr, f2, &over, nullptr, nullptr) == E);
  EXPECT(da2_norm(f1, &far, &r, &n, nullptr, nullptr, f2, &t, nullptr, nullptr) == E);
  EXPECT(da2_norm(f1, &t, &r, &n, nullptr, nullptr, f2, &wide, nullptr, nullptr) == E);
  EXPECT(da2_norm(f1, nullptr, &r, &n, nullptr, nullptr, f2, &t, nullptr, nullptr) == E);
  EXPECT(da2_norm(f1, &t, &r, &n, nullptr, nullptr, f2, nullptr, nullptr, nullptr) == E);
  EXPECT(da2_norm_bwd(f1, &t, f2, &t, &r, &n, nullptr, (float*)f3, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr) == E);
  EXPECT(da2_norm_bwd(f1, &t, f2, &t, &r, &n, nullptr, (float*)f3, nullptr, nullptr, f4, nullptr, f1, 0, nullptr) == W);
  const da2_norm_desc inf{DA2_NORM_LAYER, DA2_FP32, 0, 0, 0, INFINITY}, odd{DA2_NORM_LAYER, DA2_FP32, 0, 0, INT64_MAX, 0.0};
  EXPECT(da2_norm(f1, &t, &r, &inf, nullptr, nullptr, f2, &t, nullptr, nullptr) == E);
  EXPECT(da2_norm(f1, &t, &r, &odd, nullptr, nullptr, f2, &t, nullptr, nullptr) == E);

  // rotary positions: every scaling over the widths, written to buffers of the exact size
  for (int32_t scaling = 0; scaling < 4; ++scaling)
    for (int32_t D : {2, 4, 62, 128, 65536}) {
      const da2_rope_desc d{DA2_ROPE_HALF, D, 1, {D, 0, 0}};
      std::vector<double> turns(D / 2);
      double scale = 0;
      for (double base : {1.0000001, 10000.0, 1e300}) {
        const da2_rope_freq f{scaling, 4096, base, scaling ? 8.0 : 1.0, 32.0, 1.0};
        EXPECT(da2_rope_plan(&d, &f, turns.data(), &scale) == DA2_OK && std::isfinite(scale));
        for (double x : turns) EXPECT(std::isfinite(x) && x >= 0.0 && x < 0.16);
      }
    }
  const da2_rope_desc d{DA2_ROPE_HALF, 64, 1, {64, 0, 0}};
  const da2_rope_desc bad[] = {{2, 64, 1, {64, 0, 0}}, {0, 64, 0, {64, 0, 0}}, {0, 64, 4, {64, 0, 0}}, {0, 64, 2, {64, 0, 0}},
                               {0, 64, 1, {INT32_MAX, 0, 0}}, {0, INT32_MAX, 3, {INT32_MAX - 1, INT32_MAX - 1, INT32_MAX - 1}},
                               {0, 1, 1, {2, 0, 0}}, {0, 64, 1, {-2, 0, 0}}};
  const da2_rope_rows rr{2, 3, 3, 5, 64, 0, 0, 0};
  for (const auto& b : bad)
    EXPECT(da2_rope(&b, (double*)f1, 1.0, (int32_t*)f1, 0, &rr, f1, &t, f2, &t, f3, &t, f4, &t, nullptr) == E);
  for (const da2_rope_rows& q : {da2_rope_rows{0, 3, 3, 5, 64, 0, 0, 0}, da2_rope_rows{2, INT32_MAX, INT32_MAX, 5, 64, 0, 0, 0},
                                 da2_rope_rows{65535, 3, 3, INT32_MAX, 64, 0, 0, 0}, da2_rope_rows{2, 3, 3, 5, 65, 0, 0, 0},
                                 da2_rope_rows{2, 3, 3, 5, 64, 3, 3, 0}})
    EXPECT(da2_rope(&d, (double*)f1, 1.0, (int32_t*)f1, 0, &q, f1, &t, f2, &t, f3, &t, f4, &t, nullptr) == E);
  EXPECT(da2_rope(&d, (double*)f1, 1.0, (int32_t*)f1, INT64_MAX, &rr, f1, &t, f2, &t, f3, &t, f4, &t, nullptr) == E);

  // differential attention
  const da2_diff_problem p{2, 4, 2, 5, 7, 64, 1, 0, 0.125};
  EXPECT(da2_diff_ws_bytes(&p, 0, &bytes) == DA2_OK && da2_diff_ws_bytes(&p, 1, &bytes) == DA2_OK && bytes > 0);
  for (int32_t N : {1, 64, 65, 4096, 1 << 20})
    for (int32_t M : {1, 255, 16384, 1 << 30})
      for (int32_t G : {1, 7}) {
        const da2_diff_problem big{1, G, 1, N, M, 128, 0, 0, 1.0};
        EXPECT(da2_diff_ws_bytes(&big, 1, &bytes) == DA2_OK && bytes > 0);
      }
  for (const da2_diff_problem& q :
       {da2_diff_problem{0, 4, 2, 5, 7, 64, 0, 0, 1.0}, da2_diff_problem{2, 4, 3, 5, 7, 64, 0, 0, 1.0},
        da2_diff_problem{2, 4, 0, 5, 7, 64, 0, 0, 1.0}, da2_diff_problem{2, 4, 2, 5, INT32_MAX, 64, 0, 0, 1.0},
        da2_diff_problem{65535, INT32_MAX, INT32_MAX, 1, 1, 64, 0, 0, 1.0}, da2_diff_problem{2, 4, 2, 5, 7, 64, 2, 0, 1.0},
        da2_diff_problem{2, 4, 2, 5, 7, 64, 0, 0, NAN}, da2_diff_problem{65535, 65535, 65535, 1, 1, 64, 0, 0, 1.0},
        da2_diff_problem{1, 65535, 1, 32768, 1, 64, 0, 0, 1.0}})
    EXPECT(da2_diff_ws_bytes(&q, 1, &bytes) == E);
  const da2_diff_problem d96{2, 4, 2, 5, 7, 96, 0, 0, 1.0};
  EXPECT(da2_diff_ws_bytes(&d96, 0, &bytes) == U);
  const da2_tensor q = T(2, 4, 5, 64, DA2_BF16), k = T(2, 2, 7, 64, DA2_BF16), q32 = T(2, 4, 5, 64, DA2_FP32);
  EXPECT(da2_diff_attn(&p, f1, &q, f2, &k, f3, &k, nullptr, nullptr, nullptr, f4, &q, nullptr, nullptr, 0, nullptr) == E);
  EXPECT(da2_diff_attn(&p, f1, &q32, f2, &k, f3, &k, (float*)f1, nullptr, nullptr, f4, &q, nullptr, nullptr, 0, nullptr) == U);
  EXPECT(da2_diff_attn(&p, f1, &q, f2, &k, f3, &k, (float*)f1, nullptr, nullptr, f1, &q, nullptr, nullptr, 0, nullptr) == E);
  EXPECT(da2_diff_attn_bwd(&p, f1, &q, f2, &k, f3, &k, (float*)f1, nullptr, nullptr, (float*)f1, f4, &q, (void*)0x5000, &q, (void*)0x6000,
                           &k, (void*)0x7000, &k, (float*)f1, f1, 0, nullptr) == W);
  EXPECT(da2_diff_attn_bwd(&p, f1, &q, f2, &k, f3, &k, (float*)f1, nullptr, nullptr, nullptr, f4, &q, (void*)0x5000, &q, (void*)0x6000, &k,
                           (void*)0x7000, &k, (float*)f1, f1, 1 << 30, nullptr) == E);
  if (failures) return 1;
  std::printf("token ABI checks passed\n");
  return 0;
}
