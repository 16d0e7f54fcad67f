// Rotary positions: a token's cosines and sines, the rotation of a pair and where a row's
// pairs lie, for the kernels that rotate.
#pragma once

#include "token.hpp"

namespace da2 {

// n elements (16 bytes, or one) at p as floats, and back.
template <typename T, int V>
__device__ inline void get(const T* p, float* x) {
  if constexpr (V > 1) {
    load_vec(p, x);
  } else {
    x[0] = static_cast<float>(*p);
  }
}
template <typename T, int V>
__device__ inline void put(T* p, const float* x) {
  if constexpr (V > 1) {
    store_vec(p, x);
  } else {
    *p = static_cast<T>(x[0]);
  }
}

// cos and sin of pairs [p, p + P) of token n of sample b, times the scale; pairs from rot / 2 on get none.
template <int P>
__device__ inline void angles(const RopeArgs& a, int b, int n, int p, float* c, float* s) {
  int at[3];
  if (a.pos) {
    const int32_t* q = a.pos + b * a.pos_sb + static_cast<int64_t>(n) * a.axes;
    at[0] = q[0];
    at[1] = a.axes > 1 ? q[1] : 0;
    at[2] = a.axes > 2 ? q[2] : 0;
  } else if (a.axes == 1) {
    at[0] = n;
    at[1] = at[2] = 0;
  } else {
    const int row = n / a.grid_w, x = n - row * a.grid_w;
    if (a.axes == 2) {
      at[0] = row;
      at[1] = x;
      at[2] = 0;
    } else {
      at[0] = row / a.grid_h;
      at[1] = row - at[0] * a.grid_h;
      at[2] = x;
    }
  }
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (2 * (p + i) >= a.rot) break;
    const int where = p + i < a.pair0 ? at[0] : p + i < a.pair1 ? at[1] : at[2];
    const double t = a.turns[p + i] * where, rest = __builtin_fma(a.turns[p + i], static_cast<double>(where), -t);
    const double f = (t - __builtin_rint(t)) + (rest - __builtin_rint(rest));
    float sn, cs;
    sincospif(2.0f * static_cast<float>(f - __builtin_rint(f)), &sn, &cs);
    c[i] = cs * a.scale;
    s[i] = sn * (a.scale * a.sign);
  }
}

__device__ inline void turn(float& a, float& b, float c, float s) {
  const float x = __builtin_fmaf(a, c, -(b * s));
  b = __builtin_fmaf(a, s, b * c);
  a = x;
}

}  // namespace da2
