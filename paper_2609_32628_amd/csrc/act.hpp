// Activations of the projections and their derivatives, in float32, and eight values
// at a time of rows that may end inside them. Results are rounded to 16 bits after, so
// exponentials come from v_exp_f32 (relative error of e^x below |x| 2^-23) and quotients
// from v_rcp_f32.
#pragma once

#include "layer.hpp"
#include "tile.hpp"

namespace da2 {

__device__ inline float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }
__device__ inline float rcp_fast(float x) { return __builtin_amdgcn_rcpf(x); }

// Standard normal distribution function of z and exp(-z^2 / 2). The tail is
// erfc(x) / 2 with erfc(x) = exp(-x^2) q(1 / (1 + x / 2)), x = |z| / sqrt 2: q is a polynomial
// fitted to exp(x^2) erfc(x) over x in [0, 12], relative error 2.3e-6 in float32, so the small
// values of the negative side keep their digits.
__device__ inline float normal_cdf(float z, float& e) {
  e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
  const float t = rcp_fast(__builtin_fmaf(__builtin_fabsf(z), 0.35355339059327376f, 1.0f));
  float q = 0.08493691682815552f;
  q = __builtin_fmaf(q, t, -0.34534457325935364f);
  q = __builtin_fmaf(q, t, 0.3734673857688904f);
  q = __builtin_fmaf(q, t, 0.048874229192733765f);
  q = __builtin_fmaf(q, t, 0.2774653434753418f);
  q = __builtin_fmaf(q, t, 0.27831903100013733f);
  q = __builtin_fmaf(q, t, 0.2822796106338501f);
  const float tail = 0.5f * e * (q * t);
  return z < 0.0f ? tail : 1.0f - tail;
}

// f(z) and, where asked for, f'(z).
template <int ACT, bool D>
__device__ inline float act_one(float z, float& d) {
  if constexpr (ACT == DA2_ACT_RELU) {
    // a NaN stays one, in both; -inf gives 0
    if (D) d = z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;
    return z < 0.0f ? 0.0f : z;
  } else if constexpr (ACT == DA2_ACT_GELU) {
    float e;
    const float p = normal_cdf(z, e);
    if (D) d = __builtin_fmaf(z, e * 0.39894228040143268f, p);
    return z * p;
  } else if constexpr (ACT == DA2_ACT_GELU_TANH) {  // z (1 + tanh u) / 2 = z / (1 + exp(-2 u))
    constexpr float a = 2 * 0.79788456080286536f, b = a * 0.044715f;
    const float zz = z * z, p = rcp_fast(1.0f + exp_fast(-z * __builtin_fmaf(zz, b, a)));
    if (D) {
      // beyond 32 p is 0 or 1 and p - p p is 0, but its factor of z^3 would be infinite from 2^64 on, and 0 times that a NaN
      const float c = __builtin_amdgcn_fmed3f(z, -32.0f, 32.0f);
      d = __builtin_fmaf(c * (p - p * p), __builtin_fmaf(c * c, 3 * b, a), p);
    }
    return z * p;
  } else if constexpr (ACT == DA2_ACT_SILU) {
    const float p = rcp_fast(1.0f + exp_fast(-z));
    if (D) d = __builtin_fmaf(z, p - p * p, p);
    return z * p;
  } else if constexpr (ACT == DA2_ACT_SIGMOID) {
    // from the smaller side, where 1 - p would have no digits left (p - p p is off by 6% at 16 and 0 from 17 on)
    const float e = exp_fast(-__builtin_fabsf(z)), p = rcp_fast(1.0f + e);
    if (D) d = e * p * p;
    return z < 0.0f ? e * p : p;
  } else {
    if (D) d = 1.0f;
    return z;
  }
}
// Calls f<ACT>() (one branch for the whole wave).
template <typename F>
__device__ inline void with_act(int act, F&& f) {
  switch (act) {
    case DA2_ACT_RELU: return f.template operator()<DA2_ACT_RELU>();
    case DA2_ACT_GELU: return f.template operator()<DA2_ACT_GELU>();
    case DA2_ACT_GELU_TANH: return f.template operator()<DA2_ACT_GELU_TANH>();
    case DA2_ACT_SILU: return f.template operator()<DA2_ACT_SILU>();
    case DA2_ACT_SIGMOID: return f.template operator()<DA2_ACT_SIGMOID>();
    default: return f.template operator()<DA2_ACT_NONE>();
  }
}
__device__ inline void act8(int act, float* z) {
  with_act(act, [&]<int ACT>() {
    float d;
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = act_one<ACT, false>(z[i], d);
  });
}

// Stores the first n of eight values.
template <typename T>
__device__ inline void store8(void* p, int64_t at, int n, const float* x) {
  store_part(static_cast<T*>(p) + at, n, x);
}

// Stores the first n of eight floats.
__device__ inline void store_eight(float* p, int n, const float* x) {
  store_part(p, n, x);
  store_part(p + 4, n - 4, x + 4);
}

// Element offset of feature f of rows whose features are blocks of C, sh apart.
__device__ inline int64_t feature_at(int f, int H, int C, int64_t sh) {
  if (H == 1) return f;
  const int h = f / C;
  return h * sh + (f - h * C);
}

// Where a row's outputs, residual, gate and sums lie.
template <typename T, bool GLU>
struct RowPlace {
  T* y;
  const T *r, *gate;
  float* z;
  RowPlace() = default;
  __device__ RowPlace(const Finish& e, int64_t m) {
    const int b = static_cast<int>(static_cast<uint32_t>(m) / static_cast<uint32_t>(e.N));
    const int n = static_cast<int>(m - static_cast<int64_t>(b) * e.N);
    y = static_cast<T*>(e.y.p) + b * e.y.sb + n * e.y.sn;
    r = e.r.p ? static_cast<const T*>(e.r.p) + b * e.r.sb + n * e.r.sn : nullptr;
    gate = e.gate ? static_cast<const T*>(e.gate) + b * e.gate_sb : nullptr;
    z = e.z ? e.z + m * (GLU ? 2 : 1) * e.z_ld : nullptr;
  }
};

// Eight elements at p, of which n (at least one) are there, as they lie in memory; behind those the last one again.
template <typename T>
__device__ inline uint4 raw8(const T* p, int n) {
  uint4 v;
  if (n >= 8) {
    __builtin_memcpy(&v, p, 16);
  } else {
    const uint16_t* e = reinterpret_cast<const uint16_t*>(p);
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = e[min(i, n - 1)];
    v = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
  }
  return v;
}
// The first n of the eight elements of a 16-byte chunk, zeros behind them.
__device__ inline uint4 first8(const uint4& v, int n) {
  const auto keep = [&](uint32_t w, int i) { return n >= 2 * i + 2 ? w : n == 2 * i + 1 ? w & 0xFFFFu : 0u; };
  return make_uint4(keep(v.x, 0), keep(v.y, 1), keep(v.z, 2), keep(v.w, 3));
}
template <typename T>
__device__ inline float element(const uint4& v, int i) {
  return static_cast<float>(__builtin_bit_cast(Chunk<T>, v).v[i]);
}

// What the epilogue reads for features [f8, f8 + 8) of a row, asked for ahead. They lie in 32 features from fb on, a number
// that is the same for the whole wave, or fb = f8.
template <typename T, bool GLU>
struct Beside {
  uint4 bias, bias_u, gate, r;
  int64_t y;  // element offset of the outputs in the row
  Beside() = default;
  __device__ Beside(const Finish& e, const RowPlace<T, GLU>& row, int f8, int fb) {
    const int left = e.F - f8;
    // features are blocks of Cy; 32 of them lie in one where blocks are whole 32s
    const int h = e.Hy == 1 ? 0 : e.Cy % 32 == 0 ? fb / e.Cy : f8 / e.Cy, c = f8 - h * e.Cy;
    y = h * e.y.sh + c;
    if (e.bias) {
      bias = raw8(static_cast<const T*>(e.bias) + f8, left);
      if constexpr (GLU) bias_u = raw8(static_cast<const T*>(e.bias) + e.F + f8, left);
    }
    if (!GLU && e.gate) gate = raw8(row.gate + f8, left);
    if (!GLU && e.r.p) r = raw8(row.r + h * e.r.sh + c, left);
  }
};

// The factor of the sums, the same for all: through the scalar cache, since a vector load would wait for the copies issued before it.
template <typename T, bool GLU>
__device__ inline float back_of(const Finish& e) {
  if (GLU || !kScaledDz<T> || !e.back) return 1.0f;
  return *(const __attribute__((address_space(4))) float*)e.back;
}

// Features [f8, f8 + 8) of a row from their sums v (gated block: v and u).
template <typename T, bool GLU>
__device__ inline void finish8(const Finish& e, const RowPlace<T, GLU>& row, const Beside<T, GLU>& x, float back, float* v, float* u, int f8) {
  const int left = e.F - f8;
  if (!GLU && kScaledDz<T> && back != 1.0f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= back;
  }
  if (e.bias) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] += element<T>(x.bias, i);
      if constexpr (GLU) u[i] += element<T>(x.bias_u, i);
    }
  }
  if (e.z) {
    store_eight(row.z + f8, left, v);
    if constexpr (GLU) store_eight(row.z + e.z_ld + f8, left, u);
  }
  act8(e.act, v);
  if constexpr (GLU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= u[i];
  } else {
    if (e.gate) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= element<T>(x.gate, i);
    }
    if (e.r.p) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += element<T>(x.r, i);
    }
  }
  store8<T>(row.y, x.y, left, v);
}

}  // namespace da2
