// Host checks that the entry points of the token operators share: tensor descriptors
// against extents, rotary descriptors. Internal to libda2.
#pragma once

#include <algorithm>
#include <utility>

#include "host_util.hpp"
#include "token.hpp"

namespace da2 {

inline bool dtype_ok(int32_t t) { return t == DA2_BF16 || t == DA2_FP32 || t == DA2_FP16; }

// Extents of a [B, H, N, C] tensor.
struct Ext {
  int64_t B, H, N, C;
};

inline int32_t check_ext(const Ext& e) {
  if (e.B < 1 || e.H < 1 || e.N < 1 || e.C < 1) return DA2_ERR_INVALID_ARG;
  if (e.B > 65535 || e.H * e.N > (1ll << 31) - 1) return DA2_ERR_INVALID_ARG;
  return DA2_OK;
}

// A descriptor against the extents; an output's rows must not overlap: in the
// order of their strides, each dimension's rows end before its next begins.
inline int32_t check_view(const da2_tensor* t, const Ext& e, int32_t dtype, bool out) {
  if (!t || !dtype_ok(t->dtype) || t->dtype != dtype) return DA2_ERR_INVALID_ARG;
  std::pair<int64_t, int64_t> d[3] = {{t->stride_b, e.B}, {t->stride_h, e.H}, {t->stride_n, e.N}};
  for (auto& s : d) {
    if (s.second == 1) s.first = 0;
    if (s.first < 0 || s.first > (1ll << 40)) return DA2_ERR_INVALID_ARG;
  }
  if (!out) return DA2_OK;
  std::sort(d, d + 3);
  int64_t span = e.C;
  for (const auto& s : d) {
    if (s.second == 1) continue;
    if (s.first < span) return DA2_ERR_INVALID_ARG;
    // no memory holds more elements than that, and no later stride could be as large
    if (s.first > ((1ll << 60) - span) / (s.second - 1)) return DA2_ERR_INVALID_ARG;
    span += s.first * (s.second - 1);
  }
  return DA2_OK;
}

inline bool same_strides(const da2_tensor* a, const da2_tensor* b, const Ext& e) {
  return (e.B == 1 || a->stride_b == b->stride_b) && (e.H == 1 || a->stride_h == b->stride_h) &&
         (e.N == 1 || a->stride_n == b->stride_n);
}

// Kernels read no stride of an extent of 1 but multiply it by zero.
inline View view(const void* p, const da2_tensor* t) { return View{p, t->stride_b, t->stride_h, t->stride_n}; }
inline OutView out_view(void* p, const da2_tensor* t) { return OutView{p, t->stride_b, t->stride_h, t->stride_n}; }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Rotated channels of a block, or -1 for a descriptor that is not one.
inline int64_t rope_rot(const da2_rope_desc* r) {
  if (!r || (r->layout != DA2_ROPE_INTERLEAVED && r->layout != DA2_ROPE_HALF)) return -1;
  if (r->axes < 1 || r->axes > 3 || r->block < 2) return -1;
  int64_t rot = 0;
  for (int i = 0; i < 3; ++i) {
    const int32_t D = r->rot_axis[i];
    if (i < r->axes ? (D < 2 || D % 2) : D != 0) return -1;
    rot += D;
  }
  return rot <= r->block && r->block <= 65536 ? rot : -1;
}

}  // namespace da2
