// Shared by the token operators (row norms, rotary positions, differential
// attention): element types, 16-byte chunks at any alignment, tensor views and
// the host's descriptor checks. Internal to libda2.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/da2.h"

namespace da2 {

// A [B, H, N, C] tensor with C contiguous; strides in elements.
struct View {
  const void* p;
  int64_t sb, sh, sn;
};
struct OutView {
  void* p;
  int64_t sb, sh, sn;
};

// Element types and their arithmetic. Conversions to 16 bits round to nearest even.
typedef __bf16 bf16_t;
typedef _Float16 fp16_t;

template <typename T>
constexpr int kVec = 16 / static_cast<int>(sizeof(T));  // elements of a 16-byte chunk

// 16 bytes at the element's alignment: gfx950 loads and stores them with one
// instruction wherever they start.
template <typename T>
struct Chunk {
  T v[kVec<T>];
};

template <typename T>
__device__ inline void load_vec(const T* p, float* x) {
  Chunk<T> c;
  __builtin_memcpy(&c, p, 16);
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) x[i] = static_cast<float>(c.v[i]);
}
template <typename T>
__device__ inline void store_vec(T* p, const float* x) {
  Chunk<T> c;
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) c.v[i] = static_cast<T>(x[i]);
  __builtin_memcpy(p, &c, 16);
}
// The first n elements of a chunk (the others read as zero); n may be <= 0 or more than the chunk holds.
template <typename T>
__device__ inline void load_part(const T* p, int n, float* x) {
  if (n >= kVec<T>) {
    load_vec(p, x);
    return;
  }
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) x[i] = i < n ? static_cast<float>(p[i]) : 0.0f;
}
template <typename T>
__device__ inline void store_part(T* p, int n, const float* x) {
  if (n >= kVec<T>) {
    store_vec(p, x);
    return;
  }
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i)
    if (i < n) p[i] = static_cast<T>(x[i]);
}

// Calls f with a value of the element type of dtype (checked on the host before).
template <typename F>
inline hipError_t by_dtype(int32_t dtype, F&& f) {
  switch (dtype) {
    case DA2_BF16: return f(bf16_t{});
    case DA2_FP16: return f(fp16_t{});
    default: return f(float{});
  }
}

// ---- row norms (norm.hip) --------------------------------------------------------
struct NormArgs {
  View x, dy;
  OutView y, dx;  // null pointers: not asked for
  const void *w, *b;
  void *dw, *db;
  float* stats;         // written by the forward pass
  const float* rstats;  // read by the backward pass
  float* ws;
  int B, H, N, C;
  int dtype, wdtype, kind;
  float plus;           // 0 or 1, added to w
  int64_t w_sb;         // elements between the samples' weights; 0: shared
  double eps;
};
// Partial sums of the weight gradients: float32 [groups][parts][2][C]; a group
// is a sample of adaptive weights, or all rows.
int64_t norm_parts(int64_t rows, int64_t groups, int C, int dtype);
hipError_t launch_norm(const NormArgs& a, hipStream_t stream);
hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t stream);

// ---- rotary positions (rope.hip) ---------------------------------------------------
struct RopeArgs {
  View q, k;
  OutView qo, ko;
  const double* turns;
  const int32_t* pos;
  int64_t pos_sb;
  int B, Hq, Hk, N, d, block, rot;
  int axes, pair0, pair1;  // pairs of axis 0, and of axes 0 and 1 together
  int grid_h, grid_w;
  int layout, dtype;
  float scale, sign;       // sign of the sine: -1 turns back
  bool q_in_place, k_in_place;
};
hipError_t launch_rope(const RopeArgs& a, hipStream_t stream);

// ---- differential attention (diff_fwd.hip, diff_bwd.hip) ------------------------------
struct DiffArgs {
  View q, k, v;
  OutView o;
  const float* lam;
  const int32_t *kv_lens, *q_start;  // null: M keys; the queries are the last ones
  float* lse;           // written by the forward pass, or null
  float* ws;
  int B, Hq, Hk, N, M, d;
  int causal, dtype;
  float scale;
  // backward pass
  View dout;
  const float* rlse;
  OutView dq, dk, dv;
  float* dlam;
};
int64_t diff_fwd_ws_bytes(int B, int Hq, int Hk, int N, int M, int d);
int64_t diff_bwd_ws_bytes(int B, int Hq, int Hk, int N, int M, int d);
hipError_t launch_diff_fwd(const DiffArgs& a, hipStream_t stream);
hipError_t launch_diff_bwd(const DiffArgs& a, hipStream_t stream);

}  // namespace da2
