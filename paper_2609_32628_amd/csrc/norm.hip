// Row norms (layer norm, RMS norm), forward and backward.
//
// Forward: mean, then the mean of (x - mean)^2 from the same registers (two passes
// over registers, one over memory; no E[x^2] - mean^2, which loses what a large
// mean covers), y = (x - mean) rstd f + b.
// Backward: with g = dy f and xh = (x - mean) rstd,
//   dx = rstd (g - mean(g) - xh mean(g xh)),  dw = sum dy xh,  db = sum dy.
//
// Both are bound by memory: x in and y out, or x and dy in and dx out. A row
// stays in the registers of the threads that share it: TPR threads with K
// chunks of 16 bytes each, from part of a wave for narrow rows (a head's 64 or
// 128 channels) to a workgroup of 512 threads. Rows wider than that (4 chunks
// for each of 512 threads) are read again from the caches for each pass.
// The weight gradients are summed in registers over the rows of a workgroup,
// written as one partial row per workgroup and added up by a second kernel, so
// that their order is fixed.
#include "token.hpp"

namespace da2 {

namespace {

constexpr int kThreads = 256;   // workgroup of the rows that fit a wave or 256 threads
constexpr int kMaxK = 4;        // chunks per thread
constexpr int kLong = 512;      // workgroup of wider rows (1,024 threads would leave the gradients 128 registers)

struct RowAt {
  int64_t x, y, dy, dx, row;
};

// Where row r of group grp is (grouped: a group is a sample; else rows run over the samples).
__device__ inline RowAt row_at(const NormArgs& a, int64_t r, int grp, bool grouped) {
  const uint32_t hn = static_cast<uint32_t>(a.H) * static_cast<uint32_t>(a.N);
  uint32_t b = static_cast<uint32_t>(grp), rem = static_cast<uint32_t>(r);
  if (!grouped) {
    b = rem / hn;
    rem -= b * hn;
  }
  uint32_t h = 0, n = rem;
  if (a.H > 1) {
    h = rem / static_cast<uint32_t>(a.N);
    n = rem - h * static_cast<uint32_t>(a.N);
  }
  RowAt o;
  o.x = b * a.x.sb + h * a.x.sh + n * a.x.sn;
  o.y = b * a.y.sb + h * a.y.sh + n * a.y.sn;
  o.dy = b * a.dy.sb + h * a.dy.sh + n * a.dy.sn;
  o.dx = b * a.dx.sb + h * a.dx.sh + n * a.dx.sn;
  o.row = static_cast<int64_t>(b) * hn + rem;
  return o;
}

// n weights (or biases) from element j of the group's on, as floats.
template <int V>
__device__ inline void load_weights(const void* w, int dtype, int64_t j, int n, float* out) {
  if (dtype == DA2_FP32) {
    const float* p = static_cast<const float*>(w) + j;
    if (n >= V) {
      Chunk<float> c[V / 4];
      __builtin_memcpy(c, p, 4 * V);
#pragma unroll
      for (int i = 0; i < V; ++i) out[i] = c[i / 4].v[i % 4];
      return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = i < n ? p[i] : 0.0f;
    return;
  }
  const uint16_t* p = static_cast<const uint16_t*>(w) + j;
  uint16_t bits[V];
  if (n >= V) {
    __builtin_memcpy(bits, p, 2 * V);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) bits[i] = i < n ? p[i] : 0;
  }
#pragma unroll
  for (int i = 0; i < V; ++i)
    out[i] = dtype == DA2_BF16 ? __uint_as_float(static_cast<uint32_t>(bits[i]) << 16)
                               : static_cast<float>(__builtin_bit_cast(fp16_t, bits[i]));
}

__device__ inline void store_weight(void* w, int dtype, int64_t j, float v) {
  if (dtype == DA2_FP32) {
    static_cast<float*>(w)[j] = v;
  } else if (dtype == DA2_BF16) {
    static_cast<bf16_t*>(w)[j] = static_cast<bf16_t>(v);
  } else {
    static_cast<fp16_t*>(w)[j] = static_cast<fp16_t>(v);
  }
}

// Sums of N values over the TPR threads that share a row; every thread gets them.
template <int TPR, int N>
__device__ inline void row_sum(float (&v)[N], float* lds) {
#pragma unroll
  for (int o = (TPR < 64 ? TPR : 64) / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], o, 64);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    const int wave = threadIdx.x / 64;
    __syncthreads();  // the last sums have been read
    if (threadIdx.x % 64 == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) lds[wave * N + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = lds[i];
#pragma unroll
      for (int w = 1; w < W; ++w) s += lds[w * N + i];
      v[i] = s;
    }
  }
}

template <int TPR>
constexpr int block_of() {
  return TPR > kThreads ? TPR : kThreads;
}

template <typename T, int TPR, int K>
__global__ __launch_bounds__(block_of<TPR>()) void norm_kernel(NormArgs a, int64_t rows, int grouped) {
  constexpr int V = kVec<T>, RPB = block_of<TPR>() / TPR;
  __shared__ float lds[TPR > 64 ? TPR / 64 : 1];
  const int lane = threadIdx.x % TPR, grp = blockIdx.y;
  const float inv = 1.0f / static_cast<float>(a.C);
  const int64_t w0 = grp * a.w_sb;
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * RPB; r0 < rows; r0 += static_cast<int64_t>(gridDim.x) * RPB) {
    int64_t r = r0 + threadIdx.x / TPR;
    const bool live = r < rows;  // every thread takes part in the sums
    r = live ? r : rows - 1;
    const RowAt at = row_at(a, r, grp, grouped);
    const T* x = static_cast<const T*>(a.x.p) + at.x;
    float v[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int j = (lane + k * TPR) * V;
      load_part(x + j, a.C - j, v[k]);
    }
    float mean = 0.0f;
    if (a.kind == DA2_NORM_LAYER) {
      float s[1] = {0.0f};
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) s[0] += v[k][i];
      row_sum<TPR>(s, lds);
      mean = s[0] * inv;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int n = a.C - (lane + k * TPR) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[k][i] = i < n ? v[k][i] - mean : 0.0f;
        q[0] = __builtin_fmaf(v[k][i], v[k][i], q[0]);
      }
    }
    row_sum<TPR>(q, lds);
    const float rstd = 1.0f / __builtin_sqrtf(q[0] * inv + static_cast<float>(a.eps));
    if (!live) continue;
    if (a.stats && lane == 0) {
      a.stats[2 * at.row] = mean;
      a.stats[2 * at.row + 1] = rstd;
    }
    T* y = static_cast<T*>(a.y.p) + at.y;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int j = (lane + k * TPR) * V, n = a.C - j;
      float f[V], o[V];
      if (a.w) load_weights<V>(a.w, a.wdtype, w0 + j, n, f);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        o[i] = v[k][i] * rstd;
        if (a.w) o[i] *= f[i] + a.plus;
      }
      if (a.b) {
        load_weights<V>(a.b, a.wdtype, w0 + j, n, f);
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] += f[i];
      }
      store_part(y + j, n, o);
    }
  }
}

// Rows that do not fit a workgroup's registers: one workgroup per row, one pass over the row for each of the mean, the
// variance and the output (the later ones from the caches).
template <typename T>
__device__ inline void norm_long_row(const NormArgs& a, int64_t r, int grp, bool grouped, float* lds) {
  constexpr int V = kVec<T>;
  const RowAt at = row_at(a, r, grp, grouped);
  const T* x = static_cast<const T*>(a.x.p) + at.x;
  const float inv = 1.0f / static_cast<float>(a.C);
  float mean = 0.0f, v[V];
  if (a.kind == DA2_NORM_LAYER) {
    float s[1] = {0.0f};
    for (int64_t j = threadIdx.x * V; j < a.C; j += kLong * V) {
      load_part(x + j, static_cast<int>(a.C - j), v);
#pragma unroll
      for (int i = 0; i < V; ++i) s[0] += v[i];
    }
    row_sum<kLong>(s, lds);
    mean = s[0] * inv;
  }
  float q[1] = {0.0f};
  for (int64_t j = threadIdx.x * V; j < a.C; j += kLong * V) {
    const int n = static_cast<int>(a.C - j);
    load_part(x + j, n, v);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float d = i < n ? v[i] - mean : 0.0f;
      q[0] = __builtin_fmaf(d, d, q[0]);
    }
  }
  row_sum<kLong>(q, lds);
  const float rstd = 1.0f / __builtin_sqrtf(q[0] * inv + static_cast<float>(a.eps));
  if (a.stats && threadIdx.x == 0) {
    a.stats[2 * at.row] = mean;
    a.stats[2 * at.row + 1] = rstd;
  }
  T* y = static_cast<T*>(a.y.p) + at.y;
  const int64_t w0 = grp * a.w_sb;
  for (int64_t j = threadIdx.x * V; j < a.C; j += kLong * V) {
    const int n = static_cast<int>(a.C - j);
    float f[V];
    load_part(x + j, n, v);
    if (a.w) load_weights<V>(a.w, a.wdtype, w0 + j, n, f);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      v[i] = (v[i] - mean) * rstd;
      if (a.w) v[i] *= f[i] + a.plus;
    }
    if (a.b) {
      load_weights<V>(a.b, a.wdtype, w0 + j, n, f);
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] += f[i];
    }
    store_part(y + j, n, v);
  }
}

template <typename T>
__global__ __launch_bounds__(kLong) void norm_long_kernel(NormArgs a, int64_t rows, int grouped) {
  __shared__ float lds[kLong / 64];
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) norm_long_row<T>(a, r, blockIdx.y, grouped, lds);
}

// ---- backward ------------------------------------------------------------------
// A workgroup walks the rows blockIdx.x * RPB + {0 .. RPB-1}, then gridDim.x * RPB further, and so on; SUMS: with the
// weights' gradients.
template <typename T, int TPR, int K, bool SUMS>
__global__ __launch_bounds__(block_of<TPR>()) void norm_bwd_kernel(NormArgs a, int64_t rows, int grouped) {
  constexpr int V = kVec<T>, BLOCK = block_of<TPR>(), RPB = BLOCK / TPR;
  __shared__ float lds[TPR > 64 ? 2 * TPR / 64 : 1];
  const int lane = threadIdx.x % TPR, grp = blockIdx.y;
  const float inv = 1.0f / static_cast<float>(a.C);
  const int64_t w0 = grp * a.w_sb;
  float f[K][V], sw[SUMS ? K : 1][V], sb[SUMS ? K : 1][V];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int j = (lane + k * TPR) * V;
#pragma unroll
    for (int i = 0; i < V; ++i) f[k][i] = 1.0f - a.plus;
    if (a.w) load_weights<V>(a.w, a.wdtype, w0 + j, a.C - j, f[k]);
#pragma unroll
    for (int i = 0; i < V; ++i) f[k][i] += a.plus;
  }
  if constexpr (SUMS)
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) sw[k][i] = sb[k][i] = 0.0f;

  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * RPB; r0 < rows; r0 += static_cast<int64_t>(gridDim.x) * RPB) {
    int64_t r = r0 + threadIdx.x / TPR;
    const bool live = r < rows;
    r = live ? r : rows - 1;
    const RowAt at = row_at(a, r, grp, grouped);
    const T* x = static_cast<const T*>(a.x.p) + at.x;
    const T* dy = static_cast<const T*>(a.dy.p) + at.dy;
    float xh[K][V], g[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int j = (lane + k * TPR) * V;
      load_part(x + j, a.C - j, xh[k]);
      load_part(dy + j, live ? a.C - j : 0, g[k]);  // rows behind the last add nothing
    }
    const float mean = a.rstats[2 * at.row], rstd = a.rstats[2 * at.row + 1];
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int n = live ? a.C - (lane + k * TPR) * V : 0;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        xh[k][i] = i < n ? (xh[k][i] - mean) * rstd : 0.0f;
        if constexpr (SUMS) {
          sw[k][i] = __builtin_fmaf(g[k][i], xh[k][i], sw[k][i]);
          sb[k][i] += g[k][i];
        }
        g[k][i] *= f[k][i];
        s[0] += g[k][i];
        s[1] = __builtin_fmaf(g[k][i], xh[k][i], s[1]);
      }
    }
    if (!a.dx.p) continue;
    row_sum<TPR>(s, lds);
    if (!live) continue;
    const float m0 = a.kind == DA2_NORM_LAYER ? s[0] * inv : 0.0f, m1 = s[1] * inv;
    T* dx = static_cast<T*>(a.dx.p) + at.dx;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int j = (lane + k * TPR) * V;
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = rstd * (g[k][i] - __builtin_fmaf(xh[k][i], m1, m0));
      store_part(dx + j, a.C - j, o);
    }
  }
  if constexpr (SUMS) {
    // the workgroup's rows are added up: over the row groups of a wave, then over its waves
    float* part = a.ws + (static_cast<int64_t>(grp) * gridDim.x + blockIdx.x) * 2 * a.C;
    constexpr int SPAN = TPR < 64 ? TPR : 64;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int o = SPAN; o < 64; o <<= 1) {
          sw[k][i] += __shfl_xor(sw[k][i], o, 64);
          sb[k][i] += __shfl_xor(sb[k][i], o, 64);
        }
    constexpr int WAVES = TPR <= 64 ? BLOCK / 64 : 1;  // waves that hold the same columns
    if constexpr (WAVES == 1) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int j = (lane + k * TPR) * V;
#pragma unroll
        for (int q = 0; q < V; q += 4) {
          store_part(part + j + q, a.C - j - q, sw[k] + q);
          store_part(part + a.C + j + q, a.C - j - q, sb[k] + q);
        }
      }
    } else {
      __shared__ float cols[WAVES][2][SPAN * V];
      const int wave = threadIdx.x / 64;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (k) __syncthreads();
        if (threadIdx.x % 64 < SPAN)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            cols[wave][0][lane * V + i] = sw[k][i];
            cols[wave][1][lane * V + i] = sb[k][i];
          }
        __syncthreads();
        for (int e = threadIdx.x; e < 2 * SPAN * V; e += BLOCK) {
          const int which = e / (SPAN * V), c = e % (SPAN * V), j = k * TPR * V + c;
          float t = cols[0][which][c];
#pragma unroll
          for (int w = 1; w < WAVES; ++w) t += cols[w][which][c];
          if (j < a.C) part[which * a.C + j] = t;
        }
      }
    }
  }
}

// Wide rows: dx by one workgroup per row, in two passes.
template <typename T>
__device__ inline void norm_bwd_long_row(const NormArgs& a, int64_t r, int grp, bool grouped, float* lds) {
  constexpr int V = kVec<T>;
  const RowAt at = row_at(a, r, grp, grouped);
  const T* x = static_cast<const T*>(a.x.p) + at.x;
  const T* dy = static_cast<const T*>(a.dy.p) + at.dy;
  T* dx = static_cast<T*>(a.dx.p) + at.dx;
  const float inv = 1.0f / static_cast<float>(a.C);
  const float mean = a.rstats[2 * at.row], rstd = a.rstats[2 * at.row + 1];
  const int64_t w0 = grp * a.w_sb;
  float s[2] = {0.0f, 0.0f}, xh[V], g[V], f[V];
  auto at_chunk = [&](int64_t j) {
    const int n = static_cast<int>(a.C - j);
    load_part(x + j, n, xh);
    load_part(dy + j, n, g);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = 1.0f - a.plus;
    if (a.w) load_weights<V>(a.w, a.wdtype, w0 + j, n, f);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      xh[i] = i < n ? (xh[i] - mean) * rstd : 0.0f;
      g[i] = i < n ? g[i] * (f[i] + a.plus) : 0.0f;
    }
  };
  for (int64_t j = threadIdx.x * V; j < a.C; j += kLong * V) {
    at_chunk(j);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      s[0] += g[i];
      s[1] = __builtin_fmaf(g[i], xh[i], s[1]);
    }
  }
  row_sum<kLong>(s, lds);
  const float m0 = a.kind == DA2_NORM_LAYER ? s[0] * inv : 0.0f, m1 = s[1] * inv;
  for (int64_t j = threadIdx.x * V; j < a.C; j += kLong * V) {
    at_chunk(j);
    float o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = rstd * (g[i] - __builtin_fmaf(xh[i], m1, m0));
    store_part(dx + j, static_cast<int>(a.C - j), o);
  }
}

template <typename T>
__global__ __launch_bounds__(kLong) void norm_bwd_long_kernel(NormArgs a, int64_t rows, int grouped) {
  __shared__ float lds[2 * kLong / 64];
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) norm_bwd_long_row<T>(a, r, blockIdx.y, grouped, lds);
}

// Wide rows: partial sums of the weights' gradients. A workgroup takes 256 chunks of columns and every gridDim.x-th row.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_cols_kernel(NormArgs a, int64_t rows, int grouped, int tiles) {
  constexpr int V = kVec<T>;
  const int grp = blockIdx.y, tile = blockIdx.x % tiles, part_i = blockIdx.x / tiles, parts = gridDim.x / tiles;
  const int64_t j = (static_cast<int64_t>(tile) * kThreads + threadIdx.x) * V;
  const int n = static_cast<int>(a.C - j);
  if (n <= 0) return;
  float sw[V] = {}, sb[V] = {}, x[V], g[V];
  for (int64_t r = part_i; r < rows; r += parts) {
    const RowAt at = row_at(a, r, grp, grouped);
    const float mean = a.rstats[2 * at.row], rstd = a.rstats[2 * at.row + 1];
    load_part(static_cast<const T*>(a.x.p) + at.x + j, n, x);
    load_part(static_cast<const T*>(a.dy.p) + at.dy + j, n, g);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      sw[i] = __builtin_fmaf(g[i], (x[i] - mean) * rstd, sw[i]);
      sb[i] += g[i];
    }
  }
  float* part = a.ws + (static_cast<int64_t>(grp) * parts + part_i) * 2 * a.C;
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < n) {
      part[j + i] = sw[i];
      part[a.C + j + i] = sb[i];
    }
}

// The partial rows of a group added up: a workgroup takes 64 columns of dw or db; its four waves take every fourth
// partial, and their sums are added in order.
__global__ __launch_bounds__(kThreads) void norm_reduce_kernel(NormArgs a, int parts) {
  __shared__ float sums[kThreads];
  const int grp = blockIdx.y, which = blockIdx.z, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  void* out = which ? a.db : a.dw;
  if (!out) return;
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 64 + lane;
  float t = 0.0f;
  if (c < a.C) {
    const float* p = a.ws + (static_cast<int64_t>(grp) * parts * 2 + which) * a.C + c;
#pragma unroll 8
    for (int i = wave; i < parts; i += kThreads / 64) t += p[static_cast<int64_t>(i) * 2 * a.C];
  }
  sums[threadIdx.x] = t;
  __syncthreads();
  if (wave == 0 && c < a.C)
    store_weight(out, a.wdtype, grp * a.w_sb + c, (sums[lane] + sums[64 + lane]) + (sums[128 + lane] + sums[192 + lane]));
}

// Threads per row and chunks per thread for rows of nv chunks: part of a wave as
// far as one chunk a thread goes, then a wave, 256 and 512 threads with up to 4.
struct Shape {
  int tpr, k;  // k = 0: the row does not fit
};
Shape shape_of(int C, int vec) {
  const int nv = (C - 1) / vec + 1;
  if (nv <= 64) {
    int t = 1;
    while (t < nv) t *= 2;
    return {t, 1};
  }
  for (int t : {64, 256, kLong})
    if (nv <= kMaxK * t) return {t, (nv + t - 1) / t};
  return {kLong, 0};
}

// Calls f<TPR, K>() for the shape.
template <typename F>
hipError_t with_shape(Shape s, F&& f) {
  switch (s.tpr) {
    case 1: return f.template operator()<1, 1>();
    case 2: return f.template operator()<2, 1>();
    case 4: return f.template operator()<4, 1>();
    case 8: return f.template operator()<8, 1>();
    case 16: return f.template operator()<16, 1>();
    case 32: return f.template operator()<32, 1>();
    case 64:
      if (s.k == 1) return f.template operator()<64, 1>();
      if (s.k == 2) return f.template operator()<64, 2>();
      if (s.k == 3) return f.template operator()<64, 3>();
      return f.template operator()<64, 4>();
    case 256:
      if (s.k == 2) return f.template operator()<256, 2>();
      if (s.k == 3) return f.template operator()<256, 3>();
      return f.template operator()<256, 4>();
    default:
      if (s.k == 2) return f.template operator()<kLong, 2>();
      if (s.k == 3) return f.template operator()<kLong, 3>();
      return f.template operator()<kLong, 4>();
  }
}

// Workgroups for n units of work: the kernels walk what is beyond (a grid dimension ends at 2^32 threads).
unsigned blocks_for(int64_t n) { return static_cast<unsigned>(n < (1 << 21) ? n : (1 << 21)); }

int rows_per_block(int tpr) { return tpr >= kThreads ? 1 : kThreads / tpr; }

}  // namespace

int64_t norm_parts(int64_t rows, int64_t groups, int C, int dtype) {
  const Shape s = shape_of(C, dtype == DA2_FP32 ? 4 : 8);
  const int64_t rpb = s.k ? rows_per_block(s.tpr) : 1;
  // a workgroup's partial row costs as much as some of its rows, so it walks 16 of
  // them at least; 1,024 workgroups fill the card
  const int64_t most = (rows + 16 * rpb - 1) / (16 * rpb), fill = (1024 + groups - 1) / groups;
  return most < fill ? most : fill;
}

hipError_t launch_norm(const NormArgs& a, hipStream_t stream) {
  const bool grouped = a.w_sb != 0;
  const int64_t all = static_cast<int64_t>(a.B) * a.H * a.N, groups = grouped ? a.B : 1, rows = all / groups;
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    const Shape s = shape_of(a.C, kVec<T>);
    if (!s.k) {
      norm_long_kernel<T><<<dim3(blocks_for(rows), groups), kLong, 0, stream>>>(a, rows, grouped);
      return hipGetLastError();
    }
    return with_shape(s, [&]<int TPR, int K>() {
      constexpr int RPB = block_of<TPR>() / TPR;
      norm_kernel<T, TPR, K><<<dim3(blocks_for((rows + RPB - 1) / RPB), groups), block_of<TPR>(), 0, stream>>>(a, rows, grouped);
      return hipGetLastError();
    });
  });
}

hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t stream) {
  const bool grouped = a.w_sb != 0, sums = a.dw || a.db;
  const int64_t all = static_cast<int64_t>(a.B) * a.H * a.N, groups = grouped ? a.B : 1, rows = all / groups;
  const int64_t parts = norm_parts(rows, groups, a.C, a.dtype);
  const hipError_t e = by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    const Shape s = shape_of(a.C, kVec<T>);
    if (!s.k) {
      const int tiles = static_cast<int>((a.C + static_cast<int64_t>(kThreads) * kVec<T> - 1) / (kThreads * kVec<T>));
      // the sums first: dX may be the memory of X or dY
      if (sums) norm_cols_kernel<T><<<dim3(parts * tiles, groups), kThreads, 0, stream>>>(a, rows, grouped, tiles);
      if (a.dx.p) norm_bwd_long_kernel<T><<<dim3(blocks_for(rows), groups), kLong, 0, stream>>>(a, rows, grouped);
      return hipGetLastError();
    }
    return with_shape(s, [&]<int TPR, int K>() {
      constexpr int RPB = block_of<TPR>() / TPR;
      if (sums) {
        norm_bwd_kernel<T, TPR, K, true><<<dim3(parts, groups), block_of<TPR>(), 0, stream>>>(a, rows, grouped);
      } else {
        norm_bwd_kernel<T, TPR, K, false>
            <<<dim3(blocks_for((rows + RPB - 1) / RPB), groups), block_of<TPR>(), 0, stream>>>(a, rows, grouped);
      }
      return hipGetLastError();
    });
  });
  if (e != hipSuccess || !sums) return e;
  norm_reduce_kernel<<<dim3((a.C + 63) / 64, groups, 2), kThreads, 0, stream>>>(a, static_cast<int>(parts));
  return hipGetLastError();
}

}  // namespace da2
