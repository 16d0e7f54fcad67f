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
// for each of 512 threads, 3 in the backward pass) are read again from the caches
// for each pass. A workgroup walks over rows and fetches the next one before it
// works on this one. (bf16, 32,760 rows of 1,536: 44 us, 4.6 TB/s; 16,380 of 5,120:
// 61 us forward and 110 backward, 5.5 and 4.6 TB/s; a copy reaches 5.0 to 5.4.)
// The weight gradients are summed in registers over the rows of a workgroup,
// written as one partial row per workgroup and added up by a second kernel, so
// that their order is fixed.
#include "common.hpp"
#include "token.hpp"

namespace da2 {

namespace {

constexpr int kFwdK = 4, kBwdK = 3;  // chunks per thread
constexpr int kThreads = 256;   // workgroup of the rows that fit a wave or 256 threads
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

// 16 bytes of a row from element j on, as they lie in memory, and their values, zeros from element C on. No branch depends
// on the lane, and nothing is done with the bytes before they are needed, so that all chunks of a thread and the next
// row's are in flight together: lanes behind the row read its last 16 bytes, and where C is no whole number of chunks
// (TAIL), the last chunk is those, shifted down. Only a thread's last chunk (`last`, a constant) may end behind the row.
template <bool TAIL, typename T>
__device__ inline uint4 fetch(const T* row, int j, int C, bool last) {
  constexpr int V = kVec<T>;
  uint4 c;
  if (!last) {
    __builtin_memcpy(&c, row + j, 16);
  } else if (!TAIL || C >= V) {
    __builtin_memcpy(&c, row + min(j, C - V), 16);
  } else {  // a row of less than a chunk: one element at a time, the last one again behind it
    T e[V];
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = row[min(i, C - 1)];
    __builtin_memcpy(&c, e, 16);
  }
  return c;
}
template <bool TAIL, typename T>
__device__ inline void unpack(const uint4& c, int j, int C, bool last, float* x) {
  constexpr int V = kVec<T>;
  uint32_t w0 = c.x, w1 = c.y, w2 = c.z, w3 = c.w;
  if (TAIL && last && C >= V) {
    const int off = min(max(j + V - C, 0), V) * static_cast<int>(sizeof(T));  // bytes that go
    if constexpr (sizeof(T) == 2) {
      const bool odd = off & 2;
      w0 = odd ? __builtin_amdgcn_alignbit(w1, w0, 16) : w0;
      w1 = odd ? __builtin_amdgcn_alignbit(w2, w1, 16) : w1;
      w2 = odd ? __builtin_amdgcn_alignbit(w3, w2, 16) : w2;
      w3 = odd ? w3 >> 16 : w3;
    }
    const bool one = off & 4, two = off & 8;
    w0 = one ? w1 : w0;
    w1 = one ? w2 : w1;
    w2 = one ? w3 : w2;
    w3 = one ? 0 : w3;
    w0 = two ? w2 : w0;
    w1 = two ? w3 : w1;
    w2 = two ? 0 : w2;
    w3 = two ? 0 : w3;
  }
  const uint4 z = make_uint4(w0, w1, w2, w3);
  const Chunk<T> e = __builtin_bit_cast(Chunk<T>, z);
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = !last || (TAIL && C < V ? j + i < C : j < C) ? static_cast<float>(e.v[i]) : 0.0f;
}

// V weights (or biases) of float32 or 16 bits from element j on as floats; behind C they are any.
template <bool TAIL, int V>
__device__ inline void load_weights(const void* w, int dtype, int64_t base, int j, int C, bool last, float* x) {
  const int es = dtype == DA2_FP32 ? 4 : 2;
  const char* p = static_cast<const char*>(w) + base * es;
  uint32_t bits[V];  // as they lie in memory, 16-bit ones in the first V / 2; or an element each
  const bool each = TAIL && last;
  if (!each) {
    p += (last ? min(j, C - V) : j) * es;
    __builtin_memcpy(bits, p, 2 * V);
    __builtin_memcpy(bits + V / 2, p + (es == 4 ? 2 * V : 0), 2 * V);
  } else if (es == 4) {
#pragma unroll
    for (int i = 0; i < V; ++i) bits[i] = reinterpret_cast<const uint32_t*>(p)[min(j + i, C - 1)];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) bits[i] = reinterpret_cast<const uint16_t*>(p)[min(j + i, C - 1)];
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t h = each ? bits[i] : bits[i / 2] >> (16 * (i % 2));
    if (dtype == DA2_FP32) {
      x[i] = __uint_as_float(bits[i]);
    } else if (dtype == DA2_BF16) {
      x[i] = __uint_as_float(h << 16);
    } else {
      x[i] = static_cast<float>(__builtin_bit_cast(fp16_t, static_cast<uint16_t>(h)));
    }
  }
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
    const int wave = threadIdx.x / 64, first = wave / W * W;  // of the row
    __syncthreads();  // the last sums have been read
    if (threadIdx.x % 64 == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) lds[wave * N + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = lds[first * N + i];
#pragma unroll
      for (int w = 1; w < W; ++w) s += lds[(first + w) * N + i];
      v[i] = s;
    }
  }
}

// Waves a SIMD that the registers of n elements a thread leave room for, and the workgroups that bring the card that many
// (256 CUs of 4 SIMDs): the kernels walk over rows with as many as run at once, so that their weights and sums stay in
// registers. (5,120 columns backward: 111 us with 512 workgroups, 144 with 768; 1,536 forward: 37 us with 1,024 and 46
// with a workgroup for each four rows.)
constexpr int fwd_waves(int n, int tpr) { return n <= 8 ? 6 : n <= 16 || (n <= 24 && tpr <= 64) ? 4 : 3; }
constexpr int bwd_waves(int n) { return n <= 8 ? 4 : n <= 16 ? 3 : 2; }
constexpr int64_t resident(int waves, int block) { return 256ll * (256 * waves / block); }

template <int TPR>
constexpr int block_of() {
  return TPR > kThreads ? TPR : kThreads;
}

template <typename T, int TPR, int K, bool TAIL>
__global__ __launch_bounds__(block_of<TPR>(), fwd_waves(K * kVec<T>, TPR)) void norm_kernel(NormArgs a, int64_t rows, int grouped) {
  constexpr int V = kVec<T>, RPB = block_of<TPR>() / TPR;
  __shared__ float lds[TPR > 64 ? block_of<TPR>() / 64 : 1];
  const int lane = threadIdx.x % TPR, grp = blockIdx.y;
  const float inv = 1.0f / static_cast<float>(a.C);
  const int64_t w0 = grp * a.w_sb, step = static_cast<int64_t>(gridDim.x) * RPB;
  // the weights stay, and the next row's chunks are on their way while a row is worked on
  uint4 raw[K] = {};
  RowAt at{}, next{};
  const auto ask = [&](int64_t r) {
    if (r >= rows) return;
    next = row_at(a, r, grp, grouped);
#pragma unroll
    for (int k = 0; k < K; ++k) raw[k] = fetch<TAIL>(static_cast<const T*>(a.x.p) + next.x, (lane + k * TPR) * V, a.C, k == K - 1);
  };
  ask(static_cast<int64_t>(blockIdx.x) * RPB + threadIdx.x / TPR);
  float f[K][V], bias[K][V];
#pragma unroll
  for (int k = 0; k < K; ++k) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      f[k][i] = 1.0f - a.plus;
      bias[k][i] = 0.0f;
    }
    if (a.w) load_weights<TAIL, V>(a.w, a.wdtype, w0, (lane + k * TPR) * V, a.C, k == K - 1, f[k]);
    if (a.b) load_weights<TAIL, V>(a.b, a.wdtype, w0, (lane + k * TPR) * V, a.C, k == K - 1, bias[k]);
#pragma unroll
    for (int i = 0; i < V; ++i) f[k][i] += a.plus;
  }
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * RPB; r0 < rows; r0 += step) {
    const bool live = r0 + threadIdx.x / TPR < rows;  // every thread takes part in the sums
    float v[K][V], mean = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) unpack<TAIL, T>(raw[k], (lane + k * TPR) * V, a.C, k == K - 1, v[k]);
    at = next;
    ask(r0 + step + threadIdx.x / TPR);
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
        v[k][i] = k < K - 1 || i < n ? v[k][i] - mean : 0.0f;
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
      const int j = (lane + k * TPR) * V;
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = __builtin_fmaf(v[k][i] * rstd, f[k][i], bias[k][i]);
      store_part(y + j, k < K - 1 ? V : a.C - j, o);
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
    if (a.w) load_weights<true, V>(a.w, a.wdtype, w0, static_cast<int>(j), a.C, j + V > a.C, f);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      v[i] = (v[i] - mean) * rstd;
      if (a.w) v[i] *= f[i] + a.plus;
    }
    if (a.b) {
      load_weights<true, V>(a.b, a.wdtype, w0, static_cast<int>(j), a.C, j + V > a.C, f);
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
template <typename T, int TPR, int K, bool TAIL, bool SUMS>
__global__ __launch_bounds__(block_of<TPR>(), SUMS ? bwd_waves(K * kVec<T>) : 2) void norm_bwd_kernel(NormArgs a, int64_t rows, int grouped) {
  constexpr int V = kVec<T>, BLOCK = block_of<TPR>(), RPB = BLOCK / TPR;
  __shared__ float lds[TPR > 64 ? 2 * block_of<TPR>() / 64 : 1];
  const int lane = threadIdx.x % TPR, grp = blockIdx.y;
  const float inv = 1.0f / static_cast<float>(a.C);
  const int64_t w0 = grp * a.w_sb;
  float f[K][V], sw[SUMS ? K : 1][V], sb[SUMS ? K : 1][V];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int j = (lane + k * TPR) * V;
#pragma unroll
    for (int i = 0; i < V; ++i) f[k][i] = 1.0f - a.plus;
    if (a.w) load_weights<TAIL, V>(a.w, a.wdtype, w0, j, a.C, k == K - 1, f[k]);
#pragma unroll
    for (int i = 0; i < V; ++i) f[k][i] += a.plus;
  }
  if constexpr (SUMS)
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) sw[k][i] = sb[k][i] = 0.0f;

  // the next row's chunks are on their way while a row is worked on
  const int64_t step = static_cast<int64_t>(gridDim.x) * RPB;
  uint4 xr[K] = {}, gr[K] = {};
  float mean = 0.0f, rstd = 0.0f;
  RowAt at{}, next{};
  const auto ask = [&](int64_t r) {
    if (r >= rows) return;
    next = row_at(a, r, grp, grouped);
    const T* x = static_cast<const T*>(a.x.p) + next.x;
    const T* dy = static_cast<const T*>(a.dy.p) + next.dy;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      xr[k] = fetch<TAIL>(x, (lane + k * TPR) * V, a.C, k == K - 1);
      gr[k] = fetch<TAIL>(dy, (lane + k * TPR) * V, a.C, k == K - 1);
    }
    mean = a.rstats[2 * next.row];
    rstd = a.rstats[2 * next.row + 1];
  };
  ask(static_cast<int64_t>(blockIdx.x) * RPB + threadIdx.x / TPR);
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * RPB; r0 < rows; r0 += step) {
    const bool live = r0 + threadIdx.x / TPR < rows;
    float xh[K][V], g[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      unpack<TAIL, T>(xr[k], (lane + k * TPR) * V, a.C, k == K - 1, xh[k]);
      unpack<TAIL, T>(gr[k], (lane + k * TPR) * V, a.C, k == K - 1, g[k]);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        xh[k][i] = (xh[k][i] - mean) * rstd;
        g[k][i] = live ? g[k][i] : 0.0f;  // rows behind the last add nothing, nor do elements behind C: they are zeros
      }
    }
    const float scale = rstd;
    at = next;
    ask(r0 + step + threadIdx.x / TPR);
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
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
      for (int i = 0; i < V; ++i) o[i] = scale * (g[k][i] - __builtin_fmaf(xh[k][i], m1, m0));
      store_part(dx + j, k < K - 1 ? V : a.C - j, o);
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
    constexpr int WAVES = BLOCK / (TPR < 64 ? 64 : TPR);  // rows of the workgroup (groups of rows of a wave) that hold the same columns
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
      constexpr int SHARE = TPR < 64 ? 64 : TPR, COLS = TPR * V;
      __shared__ float cols[WAVES][2][COLS];
      const int wave = threadIdx.x / SHARE;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (k) __syncthreads();
        if (threadIdx.x % SHARE < TPR)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            cols[wave][0][lane * V + i] = sw[k][i];
            cols[wave][1][lane * V + i] = sb[k][i];
          }
        __syncthreads();
        for (int e = threadIdx.x; e < 2 * COLS; e += BLOCK) {
          const int which = e / COLS, c = e % COLS, j = k * COLS + c;
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
    if (a.w) load_weights<true, V>(a.w, a.wdtype, w0, static_cast<int>(j), a.C, j + V > a.C, f);
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

// The partial rows of a group added up: a workgroup takes 32 columns of dw or db; its threads take every eighth partial,
// and their sums are added in order.
__global__ __launch_bounds__(kThreads) void norm_reduce_kernel(NormArgs a, int parts) {
  __shared__ float sums[8][32];
  const int grp = blockIdx.y, which = blockIdx.z, lane = threadIdx.x % 32, row = threadIdx.x / 32;
  void* out = which ? a.db : a.dw;
  if (!out) return;
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + lane;
  float t = 0.0f;
  if (c < a.C) {
    const float* p = a.ws + (static_cast<int64_t>(grp) * parts * 2 + which) * a.C + c;
#pragma unroll 8
    for (int i = row; i < parts; i += 8) t += p[static_cast<int64_t>(i) * 2 * a.C];
  }
  sums[row][lane] = t;
  __syncthreads();
  if (row == 0 && c < a.C) {
#pragma unroll
    for (int i = 1; i < 8; ++i) t += sums[i][lane];
    store_weight(out, a.wdtype, grp * a.w_sb + c, t);
  }
}

// Threads per row and chunks per thread for rows of nv chunks: part of a wave as far as one chunk a thread goes, then
// 64, 256 and 512 threads with up to max_k: 4 forward, 3 backward, whose rows, weights and sums take five times the
// registers of a chunk.
struct Shape {
  int tpr, k;  // k = 0: the row does not fit
};
Shape shape_of(int C, int vec, int max_k) {
  const int nv = (C - 1) / vec + 1;
  if (nv <= 64) {
    int t = 1;
    while (t < nv) t *= 2;
    return {t, 1};
  }
  for (int t : {64, 256, kLong})
    if (nv <= max_k * t) return {t, (nv + t - 1) / t};
  return {kLong, 0};
}

// Whether shape_of gives TPR threads with K chunks for any row: those of 256 and 512 threads have more than max_k chunks
// for each of the 64 or 256 threads before them.
template <int TPR, int K>
constexpr bool reached(int max_k) {
  return K <= max_k && (TPR <= 64 || K * TPR > max_k * (TPR == 256 ? 64 : 256));
}

// Calls f<TPR, K, TAIL>() for the shape; tail: the row's last chunk is not whole.
template <bool TAIL, typename F>
hipError_t with_shape(Shape s, F&& f) {
  switch (s.tpr) {
    case 1: return f.template operator()<1, 1, TAIL>();
    case 2: return f.template operator()<2, 1, TAIL>();
    case 4: return f.template operator()<4, 1, TAIL>();
    case 8: return f.template operator()<8, 1, TAIL>();
    case 16: return f.template operator()<16, 1, TAIL>();
    case 32: return f.template operator()<32, 1, TAIL>();
    case 64:
      if (s.k == 1) return f.template operator()<64, 1, TAIL>();
      if (s.k == 2) return f.template operator()<64, 2, TAIL>();
      if (s.k == 3) return f.template operator()<64, 3, TAIL>();
      return f.template operator()<64, 4, TAIL>();
    case 256:
      if (s.k == 1) return f.template operator()<256, 1, TAIL>();
      if (s.k == 2) return f.template operator()<256, 2, TAIL>();
      if (s.k == 3) return f.template operator()<256, 3, TAIL>();
      return f.template operator()<256, 4, TAIL>();
    default:
      if (s.k == 2) return f.template operator()<kLong, 2, TAIL>();
      if (s.k == 3) return f.template operator()<kLong, 3, TAIL>();
      return f.template operator()<kLong, 4, TAIL>();
  }
}
template <typename F>
hipError_t with_shape(Shape s, bool tail, F&& f) {
  return tail ? with_shape<true>(s, f) : with_shape<false>(s, f);
}

// Workgroups for n units of work: the kernels walk what is beyond (a grid dimension ends at 2^32 threads).
unsigned blocks_for(int64_t n) { return static_cast<unsigned>(n < (1 << 21) ? n : (1 << 21)); }

int rows_per_block(int tpr) { return tpr >= kThreads ? 1 : kThreads / tpr; }

}  // namespace

int64_t norm_parts(int64_t rows, int64_t groups, int C, int dtype) {
  const int vec = dtype == DA2_FP32 ? 4 : 8;
  const Shape s = shape_of(C, vec, kBwdK);
  const int64_t rpb = s.k ? rows_per_block(s.tpr) : 1;
  const int block = s.tpr > kThreads ? s.tpr : kThreads;
  const int64_t fill = s.k ? resident(bwd_waves(s.k * vec), block) : 1024;
  // a workgroup's partial row costs as much as some of its rows, so it walks 8 of them at least
  const int64_t most = (rows + 8 * rpb - 1) / (8 * rpb), each = (fill + groups - 1) / groups;
  return most < each ? most : each;
}

hipError_t launch_norm(const NormArgs& a, hipStream_t stream) {
  const bool grouped = a.w_sb != 0;
  const int64_t all = static_cast<int64_t>(a.B) * a.H * a.N, groups = grouped ? a.B : 1, rows = all / groups;
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    const Shape s = shape_of(a.C, kVec<T>, kFwdK);
    if (!s.k) {
      norm_long_kernel<T><<<dim3(blocks_for(rows), groups), kLong, 0, stream>>>(a, rows, grouped);
      return hipGetLastError();
    }
    return with_shape(s, a.C % kVec<T> != 0, [&]<int TPR, int K, bool TAIL>() {
      if constexpr (!reached<TPR, K>(kFwdK)) {
        return hipErrorInvalidValue;
      } else {
        constexpr int RPB = block_of<TPR>() / TPR;
        const int64_t units = (rows + RPB - 1) / RPB, fill = (resident(fwd_waves(K * kVec<T>, TPR), block_of<TPR>()) + groups - 1) / groups;
        norm_kernel<T, TPR, K, TAIL><<<dim3(static_cast<unsigned>(units < fill ? units : fill), groups), block_of<TPR>(), 0, stream>>>(a, rows, grouped);
        return hipGetLastError();
      }
    });
  });
}

hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t stream) {
  const bool grouped = a.w_sb != 0, sums = a.dw || a.db;
  const int64_t all = static_cast<int64_t>(a.B) * a.H * a.N, groups = grouped ? a.B : 1, rows = all / groups;
  const int64_t parts = norm_parts(rows, groups, a.C, a.dtype);
  const hipError_t e = by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    const Shape s = shape_of(a.C, kVec<T>, kBwdK);
    if (!s.k) {
      const int tiles = static_cast<int>((a.C + static_cast<int64_t>(kThreads) * kVec<T> - 1) / (kThreads * kVec<T>));
      // the sums first: dX may be the memory of X or dY
      if (sums) norm_cols_kernel<T><<<dim3(parts * tiles, groups), kThreads, 0, stream>>>(a, rows, grouped, tiles);
      if (a.dx.p) norm_bwd_long_kernel<T><<<dim3(blocks_for(rows), groups), kLong, 0, stream>>>(a, rows, grouped);
      return hipGetLastError();
    }
    return with_shape(s, a.C % kVec<T> != 0, [&]<int TPR, int K, bool TAIL>() {
      constexpr int RPB = block_of<TPR>() / TPR;
      if constexpr (!reached<TPR, K>(kBwdK)) {
        return hipErrorInvalidValue;
      } else if (sums) {
        norm_bwd_kernel<T, TPR, K, TAIL, true><<<dim3(parts, groups), block_of<TPR>(), 0, stream>>>(a, rows, grouped);
      } else {
        norm_bwd_kernel<T, TPR, K, TAIL, false>
            <<<dim3(blocks_for((rows + RPB - 1) / RPB), groups), block_of<TPR>(), 0, stream>>>(a, rows, grouped);
      }
      return hipGetLastError();
    });
  });
  if (e != hipSuccess || !sums) return e;
  norm_reduce_kernel<<<dim3((a.C + 31) / 32, groups, 2), kThreads, 0, stream>>>(a, static_cast<int>(parts));
  return hipGetLastError();
}

}  // namespace da2
