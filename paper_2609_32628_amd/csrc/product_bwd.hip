// What the gradients of a projection need besides products of matrices: the gradients of
// the sums, dz = dY gate f'(z) (gated block: dY u f'(g) and dY f(g)), rounded to the
// tensors' type for the products with W and X; their column sums (bias) and those of
// dY f(z) (gate) in float32 from the unrounded values; and transposed copies.
// Bound by memory: dY and z in, dz and its transpose out, 64x64 elements at a time through LDS (8,190 x 5,120 with gelu and the
// sums of a bias, bf16: 88 us for 420 MB, 4.8 TB/s; gated, 8,190 x 2 x 4,096: 143 us for 600 MB, 4.2). The transposed copies
// are what the products need, whose rows run along the sum: of W (1,280 x 5,120: 10 us) and of X.
#include "act.hpp"

namespace da2 {

namespace {

__device__ inline void load_eight(const float* p, float* x) {
  load_vec(p, x);
  load_vec(p + 4, x + 4);
}

constexpr int kTileN = 64;  // rows and columns of a tile
constexpr int kThreads = 256;
constexpr int kPitch = kTileN + 8;  // elements of a tile's row in LDS: 16-byte rows, columns over all banks

// Column chunk c (8 rows) of element col of a tile in LDS.
__device__ inline uint4 column(const uint16_t* tile, int col, int c) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = tile[(8 * c + 2 * i) * kPitch + col] | static_cast<uint32_t>(tile[(8 * c + 2 * i + 1) * kPitch + col]) << 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Writes rows [0, 64) of columns f0.. of a tile as columns at.. of the transposed copy.
__device__ inline void store_transposed(const uint16_t* tile, uint16_t* out, int64_t ld, int64_t row0, int rows, int64_t at, int64_t limit) {
  for (int i = threadIdx.x; i < kTileN * 8; i += kThreads) {
    const int col = i / 8, c = i % 8;
    if (col < rows && 8 * c < limit) {
      const uint4 v = column(tile, col, c);
      __builtin_memcpy(out + (row0 + col) * ld + at + 8 * c, &v, 16);
    }
  }
}

template <typename T, bool GLU>
__global__ __launch_bounds__(kThreads) void dz_kernel(DzArgs a, int per, int blocks) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[GLU ? 2 : 1][kTileN * kPitch];
  __shared__ float sums[kThreads / 8][kTileN];
  const int b = blockIdx.z, f0 = blockIdx.x * kTileN, c = threadIdx.x % 8, f8 = f0 + 8 * c, left = a.F - f8;
  const int64_t end = !a.dzt ? a.N : b + 1 < a.B ? a.Np : a.ldt - (a.B - 1) * a.Np;  // rows of the sample, zeros behind N
  const int tiles = static_cast<int>((end + kTileN - 1) / kTileN);
  constexpr int P = GLU ? 2 : 1;
  float sb[P][8] = {}, sg[8] = {}, gate[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) gate[i] = 1.0f;
  const auto floats = [](const uint4& v, float* x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = element<T>(v, i);
  };
  if (!GLU && a.gate && left > 0) floats(raw8(static_cast<const T*>(a.gate) + b * a.gate_sb + f8, left), gate);
  // a tile, and once more for what rounding left over
  const int first = blockIdx.y * per, some = max(min(first + per, tiles) - first, 0);
  for (int i = 0; i < some << a.lo; ++i) {
    const int t = first + (i >> a.lo), lo = i & a.lo;
    for (int h = 0; h < 2; ++h) {
      const int row = h * 32 + threadIdx.x / 8, n = t * kTileN + row;
      const bool live = n < a.N && left > 0;
      float dz[P][8] = {};
      if (live) {
        const int64_t m = static_cast<int64_t>(b) * a.N + n;
        float dy[8], z[8], u[8];
        // chunks of rows are whole in memory, and what lies behind F is taken out below
        uint4 raw;
        __builtin_memcpy(&raw, static_cast<const T*>(a.dy.p) + b * a.dy.sb + n * a.dy.sn + feature_at(f8, a.Hy, a.Cy, a.dy.sh), 16);
        floats(first8(raw, left), dy);
        if (a.z) {
          load_eight(a.z + m * P * a.z_ld + f8, z);
          if constexpr (GLU) load_eight(a.z + (m * P + 1) * a.z_ld + f8, u);
          with_act(a.act, [&]<int ACT>() {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float d;
              const float f = act_one<ACT, true>(z[i], d);
              if constexpr (GLU) {
                dz[0][i] = dy[i] * u[i] * d;
                dz[P - 1][i] = dy[i] * f;
              } else {
                dz[0][i] = dy[i] * gate[i] * d;
                if (!lo) sg[i] = __builtin_fmaf(dy[i], i < left ? f : 0.0f, sg[i]);
              }
            }
          });
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) dz[0][i] = dy[i] * gate[i];
        }
        // columns behind F hold nothing
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            dz[p][i] = i < left ? dz[p][i] : 0.0f;
            if (!lo) sb[p][i] += dz[p][i];
            const float rounded = static_cast<float>(static_cast<T>(dz[p][i]));
            if (lo) dz[p][i] = __builtin_isfinite(rounded) ? dz[p][i] - rounded : 0.0f;
          }
      }
      if (a.dz && n < a.N && f8 < a.F64) {
#pragma unroll
        for (int p = 0; p < P; ++p)
          store_vec(static_cast<T*>(a.dz) + (((static_cast<int64_t>(b) * a.N + n) * (1 + a.lo) + lo) * P + p) * a.F64 + f8, dz[p]);
      }
      if (a.dzt) {
#pragma unroll
        for (int p = 0; p < P; ++p) store_vec(reinterpret_cast<T*>(tile[p]) + row * kPitch + 8 * c, dz[p]);
      }
    }
    if (a.dzt) {
      __syncthreads();
      const int64_t n0 = static_cast<int64_t>(t) * kTileN;
#pragma unroll
      for (int p = 0; p < P; ++p)
        store_transposed(tile[p], static_cast<uint16_t*>(a.dzt), a.ldt << a.lo, p * a.F64 + f0, min(kTileN, a.F - f0), lo * a.ldt + b * a.Np + n0, end - n0);
      __syncthreads();
    }
  }
  // the block's rows added up, in the order of its threads
  const int64_t part = static_cast<int64_t>(b) * blocks + blockIdx.y;
  const auto add_up = [&](const float* s, float* out) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[threadIdx.x / 8][8 * c + i] = s[i];
    __syncthreads();
    if (threadIdx.x < kTileN && f0 + static_cast<int>(threadIdx.x) < a.F) {
      float t = 0.0f;
#pragma unroll
      for (int r = 0; r < kThreads / 8; ++r) t += sums[r][threadIdx.x];
      out[f0 + threadIdx.x] = t;
    }
  };
  if (a.pbias)
#pragma unroll
    for (int p = 0; p < P; ++p) add_up(sb[p], a.pbias + (part * P + p) * a.F);
  if (!GLU && a.pgate) add_up(sg, a.pgate + part * a.F);
}

// Sums over the parts of p[group][part][cols], 32 columns a workgroup, every 32nd part a thread (1,188 parts of 256 columns: 5.5 us;
// every eighth 9.9): column c < split goes to out0, the others to out1.
constexpr int kSumRows = 32;
template <typename T>
__global__ __launch_bounds__(32 * kSumRows) void column_sum_kernel(const float* p, int64_t parts, int64_t cols, int64_t split, T* out0, T* out1,
                                                                   int64_t out_sb) {
  __shared__ float sums[kSumRows][32];
  const int lane = threadIdx.x % 32, row = threadIdx.x / 32;
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + lane;
  float t = 0.0f;
  if (c < cols) {
    const float* q = p + blockIdx.y * parts * cols + c;
#pragma unroll 8
    for (int64_t i = row; i < parts; i += kSumRows) t += q[i * cols];
  }
  sums[row][lane] = t;
  __syncthreads();
  if (row == 0 && c < cols) {
#pragma unroll
    for (int i = 1; i < kSumRows; ++i) t += sums[i][lane];
    T* out = c < split ? out0 : out1;
    if (out) out[blockIdx.y * out_sb + (c < split ? c : c - split)] = static_cast<T>(t);
  }
}

__global__ __launch_bounds__(kThreads) void transpose_kernel(TransposeArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[kTileN * kPitch];
  const int b = blockIdx.z, k0 = blockIdx.y * kTileN;
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * kTileN, end = b + 1 < a.B ? a.Np : a.ld - (a.B - 1) * a.Np;
  if (n0 >= end) return;
  for (int i = threadIdx.x; i < kTileN * 8; i += kThreads) {
    const int row = i / 8, k = k0 + i % 8 * 8, left = a.K - k;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (n0 + row < a.s.N && left > 0)
      __builtin_memcpy(&v, static_cast<const uint16_t*>(a.s.p) + b * a.s.sb + (n0 + row) * a.s.sn + feature_at(k, a.K > a.s.C ? 2 : 1, a.s.C, a.s.sh), 16);
    __builtin_memcpy(tile + row * kPitch + i % 8 * 8, &v, 16);
  }
  __syncthreads();
  store_transposed(tile, static_cast<uint16_t*>(a.out), a.ld, k0, min(kTileN, a.K - k0), b * a.Np + n0, end - n0);
}

}  // namespace

// Workgroups along the rows of a sample: enough to fill the card, each with a partial row of the sums.
int dz_blocks(int64_t B, int64_t N, int64_t F) {
  const int64_t tiles = (N + kTileN - 1) / kTileN, others = B * ((F + kTileN - 1) / kTileN), want = (2048 + others - 1) / others;
  return static_cast<int>(want < tiles ? want : tiles);
}

hipError_t launch_dz(const DzArgs& a, hipStream_t stream) {
  const int blocks = dz_blocks(a.B, a.N, a.F);
  const int64_t last = a.dzt ? a.ldt - (a.B - 1) * a.Np : 0, rows = last > a.Np ? last : a.Np;
  const int per = static_cast<int>(((rows + kTileN - 1) / kTileN + blocks - 1) / blocks);
  const dim3 grid(static_cast<unsigned>((a.F + kTileN - 1) / kTileN), blocks, a.B);
  const hipError_t e = by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    if constexpr (sizeof(T) == 4) {
      return hipErrorInvalidValue;
    } else {
      if (a.parts == 2) {
        dz_kernel<T, true><<<grid, kThreads, 0, stream>>>(a, per, blocks);
      } else {
        dz_kernel<T, false><<<grid, kThreads, 0, stream>>>(a, per, blocks);
      }
      return hipGetLastError();
    }
  });
  if (e != hipSuccess) return e;
  const int64_t cols = static_cast<int64_t>(a.parts) * a.F, all = static_cast<int64_t>(a.B) * blocks;
  hipError_t s = hipSuccess;
  if (a.pbias) s = launch_column_sum(a.pbias, all, cols, 1, a.dtype, a.dbias, nullptr, cols, 0, stream);
  if (s == hipSuccess && a.pgate)
    s = a.dgate_sb ? launch_column_sum(a.pgate, blocks, a.F, a.B, a.dtype, a.dgate, nullptr, a.F, a.dgate_sb, stream)
                   : launch_column_sum(a.pgate, all, a.F, 1, a.dtype, a.dgate, nullptr, a.F, 0, stream);
  return s;
}

hipError_t launch_column_sum(const float* p, int64_t parts, int64_t cols, int64_t groups, int dtype, void* out0, void* out1, int64_t split,
                             int64_t out_sb, hipStream_t stream) {
  return by_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    column_sum_kernel<T><<<dim3(static_cast<unsigned>((cols + 31) / 32), static_cast<unsigned>(groups)), 32 * kSumRows, 0, stream>>>(
        p, parts, cols, split, static_cast<T*>(out0), static_cast<T*>(out1), out_sb);
    return hipGetLastError();
  });
}

hipError_t launch_transpose(const TransposeArgs& a, hipStream_t stream) {
  const int64_t last = a.ld - (a.B - 1) * a.Np, cols = last > a.Np ? last : a.Np;
  const dim3 grid(static_cast<unsigned>((cols + kTileN - 1) / kTileN), (a.K + kTileN - 1) / kTileN, a.B);
  transpose_kernel<<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace da2
