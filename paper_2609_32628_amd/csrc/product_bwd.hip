// What the gradients of a projection need besides products of matrices: the gradients of
// the sums, dz = dY gate f'(z) (gated block: dY u f'(g) and dY f(g)), rounded to the
// tensors' type (fp16: times a power of two) for the products with W and X; their column sums (bias) and those of
// dY f(z) (gate) in float32 from the unrounded values; and transposed copies.
// Bound by memory: dY and z in, dz and its transpose out, 64x64 elements at a time through LDS (8,190 x 5,120 with gelu and the
// sums of a bias, bf16: 88 us for 420 MB, 4.8 TB/s; gated, 8,190 x 2 x 4,096: 141 us for 600 MB, 4.2). The transposed copies
// are what the products need, whose rows run along the sum: of W (1,280 x 5,120: 10 us) and of X. The pass for fp16's scale
// costs 25 us at 8,190 x 5,120 and 67 at 8,190 x 2 x 4,096, gated.
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

template <typename T>
__device__ inline void unpack8(const uint4& v, float* x) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = element<T>(v, i);
}
// The gates of features [f8, f8 + left) of sample b; 1 behind them, or without gates.
template <typename T, bool GLU>
__device__ inline void gates8(const DzArgs& a, int b, int f8, int left, float* gate) {
#pragma unroll
  for (int i = 0; i < 8; ++i) gate[i] = 1.0f;
  if (!GLU && a.gate && left > 0) unpack8<T>(raw8(static_cast<const T*>(a.gate) + b * a.gate_sb + f8, left), gate);
}
// dz of features [f8, f8 + left) of token n of sample b, of a gated block both halves, zeros behind them. Where act is not null: dY in
// dy, and the activations in act (zeros without z).
template <typename T, bool GLU>
__device__ inline void dz8(const DzArgs& a, int b, int n, int f8, int left, const float* gate, float (*dz)[8], float* dy, float* act) {
  constexpr int P = GLU ? 2 : 1;
  // chunks of rows are whole in memory, and what lies behind F is taken out below
  uint4 raw;
  __builtin_memcpy(&raw, static_cast<const T*>(a.dy.p) + b * a.dy.sb + n * a.dy.sn + feature_at(f8, a.Hy, a.Cy, a.dy.sh), 16);
  unpack8<T>(first8(raw, left), dy);
  if (a.z) {
    const int64_t m = static_cast<int64_t>(b) * a.N + n;
    float z[8], u[8];
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
          if (act) act[i] = i < left ? f : 0.0f;
        }
      }
    });
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      dz[0][i] = dy[i] * gate[i];
      if (act) act[i] = 0.0f;
    }
  }
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int i = 0; i < 8; ++i) dz[p][i] = i < left ? dz[p][i] : 0.0f;
}

// The largest value that all threads of the workgroup hold.
__device__ inline float block_max(float x) {
  __shared__ float most[kThreads / 64];
  x = wave_max(x);
  if (threadIdx.x % 64 == 0) most[threadIdx.x / 64] = x;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) x = fmaxf(x, most[w]);
  return x;
}

// fp16 holds neither small nor large gradients of sums, though the products of them that are the results may be in its range: dZ
// is stored times the power of two that brings its largest finite value to [2^14, 2^15), and the products' sums are divided by
// it. (A value 2^29 times smaller still keeps its 11 digits. Without it dZ of 2^-25 is 0, and dZ above 65,504 infinite.)
// This takes a pass over dY and Z of its own, fp16 only, by n_tops workgroups in the launch of a transposed copy: the largest of
// their values each. Without a gated half no activation's derivative is over 1.13, and 1.2 dY gate is taken for dZ, which
// leaves out Z, two thirds of the bytes: where all derivatives are smaller by 2^j, values 2^(29 - j) below the largest keep their digits.
constexpr float kSteepest = 1.2f;
template <typename T, bool GLU>
__device__ inline void dz_top(DzArgs a) {
  constexpr int P = GLU ? 2 : 1;
  if constexpr (!GLU) a.z = nullptr;
  const int64_t chunks = (a.F + 7) / 8, M = static_cast<int64_t>(a.B) * a.N, all = static_cast<int64_t>(a.n_tops) * kThreads;
  const int64_t rows = all / chunks, rest = all - rows * chunks;  // from one of a thread's chunks to the next
  int64_t m = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x, c = m % chunks;
  m /= chunks;
  float top = 0.0f;
  for (; m < M; m += rows) {
    const int b = static_cast<int>(static_cast<uint32_t>(m) / static_cast<uint32_t>(a.N)), f8 = static_cast<int>(c) * 8, left = a.F - f8;
    float gate[8], dz[P][8], dy[8];
    gates8<T, GLU>(a, b, f8, left, gate);
    dz8<T, GLU>(a, b, static_cast<int>(m - static_cast<int64_t>(b) * a.N), f8, left, gate, dz, dy, nullptr);
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, __builtin_isfinite(dz[p][i]) ? __builtin_fabsf(dz[p][i]) : 0.0f);
    c += rest;
    if (c >= chunks) {
      c -= chunks;
      ++m;
    }
  }
  top = block_max(top) * (GLU ? 1.0f : kSteepest);
  if (threadIdx.x == 0) a.back[1 + blockIdx.x] = top;
}
// That power of two.
__device__ inline float scale_below(float top) {
  const int above = min(max(__builtin_amdgcn_frexp_expf(top), -100), 100);  // top < 2^above
  return __builtin_ldexpf(1.0f, 15 - above);
}

template <typename T, bool GLU>
__global__ __launch_bounds__(kThreads) void dz_kernel(DzArgs a, int per, int blocks) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[GLU ? 2 : 1][kTileN * kPitch];
  __shared__ float sums[kThreads / 8][kTileN];
  const int b = blockIdx.z, f0 = blockIdx.x * kTileN, c = threadIdx.x % 8, f8 = f0 + 8 * c, left = a.F - f8;
  const int64_t end = !a.dzt ? a.N : b + 1 < a.B ? a.Np : a.ldt - (a.B - 1) * a.Np;  // rows of the sample, zeros behind N
  const int tiles = static_cast<int>((end + kTileN - 1) / kTileN);
  constexpr int P = GLU ? 2 : 1;
  float sb[P][8] = {}, sg[8] = {}, gate[8], scale = 1.0f;
  gates8<T, GLU>(a, b, f8, left, gate);
  if constexpr (kScaledDz<T>) {
    if (a.back) {
      float top = 0.0f;
      for (int i = threadIdx.x; i < a.n_tops; i += kThreads) top = fmaxf(top, a.back[1 + i]);
      scale = scale_below(block_max(top));
      if (threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) *a.back = 1.0f / scale;
    }
  }
  // a tile, and once more for what rounding left over
  const int first = blockIdx.y * per, some = max(min(first + per, tiles) - first, 0);
  for (int i = 0; i < some << a.lo; ++i) {
    const int t = first + (i >> a.lo), lo = i & a.lo;
    for (int h = 0; h < 2; ++h) {
      const int row = h * 32 + threadIdx.x / 8, n = t * kTileN + row;
      const bool live = n < a.N && left > 0;
      float dz[P][8] = {};
      if (live) {
        float dy[8], act[8];
        dz8<T, GLU>(a, b, n, f8, left, gate, dz, dy, act);
        if (!GLU && !lo) {
#pragma unroll
          for (int i = 0; i < 8; ++i) sg[i] = __builtin_fmaf(dy[i], act[i], sg[i]);
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (!lo) sb[p][i] += dz[p][i];
            if constexpr (kScaledDz<T>) dz[p][i] *= scale;
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

// Tile x, y of sample b.
__device__ inline void transpose_tile(const TransposeArgs& a, int x, int y, int b) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[kTileN * kPitch];
  const int k0 = y * kTileN;
  const int64_t n0 = static_cast<int64_t>(x) * kTileN, end = b + 1 < a.B ? a.Np : a.ld - (a.B - 1) * a.Np;
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
__global__ __launch_bounds__(kThreads) void transpose_kernel(TransposeArgs a) { transpose_tile(a, blockIdx.x, blockIdx.y, blockIdx.z); }
// The same, and the largest gradients of the sums, in one launch: tiles lie wide x tall in each sample.
template <bool GLU>
__global__ __launch_bounds__(kThreads) void transpose_and_top_kernel(TransposeArgs a, DzArgs z, uint32_t wide, uint32_t tall) {
  if (blockIdx.x < static_cast<uint32_t>(z.n_tops)) {
    dz_top<fp16_t, GLU>(z);
  } else {
    const uint32_t i = blockIdx.x - z.n_tops, row = i / wide, b = row / tall;
    transpose_tile(a, static_cast<int>(i - row * wide), static_cast<int>(row - b * tall), static_cast<int>(b));
  }
}

}  // namespace

// Workgroups along the rows of a sample: enough to fill the card, each with a partial row of the sums.
int dz_blocks(int64_t B, int64_t N, int64_t F) {
  const int64_t tiles = (N + kTileN - 1) / kTileN, others = B * ((F + kTileN - 1) / kTileN), want = (2048 + others - 1) / others;
  return static_cast<int>(want < tiles ? want : tiles);
}

// Workgroups that look for the largest gradient.
int dz_tops(int64_t M, int64_t F) {
  const int64_t n = (M * ((F + 7) / 8) + kThreads - 1) / kThreads;
  return static_cast<int>(n < 1024 ? n : 1024);
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

hipError_t launch_transpose(const TransposeArgs& a, const DzArgs* top, hipStream_t stream) {
  const int64_t last = a.ld - (a.B - 1) * a.Np, cols = last > a.Np ? last : a.Np;
  const unsigned wide = static_cast<unsigned>((cols + kTileN - 1) / kTileN), tall = (a.K + kTileN - 1) / kTileN;
  const int64_t tiles = static_cast<int64_t>(wide) * tall * a.B;
  const bool apart = !top || top->n_tops + tiles >= 1 << 24;  // a dimension of a grid ends at 2^32 threads
  if (apart) transpose_kernel<<<dim3(wide, tall, a.B), kThreads, 0, stream>>>(a);
  if (top) {
    const unsigned blocks = top->n_tops + (apart ? 0 : static_cast<unsigned>(tiles));
    if (top->parts == 2) {
      transpose_and_top_kernel<true><<<blocks, kThreads, 0, stream>>>(a, *top, wide, tall);
    } else {
      transpose_and_top_kernel<false><<<blocks, kThreads, 0, stream>>>(a, *top, wide, tall);
    }
  }
  return hipGetLastError();
}

}  // namespace da2
