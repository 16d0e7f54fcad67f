// Shared by the kernels of differential attention: operand fragments of the
// 32x32x16 MFMAs, K/V (and Q/dO) tiles in LDS and the visibility of keys.
//
// A tile row of D channels is D/8 chunks of 16 bytes. Chunk c of row r lies at
// position c ^ swz(r), so that both reads of a tile are free of bank conflicts:
//   - rows as an operand's 32 rows (ds_read_b128: one chunk of 16 rows at a time),
//   - columns as an operand's 32 rows (ds_read_b64_tr_b16: 16 lanes read 4 rows
//     of 16 columns and get 4 rows of one column each).
// The 32 rows of the first operand are taken in the order kappa(l) = 16 ((l/4)%2)
// + 4 (l/8) + l%4, so that accumulator register i of lane half g belongs to tile
// row 16 g + i: eight consecutive registers are the second operand of the next
// product as they are, whose 16-row step s takes rows 16 g + 8 s + e.
#pragma once

#include "tile.hpp"

namespace da2 {
namespace diff {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// Running maximum before the first key: finite, so that differences with it are,
// and below every score times the scale.
constexpr float kNoMax = -3.0e38f;

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The sum of eight values of T and s.
template <typename T>
__device__ inline float add8(const s16x8& x, float s) {
  typedef T Tx2 __attribute__((ext_vector_type(2)));
  const uint4 w = __builtin_bit_cast(uint4, x);
  const uint32_t pair[4] = {w.x, w.y, w.z, w.w};
  const Tx2 one = {static_cast<T>(1.0f), static_cast<T>(1.0f)};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (__is_same(T, bf16_t)) {
      s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(Tx2, pair[i]), one, s, false);
    } else {
      s = __builtin_amdgcn_fdot2(__builtin_bit_cast(Tx2, pair[i]), one, s, false);
    }
  }
  return s;
}

// ---- tiles in LDS -----------------------------------------------------------------
template <int D>
struct Tile {
  static constexpr int kChunks = D / 8;      // 16-byte chunks of a row
  static constexpr int kRow = 2 * D;         // bytes of a row
  static constexpr int kRowsPerCopy = 64 / kChunks;  // rows of one 1 KB copy
  __device__ static int swz(int r) {
    const int hi = D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2;
    return hi | ((r >> 2) & 1) | ((((r >> 3) ^ (r >> 4)) & 1) << 1);
  }
};

__device__ inline int kappa(int l) { return 16 * ((l / 4) % 2) + 4 * (l / 8) + l % 4; }

// Reader of a tile's rows: chunk 2 c + g of rows 32 j + order[lane%32] of the tile at `at`, a multiple of a row's bytes.
// The position of a chunk differs from another's in the address bits below a row only, so it is an exclusive or there.
template <int D>
struct RowReader {
  uint32_t first;
  __device__ RowReader(int lane, bool permuted) {
    const int r = permuted ? kappa(lane % 32) : lane % 32;
    first = r * Tile<D>::kRow + ((static_cast<uint32_t>(lane / 32) ^ Tile<D>::swz(r)) << 4);
  }
  __device__ s16x8 read(uint32_t at, int j, int c) const {
    return read_b128(((at + first) ^ (c << 5)) + j * 32 * Tile<D>::kRow);
  }
};

// Reader of a tile's columns: columns 32 t + lane%32, rows 32 j + 16 g + 8 s + [0, 8).
template <int D>
struct ColReader {
  uint32_t first;
  __device__ explicit ColReader(int lane) {
    const int g = lane / 32, i = lane % 16, r = 16 * g + i / 4;
    // the chunk inside 32 columns, with the row's swizzle for s = 0 and its first four rows
    first = r * Tile<D>::kRow + (((2 * ((lane / 16) % 2) + (i % 4) / 2) ^ Tile<D>::swz(r)) << 4) + (i % 2) * 8;
  }
  __device__ s16x8 read(uint32_t at, int j, int t, int s) const {
    // rows + 8 s flip the swizzle's second bit, rows + 4 its first
    const uint32_t y = (at + first) ^ (t << 6) ^ (s << 5);
    const int rows = (j * 32 + 8 * s) * Tile<D>::kRow;
    const s16x4 a = read_tr(y + rows), b = read_tr((y ^ 16) + rows + 4 * Tile<D>::kRow);
    return s16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  }
};

// Asynchronous copy of tile rows into LDS: 1 KB (kRowsPerCopy rows) per call and
// wave. The wave's rows start at LDS byte `lds` (a row of the tile that is a
// multiple of kRowsPerCopy); rows behind `last` repeat it, so nothing beyond the
// tensor's valid rows is read and the tile holds no stray values.
template <int D>
__device__ inline void copy_rows(const void* base, int64_t row_bytes, int row, int last, int lane, uint32_t lds) {
  constexpr int C = Tile<D>::kChunks;
  const int r = row + lane / C;
  const int chunk = (lane % C) ^ Tile<D>::swz(r);
  const uint32_t voff = static_cast<uint32_t>(min(r, last)) * static_cast<uint32_t>(row_bytes) + chunk * 16;
  copy_1k(base, voff, __builtin_amdgcn_readfirstlane(lds));
}

// A workgroup's shape by how many waves share a row's keys, every SHARE-th 32 of a tile each: 4 waves with 128 rows and
// 64-key tiles (1), 8 waves with 128 rows (2) or 64 rows (4) and 128-key tiles.
template <int SHARE>
struct Many {
  static constexpr int kGroups = SHARE == 1 ? 4 : 8 / SHARE;  // of 32 rows
  static constexpr int kRows = 32 * kGroups, kWaves = kGroups * SHARE, kKeys = SHARE == 1 ? 64 : 128;
};

// ---- which keys a query sees ------------------------------------------------------
struct Visible {
  int len;        // valid keys of the sample
  int64_t start;  // position of its first query
};
__device__ inline Visible visible(const DiffArgs& a, int b) {
  Visible s;
  s.len = a.kv_lens ? min(max(a.kv_lens[b], 0), a.M) : a.M;
  s.start = a.q_start ? a.q_start[b] : static_cast<int64_t>(s.len) - a.N;
  // keys that no query sees are not there: in a tile, a weight of zero would still meet what they hold
  if (a.causal && s.start + a.N < s.len) s.len = static_cast<int>(s.start + a.N < 0 ? 0 : s.start + a.N);
  return s;
}
// Query n sees the keys below this.
__device__ inline int key_limit(const DiffArgs& a, const Visible& s, int n) {
  if (!a.causal) return s.len;
  const int64_t e = s.start + n + 1;
  return static_cast<int>(e < 0 ? 0 : e < s.len ? e : s.len);
}

__device__ inline float max16(const f32x16& v) {
  const float a = fmaxf(fmaxf(v[0], v[1]), v[2]), b = fmaxf(fmaxf(v[3], v[4]), v[5]);
  const float c = fmaxf(fmaxf(v[6], v[7]), v[8]), d = fmaxf(fmaxf(v[9], v[10]), v[11]);
  const float e = fmaxf(fmaxf(v[12], v[13]), v[14]);
  return fmaxf(fmaxf(fmaxf(fmaxf(a, b), c), fmaxf(d, e)), v[15]);
}
// The sum of 16 values, pairwise: what it is added to then has a sixteenth of the additions in a chain, and takes up values
// that are small against it. (2^17 keys, the first 2^20.5 times the weight of each other one: a row's sum was 2.5e-3 off, and is
// less than 5e-4 off now; it costs 0.4 to 1% of a long prompt.)
__device__ inline float sum16(const float* v) {
  float t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = v[2 * i] + v[2 * i + 1];
#pragma unroll
  for (int n = 4; n > 0; n /= 2)
#pragma unroll
    for (int i = 0; i < n; ++i) t[i] = t[2 * i] + t[2 * i + 1];
  return t[0];
}
// Maximum and sum over lanes l and l ^ 32.
__device__ inline float max_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ inline float wave_max_f32(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
__device__ inline float wave_sum_f32(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Stores rows given as accumulator columns: lane%32 is the row (its address `row`), x[i] of lane half g is channel
// 8 (i/4) + 4 g + i%4 of 32. The halves trade quads, so that each lane stores 16 bytes.
template <typename T>
__device__ inline void store_columns(T* row, const float* x, bool live) {
  const int g = (threadIdx.x % 64) / 32;
#pragma unroll
  for (int k = 0; k < 4; k += 2) {
    typedef T Tx4 __attribute__((ext_vector_type(4)));
    Tx4 lo, hi;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      lo[e] = static_cast<T>(x[4 * k + e]);
      hi[e] = static_cast<T>(x[4 * k + 4 + e]);
    }
    const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
    const auto p = __builtin_amdgcn_permlane32_swap(a.x, b.x, false, false);
    const auto q = __builtin_amdgcn_permlane32_swap(a.y, b.y, false, false);
    if (live) *reinterpret_cast<uint4*>(row + 8 * (k + g)) = make_uint4(p[0], q[0], p[1], q[1]);
  }
}

}  // namespace diff
}  // namespace da2
