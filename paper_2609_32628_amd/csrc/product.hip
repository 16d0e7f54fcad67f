// Products of token rows with weight rows, with bias, activation, gate and residual in
// the epilogue, or both halves of a gated block at once: Z = X W' by tiles of features
// times tokens.
//
// The product is transposed, features times tokens: an accumulator's registers are
// then features of one token, four in a row, and lanes l and l ^ 32 trade quads so that
// the epilogue works on eight features in a row of one token with 16-byte accesses.
// A tile takes K in steps of 64: 128 bytes of each row, brought into LDS by
// asynchronous copies while the step before is multiplied. Chunk c (16 bytes) of row r
// lies at position c ^ (r / 2 % 8), so that the 16 rows of a read meet all banks.
// In a gated block a wave's feature rows are half gate, half up, of the same features.
#include <algorithm>

#include "act.hpp"

namespace da2 {

namespace {

constexpr int kStep = 64;               // elements of K a step
constexpr int kRowBytes = 2 * kStep;    // of a tile's row in LDS

__device__ inline int swz(int r) { return (r >> 1) & 7; }

// Element offset of row r.
__device__ inline int64_t row_at(const Side& s, int64_t r) {
  const uint32_t b = static_cast<uint32_t>(r) / static_cast<uint32_t>(s.N);
  return b * s.sb + (static_cast<uint32_t>(r) - b * static_cast<uint32_t>(s.N)) * s.sn;
}
// The least element offset of rows [r, last].
__device__ inline int64_t first_at(const Side& s, int64_t r, int64_t last) {
  const uint32_t b = static_cast<uint32_t>(r) / static_cast<uint32_t>(s.N);
  const int64_t here = row_at(s, r);
  return static_cast<uint32_t>(last) / static_cast<uint32_t>(s.N) > b ? min(here, (b + 1) * s.sb) : here;
}

// Walks K in steps along rows whose elements lie in blocks of C.
struct Walk {
  const char* at;
  int64_t jump;  // bytes from a block's last step to the next block's first
  int in, C;
  __device__ Walk(const Side& s, int64_t row, int k) {
    const int h = k / s.C;
    in = k - h * s.C;
    C = s.C;
    at = static_cast<const char*>(s.p) + 2 * (row + h * s.sh + in);
    jump = 2 * (s.sh - s.C + kStep);
  }
  __device__ void next() {
    in += kStep;
    at += in == C ? jump : kRowBytes;
    in = in == C ? 0 : in;
  }
};

enum Mode { kLinear, kGated, kPartial };

template <int TW, int TT, int WW, int WT>
struct Shape {
  static constexpr int kWaves = WW * WT, kW = TW / WW / 32, kT = TT / WT / 32;  // 32x32 blocks of a wave
  static constexpr int kTile = (TW + TT) * kRowBytes;                           // LDS bytes of a step
  static constexpr int kCopyW = TW / 8 / kWaves, kCopyT = TT / 8 / kWaves;      // 1 KB copies a wave makes
};

// Feature row of a tile's row q of the weights' side (gated: a wave's first half are part 0's).
template <int MODE, int TW, int WW>
__device__ inline int64_t weight_row(int tile, int q, int64_t R, int F) {
  if constexpr (MODE == kGated) {
    constexpr int span = TW / WW, half = span / 2;
    const int in = q % span, f = tile * (TW / 2) + q / span * half + in % half;
    return static_cast<int64_t>(in / half) * F + min(f, F - 1);
  } else {
    const int64_t r = static_cast<int64_t>(tile) * TW + q;
    return r < R ? r : R - 1;
  }
}

template <typename T, int MODE, int TW, int TT, int WW, int WT>
__global__ __launch_bounds__(64 * WW * WT, 2) void product_kernel(ProductArgs a, int tiles_w, int tiles_t, int splits) {
  using S = Shape<TW, TT, WW, WT>;
  __shared__ __attribute__((aligned(1024))) char lds[2 * S::kTile];
  const uint32_t lds0 = lds_offset(lds);
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int wave_w = wave % WW, wave_t = wave / WW;
  const int tiles = tiles_w * tiles_t, unit = unit_of(blockIdx.x, tiles * splits);
  if (unit < 0) return;
  const int split = unit / tiles, tile = unit - split * tiles;
  // tiles in groups of 8 token tiles, token tiles first: those that run at once share rows in their XCD's L2
  const int group = tile / (8 * tiles_w), in_group = tile - group * 8 * tiles_w, wide = min(8, tiles_t - group * 8);
  const int tile_w = in_group / wide, tile_t = group * 8 + in_group - tile_w * wide;
  const int64_t R = static_cast<int64_t>(a.parts) * a.f.F, m0 = static_cast<int64_t>(tile_t) * TT;

  const int steps_all = (a.K + kStep - 1) / kStep, per = (steps_all + splits - 1) / splits;
  const int step0 = split * per, steps = min(per, steps_all - step0);

  // byte offsets of the chunks that this lane copies, from the tile's lowest row; rows behind the last repeat it
  const int64_t w_first = MODE == kGated ? row_at(a.w, weight_row<MODE, TW, WW>(tile_w, 0, R, a.f.F))
                                         : first_at(a.w, weight_row<MODE, TW, WW>(tile_w, 0, R, a.f.F),
                                                    weight_row<MODE, TW, WW>(tile_w, TW - 1, R, a.f.F));
  const int64_t t_first = first_at(a.t, m0, min(m0 + TT, a.M) - 1);
  uint32_t off_w[S::kCopyW], off_t[S::kCopyT];
#pragma unroll
  for (int i = 0; i < S::kCopyW; ++i) {
    const int q = (i * S::kWaves + wave) * 8 + lane / 8, chunk = (lane % 8) ^ swz(q);
    off_w[i] = static_cast<uint32_t>(2 * (row_at(a.w, weight_row<MODE, TW, WW>(tile_w, q, R, a.f.F)) - w_first)) + chunk * 16;
  }
#pragma unroll
  for (int i = 0; i < S::kCopyT; ++i) {
    const int q = (i * S::kWaves + wave) * 8 + lane / 8, chunk = (lane % 8) ^ swz(q);
    off_t[i] = static_cast<uint32_t>(2 * (row_at(a.t, min(m0 + q, a.M - 1)) - t_first)) + chunk * 16;
  }
  Walk walk_w(a.w, w_first, step0 * kStep), walk_t(a.t, t_first, step0 * kStep);

  // brings step s into buffer s % 2
  const auto fetch = [&](int s) {
    const uint32_t to = lds0 + (s & 1) * S::kTile;
    const int k = (step0 + s) * kStep;
    if (k + kStep <= a.K) {
#pragma unroll
      for (int i = 0; i < S::kCopyW; ++i) copy_1k(walk_w.at, off_w[i], to + (i * S::kWaves + wave) * 1024);
#pragma unroll
      for (int i = 0; i < S::kCopyT; ++i) copy_1k(walk_t.at, off_t[i], to + TW * kRowBytes + (i * S::kWaves + wave) * 1024);
    } else {  // the end of K inside a step: through registers, zeros behind it
      const auto part = [&](const char* at, uint32_t off, uint32_t dst, int q) {
        const int left = a.K - k - ((lane % 8) ^ swz(q)) * 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        const char* p = at + off;
        if (left >= 8) {
          v = *reinterpret_cast<const uint4*>(p);
        } else if (left > 0) {
          uint32_t e[4] = {};
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i < left) e[i / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(p)[i]) << (16 * (i % 2));
          v = make_uint4(e[0], e[1], e[2], e[3]);
        }
        *reinterpret_cast<uint4*>(lds + (dst - lds0) + lane * 16) = v;
      };
#pragma unroll
      for (int i = 0; i < S::kCopyW; ++i)
        part(walk_w.at, off_w[i], to + (i * S::kWaves + wave) * 1024, (i * S::kWaves + wave) * 8 + lane / 8);
#pragma unroll
      for (int i = 0; i < S::kCopyT; ++i)
        part(walk_t.at, off_t[i], to + TW * kRowBytes + (i * S::kWaves + wave) * 1024, (i * S::kWaves + wave) * 8 + lane / 8);
    }
    walk_w.next();
    walk_t.next();
  };

  f32x16 acc[S::kW][S::kT];
#pragma unroll
  for (int i = 0; i < S::kW; ++i)
#pragma unroll
    for (int j = 0; j < S::kT; ++j) acc[i][j] = f32x16{};

  // chunk 2 s + lane / 32 of a wave's rows: the positions differ in the address bits of a row's chunks only
  const uint32_t read = (lane % 32) * kRowBytes + (((lane / 32) ^ swz(lane % 32)) << 4);
  const uint32_t read_w = wave_w * S::kW * 32 * kRowBytes + read, read_t = TW * kRowBytes + wave_t * S::kT * 32 * kRowBytes + read;
  if (steps > 0) fetch(0);
  for (int s = 0; s < steps; ++s) {
    wait_copies();
    barrier();
    if (s + 1 < steps) fetch(s + 1);
    const uint32_t at = lds0 + (s & 1) * S::kTile;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      s16x8 w[S::kW], t[S::kT];
#pragma unroll
      for (int i = 0; i < S::kW; ++i) w[i] = read_b128(((at + read_w) ^ (c << 5)) + i * 32 * kRowBytes);
#pragma unroll
      for (int j = 0; j < S::kT; ++j) t[j] = read_b128(((at + read_t) ^ (c << 5)) + j * 32 * kRowBytes);
#pragma unroll
      for (int i = 0; i < S::kW; ++i)
#pragma unroll
        for (int j = 0; j < S::kT; ++j) acc[i][j] = mma<T>(w[i], t[j], acc[i][j]);
    }
  }

  const int g = lane / 32;
#pragma unroll
  for (int j = 0; j < S::kT; ++j) {
    const int64_t m = m0 + (wave_t * S::kT + j) * 32 + lane % 32;
    const bool live = m < a.M;
    const int b = static_cast<int>(static_cast<uint32_t>(live ? m : 0) / static_cast<uint32_t>(a.f.N));
    const int n = static_cast<int>((live ? m : 0) - static_cast<int64_t>(b) * a.f.N);
    // eight features in a row of the lane's token: quads k and k + 1 of the lane halves
    const auto eight = [&](const f32x16& x, int k, float* v) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[4 * k + e]), __float_as_uint(x[4 * k + 4 + e]), false, false);
        v[e] = __uint_as_float(p[0]);
        v[4 + e] = __uint_as_float(p[1]);
      }
    };
    constexpr int blocks = MODE == kGated ? S::kW / 2 : S::kW;
#pragma unroll
    for (int i = 0; i < blocks; ++i)
#pragma unroll
      for (int k = 0; k < 4; k += 2) {
        float v[8], u[8];
        eight(acc[i][j], k, v);
        if constexpr (MODE == kGated) eight(acc[i + blocks][j], k, u);
        const int64_t f8 = (static_cast<int64_t>(tile_w) * WW + wave_w) * (32 * blocks) + i * 32 + 8 * (k + g);
        if constexpr (MODE == kPartial) {
          if (live && f8 < R) {
            float* to = a.ws + (static_cast<int64_t>(split) * a.M + m) * ((R + 7) / 8 * 8) + f8;
            store_vec(to, v);
            store_vec(to + 4, v + 4);
          }
        } else if (live && f8 < a.f.F) {
          finish8<T, MODE == kGated>(a.f, v, u, m, b, n, static_cast<int>(f8));
        }
      }
  }
}

// The partial sums of a split product added up in order, and the epilogue: a thread for eight features of a row.
template <typename T, bool GLU>
__global__ __launch_bounds__(256) void product_join_kernel(ProductArgs a, int splits) {
  const uint32_t chunks = (a.f.F + 7) / 8;
  const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, m = id / chunks;
  if (m >= a.M) return;
  const int f8 = static_cast<int>(id - m * chunks) * 8;
  const int64_t R = (static_cast<int64_t>(a.parts) * a.f.F + 7) / 8 * 8;
  float v[8] = {}, u[8] = {};
  for (int s = 0; s < splits; ++s) {
    const float* p = a.ws + (s * a.M + m) * R + f8;
    float x[8];
    load_vec(p, x);
    load_vec(p + 4, x + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += x[i];
    if constexpr (GLU) {
      load_part(p + a.f.F, a.f.F - f8, x);
      load_part(p + a.f.F + 4, a.f.F - f8 - 4, x + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] += x[i];
    }
  }
  const int b = static_cast<int>(m / a.f.N);
  finish8<T, GLU>(a.f, v, u, m, b, static_cast<int>(m - static_cast<int64_t>(b) * a.f.N), f8);
}

// How a product is cut: big tiles or small ones, and parts of K.
struct Plan {
  bool big;
  int splits;
};
Plan plan_of(int64_t M, int64_t R, int64_t K) {
  const int64_t big = ((M + 255) / 256) * ((R + 255) / 256), small = ((M + 127) / 128) * ((R + 127) / 128);
  const int64_t steps = (K + kStep - 1) / kStep;
  if (big >= 256) return {true, 1};
  int64_t splits = 1;
  while (small * splits * 2 <= 512 && steps / (splits * 2) >= 8) splits *= 2;
  const int64_t per = (steps + splits - 1) / splits;
  return {false, static_cast<int>((steps + per - 1) / per)};
}

template <typename T, int MODE, int TW, int TT, int WW, int WT>
hipError_t launch_tiles(const ProductArgs& a, int64_t features, int splits, hipStream_t stream) {
  using S = Shape<TW, TT, WW, WT>;
  const int64_t tw = (features + TW - 1) / TW, tt = (a.M + TT - 1) / TT;
  const auto kernel = product_kernel<T, MODE, TW, TT, WW, WT>;
  kernel<<<grid_of(static_cast<int>(tw * tt * splits)), 64 * S::kWaves, 0, stream>>>(a, static_cast<int>(tw), static_cast<int>(tt), splits);
  return hipGetLastError();
}

template <typename T, int MODE>
hipError_t launch_plan(const ProductArgs& a, const Plan& p, hipStream_t stream) {
  // a gated tile's rows are two for each feature
  const int64_t features = MODE == kGated ? 2 * static_cast<int64_t>(a.f.F) : static_cast<int64_t>(a.parts) * a.f.F;
  return p.big ? launch_tiles<T, MODE, 256, 256, 2, 4>(a, features, p.splits, stream)
               : launch_tiles<T, MODE, 128, 128, 2, 2>(a, features, p.splits, stream);
}

}  // namespace

int64_t product_ws_bytes(int64_t M, int64_t N, int64_t F, int64_t K, int parts) {
  const auto of = [&](int64_t rows) {
    const Plan p = plan_of(rows, F * parts, K);
    return p.splits > 1 ? 4 * p.splits * rows * ((F * parts + 7) / 8 * 8) : 0;
  };
  return M == N ? of(M) : std::max(of(M), of(N));
}

hipError_t launch_product(const ProductArgs& a, hipStream_t stream) {
  // A tile addresses its token rows by 32 bits from the lowest. Samples further apart than that go one by one.
  const int64_t samples = a.M / a.t.N;
  if (samples > 1 && (std::min<int64_t>(samples, 256 / a.t.N + 2) * a.t.sb + a.t.N * a.t.sn) >> 31) {
    for (int64_t b = 0; b < samples; ++b) {
      ProductArgs one = a;
      const auto skip = [&](const void* p, int64_t n) { return p ? static_cast<const char*>(p) + 2 * b * n : nullptr; };
      one.M = a.t.N;
      one.t.p = skip(a.t.p, a.t.sb);
      one.f.gate = skip(a.f.gate, a.f.gate_sb);
      one.f.r.p = skip(a.f.r.p, a.f.r.sb);
      one.f.y.p = const_cast<char*>(skip(a.f.y.p, a.f.y.sb));
      if (a.f.z) one.f.z += b * a.t.N * a.parts * a.f.z_ld;
      const hipError_t e = launch_product(one, stream);
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  const Plan p = plan_of(a.M, static_cast<int64_t>(a.f.F) * a.parts, a.K);
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    if constexpr (sizeof(T) == 4) {
      return hipErrorInvalidValue;
    } else {
      if (p.splits == 1) return a.parts == 2 ? launch_plan<T, kGated>(a, p, stream) : launch_plan<T, kLinear>(a, p, stream);
      hipError_t e = launch_plan<T, kPartial>(a, p, stream);
      if (e != hipSuccess) return e;
      const int64_t threads = a.M * ((a.f.F + 7) / 8);
      const unsigned blocks = static_cast<unsigned>((threads + 255) / 256);
      if (a.parts == 2) {
        product_join_kernel<T, true><<<blocks, 256, 0, stream>>>(a, p.splits);
      } else {
        product_join_kernel<T, false><<<blocks, 256, 0, stream>>>(a, p.splits);
      }
      return hipGetLastError();
    }
  });
}

}  // namespace da2
