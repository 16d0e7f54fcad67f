// Differential attention, forward.
//
//   O = (softmax(c Q1 K1^T) - lambda softmax(c Q2 K2^T)) V
//
// One pass over the keys with a running maximum and sum for each of the two maps:
// both maps' scores come from one K tile (the halves of its channels) and both
// weight V with one V tile, so a tile is read once for both. The products are
// transposed (S^T = K Q^T, O^T = V^T P^T): a lane holds one query, so the softmax
// statistics need no more than one exchange between the lane halves, and the
// weights are the next product's operand as they are.
//
// The rows of a key head's Hq/Hk query heads are taken together (row r is head
// r % G of token r / G), so that few tokens fill a tile and share its keys.
// A wave owns 32 rows and both maps (2 x D/32 x 16 accumulator registers):
//   - many rows: 4 waves with 128 rows walk 64-key tiles that they share, or 8
//     waves, of which two or four share a row's keys, walk 128-key tiles;
//   - few rows (up to 64): 4 waves with the same 32 rows walk the 32-key quarters
//     of 128-key tiles, each its own, and are joined at the end.
// Where that leaves CUs idle the keys are split over workgroups; a second kernel
// joins the parts. (bf16, 16,380 tokens of 12 heads, d = 128: 2.31 to 2.43 ms from
// one card to another, 1.02 to 1.07 PFLOP/s, bound by products and exponentials,
// which share the issue slots; one token over 16 caches of up to 16,384 keys, 8 key
// heads: 161 us, 5.1 TB/s.)
#include "diff.hpp"

namespace da2 {

namespace {

using namespace diff;

constexpr int kThreads = 256;

// How a problem is cut: row tiles and key splits (host and kernels).
struct Cut {
  bool few;    // few rows: waves share rows and take different keys
  int tiles;   // row tiles of a key head
  int splits;  // parts of the keys
};
Cut cut_of(int B, int Hq, int Hk, int N, int M) {
  const int64_t rows = static_cast<int64_t>(N) * (Hq / Hk);
  Cut c;
  c.few = rows <= 64;
  c.tiles = static_cast<int>(c.few ? (rows + 31) / 32 : (rows + 127) / 128);
  const int64_t units = static_cast<int64_t>(B) * Hk * c.tiles;
  // One workgroup a CU, which is what LDS holds of few rows, and parts that take longer to walk than to join. Few rows (one
  // sample of 32,768 keys, 8 key heads: 41 us with half as many workgroups, 44 with one a CU, 64 with two; 8 samples of
  // 8,192, 12 heads: 113, 74 and 80): 256 keys. Many rows: 128 keys take a workgroup of 128 rows 2.5 us, and a launch and
  // the parts' way through memory 5 us and more, so parts have 512 keys (from 1,536 on) where the tiles leave most CUs idle
  // and 2,048 else (32 tiles against 1,024 keys: 24 us whole and 26 in two parts; 64 against 2,048: 42 whole, 40 in two, 36
  // in four; 128 against 2,048: 44 whole and 49 in two; near the borders it loses: 8 against 1,535 30.9 whole and
  // 28.4 in two parts, 96 against 3,000 59.0 and 56.7).
  int64_t s = 256 / units, most = c.few ? (M + 255) / 256 : units <= 64 && M >= 1536 ? M / 512 : M / 2048;
  s = s < most ? s : most;
  c.splits = static_cast<int>(s < 1 ? 1 : s);
  return c;
}

// Floats of a row's part of few rows: its unnormalised outputs, maxima and sums. Vectors of 4 of a 32-row part of many
// rows: its statistics and its 2 D/32 accumulators.
template <int D>
constexpr int kPart = 2 * D + 4;
template <int D>
constexpr int kBlock = 64 * (1 + 2 * D / 32 * 4);

// 32 rows (a lane's query is lane%32) against 32 keys of a K and a V tile in LDS.
template <typename T, int D>
struct Rows32 {
  static constexpr int S = D / 32;  // 16-channel steps of a map
  static constexpr int C = D / 32;  // 32-channel tiles of V
  // A key's weight is 2^(score - m); a new maximum's is 2^kTop, and the largest 2^kMost. Weights are rounded to T: fp16 has
  // numbers up to 2^15 but few below 2^-14, which a long row's many small weights are (2^17 keys 2^-25 each of the first
  // one's weight, 0.3% of the row together, came out as zeros).
  static constexpr float kTop = __is_same(T, fp16_t) ? 11.0f : 0.0f, kMost = __is_same(T, fp16_t) ? 15.0f : 8.0f;
  s16x8 q[2][S];
  f32x16 u[2][C];
  float m[2], l[2];
  RowReader<D> rows;
  ColReader<D> cols;
  int lane;

  __device__ Rows32(int lane_) : rows(lane_, true), cols(lane_), lane(lane_) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      m[i] = kNoMax;
      l[i] = 0.0f;
#pragma unroll
      for (int t = 0; t < C; ++t) u[i][t] = f32x16{};
    }
  }
  __device__ void load_query(const T* row) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int s = 0; s < S; ++s)
        q[i][s] = *reinterpret_cast<const s16x8*>(row + i * (D / 2) + 16 * s + 8 * (lane / 32));
  }
  // Scores of both maps with keys [key, key + 32), at rows 32 j of the tile kt; limit: the lane's query sees the keys
  // below it.
  __device__ void scores(f32x16 (&x)[2], uint32_t kt, int j, int key, int limit, bool mask) const {
    x[0] = x[1] = f32x16{};
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int i = 0; i < 2; ++i) x[i] = mma<T>(rows.read(kt, j, i * S + s), q[i][s], x[i]);
    if (mask) {
      const int left = limit - key - 16 * (lane / 32);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[i][e] = e < left ? x[i][e] : -__builtin_inff();
    }
  }
  // The maximum is a reference for the exponentials only: it follows when a weight would pass 2^kMost, up to which the
  // weights' float32 sums and 16-bit values hold them, so that the accumulators are rarely rescaled.
  __device__ void follow(const f32x16 (&x)[2], float c) {
    float top[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) top[i] = max_halves(max16(x[i])) * c;
    if (__any(top[0] > m[0] + kMost || top[1] > m[1] + kMost)) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float to = fmaxf(m[i], top[i] - kTop), f = exp2_fast(m[i] - to);
        m[i] = to;
        l[i] *= f;
#pragma unroll
        for (int t = 0; t < C; ++t) u[i][t] *= f;
      }
    }
  }
  __device__ void weights(s16x8 (&p)[2][2], const f32x16 (&x)[2], float c) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float w[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) w[e] = exp2_fast(__builtin_fmaf(x[i][e], c, -m[i]));
      l[i] += sum16(w);
      p[i][0] = pack8<T>(w);
      p[i][1] = pack8<T>(w + 8);
    }
  }
  __device__ void values(const s16x8 (&p)[2][2], uint32_t vt, int j) {
#pragma unroll
    for (int t = 0; t < C; ++t)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const s16x8 v = cols.read(vt, j, t, s);
        u[0][t] = mma<T>(v, p[0][s], u[0][t]);
        u[1][t] = mma<T>(v, p[1][s], u[1][t]);
      }
  }
  __device__ void step(uint32_t kt, uint32_t vt, int j, int key, int limit, bool mask, float c) {
    f32x16 x[2];
    s16x8 p[2][2];
    scores(x, kt, j, key, limit, mask);
    follow(x, c);
    weights(p, x, c);
    values(p, vt, j);
  }
};

template <typename T>
__device__ inline T* row_ptr(const OutView& o, int b, int h, int n) {
  return static_cast<T*>(o.p) + b * o.sb + h * o.sh + n * o.sn;
}

// Only a sum without a key is the zero of all bits; by its bits, so that a NaN of the caller's stays one.
__device__ inline void store_lse(const DiffArgs& a, int b, int h, int n, int i, float m, float l) {
  a.lse[((static_cast<int64_t>(b) * a.Hq + h) * 2 + i) * a.N + n] =
      __float_as_uint(l) ? kLn2 * (m + __builtin_amdgcn_logf(l)) : -__builtin_inff();
}

// Output of one row from its accumulators as columns (see store_columns) and its whole sums l.
template <typename T, int D>
__device__ inline void finish_rows(const DiffArgs& a, Rows32<T, D>& r, int b, int h, int n, bool live) {
  float inv[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float l = r.l[i];
    inv[i] = l > 0.0f ? 1.0f / l : 0.0f;
    if (a.lse && live && r.lane < 32) store_lse(a, b, h, n, i, r.m[i], l);
  }
  const float f = a.lam[h] * inv[1];
  T* o = row_ptr<T>(a.o, b, h, n);
#pragma unroll
  for (int t = 0; t < D / 32; ++t) {
    float x[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = r.u[0][t][e] * inv[0] - r.u[1][t][e] * f;
    store_columns(o + 32 * t, x, live);
  }
}

// One element (channel ch, given) of a row from its parts: (U1, U2) sums and the statistics.
template <typename T>
__device__ inline void finish_element(const DiffArgs& a, int b, int h, int n, int ch, float u1, float u2, float l1, float l2) {
  const float i1 = l1 > 0.0f ? 1.0f / l1 : 0.0f, i2 = l2 > 0.0f ? 1.0f / l2 : 0.0f;
  row_ptr<T>(a.o, b, h, n)[ch] = static_cast<T>(u1 * i1 - u2 * (a.lam[h] * i2));
}

template <typename T, int D, int SHARE>
__global__ __launch_bounds__(64 * Many<SHARE>::kWaves, 2) void diff_many_kernel(DiffArgs a, int tiles, int splits, int units) {
  constexpr int GROUPS = Many<SHARE>::kGroups, ROWS = Many<SHARE>::kRows;
  constexpr int K = Many<SHARE>::kKeys, WAVES = Many<SHARE>::kWaves, BYTES = K * Tile<D>::kRow, R = Tile<D>::kRowsPerCopy, C = D / 32;
  __shared__ __align__(256) char lds[2][2][BYTES];  // [buffer][K, V]
  const int unit = unit_of(blockIdx.x, units);
  if (unit < 0) return;
  const int split = unit % splits;
  // the last rows see most keys under a causal mask: they go first
  const int tile = tiles - 1 - unit / splits % tiles;
  const int bh = unit / splits / tiles;
  const int b = bh / a.Hk, hk = bh % a.Hk, G = a.Hq / a.Hk;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int group = wave % GROUPS, share = wave / GROUPS;
  const uint32_t rows = static_cast<uint32_t>(a.N) * G, row0 = static_cast<uint32_t>(tile) * ROWS + 32 * group;
  const auto token = [&](uint32_t r) { return static_cast<int>(min(r, rows - 1) / static_cast<uint32_t>(G)); };
  const bool live = row0 + lane % 32 < rows;
  const uint32_t row = min(row0 + lane % 32, rows - 1);
  const int n = token(row), h = hk * G + static_cast<int>(row) - n * G;
  const Visible vis = visible(a, b);
  const int limit = key_limit(a, vis, n);
  const int low = key_limit(a, vis, token(row0)), high = key_limit(a, vis, token(row0 + 31));  // of the wave
  int end = key_limit(a, vis, token(static_cast<uint32_t>(tile) * ROWS + ROWS - 1));                                      // of the workgroup
  int key = 0;
  if (splits > 1) {
    const int part = ((end + splits - 1) / splits + K - 1) / K * K;
    key = min(split * part, end);
    end = min(key + part, end);
  }
  Rows32<T, D> r(lane);
  r.load_query(static_cast<const T*>(a.q.p) + b * a.q.sb + h * a.q.sh + n * a.q.sn);
  const T* kp = static_cast<const T*>(a.k.p) + b * a.k.sb + hk * a.k.sh;
  const T* vp = static_cast<const T*>(a.v.p) + b * a.v.sb + hk * a.v.sh;
  const float c = a.scale * kLog2e;
  const auto copy = [&](int at, int buf) {
#pragma unroll
    for (int i = 0; i < K / R / WAVES; ++i) {
      const int first = (wave * (K / R / WAVES) + i) * R;
      copy_rows<D>(kp + at * a.k.sn, 2 * a.k.sn, first, vis.len - 1 - at, lane, lds_offset(lds[buf][0]) + first * Tile<D>::kRow);
      copy_rows<D>(vp + at * a.v.sn, 2 * a.v.sn, first, vis.len - 1 - at, lane, lds_offset(lds[buf][1]) + first * Tile<D>::kRow);
    }
  };
  if (key < end) copy(key, 0);
  for (int buf = 0; key < end; key += K, buf ^= 1) {
    wait_copies();
    barrier();  // every wave's copies have arrived, and the other buffer has been read
    if (key + K < end) copy(key + K, buf ^ 1);
    const uint32_t kt = lds_offset(lds[buf][0]) + share * 32 * Tile<D>::kRow;
    const uint32_t vt = lds_offset(lds[buf][1]) + share * 32 * Tile<D>::kRow;
#pragma unroll
    for (int j = 0; j < K / 32; j += SHARE) {
      const int at = key + 32 * (j + share);
      if (at < min(high, end)) r.step(kt, vt, j, at, limit, at + 32 > low, c);
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) r.l[i] = sum_halves(r.l[i]);
  // The other waves of a row hand their sums to the first, one map after the other, in the room of the tiles.
  if constexpr (SHARE > 1) {
    f32x4* swap = reinterpret_cast<f32x4*>(lds) + lane;
    constexpr int PER = (4 * C + 1) * 64;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      __syncthreads();
      if (share) {
        f32x4* to = swap + ((share - 1) * GROUPS + group) * PER;
#pragma unroll
        for (int t = 0; t < C; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            to[(4 * t + e) * 64] = f32x4{r.u[i][t][4 * e], r.u[i][t][4 * e + 1], r.u[i][t][4 * e + 2], r.u[i][t][4 * e + 3]};
        to[4 * C * 64] = f32x4{r.m[i], r.l[i], 0.0f, 0.0f};
      }
      __syncthreads();
      if (!share)
#pragma unroll
        for (int o = 0; o < SHARE - 1; ++o) {
          const f32x4* from = swap + (o * GROUPS + group) * PER;
          const f32x4 other = from[4 * C * 64];
          const float m = fmaxf(r.m[i], other[0]), f = exp2_fast(r.m[i] - m), g = exp2_fast(other[0] - m);
          r.m[i] = m;
          r.l[i] = r.l[i] * f + other[1] * g;
#pragma unroll
          for (int t = 0; t < C; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const f32x4 y = from[(4 * t + e) * 64];
#pragma unroll
              for (int x = 0; x < 4; ++x) r.u[i][t][4 * e + x] = r.u[i][t][4 * e + x] * f + y[x] * g;
            }
        }
    }
  }
  if (share) return;
  if (splits == 1) {
    finish_rows(a, r, b, h, n, live);
    return;
  }
  // parts lie as the registers do, a wave's 1 KB at a time
  f32x4* part = reinterpret_cast<f32x4*>(a.ws) + (static_cast<int64_t>(unit) * GROUPS + group) * kBlock<D> + lane;
  part[0] = f32x4{r.m[0], r.l[0], r.m[1], r.l[1]};
#pragma unroll
  for (int t = 0; t < C; ++t)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        part[64 * (1 + (t * 2 + i) * 4 + e)] = f32x4{r.u[i][t][4 * e], r.u[i][t][4 * e + 1], r.u[i][t][4 * e + 2], r.u[i][t][4 * e + 3]};
}

// The parts of 32 rows joined: a wave takes one tile of 32 channels.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void diff_many_join_kernel(DiffArgs a, int tiles, int splits, int blocks) {
  constexpr int C = D / 32;
  const int lane = threadIdx.x % 64, w = blockIdx.x * 4 + threadIdx.x / 64, t = w % C, block = w / C;  // block: 32 rows
  if (block >= blocks) return;
  const int group = block % 4, bh = block / 4 / tiles, tile = tiles - 1 - block / 4 % tiles;
  const int b = bh / a.Hk, hk = bh % a.Hk, G = a.Hq / a.Hk;
  const uint32_t rows = static_cast<uint32_t>(a.N) * G, row0 = tile * 128u + 32 * group;
  const bool live = row0 + lane % 32 < rows;
  const uint32_t row = min(row0 + lane % 32, rows - 1);
  const int n = row / static_cast<uint32_t>(G), h = hk * G + static_cast<int>(row) - n * G;
  const auto part = [&](int s) {
    return reinterpret_cast<const f32x4*>(a.ws) + ((static_cast<int64_t>(block / 4) * splits + s) * 4 + group) * kBlock<D> + lane;
  };
  float m[2] = {kNoMax, kNoMax}, l[2] = {0.0f, 0.0f};
  for (int s = 0; s < splits; ++s) {
    const f32x4 st = part(s)[0];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float to = fmaxf(m[i], st[2 * i]);
      l[i] = l[i] * exp2_fast(m[i] - to) + st[2 * i + 1] * exp2_fast(st[2 * i] - to);
      m[i] = to;
    }
  }
  if (a.lse && live && t == 0 && lane < 32)
#pragma unroll
    for (int i = 0; i < 2; ++i) store_lse(a, b, h, n, i, m[i], l[i]);
  float x[16] = {};
  const float f[2] = {l[0] > 0.0f ? 1.0f / l[0] : 0.0f, l[1] > 0.0f ? -a.lam[h] / l[1] : 0.0f};
  for (int s = 0; s < splits; ++s) {
    const f32x4 st = part(s)[0];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float g = exp2_fast(st[2 * i] - m[i]) * f[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4 y = part(s)[64 * (1 + (t * 2 + i) * 4 + e)];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[4 * e + k] = __builtin_fmaf(y[k], g, x[4 * e + k]);
      }
    }
  }
  store_columns(row_ptr<T>(a.o, b, h, n) + 32 * t, x, live);
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads, 1) void diff_few_kernel(DiffArgs a, int tiles, int splits, int units) {
  constexpr int K = 128, BYTES = 32 * Tile<D>::kRow, R = Tile<D>::kRowsPerCopy;
  __shared__ __align__(256) char lds[4][2][2][BYTES];  // [wave][buffer][K, V]
  __shared__ float stat[4][2][32][2];                 // [wave][map][row][m, l]
  const int unit = unit_of(blockIdx.x, units);
  if (unit < 0) return;
  const int split = unit % splits;
  const int tile = unit / splits % tiles;
  const int bh = unit / splits / tiles;
  const int b = bh / a.Hk, hk = bh % a.Hk, G = a.Hq / a.Hk;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int rows = a.N * G, row0 = 32 * tile, live_rows = min(32, rows - row0);
  const int row = row0 + min(lane % 32, live_rows - 1);
  const int n = row / G, h = hk * G + row % G;
  const Visible vis = visible(a, b);
  const int limit = key_limit(a, vis, n), low = key_limit(a, vis, row0 / G);
  int end = key_limit(a, vis, (row0 + live_rows - 1) / G), key = 0;
  if (splits > 1) {
    const int part = ((end + splits - 1) / splits + K - 1) / K * K;
    key = min(split * part, end);
    end = min(key + part, end);
  }
  Rows32<T, D> r(lane);
  r.load_query(static_cast<const T*>(a.q.p) + b * a.q.sb + h * a.q.sh + n * a.q.sn);
  const T* kp = static_cast<const T*>(a.k.p) + b * a.k.sb + hk * a.k.sh;
  const T* vp = static_cast<const T*>(a.v.p) + b * a.v.sb + hk * a.v.sh;
  const float c = a.scale * kLog2e;
  const auto copy = [&](int at, int buf) {
#pragma unroll
    for (int i = 0; i < 32 / R; ++i)
      copy_rows<D>(kp + at * a.k.sn, 2 * a.k.sn, i * R, vis.len - 1 - at, lane, lds_offset(lds[wave][buf][0]) + i * 1024);
#pragma unroll
    for (int i = 0; i < 32 / R; ++i)
      copy_rows<D>(vp + at * a.v.sn, 2 * a.v.sn, i * R, vis.len - 1 - at, lane, lds_offset(lds[wave][buf][1]) + i * 1024);
  };
  // a wave's keys are its own: it waits for its copies, and for no other wave
  key += 32 * wave;
  if (key < end) copy(key, 0);
  for (int buf = 0; key < end; key += K, buf ^= 1) {
    wait_copies();  // and the other buffer has been read
    if (key + K < end) copy(key + K, buf ^ 1);
    r.step(lds_offset(lds[wave][buf][0]), lds_offset(lds[wave][buf][1]), 0, key, limit, key + 32 > low, c);
  }
  // The waves' parts are joined in LDS, in the room of the tiles: [wave][row][map][channel].
  __syncthreads();
  float* join = reinterpret_cast<float*>(lds);
  const int row_l = lane % 32;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float l = sum_halves(r.l[i]);
    if (lane < 32) {
      stat[wave][i][row_l][0] = r.m[i];
      stat[wave][i][row_l][1] = l;
    }
    if (row_l < live_rows)
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          *reinterpret_cast<float4*>(join + ((wave * 32 + row_l) * 2 + i) * D + 32 * t + 2 * e + 4 * (lane / 32)) =
              make_float4(r.u[i][t][e], r.u[i][t][e + 1], r.u[i][t][e + 2], r.u[i][t][e + 3]);
  }
  __syncthreads();
  for (int x = threadIdx.x; x < live_rows * D; x += kThreads) {
    const int rr = x / D, ch = x % D;
    float m[2], l[2] = {0.0f, 0.0f}, u[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      m[i] = fmaxf(fmaxf(stat[0][i][rr][0], stat[1][i][rr][0]), fmaxf(stat[2][i][rr][0], stat[3][i][rr][0]));
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = exp2_fast(stat[w][i][rr][0] - m[i]);
        l[i] += f * stat[w][i][rr][1];
        u[i] += f * join[((w * 32 + rr) * 2 + i) * D + ch];
      }
    }
    const int at = row0 + rr;
    if (splits == 1) {
      const int nn = at / G, hh = hk * G + at % G;
      finish_element<T>(a, b, hh, nn, ch, u[0], u[1], l[0], l[1]);
      if (a.lse && ch < 2) store_lse(a, b, hh, nn, ch, ch ? m[1] : m[0], ch ? l[1] : l[0]);
    } else {
      float* part = a.ws + ((static_cast<int64_t>(bh) * rows + at) * splits + split) * kPart<D>;
      part[ch] = u[0];
      part[D + ch] = u[1];
      if (ch < 2) {
        part[2 * D + 2 * ch] = ch ? m[1] : m[0];
        part[2 * D + 2 * ch + 1] = ch ? l[1] : l[0];
      }
    }
  }
}

// The parts of a row joined, a workgroup a row: the parts' factors from their statistics, a part a thread; then D/2
// threads (4 channels of a map each) add up every WAYS-th part, and their sums are added in order.
constexpr int kMostParts = 256;  // as cut_of gives them
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void diff_join_kernel(DiffArgs a, int splits) {
  constexpr int TPP = D / 2, WAYS = kThreads / TPP;
  __shared__ float factor[2][kMostParts], wave_max[2][4], wave_sum[2][4];
  __shared__ __align__(16) f32x4 sums[WAYS][TPP];
  const uint32_t r = blockIdx.x;
  const int G = a.Hq / a.Hk, tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const uint32_t rows = static_cast<uint32_t>(a.N) * G, bh = r / rows, row = r - bh * rows;
  const int b = bh / a.Hk, n = row / G, h = bh % a.Hk * G + row % G;
  const float* part = a.ws + static_cast<int64_t>(r) * splits * kPart<D>;
  const bool mine = tid < splits;
  f32x4 st = {kNoMax, 0.0f, kNoMax, 0.0f};
  if (mine) st = *reinterpret_cast<const f32x4*>(part + tid * kPart<D> + 2 * D);
  float m[2], l[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float t = wave_max_f32(st[2 * i]);
    if (lane == 0) wave_max[i][wave] = t;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    m[i] = fmaxf(fmaxf(wave_max[i][0], wave_max[i][1]), fmaxf(wave_max[i][2], wave_max[i][3]));
    const float f = exp2_fast(st[2 * i] - m[i]);
    if (mine) factor[i][tid] = f;
    const float t = wave_sum_f32(mine ? f * st[2 * i + 1] : 0.0f);
    if (lane == 0) wave_sum[i][wave] = t;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) l[i] = (wave_sum[i][0] + wave_sum[i][1]) + (wave_sum[i][2] + wave_sum[i][3]);
  const int at = tid % TPP, way = tid / TPP, map = at / (D / 4);
  f32x4 u{};
#pragma unroll 4
  for (int s = way; s < splits; s += WAYS)
    u += factor[map][s] * *reinterpret_cast<const f32x4*>(part + static_cast<int64_t>(s) * kPart<D> + 4 * at);
  sums[way][at] = u;
  __syncthreads();
  if (tid < D / 4) {
    f32x4 u1 = sums[0][tid], u2 = sums[0][D / 4 + tid];
#pragma unroll
    for (int w = 1; w < WAYS; ++w) {
      u1 += sums[w][tid];
      u2 += sums[w][D / 4 + tid];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) finish_element<T>(a, b, h, n, 4 * tid + i, u1[i], u2[i], l[0], l[1]);
  }
  if (a.lse && tid < 2) store_lse(a, b, h, n, tid, tid ? m[1] : m[0], tid ? l[1] : l[0]);
}

template <typename T, int D>
hipError_t launch(const DiffArgs& a, hipStream_t stream) {
  const Cut c = cut_of(a.B, a.Hq, a.Hk, a.N, a.M);
  const int units = a.B * a.Hk * c.tiles * c.splits;
  if (c.few) {
    diff_few_kernel<T, D><<<grid_of(units), kThreads, 0, stream>>>(a, c.tiles, c.splits, units);
  } else {
    // Waves that share a row's keys pay where 4-wave workgroups leave SIMDs with one wave or none, or a causal mask leaves
    // the last of them alone: 192 tiles of 2,048 keys 67 -> 50 us, 384 causal ones of up to 4,096 168 -> 114, but 384
    // without a mask 177 -> 197. Four of them, on half the rows, pay while each half still finds a CU of its own: 64 tiles
    // of 1,024 keys 28 -> 25 us, 126 of 777 keys of 64 channels 18.2 -> 14.7, but 192 of 1,024 keys 29 -> 47.
    if (units > (a.causal ? 512 : 256)) {
      diff_many_kernel<T, D, 1><<<grid_of(units), kThreads, 0, stream>>>(a, c.tiles, c.splits, units);
    } else if (units > 128 || c.splits > 1) {
      diff_many_kernel<T, D, 2><<<grid_of(units), 2 * kThreads, 0, stream>>>(a, c.tiles, c.splits, units);
    } else {
      const int tiles = static_cast<int>((static_cast<int64_t>(a.N) * (a.Hq / a.Hk) + 63) / 64), n = a.B * a.Hk * tiles;
      diff_many_kernel<T, D, 4><<<grid_of(n), 2 * kThreads, 0, stream>>>(a, tiles, 1, n);
    }
  }
  if (c.splits > 1 && !c.few) {
    const int blocks = units / c.splits * 4;
    diff_many_join_kernel<T, D><<<(blocks * (D / 32) + 3) / 4, kThreads, 0, stream>>>(a, c.tiles, c.splits, blocks);
  } else if (c.splits > 1) {
    diff_join_kernel<T, D><<<static_cast<unsigned>(a.B) * a.Hq * a.N, kThreads, 0, stream>>>(a, c.splits);  // at most 256 tiles of 32 rows
  }
  return hipGetLastError();
}

}  // namespace

int64_t diff_fwd_ws_bytes(int B, int Hq, int Hk, int N, int M, int d) {
  const Cut c = cut_of(B, Hq, Hk, N, M);
  if (c.splits == 1) return 0;
  if (c.few) return 4ll * B * Hq * N * c.splits * (2 * d + 4);
  return 16ll * B * Hk * c.tiles * c.splits * 4 * (d == 128 ? kBlock<128> : kBlock<64>);
}

hipError_t launch_diff_fwd(const DiffArgs& a, hipStream_t stream) {
  if (a.dtype == DA2_BF16) return a.d == 128 ? launch<bf16_t, 128>(a, stream) : launch<bf16_t, 64>(a, stream);
  return a.d == 128 ? launch<fp16_t, 128>(a, stream) : launch<fp16_t, 64>(a, stream);
}

}  // namespace da2
