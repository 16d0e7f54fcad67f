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
//   - many rows: 4 waves with 128 rows walk 64-key tiles that they share;
//   - few rows (up to 64): 4 waves with the same 32 rows walk the 32-key quarters
//     of 128-key tiles, each its own, and are joined at the end.
// Where that leaves CUs idle the keys are split over workgroups; a second kernel
// joins the parts.
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
  // two workgroups a CU; a part of fewer than 256 keys costs more to join than to walk
  int64_t s = 512 / units, most = (M + 255) / 256;
  s = s < most ? s : most;
  c.splits = static_cast<int>(s < 1 ? 1 : s);
  return c;
}

// One part of a row: its unnormalised outputs, maxima and sums.
template <int D>
constexpr int kPart = 2 * D + 4;

// 32 rows (a lane's query is lane%32) against 32 keys of a K and a V tile in LDS.
template <typename T, int D>
struct Rows32 {
  static constexpr int S = D / 32;  // 16-channel steps of a map
  static constexpr int C = D / 32;  // 32-channel tiles of V
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
  // Keys [key, key + 32) at rows 32 j of the tiles kt and vt; limit: the lane's query sees the keys below it.
  __device__ void step(uint32_t kt, uint32_t vt, int j, int key, int limit, bool mask, float c) {
    s16x8 p[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f32x16 x{};
#pragma unroll
      for (int s = 0; s < S; ++s) x = mma<T>(rows.read(kt, j, i * S + s), q[i][s], x);
      if (mask) {
        const int left = limit - key - 16 * (lane / 32);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = e < left ? x[e] : -__builtin_inff();
      }
      // The maximum is a reference for the exponentials only: it follows when a score passes it by 2^8, which the
      // weights' float32 sums and 16-bit values hold, so that the accumulators are rarely rescaled.
      const float top = max_halves(max16(x)) * c;
      if (__any(top > m[i] + 8.0f)) {
        const float to = fmaxf(m[i], top), f = exp2_fast(m[i] - to);
        m[i] = to;
        l[i] *= f;
#pragma unroll
        for (int t = 0; t < C; ++t) u[i][t] *= f;
      }
      float w[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        w[e] = exp2_fast(__builtin_fmaf(x[e], c, -m[i]));
        l[i] += w[e];
      }
      p[i][0] = pack8<T>(w);
      p[i][1] = pack8<T>(w + 8);
    }
#pragma unroll
    for (int t = 0; t < C; ++t)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const s16x8 v = cols.read(vt, j, t, s);
        u[0][t] = mma<T>(v, p[0][s], u[0][t]);
        u[1][t] = mma<T>(v, p[1][s], u[1][t]);
      }
  }
};

template <typename T>
__device__ inline T* row_ptr(const OutView& o, int b, int h, int n) {
  return static_cast<T*>(o.p) + b * o.sb + h * o.sh + n * o.sn;
}

__device__ inline void store_lse(const DiffArgs& a, int b, int h, int n, int i, float m, float l) {
  a.lse[((static_cast<int64_t>(b) * a.Hq + h) * 2 + i) * a.N + n] =
      l > 0.0f ? kLn2 * (m + __builtin_amdgcn_logf(l)) : -__builtin_inff();
}

// Output of one row from its accumulators as columns (see store_columns).
template <typename T, int D>
__device__ inline void finish_rows(const DiffArgs& a, Rows32<T, D>& r, int b, int h, int n, bool live) {
  float inv[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float l = sum_halves(r.l[i]);
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

template <typename T, int D>
__global__ __launch_bounds__(kThreads, 2) void diff_many_kernel(DiffArgs a, int tiles, int splits, int64_t units) {
  constexpr int K = 64, BYTES = K * Tile<D>::kRow, R = Tile<D>::kRowsPerCopy;
  __shared__ __align__(256) char lds[2][2][BYTES];  // [buffer][K, V]
  const int64_t unit = unit_of(blockIdx.x, units);
  if (unit < 0) return;
  const int split = static_cast<int>(unit % splits);
  // the last rows see most keys under a causal mask: they go first
  const int tile = tiles - 1 - static_cast<int>(unit / splits % tiles);
  const int64_t bh = unit / splits / tiles;
  const int b = static_cast<int>(bh / a.Hk), hk = static_cast<int>(bh % a.Hk), G = a.Hq / a.Hk;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t rows = static_cast<int64_t>(a.N) * G, row0 = static_cast<int64_t>(tile) * 128 + 32 * wave;
  const auto token = [&](int64_t r) { return static_cast<int>((r < rows ? r : rows - 1) / G); };
  const int64_t row = row0 + lane % 32;
  const bool live = row < rows;
  const int n = token(row), h = hk * G + static_cast<int>((live ? row : rows - 1) % G);
  const Visible vis = visible(a, b);
  const int limit = key_limit(a, vis, n);
  const int low = key_limit(a, vis, token(row0)), high = key_limit(a, vis, token(row0 + 31));  // of the wave
  int end = key_limit(a, vis, token(static_cast<int64_t>(tile) * 128 + 127));                 // of the workgroup
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
    for (int i = 0; i < K / R / 4; ++i) {
      const int first = (wave * (K / R / 4) + i) * R;
      copy_rows<D>(kp + at * a.k.sn, 2 * a.k.sn, first, vis.len - 1 - at, lane, lds_offset(lds[buf][0]) + first * Tile<D>::kRow);
      copy_rows<D>(vp + at * a.v.sn, 2 * a.v.sn, first, vis.len - 1 - at, lane, lds_offset(lds[buf][1]) + first * Tile<D>::kRow);
    }
  };
  if (key < end) copy(key, 0);
  for (int buf = 0; key < end; key += K, buf ^= 1) {
    wait_copies();
    barrier();  // every wave's copies have arrived, and the other buffer has been read
    if (key + K < end) copy(key + K, buf ^ 1);
    const uint32_t kt = lds_offset(lds[buf][0]), vt = lds_offset(lds[buf][1]);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int at = key + 32 * j;
      if (at < min(high, end)) r.step(kt, vt, j, at, limit, at + 32 > low, c);
    }
  }
  if (splits == 1) {
    finish_rows(a, r, b, h, n, live);
    return;
  }
  float* part = a.ws + ((bh * rows + (live ? row : rows - 1)) * splits + split) * kPart<D>;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float l = sum_halves(r.l[i]);
    if (live && lane < 32) {
      part[2 * D + 2 * i] = r.m[i];
      part[2 * D + 2 * i + 1] = l;
    }
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        if (live)
          *reinterpret_cast<float4*>(part + i * D + 32 * t + 2 * e + 4 * (lane / 32)) =
              make_float4(r.u[i][t][e], r.u[i][t][e + 1], r.u[i][t][e + 2], r.u[i][t][e + 3]);
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads, 1) void diff_few_kernel(DiffArgs a, int tiles, int splits, int64_t units) {
  constexpr int K = 128, BYTES = 32 * Tile<D>::kRow, R = Tile<D>::kRowsPerCopy;
  __shared__ __align__(256) char lds[4][2][2][BYTES];  // [wave][buffer][K, V]
  __shared__ float stat[4][2][32][2];                 // [wave][map][row][m, l]
  const int64_t unit = unit_of(blockIdx.x, units);
  if (unit < 0) return;
  const int split = static_cast<int>(unit % splits);
  const int tile = static_cast<int>(unit / splits % tiles);
  const int64_t bh = unit / splits / tiles;
  const int b = static_cast<int>(bh / a.Hk), hk = static_cast<int>(bh % a.Hk), G = a.Hq / a.Hk;
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
      float* part = a.ws + ((bh * rows + at) * splits + split) * kPart<D>;
      part[ch] = u[0];
      part[D + ch] = u[1];
      if (ch < 2) {
        part[2 * D + 2 * ch] = ch ? m[1] : m[0];
        part[2 * D + 2 * ch + 1] = ch ? l[1] : l[0];
      }
    }
  }
}

// The parts of each row joined: D threads a row.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void diff_join_kernel(DiffArgs a, int splits, int64_t rows_all) {
  const int64_t r = static_cast<int64_t>(blockIdx.x) * (kThreads / D) + threadIdx.x / D;
  if (r >= rows_all) return;
  const int ch = threadIdx.x % D, G = a.Hq / a.Hk;
  const int64_t rows = static_cast<int64_t>(a.N) * G, bh = r / rows, row = r - bh * rows;
  const int b = static_cast<int>(bh / a.Hk), n = static_cast<int>(row / G);
  const int h = static_cast<int>(bh % a.Hk) * G + static_cast<int>(row % G);
  const float* part = a.ws + r * splits * kPart<D>;
  float m[2] = {kNoMax, kNoMax}, l[2] = {0.0f, 0.0f}, u[2] = {0.0f, 0.0f};
  for (int s = 0; s < splits; ++s)
#pragma unroll
    for (int i = 0; i < 2; ++i) m[i] = fmaxf(m[i], part[s * kPart<D> + 2 * D + 2 * i]);
  for (int s = 0; s < splits; ++s, part += kPart<D>)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float f = exp2_fast(part[2 * D + 2 * i] - m[i]);
      l[i] += f * part[2 * D + 2 * i + 1];
      u[i] += f * part[i * D + ch];
    }
  finish_element<T>(a, b, h, n, ch, u[0], u[1], l[0], l[1]);
  if (a.lse && ch < 2) store_lse(a, b, h, n, ch, ch ? m[1] : m[0], ch ? l[1] : l[0]);
}

template <typename T, int D>
hipError_t launch(const DiffArgs& a, hipStream_t stream) {
  const Cut c = cut_of(a.B, a.Hq, a.Hk, a.N, a.M);
  const int64_t units = static_cast<int64_t>(a.B) * a.Hk * c.tiles * c.splits;
  if (c.few) {
    diff_few_kernel<T, D><<<grid_of(units), kThreads, 0, stream>>>(a, c.tiles, c.splits, units);
  } else {
    diff_many_kernel<T, D><<<grid_of(units), kThreads, 0, stream>>>(a, c.tiles, c.splits, units);
  }
  if (c.splits > 1) {
    const int64_t rows = static_cast<int64_t>(a.B) * a.Hq * a.N;
    diff_join_kernel<T, D><<<static_cast<unsigned>((rows + kThreads / D - 1) / (kThreads / D)), kThreads, 0, stream>>>(
        a, c.splits, rows);
  }
  return hipGetLastError();
}

}  // namespace

int64_t diff_fwd_ws_bytes(int B, int Hq, int Hk, int N, int M, int d) {
  const Cut c = cut_of(B, Hq, Hk, N, M);
  return c.splits == 1 ? 0 : 4ll * B * Hq * N * c.splits * (2 * d + 4);
}

hipError_t launch_diff_fwd(const DiffArgs& a, hipStream_t stream) {
  if (a.dtype == DA2_BF16) return a.d == 128 ? launch<bf16_t, 128>(a, stream) : launch<bf16_t, 64>(a, stream);
  return a.d == 128 ? launch<fp16_t, 128>(a, stream) : launch<fp16_t, 64>(a, stream);
}

}  // namespace da2
