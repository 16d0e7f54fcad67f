// Differential attention, backward.
//
// With P1, P2 the softmax maps, dP = dO V^T and del_i the row sums of P_i dP:
//   dS1 = P1 (dP - del1),  dS2 = -lambda P2 (dP - del2),
//   dQ_i = c dS_i K_i,  dK_i = c dS_i^T Q_i,  dV = (P1 - lambda P2)^T dO,
//   dlambda = -sum of del2.
// The maps are computed again from the scores and the forward pass's log sums.
//
// del_i equals dO . (output of map i), but outputs stored in 16 bits are too
// coarse for it: their rounding moves every dS_i of a row the same way, which
// the middle of K does not cancel (2.5 times the error of the gradients' own
// rounding, measured), and dlambda is a sum in which most of del2 cancels. So
// the rows are walked twice: once for del_i, in float32 from unrounded weights,
// then for dQ. (Not tried: one walk with a del from such outputs, and what it was
// off by, summed on the way, taken out of dQ with the weights' own sum of K.)
//
// Two kernels: dQ, where a wave keeps 32 queries and walks over the keys; dK and
// dV, where a wave keeps 32 keys and walks over the queries. Each recomputes the
// scores and dP, and neither adds into memory, so the results do not depend on
// the order of workgroups and nothing has to be cleared. In multiply-adds of d
// per pair: 2 for del, 3 for dQ, 4 for dK and dV, where one pass over both sides
// (which would need sums in memory) takes 5 beside del. (bf16, 2 x 2,048 causal
// tokens, 12 heads on 4 key heads, d = 128: dQ 114 us, dK and dV 85, joined in 17.)
//
// The weights and score gradients are rounded to 16 bits for their products. In
// fp16 that would lose them: a weight is about one over the number of keys, and dS
// that times dO, so over 4,096 keys a dO of 1e-4 leaves dS a few bits of fp16's
// subnormal numbers (error of dQ 2.4%, of dQ's own rounding 0.2%), and one of 1e4
// overflows. So fp16 products take them times a power of two, which their float32
// sums give back: dS of a row in dQ by the row's largest |dP|; in dK and dV, whose
// sums run over rows, dS by a key head's largest |dP| and the weights by its
// largest |lambda|. |dS| is at most 2 P |dP| (times |lambda| in the second map),
// so they stay below 2^15.
#include <algorithm>
#include <type_traits>

#include "diff.hpp"

namespace da2 {

namespace {

using namespace diff;

constexpr int kThreads = 256;

// Statistics of the rows of a head, 64 at a time, as dK and dV take them:
//   - minus the log sums of both maps in units of the raw scores, where the sums of the scores start, so that their
//     exponentials are the weights (the second map's with |lambda| in its log sum);
//   - minus del1, where dP's sums start; and del1 - del2 with lambda's sign turned, so that
//     sgn dP' = (-sgn lambda) (dP - del1) + this is the second map's factor.
// Rows from N on hold values that make every weight zero.
constexpr int kStat = 4 * 64;  // floats of 64 rows: [4][64]
constexpr int64_t padded(int64_t n) { return (n + 63) / 64 * 64; }
__device__ inline float* stat_at(float* stat, int64_t bh, int64_t n, int N) {
  return stat + (bh * (padded(N) / 64) + n / 64) * kStat + n % 64;
}
__device__ inline float minus_sign(float lambda) { return lambda < 0.0f ? 1.0f : -1.0f; }
__device__ inline void put_stat(float* s, float l1, float l2, float d1, float d2, float lambda, float c) {
  s[0] = -l1;
  s[64] = __builtin_amdgcn_logf(fabsf(lambda)) / c - l2;
  s[128] = -d1;
  s[192] = (d1 - d2) * minus_sign(lambda);
}
constexpr float kNever = __builtin_inff();

// A value at a wave-uniform address that the kernel does not write, through the scalar cache: a vector load would wait
// for the copies issued before it.
__device__ inline float load_uniform(const float* p) { return *(const __attribute__((address_space(4))) float*)p; }

// Whether products of T take scaled weights and score gradients.
template <typename T>
constexpr bool kScaled = __is_same(T, fp16_t);
// e with |x| < 2^e and, unless that leaves the range in which 2^e and 2^-e are floats with room to spare, 2^e <= 2 |x|.
__device__ inline int exponent_above(float x) { return min(max(__builtin_amdgcn_frexp_expf(x), -100), 100); }

// 16 floats of LDS, the same for all lanes of a half.
__device__ inline f32x16 read16(const float* p) {
  f32x16 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p + 4 * i);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[4 * i + e] = v[e];
  }
  return x;
}

// dlambda of a head: minus the sum of its rows' del2, in float64 and in a fixed order.
template <int THREADS>
__device__ inline void sum_dlam(const DiffArgs& a, float* stat, int h, double* sums) {
  double t = 0.0;
  for (int b = 0; b < a.B; ++b)
#pragma unroll 4
    for (int n = threadIdx.x; n < a.N; n += THREADS) {
      const float* s = stat_at(stat, static_cast<int64_t>(b) * a.Hq + h, n, a.N);
      t += -static_cast<double>(s[128]) - s[192] * minus_sign(a.lam[h]);
    }
  sums[threadIdx.x] = t;
  __syncthreads();
  for (int o = THREADS / 2; o > 0; o >>= 1) {
    if (threadIdx.x < o) sums[threadIdx.x] += sums[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) a.dlam[h] = static_cast<float>(-sums[0]);
}

// The largest values of a key head's n tops, into the first of as many slots. For more of them than dK and dV's workgroups
// have threads: a loop over them there takes registers that the loop over the queries needs.
constexpr int kMostTops = kThreads;
__global__ __launch_bounds__(kThreads) void diff_tops_kernel(const float2* tops, int n, float2* out) {
  __shared__ float most[2][kThreads / 64];
  const float2* top = tops + static_cast<int64_t>(blockIdx.x) * n;
  float t = 0.0f, l = 0.0f;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    t = fmaxf(t, top[i].x);
    l = fmaxf(l, top[i].y);
  }
  t = wave_max_f32(t);
  l = wave_max_f32(l);
  if (threadIdx.x % 64 == 0) {
    most[0][threadIdx.x / 64] = t;
    most[1][threadIdx.x / 64] = l;
  }
  __syncthreads();
  if (threadIdx.x == 0)
    out[blockIdx.x] = make_float2(fmaxf(fmaxf(most[0][0], most[0][1]), fmaxf(most[0][2], most[0][3])),
                                  fmaxf(fmaxf(most[1][0], most[1][1]), fmaxf(most[1][2], most[1][3])));
}

// dK and dV of 128 keys: 4 waves with 32 keys each; 32 queries of one head at a time in LDS. A wave's keys are in
// registers, its values in LDS: both in registers would leave one wave a SIMD at d = 128. HALVES = 2: twice the waves,
// the second four with the same keys and every other tile of queries. The first workgroups, a multiple of 8, sum dlambda
// beside them.
template <typename T, int D, int HALVES>
__global__ __launch_bounds__(HALVES * kThreads, D == 64 && HALVES == 1 ? 3 : 2) void diff_dkv_kernel(
    DiffArgs a, float* stat, const float2* tops, int n_tops, float* sums, int tiles, int parts, int units, int lambdas) {
  constexpr int S = D / 32, Q = 32, BYTES = Q * Tile<D>::kRow, R = Tile<D>::kRowsPerCopy;
  __shared__ __align__(256) char lds[2][HALVES][2][BYTES];  // [buffer][half][Q, dO]
  __shared__ __align__(256) char val[4 * BYTES];            // the workgroup's rows of V
  __shared__ __align__(16) float st[2][HALVES][4][Q];
  __shared__ float most[2][4 * HALVES];  // |dP| and |lambda|, by wave
  if (static_cast<int>(blockIdx.x) < lambdas) {
    if (static_cast<int>(blockIdx.x) < a.Hq) sum_dlam<HALVES * kThreads>(a, stat, blockIdx.x, reinterpret_cast<double*>(lds));
    return;
  }
  const int unit = unit_of(blockIdx.x - lambdas, units);
  if (unit < 0) return;
  // the first keys are seen by most queries under a causal mask: they go first
  const int part = unit % parts, tile = unit / parts % tiles, bh = unit / parts / tiles;
  const int b = bh / a.Hk, hk = bh % a.Hk, G = a.Hq / a.Hk;
  const int lane = threadIdx.x % 64, g = lane / 32, half = __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64) % 4;
  const Visible vis = visible(a, b);
  const int key0 = tile * 128 + 32 * wave, key = key0 + lane % 32;

  f32x16 dv[S], dk[2][S / 2];
#pragma unroll
  for (int t = 0; t < S; ++t) dv[t] = dk[t / (S / 2)][t % (S / 2)] = f32x16{};

  if constexpr (kScaled<T>) {
    const float2 x = tops[static_cast<int64_t>(bh) * n_tops + min(static_cast<int>(threadIdx.x), n_tops - 1)];
    const float t = wave_max_f32(x.x), l = wave_max_f32(x.y);
    if (lane == 0) {
      most[0][threadIdx.x / 64] = t;
      most[1][threadIdx.x / 64] = l;
    }
    __syncthreads();
  }
  // Exponents of the scales of the weights and of dS; read again where they are needed, which spares registers.
  const auto scales = [&](int& kw, int& ks) {
    float t = most[0][0], l = most[1][0];
#pragma unroll
    for (int i = 1; i < 4 * HALVES; ++i) {
      t = fmaxf(t, most[0][i]);
      l = fmaxf(l, most[1][i]);
    }
    kw = 14 - min(max(exponent_above(l), 0), 20);  // 1 + |lambda| < 2^(15 - kw)
    ks = kw - exponent_above(t);
  };

  // queries that see the tile's first key
  const int64_t seen = a.causal ? tile * 128 - vis.start : 0;
  const int n_first = static_cast<int>(seen < 0 ? 0 : seen < a.N ? seen : a.N) / Q * Q;
  const int n_tiles = tile * 128 < vis.len && seen < a.N ? (a.N - n_first + Q - 1) / Q : 0;
  // this part of them, over all heads
  const int each = (G * n_tiles + parts - 1) / parts, begin = part * each, total = min(begin + each, G * n_tiles);

  if (begin < total) {
    s16x8 kf[2][S];
    {
      const int64_t row = min(key, vis.len - 1);
      const T* kp = static_cast<const T*>(a.k.p) + b * a.k.sb + hk * a.k.sh + row * a.k.sn + 8 * g;
#pragma unroll
      for (int c = 0; c < 2 * S; ++c) kf[c / S][c % S] = *reinterpret_cast<const s16x8*>(kp + 16 * c);
    }
    const T* vp = static_cast<const T*>(a.v.p) + b * a.v.sb + hk * a.v.sh + static_cast<int64_t>(tile) * 128 * a.v.sn;
#pragma unroll
    for (int i = half; i < Q / R; i += HALVES)  // each wave its own rows
      copy_rows<D>(vp, 2 * a.v.sn, Q * wave + i * R, vis.len - 1 - tile * 128, lane, lds_offset(val) + wave * BYTES + i * 1024);
    const uint32_t vt = lds_offset(val) + wave * BYTES;
    const RowReader<D> rows(lane, true), keys(lane, false);
    const ColReader<D> cols(lane);
    const float c = a.scale * kLog2e;
    float raise = 0.0f, to_w = 1.0f;  // p is a weight times 2^raise
    if constexpr (kScaled<T>) {
      int kw, ks;
      scales(kw, ks);
      raise = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(static_cast<float>(ks))));
      to_w = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(__builtin_ldexpf(1.0f, kw - ks))));
    }
    const auto copy = [&](int at, int buf) {
      int ln = lane;
      // The offsets are formed at every step: kept over the loop, they take the registers that a third wave needs (fp16, 768
      // tiles of 8,192 queries 1,460 -> 1,395 us for the backward pass, 384 causal ones 293 -> 302).
      if constexpr (kScaled<T> && D == 64 && HALVES == 1) asm volatile("" : "+v"(ln));
      const int h = hk * G + at / n_tiles, n0 = n_first + at % n_tiles * Q;
      const T* qp = static_cast<const T*>(a.q.p) + b * a.q.sb + h * a.q.sh + n0 * a.q.sn;
      const T* op = static_cast<const T*>(a.dout.p) + b * a.dout.sb + h * a.dout.sh + n0 * a.dout.sn;
      // 2 Q / R copies of 1 KB: each wave takes its share of Q's and of dO's rows
#pragma unroll
      for (int i = wave; i < Q / R; i += 4) {
        copy_rows<D>(qp, 2 * a.q.sn, i * R, a.N - 1 - n0, ln, lds_offset(lds[buf][half][0]) + i * 1024);
        copy_rows<D>(op, 2 * a.dout.sn, i * R, a.N - 1 - n0, ln, lds_offset(lds[buf][half][1]) + i * 1024);
      }
      if (wave == 0 && ln < Q)  // four times 32 floats
        copy_1k(stat_at(stat, static_cast<int64_t>(b) * a.Hq + h, n0, a.N), (ln / 8) * 256 + (ln % 8) * 16,
                __builtin_amdgcn_readfirstlane(lds_offset(st[buf][half])));
    };
    if (begin + half < total) copy(begin + half, 0);
    for (int at = begin + half, buf = 0; at - half < total; at += HALVES, buf ^= 1) {
      wait_copies();
      barrier();  // every wave's copies have arrived, and the other buffer has been read
      if (at + HALVES < total) copy(at + HALVES, buf ^ 1);
      if (HALVES == 2 && at >= total) continue;  // the last tile is the first half's
      const int n = n_first + at % n_tiles * Q;
      // the wave's first key is seen by none of the 32 queries
      if (a.causal && key0 > vis.start + n + 31) continue;
      const float minus = minus_sign(load_uniform(a.lam + hk * G + at / n_tiles));
      const uint32_t qt = lds_offset(lds[buf][half][0]), ot = lds_offset(lds[buf][half][1]);
      // query n + 16 g + e sees the key from e = first on
      const int64_t behind = key - vis.start - n - 16 * g;
      const int first = static_cast<int>(behind < 0 ? 0 : behind < 16 ? behind : 16);
      const bool hidden = a.causal && key0 + 31 > vis.start + n;  // the wave's last key from some of the queries
      f32x16 dp = read16(&st[buf][half][2][16 * g]);  // dP - del1
#pragma unroll
      for (int s = 0; s < 2 * S; ++s) dp = mma<T>(rows.read(ot, 0, s), keys.read(vt, 0, s), dp);
      s16x8 df[2][2];
      float w[16];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f32x16 x = read16(&st[buf][half][i][16 * g]);
#pragma unroll
        for (int s = 0; s < S; ++s) x = mma<T>(rows.read(qt, 0, i * S + s), kf[i][s], x);
        if (hidden)
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] = e < first ? -__builtin_inff() : x[e];
        float d[16];
        if (i) {  // (-sgn lambda) (dP - del2)
          const f32x16 y = read16(&st[buf][half][3][16 * g]);
#pragma unroll
          for (int e = 0; e < 16; ++e) dp[e] = __builtin_fmaf(dp[e], minus, y[e]);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          if constexpr (kScaled<T>) {
            const float p = exp2_fast(__builtin_fmaf(x[e], c, raise));
            w[e] = i ? __builtin_fmaf(p, minus * to_w, w[e]) : p * to_w;
            d[e] = p * dp[e];
          } else {
            const float p = exp2_fast(x[e] * c);
            w[e] = i ? __builtin_fmaf(p, minus, w[e]) : p;
            d[e] = p * dp[e];
          }
        }
        df[i][0] = pack8<T>(d);
        df[i][1] = pack8<T>(d + 8);
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const s16x8 wf = pack8<T>(w + 8 * s);
#pragma unroll
        for (int t = 0; t < S; ++t) {
          dv[t] = mma<T>(wf, cols.read(ot, 0, t, s), dv[t]);
          f32x16& k = dk[t / (S / 2)][t % (S / 2)];
          k = mma<T>(df[t / (S / 2)][s], cols.read(qt, 0, t, s), k);
        }
      }
    }
  }
  if constexpr (HALVES == 2) {
    // the second half's sums, dV's first, go to the first half's waves in the room of the tiles
    f32x4* swap = reinterpret_cast<f32x4*>(lds) + wave * 4 * S * 64 + lane;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
      wait_copies();
      __syncthreads();
#pragma unroll
      for (int t = 0; t < S; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x16& x = pass ? dk[t / (S / 2)][t % (S / 2)] : dv[t];
          if (half) swap[(4 * t + e) * 64] = f32x4{x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]};
        }
      __syncthreads();
#pragma unroll
      for (int t = 0; t < S; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f32x16& x = pass ? dk[t / (S / 2)][t % (S / 2)] : dv[t];
          if (!half) {
            const f32x4 y = swap[(4 * t + e) * 64];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[4 * e + k] += y[k];
          }
        }
    }
    if (half) return;
  }
  if constexpr (kScaled<T>) {
    int kw, ks;
    scales(kw, ks);
    const float fw = __builtin_ldexpf(1.0f, -kw), fs = __builtin_ldexpf(1.0f, -ks);
#pragma unroll
    for (int t = 0; t < S; ++t) {
      dv[t] *= fw;
      dk[t / (S / 2)][t % (S / 2)] *= fs;
    }
  }
  // accumulator register e: key 8 (e/4) + 4 g + e%4, lane%32: channel
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int kk = key0 + 8 * (e / 4) + 4 * g + e % 4;
    if (kk >= a.M) continue;
    if (parts > 1) {
      float* s = sums + ((static_cast<int64_t>(part) * a.B * a.Hk + bh) * a.M + kk) * 2 * D + lane % 32;
#pragma unroll
      for (int t = 0; t < S; ++t) {
        s[32 * t] = dk[t / (S / 2)][t % (S / 2)][e];
        s[D + 32 * t] = dv[t][e];
      }
      continue;
    }
    const bool valid = kk < vis.len;
    T* kp = static_cast<T*>(a.dk.p) + b * a.dk.sb + hk * a.dk.sh + kk * a.dk.sn + lane % 32;
    T* vp = static_cast<T*>(a.dv.p) + b * a.dv.sb + hk * a.dv.sh + kk * a.dv.sn + lane % 32;
#pragma unroll
    for (int t = 0; t < S; ++t) {
      kp[32 * t] = static_cast<T>(valid ? dk[t / (S / 2)][t % (S / 2)][e] * a.scale : 0.0f);
      vp[32 * t] = static_cast<T>(valid ? dv[t][e] : 0.0f);
    }
  }
}

// The parts of dK and dV added up in order: D/4 threads a key, with 4 channels of each.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void diff_dkv_join_kernel(DiffArgs a, const float* sums, int parts, int64_t keys) {
  constexpr int TPK = D / 4;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * (kThreads / TPK) + threadIdx.x / TPK;
  if (r >= keys) return;
  const int bh = static_cast<uint32_t>(r) / static_cast<uint32_t>(a.M), kk = static_cast<uint32_t>(r) - bh * a.M;
  const int b = bh / a.Hk, hk = bh % a.Hk;
  const int ch = threadIdx.x % TPK * 4;
  f32x4 k{}, v{};
  if (kk < visible(a, b).len)
    for (int p = 0; p < parts; ++p) {
      const float* s = sums + (p * keys + r) * 2 * D + ch;
      k += *reinterpret_cast<const f32x4*>(s);
      v += *reinterpret_cast<const f32x4*>(s + D);
    }
  typedef T Tx4 __attribute__((ext_vector_type(4)));
  Tx4 ko, vo;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    ko[i] = static_cast<T>(k[i] * a.scale);
    vo[i] = static_cast<T>(v[i]);
  }
  *reinterpret_cast<Tx4*>(static_cast<T*>(a.dk.p) + b * a.dk.sb + hk * a.dk.sh + kk * a.dk.sn + ch) = ko;
  *reinterpret_cast<Tx4*>(static_cast<T*>(a.dv.p) + b * a.dv.sb + hk * a.dv.sh + kk * a.dv.sn + ch) = vo;
}

// del and dQ of 128 or 64 rows (a key head's query heads together, in workgroups as in the forward pass). The keys go
// through LDS twice. The rows' statistics go to `stat`, of every 32 rows the largest |dP| and |lambda| to `tops` (kScaled
// types).
template <typename T, int D, int SHARE>
__global__ __launch_bounds__(64 * Many<SHARE>::kWaves, 2) void diff_dq_kernel(DiffArgs a, float* stat, float2* tops, int tiles, int units) {
  constexpr int S = D / 32, K = Many<SHARE>::kKeys, WAVES = Many<SHARE>::kWaves, BYTES = K * Tile<D>::kRow, R = Tile<D>::kRowsPerCopy;
  constexpr int GROUPS = Many<SHARE>::kGroups, ROWS = Many<SHARE>::kRows;
  __shared__ __align__(256) char lds[2][2][BYTES];  // [buffer][K, V]
  __shared__ float sums[SHARE][GROUPS][3 + kScaled<T>][64];
  // keys spread over those that the workgroup's rows see, and the middle of them
  constexpr int SAMPLE = 8 * WAVES * 128 / D;
  __shared__ __align__(16) T sample[SAMPLE][D];
  __shared__ __align__(16) float middle[D];
  const int unit = unit_of(blockIdx.x, units);
  if (unit < 0) return;
  const int tile = tiles - 1 - unit % tiles, bh = unit / tiles;
  const int b = bh / a.Hk, hk = bh % a.Hk, G = a.Hq / a.Hk;
  const int lane = threadIdx.x % 64, g = lane / 32, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int group = wave % GROUPS, share = wave / GROUPS;
  const uint32_t rows_all = static_cast<uint32_t>(a.N) * G, row0 = static_cast<uint32_t>(tile) * ROWS + 32 * group;
  const auto token = [&](uint32_t r) { return static_cast<int>(min(r, rows_all - 1) / static_cast<uint32_t>(G)); };
  const bool live = row0 + lane % 32 < rows_all;
  const uint32_t row = min(row0 + lane % 32, rows_all - 1);
  const int n = token(row), h = hk * G + static_cast<int>(row) - n * G;
  const Visible vis = visible(a, b);
  const int limit = key_limit(a, vis, n);
  const int low = key_limit(a, vis, token(row0)), high = key_limit(a, vis, token(row0 + 31));
  const int end = key_limit(a, vis, token(static_cast<uint32_t>(tile) * ROWS + ROWS - 1));

  if (end > 0) {
    const int ch = threadIdx.x % (D / 8) * 8;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int i = threadIdx.x / (D / 8) + r * (SAMPLE / 2);
      const int64_t at = static_cast<int64_t>(end) * i / SAMPLE;
      *reinterpret_cast<uint4*>(&sample[i][ch]) = *reinterpret_cast<const uint4*>(
          static_cast<const T*>(a.k.p) + b * a.k.sb + hk * a.k.sh + at * a.k.sn + ch);
    }
  }
  s16x8 qf[2][S], of[2 * S];
  {
    const T* qp = static_cast<const T*>(a.q.p) + b * a.q.sb + h * a.q.sh + n * a.q.sn + 8 * g;
    const T* op = static_cast<const T*>(a.dout.p) + b * a.dout.sb + h * a.dout.sh + n * a.dout.sn + 8 * g;
#pragma unroll
    for (int s = 0; s < 2 * S; ++s) {
      qf[s / S][s % S] = *reinterpret_cast<const s16x8*>(qp + 16 * s);
      of[s] = *reinterpret_cast<const s16x8*>(op + 16 * s);
    }
  }
  const int64_t bhn = static_cast<int64_t>(b) * a.Hq + h;
  float lse[2], d[3] = {0.0f, 0.0f, 0.0f}, top = 0.0f;  // del1, del2, the sum of P2; the largest |dP| that the row meets
  int ks = 0;                                     // exponent of the scale of its dS
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float l = a.rlse[(bhn * 2 + i) * a.N + n];
    lse[i] = l == -__builtin_inff() ? kNever : l * kLog2e;
  }
  f32x16 dq[2][S / 2];
  float rest[2] = {0.0f, 0.0f};  // sums of the rounded dS of each map
#pragma unroll
  for (int t = 0; t < S; ++t) dq[t / (S / 2)][t % (S / 2)] = f32x16{};
  const RowReader<D> rows(lane, true);
  const ColReader<D> cols(lane);
  const T* kp = static_cast<const T*>(a.k.p) + b * a.k.sb + hk * a.k.sh;
  const T* vp = static_cast<const T*>(a.v.p) + b * a.v.sb + hk * a.v.sh;
  const float c = a.scale * kLog2e;
  const auto copy = [&](int at, int buf) {
#pragma unroll
    for (int i = 0; i < K / R / WAVES; ++i) {
      const int r0 = (wave * (K / R / WAVES) + i) * R;
      copy_rows<D>(kp + at * a.k.sn, 2 * a.k.sn, r0, vis.len - 1 - at, lane, lds_offset(lds[buf][0]) + r0 * Tile<D>::kRow);
      copy_rows<D>(vp + at * a.v.sn, 2 * a.v.sn, r0, vis.len - 1 - at, lane, lds_offset(lds[buf][1]) + r0 * Tile<D>::kRow);
    }
  };
  // P_i dP (pass 0, summed) or dS_i (pass 1) of 32 keys at rows 32 j of the tiles
  const auto walk = [&](auto pass) {
    constexpr bool kSums = decltype(pass)::value == 0;
    if (end > 0) copy(0, 0);
    for (int key = 0, buf = 0; key < end; key += K, buf ^= 1) {
      wait_copies();
      barrier();
      if (key + K < end) copy(key + K, buf ^ 1);
      const uint32_t kt = lds_offset(lds[buf][0]), vt = lds_offset(lds[buf][1]);
#pragma unroll
      for (int jj = 0; jj < K / 32; jj += SHARE) {
        const int j = jj + share;
        const int at = key + 32 * j;
        if (at >= high) continue;
        f32x16 dp{};
#pragma unroll
        for (int s = 0; s < 2 * S; ++s) dp = mma<T>(rows.read(vt, j, s), of[s], dp);
        s16x8 df[2][2];
        const bool mask = at + 32 > low;
        const int left = limit - at - 16 * g;
        if constexpr (kSums && kScaled<T>) {
          if (mask) {
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, e < left ? fabsf(dp[e]) : 0.0f);
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(dp[e]));
          }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          f32x16 x{};
#pragma unroll
          for (int s = 0; s < S; ++s) x = mma<T>(rows.read(kt, j, i * S + s), qf[i][s], x);
          const float l = kScaled<T> && !kSums ? lse[i] - static_cast<float>(ks) : lse[i];
          float ds[16], sum = 0.0f, whole = 0.0f;  // of P dP over 16 keys, and of P
          if (mask)
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = e < left ? x[e] : -__builtin_inff();
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float p = exp2_fast(__builtin_fmaf(x[e], c, -l));
            if constexpr (kSums) {
              sum = __builtin_fmaf(p, dp[e], sum);
              if (i) whole += p;
            } else {
              ds[e] = p * (dp[e] - d[i]);
            }
          }
          if constexpr (kSums) {
            d[i] += sum;
            if (i) d[2] += whole;
          } else {
            df[i][0] = pack8<T>(ds);
            df[i][1] = pack8<T>(ds + 8);
            rest[i] = add8<T>(df[i][1], add8<T>(df[i][0], rest[i]));
          }
        }
        if constexpr (!kSums) {
#pragma unroll
          for (int t = 0; t < S; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              f32x16& q = dq[t / (S / 2)][t % (S / 2)];
              q = mma<T>(cols.read(kt, j, t, s), df[t / (S / 2)][s], q);
            }
        }
      }
    }
  };
  walk(std::integral_constant<int, 0>{});
#pragma unroll
  for (int i = 0; i < 3; ++i) d[i] = sum_halves(d[i]);
  const auto add_up = [&]<int N>(float (&v)[N]) {  // over the waves of a row, in order; each gets the sum
    if constexpr (SHARE > 1) {
#pragma unroll
      for (int i = 0; i < N; ++i) sums[share][group][i][lane] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] = sums[0][group][i][lane];
#pragma unroll
        for (int o = 1; o < SHARE; ++o) v[i] += sums[o][group][i][lane];
      }
    }
  };
  if constexpr (kScaled<T>) {
    top = max_halves(top);
    if constexpr (SHARE > 1) sums[share][group][3][lane] = top;
  }
  add_up(d);
  // del2 by what the weights sum to: the float32 log sum moves all of a row's weights by up to 2^-24 of its size, and dlambda
  // is a sum in which most of del2 may cancel (60 training cases: its error was 2.3 times that of float32 softmax maps, and
  // is 0.8 times; 0.6% of the backward pass, at d = 64 and thousands of keys up to 3.5%).
  if (d[2] > 0.0f) d[1] /= d[2];
  if constexpr (kScaled<T>) {
    if constexpr (SHARE > 1)
#pragma unroll
      for (int o = 0; o < SHARE; ++o) top = fmaxf(top, sums[o][group][3][lane]);
    ks = 14 - exponent_above(top);
    const float2 most = make_float2(wave_max_f32(top), wave_max_f32(fabsf(a.lam[h])));
    if (!share && lane == 0) tops[(static_cast<int64_t>(bh) * tiles + tile) * GROUPS + group] = most;
  }
  if (!share && live && lane < 32) put_stat(stat_at(stat, bhn, n, a.N), lse[0] / c, lse[1] / c, d[0], d[1], a.lam[h], c);
  if (tile == tiles - 1)  // rows behind the last token
    for (int x = threadIdx.x; x < G * static_cast<int>(padded(a.N) - a.N); x += 64 * WAVES)
      put_stat(stat_at(stat, static_cast<int64_t>(b) * a.Hq + hk * G + x % G, a.N + x / G, a.N), kNever, kNever, 0.0f, 0.0f, 1.0f, 1.0f);
  wait_copies();
  barrier();  // the tiles have been read
  walk(std::integral_constant<int, 1>{});
  // A row's dS sum to zero, its rounded dS do not quite: what they sum to, times a middle of the keys, is taken out of dQ, so
  // that the rounding meets what the keys differ by and not what they share (keys whose mean is half their spread: dQ's error
  // is 1.45 times that of rounding dQ alone, and 1.52 times without this; keys whose mean is 8 times their spread: 1.4 and 8
  // times. It costs 2% of the backward pass). The middle is, channel by channel, the median of eight means of every eighth
  // sampled key: as long as most of the eight hold ordinary keys it lies among those, so that no single key moves it far,
  // however large (2,048 keys, the first 20 or 100 times as large as the others and not attended to: 1.50 times; with the
  // mean of as many keys 1.7 and 3.7).
#pragma unroll
  for (int i = 0; i < 2; ++i) rest[i] = sum_halves(rest[i]);
  __syncthreads();
  if (threadIdx.x < D) {
    float v[8] = {};
    if (end > 0)
#pragma unroll
      for (int i = 0; i < SAMPLE; ++i) v[i % 8] += static_cast<float>(sample[i][threadIdx.x]);
    // the three largest go to the end and the three smallest to the front
    const auto order = [&](int i) {
      const float lo = fminf(v[i], v[i + 1]);
      v[i + 1] = fmaxf(v[i], v[i + 1]);
      v[i] = lo;
    };
#pragma unroll
    for (int k = 0; k < 3; ++k) {
#pragma unroll
      for (int i = k; i < 7 - k; ++i) order(i);
#pragma unroll
      for (int i = 5 - k; i >= k; --i) order(i);
    }
    middle[threadIdx.x] = (v[3] + v[4]) * (4.0f / SAMPLE);
  }
  add_up(rest);
  if constexpr (SHARE > 1) {
    f32x4* swap = reinterpret_cast<f32x4*>(lds) + lane;
    constexpr int PER = 4 * S * 64;
    if (share) {
      f32x4* to = swap + ((share - 1) * GROUPS + group) * PER;
#pragma unroll
      for (int t = 0; t < S; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x16& q = dq[t / (S / 2)][t % (S / 2)];
          to[(4 * t + e) * 64] = f32x4{q[4 * e], q[4 * e + 1], q[4 * e + 2], q[4 * e + 3]};
        }
    }
  }
  __syncthreads();
  if (share) return;
  if constexpr (SHARE > 1) {
    const f32x4* swap = reinterpret_cast<const f32x4*>(lds) + lane;
    constexpr int PER = 4 * S * 64;
#pragma unroll
    for (int o = 0; o < SHARE - 1; ++o)
#pragma unroll
      for (int t = 0; t < S; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x4 y = swap[(o * GROUPS + group) * PER + (4 * t + e) * 64];
#pragma unroll
          for (int x = 0; x < 4; ++x) dq[t / (S / 2)][t % (S / 2)][4 * e + x] += y[x];
        }
  }
  const float back = kScaled<T> ? __builtin_ldexpf(a.scale, -ks) : a.scale, f[2] = {back, -a.lam[h] * back};
  T* out = static_cast<T*>(a.dq.p) + b * a.dq.sb + h * a.dq.sh + n * a.dq.sn;
#pragma unroll
  for (int t = 0; t < S; ++t) {
    float x[16];
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const f32x4 m = *reinterpret_cast<const f32x4*>(&middle[32 * t + 2 * e + 4 * g]);
#pragma unroll
      for (int y = 0; y < 4; ++y)
        x[e + y] = __builtin_fmaf(-rest[t / (S / 2)], m[y], dq[t / (S / 2)][t % (S / 2)][e + y]) * f[t / (S / 2)];
    }
    store_columns(out + 32 * t, x, live);
  }
}

int64_t stat_floats(int B, int Hq, int N) { return 4ll * B * Hq * padded(N); }
// Two for every 32 rows of the tiles of 128 (or 64), two for a key head, and the next section on a multiple of 64.
int64_t top_floats(int B, int Hk, int64_t rows) {
  const int64_t heads = static_cast<int64_t>(B) * Hk;
  return padded(2 * heads * ((rows + 127) / 128 * 4 + 1));
}

// How a key tile's queries are shared out where the tiles alone leave CUs idle: without a causal mask over two sets of
// waves of a workgroup, then over as many workgroups as bring the card one a CU; with one, over 4-wave workgroups until
// the card has 768, so that tiles that few queries see even out; of 8 query tiles at least. (Backward pass: 192 tiles of
// 1,024 queries 111 us in two parts and 106 with two sets of waves; 384 without a mask 638 and 672; 128 tiles of a causal
// step 288 us in 2 parts, 212 in 4, 191 in 6, 218 in 12, and with two sets of waves 199 at best.)
struct Share {
  int halves, parts;
};
Share dkv_share(int B, int Hq, int Hk, int N, int M, bool causal) {
  const int64_t units = static_cast<int64_t>(B) * Hk * ((M + 127ll) / 128);
  const int64_t want = (causal ? 768 : 256) / units, most = static_cast<int64_t>(Hq / Hk) * ((N + 31) / 32) / 8;
  const int64_t parts = want < most ? want : most;
  return {!causal && units <= 256 ? 2 : 1, static_cast<int>(parts < 1 ? 1 : parts)};
}

template <typename T, int D>
hipError_t launch(const DiffArgs& a, hipStream_t stream) {
  float* stat = a.ws;
  float2* tops = reinterpret_cast<float2*>(stat + stat_floats(a.B, a.Hq, a.N));
  int n_tops;  // of a key head
  const int64_t rows = static_cast<int64_t>(a.N) * (a.Hq / a.Hk);
  const int row_tiles = static_cast<int>((rows + 127) / 128), row_units = a.B * a.Hk * row_tiles;
  // as in the forward pass: 192 tiles of 2,048 keys 237 -> 207 us for the backward pass, 384 causal ones of up to 4,096
  // 518 -> 415, 384 without a mask 655 -> 699; half the rows: 64 tiles of 1,024 keys 88 -> 71, 126 of 777 keys of 64
  // channels 60 -> 51, 192 of 1,024 keys 104 -> 119
  if (row_units > (a.causal ? 512 : 256)) {
    diff_dq_kernel<T, D, 1><<<grid_of(row_units), kThreads, 0, stream>>>(a, stat, tops, row_tiles, row_units);
    n_tops = row_tiles * Many<1>::kGroups;
  } else if (row_units > 128) {
    diff_dq_kernel<T, D, 2><<<grid_of(row_units), 2 * kThreads, 0, stream>>>(a, stat, tops, row_tiles, row_units);
    n_tops = row_tiles * Many<2>::kGroups;
  } else {
    const int tiles = static_cast<int>((rows + 63) / 64), n = a.B * a.Hk * tiles;
    diff_dq_kernel<T, D, 4><<<grid_of(n), 2 * kThreads, 0, stream>>>(a, stat, tops, tiles, n);
    n_tops = tiles * Many<4>::kGroups;
  }
  const int key_tiles = static_cast<int>((a.M + 127ll) / 128);
  const Share share = dkv_share(a.B, a.Hq, a.Hk, a.N, a.M, a.causal);
  const int parts = share.parts;
  const int64_t keys = static_cast<int64_t>(a.B) * a.Hk * a.M;  // at most 768 tiles of 128 where they are joined
  const int key_units = a.B * a.Hk * key_tiles * parts;
  float* sums = stat + stat_floats(a.B, a.Hq, a.N) + top_floats(a.B, a.Hk, rows);
  if (kScaled<T> && n_tops > kMostTops) {
    float2* out = tops + static_cast<int64_t>(a.B) * a.Hk * n_tops;
    diff_tops_kernel<<<a.B * a.Hk, kThreads, 0, stream>>>(tops, n_tops, out);
    tops = out;
    n_tops = 1;
  }
  const int lambdas = static_cast<int>(grid_of(a.Hq));
  if (share.halves == 1) {
    diff_dkv_kernel<T, D, 1><<<lambdas + grid_of(key_units), kThreads, 0, stream>>>(a, stat, tops, n_tops, sums, key_tiles, parts, key_units, lambdas);
  } else {
    diff_dkv_kernel<T, D, 2><<<lambdas + grid_of(key_units), 2 * kThreads, 0, stream>>>(a, stat, tops, n_tops, sums, key_tiles, parts, key_units, lambdas);
  }
  if (parts > 1)
    diff_dkv_join_kernel<T, D><<<static_cast<unsigned>((keys + 1024 / D - 1) / (1024 / D)), kThreads, 0, stream>>>(a, sums, parts, keys);
  return hipGetLastError();
}

}  // namespace

int64_t diff_bwd_ws_bytes(int B, int Hq, int Hk, int N, int M, int d) {
  const int64_t parts = std::max(dkv_share(B, Hq, Hk, N, M, false).parts, dkv_share(B, Hq, Hk, N, M, true).parts);
  return 4 * (stat_floats(B, Hq, N) + top_floats(B, Hk, static_cast<int64_t>(N) * (Hq / Hk)) + (parts > 1 ? parts * B * Hk * M * 2 * d : 0));
}

hipError_t launch_diff_bwd(const DiffArgs& a, hipStream_t stream) {
  if (a.dtype == DA2_BF16) return a.d == 128 ? launch<bf16_t, 128>(a, stream) : launch<bf16_t, 64>(a, stream);
  return a.d == 128 ? launch<fp16_t, 128>(a, stream) : launch<fp16_t, 64>(a, stream);
}

}  // namespace da2
