// Norm of the heads of Q and K and rotary positions in one pass, forward and backward.
//
// Forward: y = R(pos) (f xh), xh = (x - mean) rstd over a head's d channels, f = w or 1 + w; one
// rounding. Backward, with g = R(pos)' dy: dw = sum g xh, and for h = g f
//   dx = rstd (h - xh mean(h xh) - mean(h))   (RMS: without mean(h) and mean).
// mean and rstd are computed again from x, which the backward pass reads anyway: no
// statistics are stored.
//
// Bound by memory: Q and K (and their gradients) in and out once, where a norm and a
// rotation by themselves take two passes. The threads that share a row (part of a wave)
// hold it in registers, one or two chunks of 16 bytes each; they keep their token's
// cosines and sines and both weights over all the heads that they walk, and fetch the
// next head's row before they work on this one. Rows whose width or halves are not
// whole chunks take the same kernel with single elements.
// The weights' gradients are summed in registers over a workgroup's rows, written as
// one partial row a workgroup and added up in a fixed order by a second kernel.
//
// Measured: 24 heads of 32,760 tokens, d = 128, bf16: 84 us for 402 MB, 4.8 TB/s (two norms and a rotation by themselves 127).
// 24 heads of 6,333 tokens, fp16: forward 21 us, 3.7 TB/s; backward 40 and 5.5 for the weights' sums, 2.9 TB/s (its 1,188 workgroups of
// 150 registers a thread fit the card one and a half times). fp32, 24 heads of 32,760: 158 us for 805 MB, 5.1 TB/s; both passes 391.
#include "common.hpp"
#include "layer.hpp"
#include "rope.hpp"

namespace da2 {

namespace {

constexpr int kThreads = 256;

// V weights of any type from element at on.
template <typename U, int V>
__device__ inline void weights_of(const void* w, int at, float* x) {
  struct Some {
    U v[V];
  } c;
  __builtin_memcpy(&c, static_cast<const U*>(w) + at, sizeof c);
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = static_cast<float>(c.v[i]);
}
template <int V>
__device__ inline void load_weights(const void* w, int dtype, int at, float plus, float* x) {
  if (!w) {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = 1.0f;
    return;
  }
  if (dtype == DA2_FP32) weights_of<float, V>(w, at, x);
  else if (dtype == DA2_BF16) weights_of<bf16_t, V>(w, at, x);
  else weights_of<fp16_t, V>(w, at, x);
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] += plus;
}

// Where a unit of a row lies: its chunk, the chunk of the pairs' second halves, and its first pair.
template <int V, bool HALF>
struct Unit {
  static constexpr int P = HALF ? V : (V > 1 ? V / 2 : 1);  // pairs
  static constexpr bool kTwo = HALF || V == 1;              // second halves are a chunk of their own
  int i, j, pair;
  bool live, moves;
  Unit() = default;
  __device__ Unit(const RopeArgs& a, int units, int u) {
    live = u < units * (a.d / a.block);
    const int k = live ? u / units : 0, r = live ? u - k * units : 0;
    const int turning = HALF ? a.rot / 2 / V : (V > 1 ? (a.rot + V - 1) / V : a.rot / 2);
    moves = r >= turning;
    pair = 0;
    if (moves) {
      i = (HALF || V == 1 ? a.rot : turning * V) + (r - turning) * V;
    } else if (HALF) {
      i = pair = r * V;
    } else {
      pair = r * P;
      i = 2 * pair;
    }
    i += k * a.block;
    j = HALF ? i + a.rot / 2 : i + 1;
  }
  __device__ bool two() const { return kTwo && live && !moves; }
};

// Sums over the TPR threads of a row.
template <int TPR, int N>
__device__ inline void row_sum(float (&v)[N]) {
#pragma unroll
  for (int o = TPR / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], o, 64);
}

// A thread's share of a row as it lies in memory: it stays so while it is on its way.
template <typename T, int V, bool HALF, int K>
struct Fetched {
  struct Some {
    T v[V];
  };
  static constexpr int C = Unit<V, HALF>::kTwo ? 2 : 1;
  Some c[K][C];
  __device__ void load(const T* row, const Unit<V, HALF>* u) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      c[k][0] = Some{};
      if constexpr (C > 1) c[k][1] = Some{};
      if (u[k].live) __builtin_memcpy(&c[k][0], row + u[k].i, sizeof(Some));
      if constexpr (C > 1)
        if (u[k].two()) __builtin_memcpy(&c[k][1], row + u[k].j, sizeof(Some));
    }
  }
};

// A thread's share of a row: W values of each of K units, the first V of chunk i and the others of chunk j.
template <typename T, int V, bool HALF, int K>
struct Share {
  static constexpr int W = Unit<V, HALF>::kTwo ? 2 * V : V;
  float v[K][W];
  __device__ explicit Share(const Fetched<T, V, HALF, K>& f) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < W; ++e) v[k][e] = static_cast<float>(f.c[k][e / V].v[e % V]);
  }
  __device__ void store(T* row, const Unit<V, HALF>* u) const {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (u[k].live) put<T, V>(row + u[k].i, v[k]);
      if constexpr (W > V)
        if (u[k].two()) put<T, V>(row + u[k].j, v[k] + V);
    }
  }
  // Whether value e of unit k is one of the row's.
  __device__ static bool holds(const Unit<V, HALF>& u, int e) { return e < V ? u.live : u.two(); }
  __device__ void rotate(const RopeArgs& a, const Unit<V, HALF>* u, const float (*c)[Unit<V, HALF>::P], const float (*s)[Unit<V, HALF>::P]) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (u[k].moves || !u[k].live) continue;
      if constexpr (W > V) {
#pragma unroll
        for (int e = 0; e < V; ++e) turn(v[k][e], v[k][V + e], c[k][e], s[k][e]);
      } else {
#pragma unroll
        for (int e = 0; e < Unit<V, HALF>::P; ++e)
          if (2 * (u[k].pair + e) < a.rot) turn(v[k][2 * e], v[k][2 * e + 1], c[k][e], s[k][e]);
      }
    }
  }
  // The row's mean taken out (layer norm), and 1 / sqrt(variance + eps).
  template <int TPR>
  __device__ float normalize(const QkArgs& a, const Unit<V, HALF>* u) {
    const float inv = 1.0f / static_cast<float>(a.r.d);
    if (a.kind == DA2_NORM_LAYER) {
      float m[1] = {0.0f};
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < W; ++e) m[0] += v[k][e];
      row_sum<TPR>(m);
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < W; ++e) v[k][e] = holds(u[k], e) ? v[k][e] - m[0] * inv : 0.0f;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < W; ++e) q[0] = __builtin_fmaf(v[k][e], v[k][e], q[0]);
    row_sum<TPR>(q);
    return 1.0f / __builtin_sqrtf(q[0] * inv + static_cast<float>(a.eps));
  }
};

template <int V, bool HALF, int K>
__device__ inline void load_factors(const QkArgs& a, const void* w, const Unit<V, HALF>* u, float (*f)[Unit<V, HALF>::kTwo ? 2 * V : V]) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (u[k].live) load_weights<V>(w, a.wdtype, u[k].i, a.plus, f[k]);
    if constexpr (Unit<V, HALF>::kTwo)
      if (u[k].two()) load_weights<V>(w, a.wdtype, u[k].j, a.plus, f[k] + V);
  }
}

// What a thread keeps of its token: where its units lie, and their cosines and sines.
template <typename T, int V, bool HALF, int TPR, int K>
struct Token {
  using U = Unit<V, HALF>;
  U u[K];
  float c[K][U::P], s[K][U::P];
  int b, n;
  __device__ Token(const RopeArgs& a, int units) {
#pragma unroll
    for (int k = 0; k < K; ++k) u[k] = U(a, units, threadIdx.x % TPR + k * TPR);
  }
  __device__ void move_to(const RopeArgs& a, uint32_t token) {
    b = token / static_cast<uint32_t>(a.N);
    n = token - static_cast<uint32_t>(b) * a.N;
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (u[k].live && !u[k].moves) angles<U::P>(a, b, n, u[k].pair, c[k], s[k]);
  }
  __device__ const T* row(const View& v, int h) const { return static_cast<const T*>(v.p) + b * v.sb + h * v.sh + n * v.sn; }
  __device__ T* row(const OutView& v, int h) const { return static_cast<T*>(v.p) + b * v.sb + h * v.sh + n * v.sn; }
};

// units: of a block; heads: that a thread walks.
template <typename T, int V, bool HALF, int TPR, int K>
__global__ __launch_bounds__(kThreads) void qk_kernel(QkArgs a, int units, int heads) {
  using S = Share<T, V, HALF, K>;
  const uint32_t token = blockIdx.x * (kThreads / TPR) + threadIdx.x / TPR;
  if (token >= static_cast<uint64_t>(a.r.B) * a.r.N) return;  // all the threads of a row
  Token<T, V, HALF, TPR, K> at(a.r, units);
  const int h0 = blockIdx.y * heads, h1 = min(h0 + heads, a.r.Hq + a.r.Hk);
  const auto walk = [&](const View& in, const OutView& out, const void* w, int from, int to) {
    if (from >= to) return;
    Fetched<T, V, HALF, K> next;
    next.load(at.row(in, from), at.u);
    float f[K][S::W];
    load_factors<V, HALF, K>(a, w, at.u, f);
    for (int h = from; h < to; ++h) {
      S x(next);
      if (h + 1 < to) next.load(at.row(in, h + 1), at.u);
      const float r = x.template normalize<TPR>(a, at.u);
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < S::W; ++e) x.v[k][e] *= r * f[k][e];
      x.rotate(a.r, at.u, at.c, at.s);
      x.store(at.row(out, h), at.u);
    }
  };
  at.move_to(a.r, token);
  walk(a.r.q, a.r.qo, a.wq, h0, min(h1, a.r.Hq));
  walk(a.r.k, a.r.ko, a.wk, max(h0 - a.r.Hq, 0), h1 - a.r.Hq);
}

// A workgroup has heads of Q alone (blockIdx.y below q_parts) or of K, and so one set of weights and sums.
template <typename T, int V, bool HALF, int TPR, int K>
__global__ __launch_bounds__(kThreads) void qk_bwd_kernel(QkArgs a, int units, int heads, int q_parts) {
  using S = Share<T, V, HALF, K>;
  Token<T, V, HALF, TPR, K> at(a.r, units);
  const bool is_q = static_cast<int>(blockIdx.y) < q_parts;
  const int h0 = (static_cast<int>(blockIdx.y) - (is_q ? 0 : q_parts)) * heads, h1 = min(h0 + heads, is_q ? a.r.Hq : a.r.Hk);
  const View in = is_q ? a.xq : a.xk, grad = is_q ? a.r.q : a.r.k;
  const OutView out = is_q ? a.r.qo : a.r.ko;
  const float inv = 1.0f / static_cast<float>(a.r.d);
  float f[K][S::W], sum[K][S::W];
  load_factors<V, HALF, K>(a, is_q ? a.wq : a.wk, at.u, f);
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int e = 0; e < S::W; ++e) sum[k][e] = 0.0f;
  const auto walk = [&] {
    Fetched<T, V, HALF, K> nx, ng;
    nx.load(at.row(in, h0), at.u);
    ng.load(at.row(grad, h0), at.u);
    for (int h = h0; h < h1; ++h) {
      S x(nx), g(ng);
      if (h + 1 < h1) {
        nx.load(at.row(in, h + 1), at.u);
        ng.load(at.row(grad, h + 1), at.u);
      }
      const float r = x.template normalize<TPR>(a, at.u);
      g.rotate(a.r, at.u, at.c, at.s);
      float m[2] = {0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < S::W; ++e) {
          x.v[k][e] *= r;
          // a value that is none of the row's is zero, but a row of infinite rstd would make it a NaN
          if (S::holds(at.u[k], e)) {
            sum[k][e] = __builtin_fmaf(g.v[k][e], x.v[k][e], sum[k][e]);
            g.v[k][e] *= f[k][e];
            m[0] += g.v[k][e];
            m[1] = __builtin_fmaf(g.v[k][e], x.v[k][e], m[1]);
          }
        }
      row_sum<TPR>(m);
      const float m0 = a.kind == DA2_NORM_LAYER ? m[0] * inv : 0.0f, m1 = m[1] * inv;
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < S::W; ++e) x.v[k][e] = r * (g.v[k][e] - __builtin_fmaf(x.v[k][e], m1, m0));
      x.store(at.row(out, h), at.u);
    }
  };
  const uint64_t tokens = static_cast<uint64_t>(a.r.B) * a.r.N;
  for (uint64_t token = blockIdx.x * (kThreads / TPR) + threadIdx.x / TPR; token < tokens; token += gridDim.x * (kThreads / TPR)) {
    at.move_to(a.r, static_cast<uint32_t>(token));
    walk();
  }
  if (!a.dwq && !a.dwk) return;
  // the rows that a wave holds, then the waves
  __shared__ float cols[kThreads / 64][kQkMaxD];
  const int wave = threadIdx.x / 64;
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int e = 0; e < S::W; ++e) {
#pragma unroll
      for (int o = TPR; o < 64; o <<= 1) sum[k][e] += __shfl_xor(sum[k][e], o, 64);
      if (threadIdx.x % 64 < TPR && S::holds(at.u[k], e)) cols[wave][e < V ? at.u[k].i + e : at.u[k].j + (e - V)] = sum[k][e];
    }
  __syncthreads();
  float* part = a.ws + (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * 2 * a.r.d;
  for (int i = threadIdx.x; i < a.r.d; i += kThreads) {
    float t = cols[0][i];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) t += cols[w][i];
    part[i] = is_q ? t : 0.0f;
    part[a.r.d + i] = is_q ? 0.0f : t;
  }
}

constexpr int kWide = 512, kMaxParts = 3 * kWide;  // workgroups of the backward pass: along the tokens, and in all at most

// Units of a block for chunks of V.
int units_of(const RopeArgs& r, int V) {
  if (V == 1) return r.rot / 2 + (r.block - r.rot);
  return r.layout == DA2_ROPE_HALF ? r.rot / 2 / V + (r.block - r.rot) / V : r.block / V;
}
bool whole(const RopeArgs& r, int V) {
  return r.layout == DA2_ROPE_HALF ? (r.rot / 2) % V == 0 && (r.block - r.rot) % V == 0 : r.block % V == 0;
}

// Calls f<T, V, HALF, TPR, K>(units): threads a row and units a thread.
template <typename F>
hipError_t with_shape(const RopeArgs& r, F&& f) {
  return by_dtype(r.dtype, [&](auto t) {
    using T = decltype(t);
    constexpr int V = kVec<T>;
    const auto layout = [&]<bool HALF>() {
      if (whole(r, V)) {
        const int units = units_of(r, V), all = units * (r.d / r.block);
        if (all <= 8) return f.template operator()<T, V, HALF, 8, 1>(units);
        if (all <= 16) return f.template operator()<T, V, HALF, 16, 1>(units);
        if (all <= 32) return f.template operator()<T, V, HALF, 32, 1>(units);
        if (all <= 64) return f.template operator()<T, V, HALF, 64, 1>(units);
        return f.template operator()<T, V, HALF, 64, 2>(units);
      }
      const int units = units_of(r, 1), all = units * (r.d / r.block);
      if (all <= 64) return f.template operator()<T, 1, HALF, 64, 1>(units);
      if (all <= 128) return f.template operator()<T, 1, HALF, 64, 2>(units);
      return f.template operator()<T, 1, HALF, 64, 8>(units);
    };
    return r.layout == DA2_ROPE_HALF ? layout.template operator()<true>() : layout.template operator()<false>();
  });
}

}  // namespace

int64_t qk_ws_bytes(int B, int Hq, int Hk, int N, int d) {
  const int64_t rows = static_cast<int64_t>(B) * N * (static_cast<int64_t>(Hq) + Hk);
  return 8 * (rows < kMaxParts ? rows : kMaxParts) * d;
}

hipError_t launch_qk(const QkArgs& a, hipStream_t stream) {
  return with_shape(a.r, [&]<typename T, int V, bool HALF, int TPR, int K>(int units) {
    const int all = a.r.Hq + a.r.Hk;
    const int64_t tokens = static_cast<int64_t>(a.r.B) * a.r.N, blocks = (tokens + kThreads / TPR - 1) / (kThreads / TPR);
    // A thread keeps its cosines and sines for as many heads as leave the card 2^18 threads, 16 waves a CU (24 heads of 6,333
    // tokens: 22 us, with 2^19 and 2^20 25 and 34).
    int64_t heads = tokens * TPR * all >> 18;
    heads = heads < 1 ? 1 : heads > all ? all : heads;
    qk_kernel<T, V, HALF, TPR, K><<<dim3(static_cast<unsigned>(blocks), static_cast<unsigned>((all + heads - 1) / heads)), kThreads, 0, stream>>>(
        a, units, static_cast<int>(heads));
    return hipGetLastError();
  });
}

hipError_t launch_qk_bwd(const QkArgs& a, hipStream_t stream) {
  int64_t parts = 0;
  const hipError_t e = with_shape(a.r, [&]<typename T, int V, bool HALF, int TPR, int K>(int units) {
    const int64_t all = a.r.Hq + a.r.Hk, tokens = static_cast<int64_t>(a.r.B) * a.r.N;
    int64_t x = (tokens + kThreads / TPR - 1) / (kThreads / TPR);
    x = x < kWide ? x : kWide;
    const int64_t most = kWide / x > 2 ? kWide / x : 2, heads = (all + most - 1) / most;
    const int64_t q_parts = (a.r.Hq + heads - 1) / heads, y = q_parts + (a.r.Hk + heads - 1) / heads;
    parts = x * y;  // at most 3 kWide
    qk_bwd_kernel<T, V, HALF, TPR, K><<<dim3(static_cast<unsigned>(x), static_cast<unsigned>(y)), kThreads, 0, stream>>>(
        a, units, static_cast<int>(heads), static_cast<int>(q_parts));
    return hipGetLastError();
  });
  if (e != hipSuccess || (!a.dwq && !a.dwk)) return e;
  return launch_column_sum(a.ws, parts, 2 * a.r.d, 1, a.wdtype, a.dwq, a.dwk, a.r.d, 0, stream);
}

}  // namespace da2
