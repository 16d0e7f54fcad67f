// Rotary positions of Q and K.
//
// Pair (a, b) of a token at position pos becomes scale (a cos t - b sin t,
// a sin t + b cos t) with t = 2 pi turns[p] pos. turns pos is a float64 product
// and what its rounding left out; whole turns are taken out of both before their
// sum is rounded to float32, so the angle is off by at most pi 2^-25 (and 2^-50)
// wherever the token is and however fast the pair turns.
//
// Bound by memory: Q and K in and out. The angles do not depend on the head, so
// a thread computes the cosines and sines of its pairs of one token once and
// walks over heads (of Q, then of K) with them; nothing is read but Q, K, the
// position and a few turns. A unit is 16 bytes of one half of the pairs: 16
// bytes of channels (interleaved), two times 16 bytes (halves), or 16 bytes of
// channels that only move. Rows whose width or halves are not whole chunks take
// the same kernel with single elements. (bf16, 24 heads of 32,760 tokens: 83 us,
// 4.9 TB/s.)
#include "rope.hpp"

namespace da2 {

namespace {

constexpr int kThreads = 256;

// units: threads per token; V: elements of a unit's chunk (16 bytes, or 1); HALF: the layout.
template <typename T, int V, bool HALF>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a, int units, int heads) {
  constexpr int P = HALF ? V : (V > 1 ? V / 2 : 1);  // pairs of a unit
  const uint32_t id = blockIdx.x * kThreads + threadIdx.x;  // below 2^32, as the host checks
  const uint32_t token = id / static_cast<uint32_t>(units);
  if (token >= static_cast<uint64_t>(a.B) * a.N) return;
  const int u = static_cast<int>(id - token * units);
  const int b = token / static_cast<uint32_t>(a.N), n = token - static_cast<uint32_t>(b) * a.N;
  // channels of the unit inside a block: i (and j, the pairs' second halves)
  const int turning = HALF ? a.rot / 2 / V : (V > 1 ? (a.rot + V - 1) / V : a.rot / 2);
  const bool moves = u >= turning;  // channels beyond rot
  int i, j = 0, pair = 0;
  if (moves) {
    i = (HALF || V == 1 ? a.rot : turning * V) + (u - turning) * V;
  } else if (HALF) {
    i = u * V;
    j = i + a.rot / 2;
    pair = i;
  } else {
    pair = u * P;
    i = 2 * pair;
    j = i + 1;  // single pairs
  }
  float c[P], s[P];
  if (!moves) angles<P>(a, b, n, pair, c, s);
  const int blocks = a.d / a.block, h1 = min(static_cast<int>(blockIdx.y + 1) * heads, a.Hq + a.Hk);
  constexpr bool PAIR = HALF || V == 1;  // the pairs' second halves are a chunk of their own
  for (int k = 0; k < blocks; ++k) {
    for (int h = blockIdx.y * heads; h < h1; ++h) {
      const bool is_q = h < a.Hq;
      if (moves && (is_q ? a.q_in_place : a.k_in_place)) continue;
      const View& in = is_q ? a.q : a.k;
      const OutView& out = is_q ? a.qo : a.ko;
      const int hh = is_q ? h : h - a.Hq;
      const T* x = static_cast<const T*>(in.p) + b * in.sb + hh * in.sh + n * in.sn + k * a.block;
      T* y = static_cast<T*>(out.p) + b * out.sb + hh * out.sh + n * out.sn + k * a.block;
      float v[V], w[V];
      get<T, V>(x + i, v);
      if (!moves) {
        if constexpr (PAIR) {
          get<T, V>(x + j, w);
#pragma unroll
          for (int e = 0; e < V; ++e) turn(v[e], w[e], c[e], s[e]);
          put<T, V>(y + j, w);
        } else {
#pragma unroll
          for (int e = 0; e < P; ++e)
            if (2 * (pair + e) < a.rot) turn(v[2 * e], v[2 * e + 1], c[e], s[e]);
        }
      }
      put<T, V>(y + i, v);
    }
  }
}

template <typename T, int V, bool HALF>
hipError_t launch(const RopeArgs& a, hipStream_t stream) {
  // threads of a token: the turning units of a block and the ones that move
  int units;
  if (V == 1) {
    units = a.rot / 2 + (a.block - a.rot);
  } else if (HALF) {
    units = a.rot / 2 / V + (a.block - a.rot) / V;
  } else {
    units = a.block / V;
  }
  const int all = a.Hq + a.Hk;
  const int64_t threads = static_cast<int64_t>(a.B) * a.N * units;
  // A thread keeps its angles for as many heads as leave the card 2^20 threads, four rounds of its 256 CUs x 16 waves (24
  // heads of 32,760 tokens: 83 us with a quarter of that, 82 with 2^20 or twice that; 40 heads of 8,000 tokens: 31, 29
  // and 38).
  int64_t heads = threads * all >> 20;
  heads = heads < 1 ? 1 : heads > all ? all : heads;
  const int64_t chunks = (all + heads - 1) / heads;
  const int64_t blocks = (threads + kThreads - 1) / kThreads;
  rope_kernel<T, V, HALF><<<dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(chunks)), kThreads, 0, stream>>>(
      a, units, static_cast<int>(heads));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, hipStream_t stream) {
  return by_dtype(a.dtype, [&](auto t) {
    using T = decltype(t);
    constexpr int V = kVec<T>;
    if (a.layout == DA2_ROPE_HALF) {
      const bool whole = (a.rot / 2) % V == 0 && (a.block - a.rot) % V == 0;
      return whole ? launch<T, V, true>(a, stream) : launch<T, 1, true>(a, stream);
    }
    return a.block % V == 0 ? launch<T, V, false>(a, stream) : launch<T, 1, false>(a, stream);
  });
}

}  // namespace da2
