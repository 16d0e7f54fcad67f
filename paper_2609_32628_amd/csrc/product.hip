// Products of token rows with weight rows, with bias, activation, gate and residual in the epilogue, or both halves of a
// gated block at once: Z = X W', Y = R + gate act(Z + bias), or act(G) U; sums in float32, one rounding.
//
// The product is transposed, features times tokens: an accumulator's four registers are then features of one token, and
// the epilogue works on eight features in a row of one token with 16-byte accesses. In a gated block a wave's feature
// rows are half gate, half up, of the same features, so that both sums meet in one lane.
//
// Tiles are 256x256 by eight waves, one workgroup a CU, or 128x128 by four, two a CU: a tile of 256 reads half of what
// one of 128 does, and leaves CUs idle where tiles are few. K goes in steps of 64, 128 bytes of each row, brought into LDS by
// asynchronous copies while the step before is multiplied: 16x16x32 products, whose operands are read from LDS a few products
// ahead of their use, and one barrier a step. Workgroups stay for as many tiles as there are, and copy the next tile's first
// step before a tile's epilogue.
//
// Measured (bf16, calls in a row, over several cards): 8,192^3 804 to 820 us, 1,341 to 1,368 TFLOP/s (a plain library product 689 to
// 702 us); 8,190 x 5,120 x 2 x 13,824 gated 1,740 to 1,854 us, 1,251 to 1,333 (the library's product without the block 1,785 to 1,814);
// 32,760 x 1,536 x 4,608 with bias 431 to 475 us, 976 to 1,076 (335 to 373). The gated large tile keeps 15 to 17 vector registers in
// scratch memory, around the loop over K, not in it.
// Bound by the copies into LDS, which share its ports with the operands' reads: without them the same loop runs at 1,534, and
// the matrix units are busy 66% of the time; and by the epilogue, during which a CU multiplies nothing: 9 us of a tile of 256,
// 1.4 a step. Tried and no faster:
// 128x128 a wave (1.05 to 1.14 PFLOP/s), tiles of 256x128 with three steps of 32 in LDS (0.96), steps of 32 with three or
// four in LDS (5% slower), workgroups that begin at different steps of K (2 to 8% slower), wave priorities, copies in one go.
#include <algorithm>
#include <utility>

#include "act.hpp"

namespace da2 {

namespace {

enum Mode { kLinear, kGated, kPartial };

constexpr int kRowBytes = 2 * kStep;  // of a tile's row
constexpr int kStage = 2048;          // LDS bytes of a wave's epilogue

// A step's rows lie in LDS in blocks of eight, as one copy of 1 KB brings them: 128 bytes of a row after the other, in the order
// of the lanes. Row
// 64 q + 16 j + 2 b + p is line 2 j + p of block 8 q + b, and a block begins 16 bytes behind the one before, so that the 16 rows of
// a read meet all banks.
constexpr int kBlock = 1024 + 16;
__device__ inline int row_of(int block, int line) { return block / 8 * 64 + line / 2 * 16 + block % 8 * 2 + line % 2; }
// LDS byte of row r's first chunk, for r below 64.
__device__ inline int line_at(int r) { return r % 16 / 2 * kBlock + (r / 16 * 2 + r % 2) * kRowBytes; }

// Element offset of row r.
__device__ inline int64_t row_at(const Side& s, int64_t r) {
  if (s.B == 1) return r * s.sn;
  const uint32_t b = static_cast<uint32_t>(r) / static_cast<uint32_t>(s.N);
  return b * s.sb + (static_cast<uint32_t>(r) - b * static_cast<uint32_t>(s.N)) * s.sn;
}
// The least element offset of rows [r, last].
__device__ inline int64_t first_at(const Side& s, int64_t r, int64_t last) {
  if (s.B == 1) return r * s.sn;
  const uint32_t b = static_cast<uint32_t>(r) / static_cast<uint32_t>(s.N);
  const int64_t here = row_at(s, r);
  return static_cast<uint32_t>(last) / static_cast<uint32_t>(s.N) > b ? min(here, (b + 1) * s.sb) : here;
}

// Walks K in steps along rows whose elements lie in blocks of C.
struct Walk {
  const char* at;
  int64_t jump;  // bytes from a block's last step to the next block's first
  int in, C;
  __device__ void start(const Side& s, int64_t row, int k) {
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

// Four copies of 1 KB to the LDS blocks from byte `to` on, by the lanes of a mask that is all or none of them (a branch would
// cut the products' schedule). The immediate offset counts for both addresses: offsets v are a block less from one to the next.
__device__ inline i32x4 buffer_at(const char* base) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  // raw buffer: 48 bits of address, no stride, 2^32 - 1 bytes, 32-bit data format
  return i32x4{__builtin_amdgcn_readfirstlane(static_cast<int>(p)), __builtin_amdgcn_readfirstlane(static_cast<int>(p >> 32 & 0xFFFF)), -1, 0x00020000};
}
__device__ inline void copy_4k(const i32x4& base, const uint32_t* v, uint32_t to) {
  asm volatile(
      "s_mov_b32 m0, %5\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %4, 0 offen lds\n\tbuffer_load_dwordx4 %1, %4, 0 offen offset:1040 lds\n\t"
      "buffer_load_dwordx4 %2, %4, 0 offen offset:2080 lds\n\tbuffer_load_dwordx4 %3, %4, 0 offen offset:3120 lds" ::"v"(v[0]),
      "v"(v[1]), "v"(v[2]), "v"(v[3]), "s"(base), "s"(__builtin_amdgcn_readfirstlane(to))
      : "memory", "m0");
}
__device__ inline void copy_4k_if(const i32x4& base, const uint32_t* v, uint32_t to, int lanes) {
  asm volatile(
      "s_mov_b32 m0, %5\n\ts_mov_b32 exec_lo, %6\n\ts_mov_b32 exec_hi, %6\n\tbuffer_load_dwordx4 %0, %4, 0 offen lds\n\t"
      "buffer_load_dwordx4 %1, %4, 0 offen offset:1040 lds\n\tbuffer_load_dwordx4 %2, %4, 0 offen offset:2080 lds\n\t"
      "buffer_load_dwordx4 %3, %4, 0 offen offset:3120 lds\n\ts_mov_b64 exec, -1" ::"v"(v[0]),
      "v"(v[1]), "v"(v[2]), "v"(v[3]), "s"(base), "s"(__builtin_amdgcn_readfirstlane(to)), "s"(__builtin_amdgcn_readfirstlane(lanes))
      : "memory", "m0");
}

template <typename T>
__device__ inline f32x4 mma16(const s16x8& a, const s16x8& b, const f32x4& c) {
  if constexpr (__is_same(T, bf16_t)) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
}

// The compiler leaves memory accesses on their side of it.
__device__ inline void in_order() { asm volatile("" ::: "memory"); }

// A workgroup's tile of TW feature rows and TT tokens, and its WW x WT waves. END: K is no whole number of steps.
template <int MODE_, bool END, int TW_, int TT_, int WW_, int WT_>
struct Shape {
  static constexpr int MODE = MODE_, TW = TW_, TT = TT_, WW = WW_, WT = WT_;
  static constexpr bool kEnd = END;
  static constexpr int kWaves = WW * WT, kW = TW / WW / 16, kT = TT / WT / 16;   // 16x16 blocks of a wave
  static constexpr int kBlocks = kW / (MODE == kGated ? 4 : 2);                  // 32s of features
  static constexpr int kCopyW = TW / 8 / kWaves, kCopyT = TT / 8 / kWaves;       // 1 KB copies a wave makes of a step
  static constexpr int kSideW = TW / 8 * kBlock;                                  // LDS bytes of a step's feature rows
  static constexpr int kTile = kSideW + TT / 8 * kBlock;                         // of a step
  static constexpr int kLds = 2 * kTile + kStage * kWaves;
  static constexpr int kPerCu = 160 * 1024 / kLds;                               // workgroups of a CU
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

// A workgroup's units of work: tiles, or parts of K of a tile. Ids go around the eight XCDs; each XCD has consecutive
// units, which its workgroups take in turn, and tiles come in groups of 8 token tiles, token tiles first: those that run
// at once share rows in their XCD's L2.
struct Units {
  int unit, end, stride;
  __device__ Units(int total) {
    const int per = (total + 7) / 8, xcd = blockIdx.x % 8;
    unit = xcd * per + blockIdx.x / 8;
    end = min((xcd + 1) * per, total);
    stride = gridDim.x / 8;
  }
};
struct Unit {
  int split, tile_w, tile_t, step0, steps;
  __device__ Unit(int unit, int tiles_w, int tiles_t, int splits, int K) {
    const int tiles = tiles_w * tiles_t;
    split = unit / tiles;
    const int tile = unit - split * tiles, group = tile / (8 * tiles_w), in_group = tile - group * 8 * tiles_w;
    const int wide = min(8, tiles_t - group * 8);
    tile_w = in_group / wide;
    tile_t = group * 8 + in_group - tile_w * wide;
    const int all = (K + kStep - 1) / kStep, per = (all + splits - 1) / splits;
    step0 = split * per;
    steps = min(per, all - step0);
  }
};

// The copies of a workgroup's steps into LDS, in order: step i goes to buffer i % 2.
template <typename S>
struct Copies {
  static constexpr int TW = S::TW, TT = S::TT;
  const ProductArgs& a;
  const int tiles_w, tiles_t, splits;
  Units units;
  int k, left, lane, wave;  // element of the next step, steps left of the unit
  uint32_t lds0, to;
  Walk walk_w, walk_t;
  uint32_t off_w[S::kCopyW], off_t[S::kCopyT];  // of the chunks that this lane copies, from the tile's lowest row

  __device__ Copies(const ProductArgs& a_, int tiles_w_, int tiles_t_, int splits_, uint32_t lds, int lane_, int wave_)
      : a(a_), tiles_w(tiles_w_), tiles_t(tiles_t_), splits(splits_), units(tiles_w_ * tiles_t_ * splits_), lane(lane_), wave(wave_), lds0(lds), to(lds) {
    left = 0;
    if (more()) start();
  }
  __device__ bool more() const { return units.unit < units.end; }
  template <bool W>
  __device__ int row(int i) const { return row_of(wave * (W ? S::kCopyW : S::kCopyT) + i, lane / 8); }  // of copy i
  __device__ void start() {
    const Unit u(units.unit, tiles_w, tiles_t, splits, a.K);
    const int64_t R = static_cast<int64_t>(a.parts) * a.f.F, m0 = static_cast<int64_t>(u.tile_t) * TT;
    const auto weight = [&](int q) { return weight_row<S::MODE, TW, S::WW>(u.tile_w, q, R, a.f.F); };
    const int64_t w_first = S::MODE == kGated ? row_at(a.w, weight(0)) : first_at(a.w, weight(0), weight(TW - 1));
    const int64_t t_first = first_at(a.t, m0, min(m0 + TT, a.M) - 1);
    // rows behind the last repeat it
#pragma unroll
    for (int i = 0; i < S::kCopyW; ++i)
      off_w[i] = static_cast<uint32_t>(2 * (row_at(a.w, weight(row<true>(i))) - w_first)) + lane % 8 * 16 + kBlock * (3 - i);
#pragma unroll
    for (int i = 0; i < S::kCopyT; ++i)
      off_t[i] = static_cast<uint32_t>(2 * (row_at(a.t, min(m0 + row<false>(i), a.M - 1)) - t_first)) + lane % 8 * 16 + kBlock * (3 - i);
    walk_w.start(a.w, w_first, u.step0 * kStep);
    walk_t.start(a.t, t_first, u.step0 * kStep);
    k = u.step0 * kStep;
    left = u.steps;
  }
  // Whether there is a next step and it is whole.
  __device__ bool whole() const { return more() && (!S::kEnd || k + kStep <= a.K); }
  // The copies of one side of the step.
  template <bool W>
  __device__ void side(int lanes) {
    const uint32_t at = to + (W ? wave * (S::kCopyW * kBlock) : S::kSideW + wave * (S::kCopyT * kBlock));
    if constexpr (S::kEnd) copy_4k_if(buffer_at((W ? walk_w.at : walk_t.at) - 3 * kBlock), W ? off_w : off_t, at, lanes);
    else copy_4k(buffer_at((W ? walk_w.at : walk_t.at) - 3 * kBlock), W ? off_w : off_t, at);
  }
  // The end of K inside a step: through registers, zeros behind it. A row's last chunk lies in its stride, and is whole in memory.
  __device__ void copy_end(char* lds) {
    constexpr int n = S::kCopyW + S::kCopyT;
    const int rest = a.K - k - lane % 8 * 8;
    uint4 v[n];
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const bool w = i < S::kCopyW;
      const int c = w ? i : i - S::kCopyW;
      const char* p = (w ? walk_w.at + off_w[w ? c : 0] : walk_t.at + off_t[w ? 0 : c]) - kBlock * (3 - c);
      v[i] = make_uint4(0, 0, 0, 0);
      if (rest > 0) v[i] = *reinterpret_cast<const uint4*>(p);
    }
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const bool w = i < S::kCopyW;
      const int c = w ? i : i - S::kCopyW;
      *reinterpret_cast<uint4*>(lds + (to - lds0) + ((w ? wave * S::kCopyW : TW / 8 + wave * S::kCopyT) + c) * kBlock + lane * 16) = first8(v[i], rest);
    }
  }
  __device__ void next() {
    to = lds0 + (to == lds0 ? S::kTile : 0);
    if (!more()) return;
    if (--left == 0) {
      units.unit += units.stride;
      if (more()) start();  // else the last step is copied again, to where it is not read
      return;
    }
    walk_w.next();
    walk_t.next();
    k += kStep;
  }
  __device__ void step(char* lds) {
    if (whole()) {
      side<true>(-1);
      side<false>(-1);
    } else if (more()) {
      copy_end(lds);
    }
    next();
  }
};

template <typename T, typename S>
__global__ __launch_bounds__(64 * S::kWaves, 2) void product_kernel(ProductArgs a, int tiles_w, int tiles_t, int splits) {
  constexpr int MODE = S::MODE, TW = S::TW, TT = S::TT, WW = S::WW;
  __shared__ __attribute__((aligned(1024))) char lds[S::kLds];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int wave_w = wave % WW, wave_t = wave / WW;
  char* const stage = lds + 2 * S::kTile + wave * kStage;
  const uint32_t lds0 = lds_offset(lds);
  const int64_t R = static_cast<int64_t>(a.parts) * a.f.F;
  Units mine(tiles_w * tiles_t * splits);
  if (mine.unit >= mine.end) return;
  Copies<S> copies(a, tiles_w, tiles_t, splits, lds0, lane, wave);
  copies.step(lds);
  const float back = back_of<T, MODE == kGated>(a.f);

  f32x4 acc[S::kW][S::kT];
  const auto clear = [&] {
#pragma unroll
    for (int i = 0; i < S::kW; ++i)
#pragma unroll
      for (int j = 0; j < S::kT; ++j) acc[i][j] = f32x4{};
  };
  clear();
  // Operand n of half h of a step: chunk 4 h + lane / 16 of 16 rows.
  const uint32_t read = line_at(lane % 16) + lane / 16 * 16;
  const uint32_t read_w = wave_w * (S::kW * 2 * kBlock) + read, read_t = S::kSideW + wave_t * (S::kT * 2 * kBlock) + read;
  const auto fetch = [&](uint32_t at, int n, int h) { return read_b128(at + n / 4 * 8 * kBlock + n % 4 * 2 * kRowBytes + h * 64); };
  static_assert(S::kCopyW == 4 && S::kCopyT == 4 && S::kT == 4);
  // A step is 2 kW operands of weights, kW of each half, one after the other with the four token operands of the half. The weights'
  // are read kLead ahead, the tokens' while the half before is multiplied.
  constexpr int kLead = 3, kAll = 2 * S::kW;
  s16x8 fw[kLead + 1], ft[2][S::kT];
  const auto mask = [&](bool whole) { return __builtin_amdgcn_readfirstlane(whole ? -1 : 0); };
  bool whole = copies.whole();
  if (whole) copies.template side<true>(-1);
  uint32_t at = lds0;
  wait_copies();
  barrier();
#pragma unroll
  for (int j = 0; j < S::kT; ++j) ft[0][j] = fetch(at + read_t, j, 0);
#pragma unroll
  for (int n = 0; n < kLead; ++n) fw[n] = fetch(at + read_w, n, 0);
  // Operand N of the step at `at`; from N = kAll - kLead on reads are of the next step, at `other`.
  const auto operand = [&]<int N>(uint32_t from) {
    constexpr int h = N / S::kW, next = (N + kLead) % kAll, tokens = N - (h + 1) * S::kW + kLead;
    fw[(N + kLead) % (kLead + 1)] = fetch(from + read_w, next % S::kW, next / S::kW);
    // the next half's token operands: two, one and one
    if constexpr (tokens == 0) {
      ft[1 - h][0] = fetch(from + read_t, 0, 1 - h);
      ft[1 - h][1] = fetch(from + read_t, 1, 1 - h);
    } else if constexpr (tokens > 0) {
      ft[1 - h][tokens + 1] = fetch(from + read_t, tokens + 1, 1 - h);
    }
    if constexpr (N == kAll - kLead + 1) copies.template side<true>(mask(whole));
    if constexpr (N == 2) copies.template side<false>(mask(whole));
#pragma unroll
    for (int j = 0; j < S::kT; ++j) acc[N % S::kW][j] = mma16<T>(fw[N % (kLead + 1)], ft[h][j], acc[N % S::kW][j]);
    __builtin_amdgcn_sched_barrier(0);
  };

  for (; mine.unit < mine.end; mine.unit += mine.stride) {
    const Unit u(mine.unit, tiles_w, tiles_t, splits, a.K);
    for (int s = 0; s < u.steps; ++s) {
      [&]<int... N>(std::integer_sequence<int, N...>) { (operand.template operator()<N>(at), ...); }(std::make_integer_sequence<int, S::kW>{});
      if (S::kEnd && copies.more() && !whole) copies.copy_end(lds);
      copies.next();
      whole = copies.whole();
      [&]<int... N>(std::integer_sequence<int, N...>) { (operand.template operator()<S::kW + N>(at), ...); }(std::make_integer_sequence<int, S::kW - kLead>{});
      // the next step has arrived, and every wave's reads of this one have been answered: its buffer takes the one after
      wait_copies();
      barrier();
      at = lds0 + (at == lds0 ? S::kTile : 0);
      [&]<int... N>(std::integer_sequence<int, N...>) { (operand.template operator()<kAll - kLead + N>(at), ...); }(std::make_integer_sequence<int, kLead>{});
    }

    // The epilogue, 16 tokens and 32 features at a time: the sums go through the wave's 2 KB of LDS, so that one piece of
    // code with 8 features of a token a lane serves all blocks (unrolled over the blocks' registers it was 170 KB of
    // instructions, whose fetches took 18 us a tile).
    const int64_t m0 = static_cast<int64_t>(u.tile_t) * TT + wave_t * S::kT * 16;
    const int f0 = (u.tile_w * WW + wave_w) * (32 * S::kBlocks), chunk = lane % 4;
    const auto put = [&](const f32x4& x, int half) {  // 16 features
      *reinterpret_cast<f32x4*>(stage + lane % 16 * 128 + (((4 * half + lane / 16) ^ (lane % 8)) << 4)) = x;
    };
    const auto take = [&](float* v) {
      const int row = lane / 4;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(stage + row * 128 + (((2 * chunk + h) ^ (row % 8)) << 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * h + e] = x[e];
      }
    };
    // Part p = t16 kBlocks + i: tokens t16 * 16 + {0..15}, features i * 32 + {0..31}. What the next part's epilogue reads is
    // asked for before this part is worked on.
    constexpr bool GLU = MODE == kGated;
    constexpr int kParts = S::kBlocks * S::kT;
    RowPlace<T, GLU> next_row{};
    Beside<T, GLU> next{};
    const auto ask = [&](int p) {
      if constexpr (MODE != kPartial) {
        const int t16 = p / S::kBlocks, i = p % S::kBlocks;
        if (i == 0) next_row = RowPlace<T, GLU>(a.f, min(m0 + t16 * 16 + lane / 4, a.M - 1));
        next = Beside<T, GLU>(a.f, next_row, min(f0 + i * 32 + 8 * chunk, a.f.F - 1), min(f0 + i * 32, a.f.F - 1));
      }
    };
    ask(0);
    // two at a time where registers allow it (32,760 x 1,536 x 4,608 with bias, both in turn on one card: 455 us instead of 477; with gate
    // and residual no difference; gated and small tiles 3 and 1% slower)
    constexpr int kTogether = MODE == kLinear && TW == 256 ? 2 : 1;
#pragma unroll kTogether
    for (int part = 0; part < kParts; ++part) {
      const int at16 = part / S::kBlocks, f8 = f0 + part % S::kBlocks * 32 + 8 * chunk;
      const RowPlace<T, GLU> row = next_row;
      const Beside<T, GLU> beside = next;
      if (part + 1 < kParts) ask(part + 1);
      // by halves: one after the other the comparisons take longer than the part
      const auto put_block = [&]<int SECOND>() {
        const auto among = [&]<int FROM, int TO>(auto&& self) {
          if constexpr (TO - FROM == 1) {
            constexpr int w = 2 * (FROM % S::kBlocks) + SECOND * (S::kW / 2);
            put(acc[w][FROM / S::kBlocks], 0);
            put(acc[w + 1][FROM / S::kBlocks], 1);
            asm volatile("; part %0" ::"n"(FROM));  // leaves that are alike would become one, with the sums in memory
          } else if (part < (FROM + TO) / 2) {
            self.template operator()<FROM, (FROM + TO) / 2>(self);
          } else {
            self.template operator()<(FROM + TO) / 2, TO>(self);
          }
        };
        among.template operator()<0, S::kBlocks * S::kT>(among);
      };
      // the wave's lanes read what others wrote: LDS takes its accesses in order, and the compiler has to leave them so
      float v[8], w[8];
      put_block.template operator()<0>();
      in_order();
      take(v);
      in_order();
      if constexpr (GLU) {
        put_block.template operator()<1>();
        in_order();
        take(w);
        in_order();
      }
      const int64_t m = m0 + at16 * 16 + lane / 4;
      if constexpr (MODE == kPartial) {
        if (m < a.M && f8 < R) {
          float* to = a.ws + (static_cast<int64_t>(u.split) * a.M + m) * ((R + 7) / 8 * 8) + f8;
          store_vec(to, v);
          store_vec(to + 4, v + 4);
        }
      } else if (m < a.M && f8 < a.f.F) {
        finish8<T, GLU>(a.f, row, beside, back, v, w, f8);
      }
    }
    clear();
  }
  wait_copies();  // LDS may become another workgroup's
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
#pragma unroll 4
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
  const RowPlace<T, GLU> row(a.f, m);
  finish8<T, GLU>(a.f, row, Beside<T, GLU>(a.f, row, f8, f8), back_of<T, GLU>(a.f), v, u, f8);
}

// ---- few tokens ------------------------------------------------------------------------
// Up to 16 tokens: the weights are read once, which bounds it. A workgroup has 16 features (of a gated block both halves) and
// all tokens; its eight waves take every eighth 64 elements of K each, straight from memory into the operands of the 16x16x32
// products, two of them on their way at a time, and their sums are added up in order in LDS.
// 4 x 5,120 x 5,120, bf16: 16 us with the launch, 52 MB of weights at 3.3 TB/s; 16 x 2,048 x 2 x 5,504, fp16: 15 us, 45 MB
// at 3.0. A load takes 64 bytes of 16 rows, and what a CU has on its way bounds it: 16 waves, or four products ahead, are no
// faster. The tokens' rows are read by every workgroup, 16 of them as many bytes as its weights: 5,120 x 5,120 takes 15 us
// for one token and 21 for 16. The gated kernel keeps 19 vector registers in scratch memory in its epilogue.
constexpr int kFew = kFewTokens, kFewWaves = 8, kAhead = 2;

// A chunk of a row, of which `left` elements are the row's; zeros behind them.
__device__ inline s16x8 load_row8(const uint16_t* p, int left) {
  uint4 v = make_uint4(0, 0, 0, 0);
  if (left > 0) v = *reinterpret_cast<const uint4*>(p);
  return __builtin_bit_cast(s16x8, first8(v, left));
}

template <typename T, bool GLU, bool LO>
__global__ __launch_bounds__(64 * kFewWaves, 4) void product_few_kernel(ProductArgs a) {
  constexpr int P = GLU ? 2 : 1;
  __shared__ __attribute__((aligned(16))) float sums[kFewWaves][kFew][16 * P + 4];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, g = lane / 16;
  const int f0 = blockIdx.x * 16;
  const uint16_t* w[P];
#pragma unroll
  for (int p = 0; p < P; ++p)
    w[p] = static_cast<const uint16_t*>(a.w.p) + row_at(a.w, min(f0 + r, a.f.F - 1) + static_cast<int64_t>(p) * a.f.F) + 8 * g;
  const bool live = r < a.M;
  const uint16_t* t = static_cast<const uint16_t*>(a.t.p) + row_at(a.t, live ? r : 0) + 8 * g;
  f32x4 acc[P] = {};
  const int blocks = (a.K + 63) / 64, whole = a.K / 64;
  const auto at = [&](int k) {  // of element k, the first of 64 in a row of t
    const int h = k / a.t.C;
    return h * a.t.sh + (k - h * a.t.C);
  };
  constexpr int L = LO ? 2 : 1;
  const auto add = [&](const s16x8 (&fw)[P][2], const s16x8 (&ft)[L][2]) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int l = L; l--;) acc[p] = mma16<T>(fw[p][c], ft[l][c], acc[p]);
  };
  int b = wave;
  for (; b + (kAhead - 1) * kFewWaves < whole; b += kAhead * kFewWaves) {
    s16x8 fw[kAhead][P][2], ft[kAhead][L][2] = {};
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int k = (b + u * kFewWaves) * 64;
      const int64_t x = at(k);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int p = 0; p < P; ++p) fw[u][p][c] = *reinterpret_cast<const s16x8*>(w[p] + k + 32 * c);
#pragma unroll
        for (int l = 0; l < L; ++l)
          if (live) ft[u][l][c] = *reinterpret_cast<const s16x8*>(t + l * a.t.sh + x + 32 * c);
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) add(fw[u], ft[u]);
  }
  for (; b < blocks; b += kFewWaves) {
    s16x8 fw[P][2], ft[L][2];
    const int k = b * 64, left = a.K - k - 8 * g;
    const int64_t x = at(k);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int p = 0; p < P; ++p) fw[p][c] = load_row8(w[p] + k + 32 * c, left - 32 * c);
#pragma unroll
      for (int l = 0; l < L; ++l) ft[l][c] = load_row8(t + l * a.t.sh + x + 32 * c, live ? left - 32 * c : 0);
    }
    add(fw, ft);
  }
  // lane: token r, features 4 g + {0..3}
#pragma unroll
  for (int p = 0; p < P; ++p) *reinterpret_cast<f32x4*>(&sums[wave][r][16 * p + 4 * g]) = acc[p];
  __syncthreads();
  const int m = threadIdx.x / 2, c = threadIdx.x % 2, f8 = f0 + 8 * c;
  if (m >= a.M || f8 >= a.f.F) return;
  float v[2][8] = {};
#pragma unroll
  for (int p = 0; p < P; ++p)
    for (int s = 0; s < kFewWaves; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[p][e] += sums[s][m][p * 16 + c * 8 + e];
  const RowPlace<T, GLU> row(a.f, m);
  finish8<T, GLU>(a.f, row, Beside<T, GLU>(a.f, row, f8, f8), back_of<T, GLU>(a.f), v[0], v[1], f8);
}

template <typename T, typename S>
hipError_t launch_tiles(const ProductArgs& a, int splits, hipStream_t stream) {
  // a gated tile's rows are two for each feature
  const int64_t features = static_cast<int64_t>(a.parts) * a.f.F;
  const int64_t tw = (features + S::TW - 1) / S::TW, tt = (a.M + S::TT - 1) / S::TT;
  // as many workgroups as run at once, in eights
  const int64_t units = (tw * tt * splits + 7) / 8 * 8, most = 256 * S::kPerCu;
  product_kernel<T, S><<<static_cast<unsigned>(units < most ? units : most), 64 * S::kWaves, 0, stream>>>(a, static_cast<int>(tw), static_cast<int>(tt), splits);
  return hipGetLastError();
}

template <typename T, int MODE, bool END>
hipError_t launch_plan(const ProductArgs& a, const Plan& p, hipStream_t stream) {
  return p.big ? launch_tiles<T, Shape<MODE, END, 256, 256, 2, 4>>(a, p.splits, stream)
               : launch_tiles<T, Shape<MODE, END, 128, 128, 2, 2>>(a, p.splits, stream);
}
template <typename T, int MODE>
hipError_t launch_plan(const ProductArgs& a, const Plan& p, hipStream_t stream) {
  return a.K % kStep ? launch_plan<T, MODE, true>(a, p, stream) : launch_plan<T, MODE, false>(a, p, stream);
}

}  // namespace

int64_t product_ws_bytes(int64_t M, int64_t N, int64_t F, int64_t K, int parts, bool lo) {
  return std::max(partial_bytes(M, F, K, parts, lo), M == N ? 0 : partial_bytes(N, F, K, parts, lo));
}

hipError_t launch_product(const ProductArgs& a, hipStream_t stream) {
  if (few_rows(a.M, a.f.F, a.K, a.parts, a.lo))
    return by_dtype(a.dtype, [&](auto t) {
      using T = decltype(t);
      if constexpr (sizeof(T) == 4) {
        return hipErrorInvalidValue;
      } else {
        const unsigned blocks = (a.f.F + 15) / 16;
        if (a.parts == 2) {
          product_few_kernel<T, true, false><<<blocks, 64 * kFewWaves, 0, stream>>>(a);
        } else if (a.lo) {
          product_few_kernel<T, false, true><<<blocks, 64 * kFewWaves, 0, stream>>>(a);
        } else {
          product_few_kernel<T, false, false><<<blocks, 64 * kFewWaves, 0, stream>>>(a);
        }
        return hipGetLastError();
      }
    });
  if (a.lo) {  // K twice over: the tokens' two blocks, and the weights again (which is too long for few rows, too)
    ProductArgs two = a;
    two.lo = false;
    two.w.C = a.K;
    two.w.sh = 0;
    two.K = 2 * a.K;
    return launch_product(two, stream);
  }
  // A tile addresses its token rows by 32 bits from the lowest. Samples further apart than that go one by one.
  const int64_t samples = a.t.B;
  if (samples > 1 && (std::min<int64_t>(samples, 256 / a.t.N + 2) * a.t.sb + a.t.N * a.t.sn + (1 << 16)) >> 31) {
    for (int64_t b = 0; b < samples; ++b) {
      ProductArgs one = a;
      const auto skip = [&](const void* p, int64_t n) { return p ? static_cast<const char*>(p) + 2 * b * n : nullptr; };
      one.M = a.t.N;
      one.t.B = 1;
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
