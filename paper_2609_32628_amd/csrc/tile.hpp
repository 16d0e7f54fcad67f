// Shared by the kernels that work on tiles in LDS: operand fragments, 32x32x16 MFMAs,
// LDS reads and asynchronous copies, and the order of work over the XCDs.
#pragma once

#include "common.hpp"
#include "token.hpp"

namespace da2 {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));

// ---- MFMA on fragments of 8 16-bit values --------------------------------------------
template <typename T>
__device__ inline f32x16 mma(const s16x8& a, const s16x8& b, const f32x16& c) {
  if constexpr (__is_same(T, bf16_t)) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
}
// Eight floats rounded to T (nearest even).
template <typename T>
__device__ inline s16x8 pack8(const float* x) {
  typedef T Tx8 __attribute__((ext_vector_type(8)));
  Tx8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = static_cast<T>(x[i]);
  return __builtin_bit_cast(s16x8, v);
}

typedef __attribute__((address_space(3))) const s16x8* lds_s16x8;
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

__device__ inline uint32_t lds_offset(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)p));
}
__device__ inline s16x8 read_b128(uint32_t at) { return *reinterpret_cast<lds_s16x8>(at); }
__device__ inline s16x4 read_tr(uint32_t at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4>(at));
}

// Asynchronous copy of 1 KB into LDS from byte `lds` on: lane l brings the 16 bytes at base + voff to lds + 16 l.
// Issued as assembly, since the compiler would wait for it before every LDS read
// that follows; the kernels wait for their copies themselves.
__device__ inline void copy_1k(const void* base, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(base), "s"(lds)
               : "memory", "m0");
}
// The wave's copies have arrived, and its reads of LDS have been answered (so that
// after a barrier no read is left that the next copy could overtake).
__device__ inline void wait_copies() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
__device__ inline void barrier() { asm volatile("s_barrier" ::: "memory"); }

// Workgroup id -> unit of work, such that each XCD (ids go around the eight of
// them) has consecutive units, which share a head's keys in its L2; -1: none.
// Units, rows of a key head and workgroups are 32-bit numbers (the host checks):
// a 64-bit division costs a short call as much as a key tile.
__device__ inline int unit_of(uint32_t id, int total) {
  const int per = (total + 7) / 8, u = static_cast<int>(id % 8) * per + static_cast<int>(id / 8);
  return u < total ? u : -1;
}
inline unsigned grid_of(int total) { return static_cast<unsigned>((total + 7) / 8 * 8); }

}  // namespace da2
