// bf16 tiles of tokens in LDS and the fragments that the matrix instruction v_mfma_f32_32x32x16_bf16 takes from them.
#pragma once
#include "common.h"

#define AB_KT 64   // tokens per LDS tile
#define LOG2E 1.4426950408889634f
#define MFMA(a, b, c) __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0)
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;

template <int D>
struct ATile {
  static constexpr int LD = D;
  static constexpr int ELEMS = AB_KT * D;
  static constexpr int BYTES = ELEMS * 2;
  static constexpr int CPR = D / 8;   // 16-byte chunks per row
  static constexpr int IPW = D / 32;  // transfers per wave per tile (4 waves)
  __device__ static __forceinline__ int swz(int r) { return (((r & 3) << 2) | ((r >> 2) & 3)) & (CPR - 1); }
  // element offset of (row r, column c), c a multiple of 4
  __device__ static __forceinline__ int off(int r, int c) { return r * LD + ((((c >> 3) ^ swz(r)) << 3) | (c & 7)); }
};

// Byte offsets inside a tile of the two kinds of fragment reads, precomputed per lane.
//   direct: row l32 (+32*mt), columns ks*16 + kg*8 .. +7              -> kdir[ks] (+ mt*32*LD*2)
//   transposed: rows 4*kg + s/4 (+8 for the second read) (+ mt*32 + 16*c), column dt*32 + h16*16 + (s%4)*4
//                                                                      -> tr0[dt], tr1[dt] (+ (mt*32+16c)*LD*2)
// The swizzle of a row only depends on row%16 through bits that the added multiples of 16 (and, for
// the direct reads, 32) leave untouched, so the additions are plain constants.
template <int D>
struct FragAddr {
  int kdir[D / 16], tr0[D / 32], tr1[D / 32];
  __device__ __forceinline__ void init(int lane) {
    using TL = ATile<D>;
    const int l32 = lane & 31, kg = lane >> 5, s16 = lane & 15, h16 = (lane >> 4) & 1;
#pragma unroll
    for (int ks = 0; ks < D / 16; ks++) kdir[ks] = TL::off(l32, ks * 16 + kg * 8) * 2;
#pragma unroll
    for (int dt = 0; dt < D / 32; dt++) {
      tr0[dt] = TL::off(4 * kg + (s16 >> 2), dt * 32 + h16 * 16 + ((s16 & 3) << 2)) * 2;
      tr1[dt] = TL::off(8 + 4 * kg + (s16 >> 2), dt * 32 + h16 * 16 + ((s16 & 3) << 2)) * 2;
    }
  }
};
// Fragment reads take a per-lane pointer (tile base + precomputed lane offset) and a compile-time
// constant byte offset, which the compiler folds into the offset field of the LDS instruction.
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
__device__ __forceinline__ bf16x8 lds_frag(const lds_char* lane_ptr, int const_off) {
  return *reinterpret_cast<const lds_bf16x8*>(lane_ptr + const_off);
}
__device__ __forceinline__ bf16x8 lds_frag_tr(const lds_char* lane_ptr0, const lds_char* lane_ptr1, int const_off) {
  s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lane_ptr0 + const_off));
  s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lane_ptr1 + const_off));
  return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
// Registers 8c..8c+7 of a 32x32 result tile as a bf16 B fragment (k-slots = rows 16c+4g+{0..3}, 16c+8+4g+{0..3}).
__device__ __forceinline__ bf16x8 pack_rows(const f32x16& t, int c) {
  bf16x8 f;
#pragma unroll
  for (int i = 0; i < 8; i++) f[i] = (bf16_t)t[8 * c + i];
  return f;
}
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
