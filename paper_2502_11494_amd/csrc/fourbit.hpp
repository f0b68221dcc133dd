// Rows held in 4 bits: blocks of 32 values of a head, each a code of a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (two bits of
// exponent, one of fraction) times the block's power of two, which is the block's scale byte e: 2^(e - 127).  This is the format of
// the matrix cores' 4-bit operands, for which the chip has conversions; a value has two significant bits, so bfloat16 and 32 bits
// hold it exactly, whatever the scale.  e is the smallest that leaves the largest value under 7, which rounds to 6 with no
// more error than one unit, the most that 4 to 6 make; a block with an infinity or NaN has e = 255 and is NaN.
#pragma once

#include "cache.hpp"
#include "k_rotate.hpp"

namespace dart {

constexpr int kBlock = 32;  // values of a scale byte; 16 bytes of codes
constexpr int kNoNumber = 255, kTopScale = 252;  // (252: 6 * 2^125, the largest that 32 bits hold)

// Values 2 * BYTE and 2 * BYTE + 1 of a word of codes.
template <int DT, int BYTE>
__device__ __forceinline__ void two_values(uint32_t codes, float scale, uint32_t* to) {
  if constexpr (DT == kBF16) {
    to[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE));
  } else {
    const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, BYTE);
    to[0] = __float_as_uint(v[0]);
    to[1] = __float_as_uint(v[1]);
  }
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }  // (the conversions take its exponent)

// A value that the compiler takes as new, so that what is made of it is made here and not kept over a loop.
__device__ __forceinline__ void made_here(uint32_t& x) { asm volatile("" : "+v"(x)); }

struct In4Bits {
  static constexpr bool kCodes = true, kPages = false;
  // Values of a load, where a thread has a share of them: 32 (a block), 16 or 8.
  static constexpr int unit(int, int share) { return share < kBlock ? share : kBlock; }
  // Whether a block may hold infinities or NaN: 253 and 254, which no append writes, take the largest codes beyond 32 bits.
  __device__ static __forceinline__ bool odd(uint32_t scale) { return scale > kTopScale; }
  __device__ static __forceinline__ bool odd(const uint8_t* scales, long at) { return odd(scales[at / kBlock]); }

  // A 16-byte piece of a row: the eight bf16 values of a word of codes, or the half-th four of them in 32 bits.
  template <int DT>
  __device__ static __forceinline__ u32x4 piece(uint32_t codes, uint32_t scale, int half) {
    const float s = scale_of(scale);
    uint32_t w[4];
    if constexpr (DT == kBF16) {
      two_values<DT, 0>(codes, s, w);
      two_values<DT, 1>(codes, s, w + 1);
      two_values<DT, 2>(codes, s, w + 2);
      two_values<DT, 3>(codes, s, w + 3);
    } else if (half == 0) {
      two_values<DT, 0>(codes, s, w);
      two_values<DT, 1>(codes, s, w + 2);
    } else {
      two_values<DT, 2>(codes, s, w);
      two_values<DT, 3>(codes, s, w + 2);
    }
    return u32x4{w[0], w[1], w[2], w[3]};
  }

  // VE (four or eight) values from element `at` of a pool on, a multiple of VE.
  template <int DT, int VE>
  __device__ static __forceinline__ Piece<DT, VE> values(const void* codes, const uint8_t* scales, long at) {
    uint32_t w = 0;
    __builtin_memcpy(&w, __builtin_assume_aligned(static_cast<const unsigned char*>(codes) + at / 2, VE / 2), VE / 2);
    const uint32_t scale = scales[at / kBlock];
    Piece<DT, VE> p;
    constexpr int kBytes = sizeof p < 16 ? sizeof p : 16;
    u32x4 x = piece<DT>(w, scale, 0);
    __builtin_memcpy(p.w, &x, kBytes);
    if constexpr (sizeof(p) > 16) {
      x = piece<DT>(w, scale, 1);
      __builtin_memcpy(p.w + 4, &x, 16);
    }
    return p;
  }
};

// Pages of 16 rows and more, a row's stride small enough for 32 bits to hold 16 of them: tiles of 16 keys that lie in one page.
struct In4BitsPages : In4Bits {
  static constexpr bool kPages = true;
};

}  // namespace dart
