// Rows to pages held in 4 bits, and back.
#pragma once

#include "fourbit.hpp"

namespace dart {

struct Hold {
  int Hkv, d, T;
  int blocks;           // of a head
  int heads_blocks;     // of all heads of a row
  uint32_t per_block;   // ceil(2^32 / blocks), 0 for one block
  const void *k, *v;    // rows (append)
  void *k_out, *v_out;  // rows (read), or nullptr
  long k_ld, v_ld;
  void *k_codes, *v_codes;
  uint8_t *k_scales, *v_scales;
};

// The largest of four lanes that hold a block.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, true);
  x = x > y ? x : y;
  y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, true);
  return x > y ? x : y;
}

// The scale byte of a block whose largest magnitude has these bits: two powers under it, one more from 1.75 on.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  const int e = (int)((top + 0x00200000u) >> 23) - 2;
  return top >= 0x7f800000u ? kNoNumber : e < 0 ? 0 : e < kTopScale ? e : kTopScale;
}

// Eight values to a word of codes: rounded to nearest, ties to the even code, to the largest where beyond it.
template <int DT>
__device__ __forceinline__ uint32_t codes_of(const Piece<DT, 8>& p, float scale) {
  uint32_t w = 0;
  if constexpr (DT == kBF16) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, p.w[0]), scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, p.w[1]), scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, p.w[2]), scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, p.w[3]), scale, 3);
  } else {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, p.get(0), p.get(1), scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, p.get(2), p.get(3), scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, p.get(4), p.get(5), scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, p.get(6), p.get(7), scale, 3);
  }
  return w;
}

// The tokens' key and value rows to their places in the pages (READ: from them).  Four lanes hold a block of 32 values, eight
// each; W waves share a token.  Memory-bound: every row is read once and written once.
template <int DT, int W, bool READ>
__global__ __launch_bounds__(256) void k_hold(Hold a, Cache c) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = wave % W;
  const long t = (long)blockIdx.x * (4 / W) + wave / W;
  if (t >= a.T) return;
  const int b = c.cu == nullptr ? (int)t : owner_of(c.cu, c.B, (int)t);
  const Seq s = sequence_of(c, b);
  const int i = (int)t - s.tok0;
  bool bad = false, put = false;
  long slot = 0;
  if (s.valid && i >= 0 && i < s.n && s.kv >= s.n) {
    slot = key_offset(c, c.pages + (long)b * c.pages_ld, s.kv - s.n + i, bad);
    put = !bad;
  }
  if (!put) {
    if (lane == 0 && part == 0) flag(c, bad ? kBadPage : kBadSequence);
    return;
  }
  const int sub = lane & 3;
  constexpr int kAtOnce = 4;  // rounds of 16 blocks whose loads are on their way together
  for (int x0 = part * 16; x0 < 2 * a.heads_blocks; x0 += kAtOnce * W * 16) {
    Piece<DT, 8> p[kAtOnce] = {};
    uint32_t w[kAtOnce], e[kAtOnce];
    long at[kAtOnce], row[kAtOnce];
    bool value[kAtOnce], on[kAtOnce], in[kAtOnce];
#pragma unroll
    for (int n = 0; n < kAtOnce; ++n) {
      const int x = x0 + n * W * 16 + (lane >> 2);
      value[n] = x >= a.heads_blocks;
      const int y = value[n] ? x - a.heads_blocks : x;
      const int h = a.per_block == 0 ? y : (int)(((uint64_t)(uint32_t)y * a.per_block) >> 32);
      const int j = y - h * a.blocks;
      on[n] = x < 2 * a.heads_blocks && (!READ || (value[n] ? a.v_out : a.k_out) != nullptr);
      in[n] = on[n] && j * kBlock + sub * 8 < a.d;  // (else filled up with zeros)
      at[n] = slot + (long)h * c.head_ld + j * kBlock + sub * 8;
      row[n] = t * (value[n] ? a.v_ld : a.k_ld) + (long)h * a.d + j * kBlock + sub * 8;
      if (READ && in[n]) {
        __builtin_memcpy(&w[n], __builtin_assume_aligned(static_cast<const unsigned char*>(value[n] ? a.v_codes : a.k_codes) + at[n] / 2, 4), 4);
        e[n] = (value[n] ? a.v_scales : a.k_scales)[at[n] / kBlock];
      }
      if (!READ && in[n]) p[n] = load_piece<DT, 8>(value[n] ? a.v : a.k, row[n]);
    }
#pragma unroll
    for (int n = 0; n < kAtOnce; ++n) {
      if (READ) {
        if (!in[n]) continue;
        void* out = value[n] ? a.v_out : a.k_out;
        const u32x4 x = In4Bits::piece<DT>(w[n], e[n], 0);
        unsigned char* to = static_cast<unsigned char*>(out) + row[n] * (DT == kBF16 ? 2 : 4);
        *reinterpret_cast<u32x4*>(to) = x;
        if (DT == kF32) *reinterpret_cast<u32x4*>(to + 16) = In4Bits::piece<DT>(w[n], e[n], 1);
        continue;
      }
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t u = __float_as_uint(p[n].get(j)) & 0x7fffffffu;
        top = top > u ? top : u;
      }
      const uint32_t scale = scale_byte(quad_max(top));
      const uint32_t codes = scale == kNoNumber ? 0u : codes_of<DT>(p[n], scale_of(scale));
      if (!on[n]) continue;
      __builtin_memcpy(__builtin_assume_aligned(static_cast<unsigned char*>(value[n] ? a.v_codes : a.k_codes) + at[n] / 2, 4), &codes, 4);
      if (sub == 0) (value[n] ? a.v_scales : a.k_scales)[at[n] / kBlock] = (uint8_t)scale;
    }
  }
}

}  // namespace dart
