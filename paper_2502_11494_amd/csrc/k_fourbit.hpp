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
// each; W waves share a token.  Memory-bound: every row is read once and written once (23 040 tokens of 32 + 32 heads of 128,
// bf16: append 94 us, 5.1 TB/s, read 70 us, 6.8 TB/s of which most is written; 32 000 of 12 + 12 heads of 80 in 32 bits 68 and 51 us, 4.2 and
// 5.6 TB/s; a few tokens 3.5 us, four dependent loads).  Rows pass the caches by (append 121 -> 94, read 92 -> 70; with 32-bit rows, whose
// lanes write every second 16 bytes at a time, the other way round: 53 -> 103); tokens in a row go to one die, whose cache joins the pieces of
// lines that they write (the append 130 -> 121).
template <int DT, int W, bool READ>
__global__ __launch_bounds__(256) void k_hold(Hold a, Cache c) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = wave % W;
  const long t = (READ && DT == kF32 ? (long)blockIdx.x : xcd_contiguous(blockIdx.x, gridDim.x)) * (4 / W) + wave / W;
  if (t >= a.T) return;
  const int sub = lane & 3;
  constexpr int kAtOnce = 4;  // rounds of 16 blocks whose loads are on their way together
  struct Round {
    int at;           // of the pages, beside the token's place and the head's
    int head;
    long row;
    bool value, on, in;  // on: a block there is; in: it has values here (else filled up with zeros)
  };
  auto round_of = [&](int x0, int n) {
    const int x = x0 + n * W * 16 + (lane >> 2);
    Round r;
    r.value = x >= a.heads_blocks;
    const int y = r.value ? x - a.heads_blocks : x;
    r.head = a.per_block == 0 ? y : (int)(((uint64_t)(uint32_t)y * a.per_block) >> 32);
    r.at = (y - r.head * a.blocks) * kBlock + sub * 8;
    r.on = x < 2 * a.heads_blocks && (!READ || (r.value ? a.v_out : a.k_out) != nullptr);
    r.in = r.on && r.at < a.d;
    r.row = t * (r.value ? a.v_ld : a.k_ld) + (long)r.head * a.d + r.at;
    return r;
  };
  Piece<DT, 8> p[kAtOnce];
  auto load_rows = [&](int x0) {
#pragma unroll
    for (int n = 0; n < kAtOnce; ++n) {
      const Round r = round_of(x0, n);
      p[n] = Piece<DT, 8>{};
      if (!r.in) continue;
      const u32x4* from = reinterpret_cast<const u32x4*>(static_cast<const unsigned char*>(r.value ? a.v : a.k) + r.row * (DT == kBF16 ? 2 : 4));
#pragma unroll
      for (int j = 0; j < (DT == kBF16 ? 1 : 2); ++j) {
        const u32x4 x = __builtin_nontemporal_load(from + j);
#pragma unroll
        for (int i = 0; i < 4; ++i) p[n].w[4 * j + i] = x[i];
      }
    }
  };
  if (!READ) load_rows(part * 16);  // (they do not wait for the token's place)

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
  for (int x0 = part * 16; x0 < 2 * a.heads_blocks; x0 += kAtOnce * W * 16) {
    if (READ) {
      uint32_t w[kAtOnce], e[kAtOnce];
#pragma unroll
      for (int n = 0; n < kAtOnce; ++n) {
        const Round r = round_of(x0, n);
        const long at = slot + (long)r.head * c.head_ld + r.at;
        w[n] = e[n] = 0;
        if (!r.in) continue;
        __builtin_memcpy(&w[n], __builtin_assume_aligned(static_cast<const unsigned char*>(r.value ? a.v_codes : a.k_codes) + at / 2, 4), 4);
        e[n] = (r.value ? a.v_scales : a.k_scales)[at / kBlock];
      }
#pragma unroll
      for (int n = 0; n < kAtOnce; ++n) {
        const Round r = round_of(x0, n);
        if (!r.in) continue;
        unsigned char* to = static_cast<unsigned char*>(r.value ? a.v_out : a.k_out) + r.row * (DT == kBF16 ? 2 : 4);
        if (DT == kBF16) {
          __builtin_nontemporal_store(In4Bits::piece<DT>(w[n], e[n], 0), reinterpret_cast<u32x4*>(to));
        } else {
          *reinterpret_cast<u32x4*>(to) = In4Bits::piece<DT>(w[n], e[n], 0);
          *reinterpret_cast<u32x4*>(to + 16) = In4Bits::piece<DT>(w[n], e[n], 1);
        }
      }
      continue;
    }
    uint32_t codes[kAtOnce], scale[kAtOnce];
#pragma unroll
    for (int n = 0; n < kAtOnce; ++n) {
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t u = __float_as_uint(p[n].get(j)) & 0x7fffffffu;
        top = top > u ? top : u;
      }
      scale[n] = scale_byte(quad_max(top));
      codes[n] = scale[n] == kNoNumber ? 0u : codes_of<DT>(p[n], scale_of(scale[n]));
    }
    const int next = x0 + kAtOnce * W * 16;
    if (next < 2 * a.heads_blocks) load_rows(next);
#pragma unroll
    for (int n = 0; n < kAtOnce; ++n) {
      const Round r = round_of(x0, n);
      const long at = slot + (long)r.head * c.head_ld + r.at;
      if (!r.on) continue;
      __builtin_memcpy(__builtin_assume_aligned(static_cast<unsigned char*>(r.value ? a.v_codes : a.k_codes) + at / 2, 4), &codes[n], 4);
      if (sub == 0) (r.value ? a.v_scales : a.k_scales)[at / kBlock] = (uint8_t)scale[n];
    }
  }
}

}  // namespace dart
