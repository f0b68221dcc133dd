// What the kernels on 4-bit pages and on eviction use of the device language beyond tests/lanes/hip/hip_runtime.h.
#pragma once

#include <hip/hip_runtime.h>

struct int2 { int x, y; };
inline int2 make_int2(int x, int y) { return {x, y}; }
inline uint2 make_uint2(unsigned x, unsigned y) { return {x, y}; }

extern dim3 lanes_grid, lanes_block;
inline void lanes_shape(dim3 grid, dim3 block, size_t, hipStream_t) { lanes_grid = grid, lanes_block = block; }
#define gridDim lanes_grid
#define blockDim lanes_block

template <class T>
T __shfl_up(T v, int by) {
  const int l = lane_now & 63;
  return from_lane(v, l >= by ? l - by : l);
}
template <class T>
T __shfl(T v, int lane) { return from_lane(v, lane & 63); }
inline int __popcll(unsigned long long x) { return __builtin_popcountll(x); }
inline int atomicAdd(int* p, int v) {
  const int old = *p;
  *p += v;
  return old;
}

// (common.hpp has it for the device's compiler only)
namespace dart {
inline long xcd_contiguous(unsigned block, unsigned blocks) { return (long)(block % 8) * (blocks / 8) + block / 8; }
}

// 4-bit values and their scales, by their definition.
typedef __bf16 lanes_bf2 __attribute__((ext_vector_type(2)));
typedef float lanes_f2 __attribute__((ext_vector_type(2)));
inline float lanes_scale(float s) {
  const uint32_t e = __float_as_uint(s) >> 23 & 255;
  return e == 255 ? NAN : ldexpf(1.f, (int)e - 127);
}
inline float lanes_value(uint32_t code, float scale) {
  static const float grid[8] = {0.f, 0.5f, 1.f, 1.5f, 2.f, 3.f, 4.f, 6.f};
  const float v = grid[code & 7] * scale;
  return code & 8 ? -v : v;
}
inline uint32_t lanes_code(float x, float scale) {
  const double y = fabs((double)x) / scale;
  const uint32_t c = (y > 0.25) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0);
  return c | (std::signbit(x) ? 8u : 0u);
}
inline lanes_f2 lanes_values(uint32_t codes, float s, int byte) {
  const float scale = lanes_scale(s);
  return lanes_f2{lanes_value(codes >> (8 * byte) & 15, scale), lanes_value(codes >> (8 * byte + 4) & 15, scale)};
}
inline lanes_bf2 lanes_values_bf16(uint32_t codes, float s, int byte) {
  const lanes_f2 v = lanes_values(codes, s, byte);  // (exact: two significant bits)
  const uint32_t w = __float_as_uint(v[0]) >> 16 | (__float_as_uint(v[1]) & 0xffff0000u);
  return __builtin_bit_cast(lanes_bf2, w);
}
inline uint32_t lanes_codes(uint32_t old, float a, float b, float s, int byte) {
  const float scale = lanes_scale(s);
  const uint32_t two = lanes_code(a, scale) | lanes_code(b, scale) << 4;
  return (old & ~(255u << (8 * byte))) | two << (8 * byte);
}
inline uint32_t lanes_codes_bf16(uint32_t old, lanes_bf2 v, float s, int byte) {
  const uint32_t w = __builtin_bit_cast(uint32_t, v);
  return lanes_codes(old, __uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u), s, byte);
}
#define __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, b) lanes_values(c, s, b)
#define __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, b) lanes_values_bf16(c, s, b)
#define __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, x, y, s, b) lanes_codes(o, x, y, s, b)
#define __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, v, s, b) lanes_codes_bf16(o, v, s, b)

#define __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, x, y, z) lanes_product_f32<32>(a, b, c)
