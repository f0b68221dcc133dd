// What the attention and rotation kernels use of the device language, on the CPU: a lane is a fiber, an
// operation across lanes is a meeting of its wave's 64, a barrier one of the workgroup.  Lanes run one at a
// time from meeting to meeting, so results do not depend on the machine; which lane of a wave goes first is
// the caller's choice (lanes.cpp).  Divergent operations across lanes are not covered: all 64 have to come.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdlib>
#include <cstring>
#include <functional>

#define __device__
#define __global__
#define __host__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __shared__ static

using std::max;
using std::min;

struct uint2 { unsigned x, y; };
struct float2 { float x, y; };
inline float2 make_float2(float x, float y) { return {x, y}; }
struct dim3 {
  unsigned x, y, z;
  dim3(unsigned a = 1, unsigned b = 1, unsigned c = 1) : x(a), y(b), z(c) {}
};
typedef void* hipStream_t;
enum hipError_t { hipSuccess = 0 };
hipError_t hipGetLastError();

// ---- lanes.cpp -----------------------------------------------------------------------------------
constexpr int kSlot = 64;  // bytes a lane brings to a meeting
struct Box {
  alignas(16) unsigned char brought[64][kSlot];
};
struct Meeting {
  Box box[2];  // in turn: what was brought to one meeting is read until the next but one begins
  int arrived, turn;
};
extern int lane_now;           // of the workgroup
extern dim3 block_now;
Meeting& wave_now();
void wave_meet();              // returns when all 64 lanes have called it
void block_meet();
void lanes_launch(const char* what, dim3 grid, dim3 block, size_t lds, hipStream_t, std::function<void()> kernel);
unsigned char* lanes_lds();

#define threadIdx (dim3((unsigned)lane_now, 0, 0))
#define blockIdx block_now

template <class T>
const Box& bring(const T& v) {
  static_assert(sizeof(T) <= kSlot, "");
  Meeting& w = wave_now();
  Box& box = w.box[w.turn & 1];
  memcpy(box.brought[lane_now & 63], &v, sizeof v);
  wave_meet();
  return box;
}
template <class T>
T brought(const Box& w, int lane, int at = 0) {
  T v;
  memcpy(&v, w.brought[lane] + at * sizeof v, sizeof v);
  return v;
}
template <class T>
T from_lane(T v, int lane) {
  return brought<T>(bring(v), lane & 63);
}

inline void __syncthreads() { block_meet(); }
inline unsigned long long __ballot(bool p) {
  const Box& w = bring(p);
  unsigned long long r = 0;
  for (int i = 0; i < 64; ++i) r |= (unsigned long long)brought<bool>(w, i) << i;
  return r;
}
inline bool __any(bool p) { return __ballot(p) != 0; }
template <class T>
T __shfl_xor(T v, int mask) { return from_lane(v, (lane_now & 63) ^ mask); }
#define __builtin_amdgcn_readfirstlane(x) from_lane(x, 0)
#define __builtin_amdgcn_readlane(x, l) from_lane(x, l)
#define __builtin_amdgcn_wave_barrier() wave_meet()
#define __builtin_amdgcn_fence(...) ((void)0)
#define __builtin_amdgcn_sched_group_barrier(...) ((void)0)

// Quad permutations and rotations of a row of 16, the ones in use.
inline int lanes_dpp(int v, int control) {
  const int l = lane_now & 63;
  int from;
  if (control < 0x100) from = (l & ~3) | ((control >> (2 * (l & 3))) & 3);
  else if (control > 0x120 && control < 0x130) from = (l & ~15) | ((l - (control - 0x120)) & 15);
  else abort();
  return from_lane(v, from);
}
#define __builtin_amdgcn_update_dpp(old, v, control, rows, banks, bound) lanes_dpp(v, control)

// Odd rows of N lanes of the first and even rows of the second change places.
struct Swapped {
  unsigned r[2];
  unsigned operator[](int i) const { return r[i]; }
};
template <int N>
Swapped lanes_swap(unsigned a, unsigned b) {
  const unsigned both[2] = {a, b};
  const Box& w = bring(both);
  const int l = lane_now & 63, low = l & ~N, high = l | N;
  const Swapped s = l & N ? Swapped{{brought<unsigned>(w, low, 1), b}} : Swapped{{a, brought<unsigned>(w, high, 0)}};
  return s;
}
#define __builtin_amdgcn_permlane16_swap(a, b, x, y) lanes_swap<16>(a, b)
#define __builtin_amdgcn_permlane32_swap(a, b, x, y) lanes_swap<32>(a, b)

// D = A B + C of one wave: A is N x K, B is K x N, N = 16 or 32.  Lane l brings kPer elements of row l % N of A, and of column
// l % N of B, from k = l / N * kPer on; it holds of column l % N of D four rows in every 4 * (64 / N), the (l / N)-th four.
template <int N, int kPer, class Acc>
Acc lanes_product(const float (&a)[kPer], const float (&b)[kPer], Acc c) {
  struct { float a[kPer], b[kPer]; } both;
  memcpy(both.a, a, sizeof both.a);
  memcpy(both.b, b, sizeof both.b);
  const Box& w = bring(both);
  constexpr int kGroups = 64 / N;
  const int l = lane_now & 63, n = l % N, g = l / N;
  for (int i = 0; i < N * N / 64; ++i) {
    const int m = 4 * kGroups * (i / 4) + 4 * g + i % 4;
    float part[kPer] = {};
    for (int k = 0; k < kGroups; ++k) {
      const float* row = reinterpret_cast<const float*>(w.brought[m + N * k]);
      const float* column = reinterpret_cast<const float*>(w.brought[n + N * k]) + kPer;
      for (int x = 0; x < kPer; ++x) part[x] += row[x] * column[x];
    }
    for (int x = 0; x < kPer; ++x) c[i] += part[x];
  }
  return c;
}
template <int N, class Acc, class Operand>
Acc lanes_product_bf16(const Operand& a, const Operand& b, Acc c) {
  uint16_t h[16];
  uint32_t u[16];
  float f[2][8];
  memcpy(h, &a, 16);
  memcpy(h + 8, &b, 16);
  for (int i = 0; i < 16; ++i) u[i] = (uint32_t)h[i] << 16;
  memcpy(f, u, sizeof f);
  return lanes_product<N>(f[0], f[1], c);
}
template <int N, class Acc>
Acc lanes_product_f32(float a, float b, Acc c) {
  const float x[1] = {a}, y[1] = {b};
  return lanes_product<N>(x, y, c);
}
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, x, y, z) lanes_product_bf16<32>(a, b, c)
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) lanes_product_bf16<16>(a, b, c)
#define __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, x, y, z) lanes_product_f32<16>(a, b, c)

// Four 16-bit elements of each of 16 lanes, transposed among them.
typedef short lanes_4 __attribute__((ext_vector_type(4)));
inline lanes_4 lanes_transposed(const void* at) {
  lanes_4 v, r;
  memcpy(&v, at, sizeof v);
  const Box& w = bring(v);
  const int l = lane_now & 63, i = l & 15;
  for (int j = 0; j < 4; ++j) r[j] = brought<short>(w, (l & ~15) + i / 4 + 4 * j, i % 4);
  return r;
}
#define __builtin_amdgcn_ds_read_tr16_b64_v4i16(p) lanes_transposed(p)

// ---- arithmetic --------------------------------------------------------------------------------------
inline float __uint_as_float(uint32_t u) { float f; memcpy(&f, &u, 4); return f; }
inline uint32_t __float_as_uint(float f) { uint32_t u; memcpy(&u, &f, 4); return u; }
inline float __int_as_float(int u) { return __uint_as_float((uint32_t)u); }
inline int __float_as_int(float f) { return (int)__float_as_uint(f); }
inline double __longlong_as_double(long long u) { double f; memcpy(&f, &u, 8); return f; }
inline long long __double_as_longlong(double f) { long long u; memcpy(&u, &f, 8); return u; }
#define __builtin_amdgcn_exp2f(x) exp2f(x)
inline float rsqrtf(float x) { return (float)(1.0 / sqrt((double)x)); }
inline void sincospif(float x, float* s, float* c) {
  *s = (float)sin(x * 3.14159265358979323846);
  *c = (float)cos(x * 3.14159265358979323846);
}
inline int atomicOr(int* p, int v) {
  const int old = *p;
  *p |= v;
  return old;
}
#define __hip_atomic_load(p, order, scope) (*(p))
#define __hip_atomic_store(p, v, order, scope) (*(p) = (v))
