// Attention over the paged cache.
#pragma once

#include "cache.hpp"
#include "k_rotate.hpp"

namespace dart {

struct Attend {
  const void *q, *k_pool, *v_pool;
  void* out;
  float* lse;  // or nullptr
  long q_ld, out_ld;
  float scale;
  int causal;
};

// One wave per (token, query head), key after key, with the running maximum and sum.  Right for
// every case; a score costs a reduction over the wave.
template <int DT>
__global__ __launch_bounds__(64) void k_attend_rows(Attend a, Cache c) {
  constexpr int kPer = 4;  // elements of a head in a lane
  const int t = blockIdx.x, head = blockIdx.y, lane = threadIdx.x;
  const int b = c.cu == nullptr ? t : owner_of(c.cu, c.B, t);
  const Seq s = sequence_of(c, b);
  int own = s.kv;
  if (a.causal) own = s.kv - s.n + (t - s.tok0) + 1;
  bool ok = s.valid && t >= s.tok0 && t < s.tok0 + s.n;
  int prefix = 0, g = 0;
  if (c.groups > 0) {
    g = owner_of(c.group_cu, c.groups, b);
    prefix = prefix_of(c, g);
    if (prefix < 0 || b < c.group_cu[g] || b >= c.group_cu[g + 1]) ok = false;
  }
  if (!ok) {
    if (lane == 0) flag(c, kBadSequence);
    own = prefix = 0;
  }
  const int h = head / (c.Hq / c.Hkv);
  auto get = [&](const void* p, long at) -> float {
    if constexpr (DT == kBF16) return __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[at] << 16);
    else return static_cast<const float*>(p)[at];
  };
  float q[kPer], o[kPer] = {};
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int e = i * kWave + lane;
    q[i] = e < c.d ? get(a.q, t * a.q_ld + (long)head * c.d + e) * a.scale : 0.f;
  }
  float m = -INFINITY, l = 0.f;
  auto pass = [&](const int* table, int n) {
    for (int j = 0; j < n; ++j) {
      bool bad;
      const long at = key_offset(c, table, j, bad) + (long)h * c.head_ld;
      if (bad && lane == 0) flag(c, kBadPage);
      float x = 0.f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int e = i * kWave + lane;
        if (e < c.d) x += q[i] * get(a.k_pool, at + e);
      }
      x = wave_sum(x);
      const float top = fmaxf(m, x), base = top == -INFINITY ? 0.f : top;
      const float keep = __expf(m - base), p = __expf(x - base);
      l = l * keep + p;
      m = top;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int e = i * kWave + lane;
        if (e < c.d) o[i] = o[i] * keep + p * get(a.v_pool, at + e);
      }
    }
  };
  if (prefix > 0) pass(c.prefix_pages + (long)g * c.prefix_ld, prefix);
  if (own > 0) pass(c.pages + (long)b * c.pages_ld, own);
  const bool none = l == 0.f;  // nothing seen, or nothing but scores of -infinity
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int e = i * kWave + lane;
    if (e >= c.d) continue;
    const float v = none ? 0.f : o[i] / l;
    const long at = t * a.out_ld + (long)head * c.d + e;
    if constexpr (DT == kBF16) static_cast<uint16_t*>(a.out)[at] = (uint16_t)bf16_pair(v, 0.f);
    else static_cast<float*>(a.out)[at] = v;
  }
  if (a.lse != nullptr && lane == 0) a.lse[(long)t * c.Hq + head] = none ? -INFINITY : m + logf(l);
}

}  // namespace dart
