// Head norm and position rotation of queries and keys, and the append of keys and values to
// their pages.
#pragma once

#include "cache.hpp"

namespace dart {

constexpr int kMaxPlanes = 4;
constexpr int kMaxPairs = 128;  // of a head of 256

struct Rotate {
  int Hq, Hkv, d, half;  // half: pairs of a head that are turned
  int T, interleaved, planes;
  int section_end[kMaxPlanes];  // pairs below section_end[p] and of no earlier plane follow plane p
  const float* inv_freq;
  const void *qw, *kw;
  float eps, scale;
  const void *q, *k, *v;
  long q_ld, k_ld, v_ld;
  const long long* pos;
  long pos_ld;
  void *q_out, *k_out;
  long q_out_ld, k_out_ld;
  float* l1;
  void *k_pool, *v_pool;  // (append)
  int lanes_shift;        // 2^lanes_shift lanes per head
  int units;              // of them in use: each holds two pieces of VE elements
};

// VE elements of a row, as loaded: bf16 pairs or 32-bit words.
template <int DT, int VE>
struct Piece {
  static constexpr int kWords = DT == kBF16 ? VE / 2 : VE;
  uint32_t w[kWords];
  __device__ __forceinline__ float get(int i) const {
    if constexpr (DT == kBF16) return i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
    else return __uint_as_float(w[i]);
  }
};
template <int DT, int VE>
__device__ __forceinline__ Piece<DT, VE> load_piece(const void* row, long at) {
  Piece<DT, VE> p;
  constexpr int kBytes = Piece<DT, VE>::kWords * 4;
  const unsigned char* src = static_cast<const unsigned char*>(row) + at * (DT == kBF16 ? 2 : 4);
  __builtin_memcpy(&p, __builtin_assume_aligned(src, kBytes), kBytes);
  return p;
}
template <int DT, int VE>
__device__ __forceinline__ void store_piece(void* row, long at, const Piece<DT, VE>& p) {
  constexpr int kBytes = Piece<DT, VE>::kWords * 4;
  unsigned char* dst = static_cast<unsigned char*>(row) + at * (DT == kBF16 ? 2 : 4);
  __builtin_memcpy(__builtin_assume_aligned(dst, kBytes), &p, kBytes);
}
// Rounded to nearest, ties to even; NaN stays one.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const bf16x2 r = __builtin_convertvector((f32x2{lo, hi}), bf16x2);
  return __builtin_bit_cast(uint32_t, r);
}
template <int DT, int VE>
__device__ __forceinline__ Piece<DT, VE> round_piece(const float (&x)[VE]) {
  Piece<DT, VE> p;
  if constexpr (DT == kBF16) {
#pragma unroll
    for (int i = 0; i < VE / 2; ++i) p.w[i] = bf16_pair(x[2 * i], x[2 * i + 1]);
  } else {
#pragma unroll
    for (int i = 0; i < VE; ++i) p.w[i] = __float_as_uint(x[i]);
  }
  return p;
}

// Memory-bound: every row is read once and written once (23 040 tokens of 32 + 32 + 32 heads of 128 to their pages: 1.13 GB
// in 211 us, 5.4 TB/s, where a large copy moves 4.8; 36 864 tokens of 28 + 4 heads 113 us, 5.3 TB/s; a single token 6.5 us,
// the launch).  W waves share a token: one or four (launch_rotate).  A head lies in 2^lanes_shift lanes of two pieces of 16
// bytes (8 where a half head of bf16 is no multiple of 8 elements; 9216 tokens take 28 us with pieces of 16 bytes, 33 with 8):
// with pairs (p, p + half) piece u of the first half and piece u of the second, so that both elements of a pair are in one
// lane and a lane meets the same angles in every head.  The angles are taken once per wave, a lane per pair:
// position * frequency in 64 bits as turns, of which the whole ones are dropped, so that a long context's positions
// lose nothing.  Norms are summed in 32 bits over a head's elements, the L1 norms of key rows in 64.
template <int DT, int VE, int W, bool APPEND>
__global__ __launch_bounds__(256) void k_norm_rotate(Rotate a, Cache c) {
  __shared__ float2 turn[4][kMaxPairs];
  __shared__ double l1_part[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int part = wave % W;
  const long t = (long)blockIdx.x * (4 / W) + wave / W;
  const bool live = t < a.T;

  const int L = 1 << a.lanes_shift, u = lane & (L - 1), per = kWave >> a.lanes_shift;
  const bool used = u < a.units && live;
  const int rot_units = a.half / VE;
  const bool turned = u < rot_units;
  const int rest = 2 * a.half + 2 * (u - rot_units) * VE;  // (past the turned pairs: two pieces in a row)
  const int at0 = turned ? (a.interleaved ? 2 * u * VE : u * VE) : rest;
  const int at1 = turned && !a.interleaved ? a.half + u * VE : at0 + VE;
  const bool two = at1 < a.d;
  const int heads = a.Hq + a.Hkv + (APPEND ? a.Hkv : 0);
  // With a wave to a token two rounds of heads are asked for before the first is worked on, the first two before the
  // angles (36 864 tokens of 28 + 4 heads 111 -> 108.5 us; four at once 110, and 32 000 of 28 + 4 + 4 then take 128 instead
  // of 112).  Four waves to a token have a few rounds each and do better the plain way (576 tokens of
  // 64 heads, 32 bits: 10.8 us, 11.2 with two rounds, 11.5 with the loads first; 23 040 of 96 heads 211, 210 and 213).
  constexpr int kAhead = W == 1 ? 2 : 1;
  Piece<DT, VE> r0[kAhead] = {}, r1[kAhead] = {};
  auto load = [&](int h0) {
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int head = h0 + x * W * per + (lane >> a.lanes_shift);
      const bool is_q = head < a.Hq, is_k = !is_q && head < a.Hq + a.Hkv;
      if (!used || head >= heads) continue;
      const void* src = is_q ? a.q : is_k ? a.k : a.v;
      const long row = t * (is_q ? a.q_ld : is_k ? a.k_ld : a.v_ld) +
                       (long)(is_q ? head : is_k ? head - a.Hq : head - a.Hq - a.Hkv) * a.d;
      r0[x] = load_piece<DT, VE>(src, row + at0);
      if (two) r1[x] = load_piece<DT, VE>(src, row + at1);
    }
  };
  if (W == 1) load(0);

  for (int p = lane; p < a.half; p += kWave) {
    float sn = 0.f, cs = 1.f;
    if (live) {
      int plane = 0;
      for (int i = 0; i + 1 < a.planes; ++i) plane += p >= a.section_end[i];
      const double turns = (double)a.pos[plane * a.pos_ld + t] * ((double)a.inv_freq[p] * 0.15915494309189533577);
      // half turns in two words: what the first leaves (under 2^-25) turns the sine and cosine of it a little further
      const double halves = 2.0 * (turns - rint(turns));
      const float first = (float)halves, rest = (float)((halves - first) * 3.14159265358979323846);
      float s0, c0;
      sincospif(first, &s0, &c0);
      sn = fmaf(c0, rest, s0);
      cs = fmaf(-s0, rest, c0);
    }
    turn[wave][p] = make_float2(cs * a.scale, sn * a.scale);
  }
  __syncthreads();

  // where the token's keys and values go
  long slot = 0;
  bool put = false;
  if (APPEND && live) {
    const int b = c.cu == nullptr ? (int)t : owner_of(c.cu, c.B, (int)t);
    const Seq s = sequence_of(c, b);
    const int i = (int)t - s.tok0;
    bool bad = false;
    if (s.valid && i >= 0 && i < s.n && s.kv >= s.n) {
      slot = key_offset(c, c.pages + (long)b * c.pages_ld, s.kv - s.n + i, bad);
      put = !bad;
    }
    if (!put && lane == 0 && part == 0) flag(c, bad ? kBadPage : kBadSequence);
  }

  float cs[VE], sn[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    const float2 v = turned && used ? turn[wave][u * VE + j] : make_float2(1.f, 0.f);
    cs[j] = v.x;
    sn[j] = v.y;
  }
  double l1 = 0.0;
  for (int h0 = part * per; h0 < heads; h0 += kAhead * W * per) {
    if (W > 1 || h0 > 0) load(h0);
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int head = h0 + x * W * per + (lane >> a.lanes_shift);
      if (h0 + x * W * per >= heads) break;
      const bool on = used && head < heads;
      const bool is_q = head < a.Hq, is_k = !is_q && head < a.Hq + a.Hkv;
      const int h = is_q ? head : is_k ? head - a.Hq : head - a.Hq - a.Hkv;
      Piece<DT, VE> p0 = r0[x], p1 = r1[x];
      if (is_q || is_k) {
        float x0[VE], x1[VE];
#pragma unroll
        for (int j = 0; j < VE; ++j) x0[j] = p0.get(j), x1[j] = p1.get(j);
        const void* w = is_q ? a.qw : a.kw;
        if (a.qw != nullptr || a.kw != nullptr) {
          float ss = 0.f;
#pragma unroll
          for (int j = 0; j < VE; ++j) ss += x0[j] * x0[j] + x1[j] * x1[j];
          for (int o = 1; o < L; o <<= 1) ss += __shfl_xor(ss, o);
          float v = ss / (float)a.d + a.eps;
          // Elements over 2^60 or so have squares that 32 bits do not hold, and those under 2^-60 squares that lose their
          // bits (which matters where eps does not outweigh them): the head and eps are then taken in other units.
          const bool far = !(v > 0x1p-90f && v < INFINITY);
          if (__any(far)) {
            const float unit = !far || w == nullptr ? 1.f : v < 1.f ? 0x1p100f : 0x1p-70f;
            ss = 0.f;
#pragma unroll
            for (int j = 0; j < VE; ++j) {
              x0[j] *= unit;
              x1[j] *= unit;
              ss += x0[j] * x0[j] + x1[j] * x1[j];
            }
            for (int o = 1; o < L; o <<= 1) ss += __shfl_xor(ss, o);
            v = ss / (float)a.d + a.eps * unit * unit;
          }
          if (on && w != nullptr) {
            const float r = rsqrtf(v);
            const Piece<DT, VE> w0 = load_piece<DT, VE>(w, at0);
            Piece<DT, VE> w1 = {};
            if (two) w1 = load_piece<DT, VE>(w, at1);
#pragma unroll
            for (int j = 0; j < VE; ++j) x0[j] = x0[j] * r * w0.get(j), x1[j] = x1[j] * r * w1.get(j);
          }
        }
        if (turned) {
          if (a.interleaved) {
#pragma unroll
            for (int j = 0; j < VE / 2; ++j) {
              const float e0 = x0[2 * j], o0 = x0[2 * j + 1], e1 = x1[2 * j], o1 = x1[2 * j + 1];
              x0[2 * j] = e0 * cs[j] - o0 * sn[j];
              x0[2 * j + 1] = o0 * cs[j] + e0 * sn[j];
              x1[2 * j] = e1 * cs[VE / 2 + j] - o1 * sn[VE / 2 + j];
              x1[2 * j + 1] = o1 * cs[VE / 2 + j] + e1 * sn[VE / 2 + j];
            }
          } else {
#pragma unroll
            for (int j = 0; j < VE; ++j) {
              const float e = x0[j], o = x1[j];
              x0[j] = e * cs[j] - o * sn[j];
              x1[j] = o * cs[j] + e * sn[j];
            }
          }
        }
        p0 = round_piece<DT, VE>(x0);
        p1 = round_piece<DT, VE>(x1);
        if (is_k && on) {  // 2*VE terms in 32 bits, their sums in 64
          float s = 0.f;
#pragma unroll
          for (int j = 0; j < VE; ++j) s += fabsf(p0.get(j)) + (two ? fabsf(p1.get(j)) : 0.f);
          l1 += (double)s;
        }
      }
      if (!on) continue;
      if (is_q || (is_k && a.k_out != nullptr)) {
        void* dst = is_q ? a.q_out : a.k_out;
        const long r = t * (is_q ? a.q_out_ld : a.k_out_ld) + (long)h * a.d;
        store_piece<DT, VE>(dst, r + at0, p0);
        if (two) store_piece<DT, VE>(dst, r + at1, p1);
      }
      if (APPEND && !is_q && put) {
        void* dst = is_k ? a.k_pool : a.v_pool;
        const long r = slot + (long)h * c.head_ld;
        store_piece<DT, VE>(dst, r + at0, p0);
        if (two) store_piece<DT, VE>(dst, r + at1, p1);
      }
    }
  }
  if (a.l1 == nullptr) return;
  l1 = wave_sum(l1);
  if (W == 1) {
    if (live && lane == 0) a.l1[t] = (float)l1;
    return;
  }
  if (lane == 0) l1_part[wave] = l1;
  __syncthreads();
  if (live && lane == 0 && part == 0) {
    for (int i = 1; i < W; ++i) l1 += l1_part[wave + i];
    a.l1[t] = (float)l1;
  }
}

}  // namespace dart
