// Host side of the attention calls of include/dart.h: argument checks, the choice of variants
// and kernel launches.  No allocation, no synchronisation.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/dart.h"
#include "cache.hpp"
#include "k_attend.hpp"
#include "k_rotate.hpp"

using namespace dart;

namespace {

dart_status make_rotate(const dart_rotation* u, Rotate& a) {
  if (!u) return DART_ERR_NULL;
  DART_TRY(check_heads(u->Hq, u->Hkv, u->d, u->dtype));
  if (u->rot < 0 || u->rot > u->d || u->rot % 8 || u->planes < 1 || u->planes > kMaxPlanes) return DART_ERR_SHAPE;
  if (!(u->eps >= 0.f) || !std::isfinite(u->eps) || !std::isfinite(u->scale)) return DART_ERR_SHAPE;
  if (u->rot > 0 && !u->inv_freq) return DART_ERR_NULL;
  if ((u->q_weight && off16(u->q_weight)) || (u->k_weight && off16(u->k_weight))) return DART_ERR_ALIGN;
  a = {};
  a.Hq = u->Hq;
  a.Hkv = u->Hkv;
  a.d = u->d;
  a.half = u->rot / 2;
  a.interleaved = u->interleaved != 0;
  a.planes = u->planes;
  int end = 0;
  for (int p = 0; p < kMaxPlanes; ++p) {
    if (u->planes > 1 && p < u->planes) {
      if (u->sections[p] < 0 || u->sections[p] > a.half - end) return DART_ERR_SHAPE;
      end += u->sections[p];
    }
    a.section_end[p] = u->planes > 1 ? end : a.half;
  }
  if (u->planes > 1 && end != a.half) return DART_ERR_SHAPE;
  a.inv_freq = u->inv_freq;
  a.qw = u->q_weight;
  a.kw = u->k_weight;
  a.eps = u->eps;
  a.scale = u->scale;
  return DART_OK;
}

template <int DT, int VE, bool APPEND>
dart_status launch_rotate(Rotate& a, const Cache& c, hipStream_t st) {
  const int rest = a.d - 2 * a.half;
  a.units = a.half / VE + (rest + 2 * VE - 1) / (2 * VE);
  a.lanes_shift = 0;
  while ((1 << a.lanes_shift) < a.units) ++a.lanes_shift;
  // Four waves share a token where there are few, or where each then has two rounds of heads or more: 36 864 tokens of
  // 32 + 32 heads 229 us with a wave each and 213 with four, 31 000 of 28 + 4 + 4 heads 114 and 154, 32 of those 8.6 and 7.9.
  // (2^24 blocks of 256 threads would be more than a launch takes)
  const int rounds = ((a.Hq + a.Hkv * (APPEND ? 2 : 1)) << a.lanes_shift) / kWave;
  if (a.T < 1024 || (rounds >= 8 && a.T < kMaxTokens))
    k_norm_rotate<DT, VE, 4, APPEND><<<dim3(a.T), dim3(256), 0, st>>>(a, c);
  else
    k_norm_rotate<DT, VE, 1, APPEND><<<dim3((a.T + 3) / 4), dim3(256), 0, st>>>(a, c);
  return launched();
}

template <bool APPEND>
dart_status rotate(Rotate& a, const Cache& c, int dtype, hipStream_t st) {
  if (dtype == DART_F32) return launch_rotate<kF32, 4, APPEND>(a, c, st);
  // pieces of 16 bytes unless a pair's two elements would then not fall to one lane
  return a.half % 8 == 0 ? launch_rotate<kBF16, 8, APPEND>(a, c, st) : launch_rotate<kBF16, 4, APPEND>(a, c, st);
}

dart_status set_rows(Rotate& a, int dtype, int T, const void* q, int64_t q_ld, const void* k, int64_t k_ld,
                     const int64_t* pos, int64_t pos_ld, void* q_out, int64_t q_out_ld, void* k_out, int64_t k_out_ld,
                     float* l1) {
  if (!pos) return DART_ERR_NULL;
  if (a.planes > 1 && pos_ld < T && pos_ld != 0) return DART_ERR_SHAPE;  // (0: the planes are alike)
  DART_TRY(check_rows(q, q_ld, (int64_t)a.Hq * a.d, dtype));
  DART_TRY(check_rows(k, k_ld, (int64_t)a.Hkv * a.d, dtype));
  DART_TRY(check_rows(q_out, q_out_ld, (int64_t)a.Hq * a.d, dtype));
  if (k_out) DART_TRY(check_rows(k_out, k_out_ld, (int64_t)a.Hkv * a.d, dtype));
  a.T = T;
  a.q = q;
  a.k = k;
  a.q_ld = q_ld;
  a.k_ld = k_ld;
  a.pos = reinterpret_cast<const long long*>(pos);
  a.pos_ld = a.planes > 1 ? pos_ld : 0;
  a.q_out = q_out;
  a.k_out = k_out;
  a.q_out_ld = q_out_ld;
  a.k_out_ld = k_out_ld;
  a.l1 = l1;
  return DART_OK;
}

template <int DT, int DP, int QW, int WM, int WK, int KT>
dart_status launch_tiles(const Attend& a, const Cache& c, const Parting& sp, hipStream_t st) {
  typedef AttendShape<DT, DP, QW, WM, WK, KT> S;
  // (one launch, or slices of the row tiles where it would have too many blocks: a launch takes the last `slots` of those left)
  const long most = kMaxBlocks / ((long)c.Hkv * sp.chunks);
  Parting left = sp;
  while (left.slots > 0) {
    const long slots = std::min(left.slots, most);
    k_attend<DT, DP, QW, WM, WK, KT><<<dim3((unsigned)(slots * c.Hkv * sp.chunks)), dim3(S::kThreads), S::kLds, st>>>(a, c, left);
    DART_TRY(launched());
    left.slots -= slots;
  }
  return DART_OK;
}

template <int DP>
dart_status launch_bf16(const Attend& a, const Cache& c, const Parting& sp, Kind kind, hipStream_t st) {
  if (kind == kFew) return launch_tiles<kBF16, DP, 16, 1, 4, 32>(a, c, sp, st);
  if constexpr (DP <= 128)
    if (kind == kWide) return launch_tiles<kBF16, DP, 32, 8, 1, 64>(a, c, sp, st);
  return launch_tiles<kBF16, DP, many_columns(kBF16, DP), 4, 1, 64>(a, c, sp, st);
}

template <int DP>
dart_status launch_f32(const Attend& a, const Cache& c, const Parting& sp, Kind kind, hipStream_t st) {
  if constexpr (DP <= 128)
    if (kind == kFew) return launch_tiles<kF32, DP, 16, 1, 4, 32>(a, c, sp, st);
  return launch_tiles<kF32, DP, many_columns(kF32, DP), 4, 1, 32>(a, c, sp, st);
}

template <int DT, int DP, int KT>
dart_status launch_both(const Attend& a, const Cache& c, const Parting& pre, const Parting& own, hipStream_t st) {
  constexpr int kLds = std::max(AttendShape<DT, DP, 16, 1, 4, 32>::kLds, AttendShape<DT, DP, many_columns(DT, DP), 4, 1, KT>::kLds);
  const long n = blocks_of(c, pre);
  k_attend_both<DT, DP, KT><<<dim3((unsigned)(n + blocks_of(c, own))), dim3(256), kLds, st>>>(a, c, pre, own, (unsigned)n);
  return launched();
}

dart_status launch_attend(const Attend& a, const Cache& c, int dtype, const Parting& sp, Kind k, hipStream_t st) {
  if (dtype == DART_BF16)
    return c.d <= 64 ? launch_bf16<64>(a, c, sp, k, st) : c.d <= 128 ? launch_bf16<128>(a, c, sp, k, st) : launch_bf16<256>(a, c, sp, k, st);
  return c.d <= 64 ? launch_f32<64>(a, c, sp, k, st) : c.d <= 128 ? launch_f32<128>(a, c, sp, k, st) : launch_f32<256>(a, c, sp, k, st);
}

}  // namespace

namespace dart {

// (SHARED: the own keys' parts are cut on the device; what reads them pays for that only then)
template <bool SHARED>
dart_status dart_attend_join_of(const Attend& a, const Cache& c, int dtype, const AttendPlan& p, hipStream_t st) {
  const JoinPlan j = plan_join(c, p.parts);
  if (dtype == DART_BF16)
    k_attend_join<kBF16, SHARED><<<dim3((unsigned)j.blocks), dim3(256), 0, st>>>(a, c, p.pre.chunk, p.pre.chunks, p.own.chunk, p.own.share,
                                                                                p.own.part_o, p.own.part_ml, j.lanes_shift, j.split_shift);
  else
    k_attend_join<kF32, SHARED><<<dim3((unsigned)j.blocks), dim3(256), 0, st>>>(a, c, p.pre.chunk, p.pre.chunks, p.own.chunk, p.own.share,
                                                                               p.own.part_o, p.own.part_ml, j.lanes_shift, j.split_shift);
  return launched();
}

dart_status dart_attend_join(const Attend& a, const Cache& c, int dtype, const AttendPlan& p, hipStream_t st) {
  return p.own.share > 0 ? dart_attend_join_of<true>(a, c, dtype, p, st) : dart_attend_join_of<false>(a, c, dtype, p, st);
}

}  // namespace dart

extern "C" {

dart_status dart_norm_rotate(const dart_rotation* rotation, int32_t T, const void* q, int64_t q_ld, const void* k,
                             int64_t k_ld, const int64_t* pos, int64_t pos_plane_stride, void* q_out, int64_t q_out_ld,
                             void* k_out, int64_t k_out_ld, float* l1_out, void* stream) {
  Rotate a;
  DART_TRY(make_rotate(rotation, a));
  if (T < 0 || T > kMaxTokens) return DART_ERR_SHAPE;
  if (T == 0) return DART_OK;
  if (!k_out) return DART_ERR_NULL;
  DART_TRY(set_rows(a, rotation->dtype, T, q, q_ld, k, k_ld, pos, pos_plane_stride, q_out, q_out_ld, k_out, k_out_ld,
                    l1_out));
  return rotate<false>(a, Cache{}, rotation->dtype, static_cast<hipStream_t>(stream));
}

dart_status dart_norm_rotate_append(const dart_rotation* rotation, const dart_cache* cache, const void* q,
                                    int64_t q_ld, const void* k, int64_t k_ld, const void* v, int64_t v_ld,
                                    const int64_t* pos, int64_t pos_plane_stride, void* q_out, int64_t q_out_ld,
                                    void* k_out, int64_t k_out_ld, float* l1_out, void* k_pool, void* v_pool,
                                    int32_t* status, void* stream) {
  Rotate a;
  Cache c;
  DART_TRY(make_rotate(rotation, a));
  DART_TRY(make_cache(cache, c));
  if (rotation->dtype != cache->dtype) return DART_ERR_DTYPE;
  if (a.Hq != c.Hq || a.Hkv != c.Hkv || a.d != c.d) return DART_ERR_SHAPE;
  if (c.T == 0 || c.B == 0) return DART_OK;
  DART_TRY(set_rows(a, rotation->dtype, c.T, q, q_ld, k, k_ld, pos, pos_plane_stride, q_out, q_out_ld, k_out, k_out_ld,
                    l1_out));
  DART_TRY(check_rows(v, v_ld, (int64_t)a.Hkv * a.d, cache->dtype));
  if (!k_pool || !v_pool) return DART_ERR_NULL;
  if (off16(k_pool) || off16(v_pool)) return DART_ERR_ALIGN;
  a.v = v;
  a.v_ld = v_ld;
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  c.status = status;
  return rotate<true>(a, c, cache->dtype, static_cast<hipStream_t>(stream));
}

size_t dart_attend_workspace_bytes(const dart_cache* cache) {
  Cache c;
  AttendPlan p;
  if (make_cache(cache, c) != DART_OK || plan_attend(c, cache->dtype, p) != DART_OK) return 0;
  return p.total;
}

dart_status dart_attend(const dart_cache* cache, const void* q, int64_t q_ld, const void* k_pool, const void* v_pool,
                        float scale, int32_t causal, void* out, int64_t out_ld, float* lse, void* ws, size_t ws_bytes,
                        int32_t* status, void* stream) {
  Cache c;
  DART_TRY(make_cache(cache, c));
  if (!std::isfinite(scale)) return DART_ERR_SHAPE;
  if (c.T == 0 || c.B == 0) return DART_OK;
  DART_TRY(check_rows(q, q_ld, (int64_t)c.Hq * c.d, cache->dtype));
  DART_TRY(check_rows(out, out_ld, (int64_t)c.Hq * c.d, cache->dtype));
  if (!k_pool || !v_pool) return DART_ERR_NULL;
  if (off16(k_pool) || off16(v_pool)) return DART_ERR_ALIGN;
  AttendPlan p;
  DART_TRY(plan_attend(c, cache->dtype, p));
  if (!ws || (reinterpret_cast<uintptr_t>(ws) % kAlign) != 0 || ws_bytes < p.total) return DART_ERR_WORKSPACE;
  c.status = status;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const Attend a = {q, k_pool, v_pool, out, lse, q_ld, out_ld, scale, causal != 0, 1.0 / (c.Hq / c.Hkv)};
  float* part_o = static_cast<float*>(ws);
  float2* part_ml = reinterpret_cast<float2*>(static_cast<unsigned char*>(ws) + p.o_ml);
  p.own.part_o = p.pre.part_o = part_o;
  p.own.part_ml = p.pre.part_ml = part_ml;
  const bool bf16 = cache->dtype == DART_BF16;
  if (p.both && bf16) {
    DART_TRY(c.d <= 64    ? (launch_both<kBF16, 64, 64>(a, c, p.pre, p.own, st))
             : c.d <= 128 ? (launch_both<kBF16, 128, 64>(a, c, p.pre, p.own, st))
                          : (launch_both<kBF16, 256, 64>(a, c, p.pre, p.own, st)));
  } else if (p.both) {
    DART_TRY(c.d <= 64 ? (launch_both<kF32, 64, 32>(a, c, p.pre, p.own, st)) : (launch_both<kF32, 128, 32>(a, c, p.pre, p.own, st)));
  } else {
    if (c.groups > 0) DART_TRY(launch_attend(a, c, cache->dtype, p.pre, p.pre_kind, st));
    DART_TRY(launch_attend(a, c, cache->dtype, p.own, p.own_kind, st));
  }
  if (p.parts == 1) return DART_OK;
  return dart_attend_join(a, c, cache->dtype, p, st);
}

}  // extern "C"
