// Host side of the calls of include/dart.h on caches held in 4 bits: argument checks, the choice of
// variants and kernel launches.  No allocation, no synchronisation.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/dart.h"
#include "cache.hpp"
#include "k_attend4.hpp"
#include "k_fourbit.hpp"

using namespace dart;

namespace {

// Codes (16 bytes to a block) and scales (a byte) of a pool.
dart_status check_pool(const void* codes, const void* scales) {
  if (!codes || !scales) return DART_ERR_NULL;
  return off16(codes) ? DART_ERR_ALIGN : DART_OK;
}

template <int DT, bool READ>
dart_status launch_hold(const Hold& a, const Cache& c, hipStream_t st) {
  // Four waves share a token where there are few; else each has its own, whose place it then finds once for all heads (23 040 tokens
  // of 32 + 32 heads, bf16: append and read 94 + 70 us, with four waves 113 + 71).
  if (a.T < 1024)
    k_hold<DT, 4, READ><<<dim3((unsigned)round_up8(a.T)), dim3(256), 0, st>>>(a, c);
  else
    k_hold<DT, 1, READ><<<dim3((unsigned)round_up8((a.T + 3) / 4)), dim3(256), 0, st>>>(a, c);
  return launched();
}

void set_hold(Hold& a, const Cache& c) {
  a.Hkv = c.Hkv;
  a.d = c.d;
  a.T = c.T;
  a.blocks = (c.d + kBlock - 1) / kBlock;
  a.heads_blocks = c.Hkv * a.blocks;
  a.per_block = a.blocks > 1 ? (uint32_t)(((1ull << 32) + a.blocks - 1) / a.blocks) : 0;
}

template <int DT, int DP, int QW, int WM, int WK, int KT, class HELD = In4Bits>
dart_status launch_tiles(const Attend& a, const Scales& scales, const Cache& c, const Parting& sp, hipStream_t st) {
  typedef AttendShape<DT, DP, QW, WM, WK, KT, HELD> S;
  const long most = kMaxBlocks / ((long)c.Hkv * sp.chunks);
  Parting left = sp;
  while (left.slots > 0) {
    const long slots = std::min(left.slots, most);
    k_attend_4bit<DT, DP, QW, WM, WK, KT, HELD><<<dim3((unsigned)(slots * c.Hkv * sp.chunks)), dim3(S::kThreads), S::kLds, st>>>(a, scales, c, left);
    DART_TRY(launched());
    left.slots -= slots;
  }
  return DART_OK;
}

template <int DT, int DP>
dart_status launch_attend(const Attend& a, const Scales& scales, const Cache& c, const Parting& sp, Kind kind, hipStream_t st) {
  if constexpr (DP <= 128)
    if (kind == kFew && codes_in_pages(c, true)) return launch_tiles<DT, DP, 16, 1, 4, 64, In4BitsPages>(a, scales, c, sp, st);
  if constexpr (DT == kBF16 || DP <= 128)
    if (kind == kFew) return launch_tiles<DT, DP, 16, 1, 4, 32>(a, scales, c, sp, st);
  if constexpr (DT == kBF16 && DP <= 128)
    if (kind == kWide) return launch_tiles<DT, DP, 32, 8, 1, 64>(a, scales, c, sp, st);
  return launch_tiles<DT, DP, many_columns(DT, DP), 4, 1, DT == kBF16 ? 64 : 32>(a, scales, c, sp, st);
}

template <int DT, int DP>
dart_status launch_both(const Attend& a, const Scales& scales, const Cache& c, const Parting& pre, const Parting& own, hipStream_t st) {
  constexpr int KT = DT == kBF16 ? 64 : 32;
  constexpr int kLds = std::max(AttendShape<DT, DP, 16, 1, 4, 32, In4Bits>::kLds, AttendShape<DT, DP, many_columns(DT, DP), 4, 1, KT, In4Bits>::kLds);
  const long n = blocks_of(c, pre);
  k_attend_4bit_both<DT, DP, KT><<<dim3((unsigned)(n + blocks_of(c, own))), dim3(256), kLds, st>>>(a, scales, c, pre, own, (unsigned)n);
  return launched();
}

template <int DT, int DP>
dart_status launch_width(const Attend& a, const Scales& scales, const Cache& c, const AttendPlan& p, hipStream_t st) {
  if constexpr (DT == kBF16 || DP <= 128)
    if (p.both) return launch_both<DT, DP>(a, scales, c, p.pre, p.own, st);
  if (c.groups > 0) DART_TRY((launch_attend<DT, DP>(a, scales, c, p.pre, p.pre_kind, st)));
  return launch_attend<DT, DP>(a, scales, c, p.own, p.own_kind, st);
}

template <int DT>
dart_status launch_all(const Attend& a, const Scales& scales, const Cache& c, const AttendPlan& p, hipStream_t st) {
  DART_TRY((c.d <= 64    ? launch_width<DT, 64>(a, scales, c, p, st)
            : c.d <= 128 ? launch_width<DT, 128>(a, scales, c, p, st)
                         : launch_width<DT, 256>(a, scales, c, p, st)));
  if (p.parts == 1) return DART_OK;
  return dart_attend_join(a, c, DT == kBF16 ? DART_BF16 : DART_F32, p, st);
}

}  // namespace

extern "C" {

dart_status dart_append_4bit(const dart_cache* cache, const void* k, int64_t k_ld, const void* v, int64_t v_ld, void* k_codes,
                             void* k_scales, void* v_codes, void* v_scales, int32_t* status, void* stream) {
  Cache c;
  DART_TRY(make_cache(cache, c, 4));
  if (c.T == 0 || c.B == 0) return DART_OK;
  DART_TRY(check_rows(k, k_ld, (int64_t)c.Hkv * c.d, cache->dtype));
  DART_TRY(check_rows(v, v_ld, (int64_t)c.Hkv * c.d, cache->dtype));
  DART_TRY(check_pool(k_codes, k_scales));
  DART_TRY(check_pool(v_codes, v_scales));
  c.status = status;
  Hold a = {};
  set_hold(a, c);
  a.k = k, a.v = v, a.k_ld = k_ld, a.v_ld = v_ld;
  a.k_codes = k_codes, a.v_codes = v_codes;
  a.k_scales = static_cast<uint8_t*>(k_scales), a.v_scales = static_cast<uint8_t*>(v_scales);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return cache->dtype == DART_BF16 ? launch_hold<kBF16, false>(a, c, st) : launch_hold<kF32, false>(a, c, st);
}

dart_status dart_read_4bit(const dart_cache* cache, const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales,
                           void* k_out, int64_t k_ld, void* v_out, int64_t v_ld, int32_t* status, void* stream) {
  Cache c;
  DART_TRY(make_cache(cache, c, 4));
  if (c.T == 0 || c.B == 0 || (!k_out && !v_out)) return DART_OK;
  if (k_out) {
    DART_TRY(check_rows(k_out, k_ld, (int64_t)c.Hkv * c.d, cache->dtype));
    DART_TRY(check_pool(k_codes, k_scales));
  }
  if (v_out) {
    DART_TRY(check_rows(v_out, v_ld, (int64_t)c.Hkv * c.d, cache->dtype));
    DART_TRY(check_pool(v_codes, v_scales));
  }
  c.status = status;
  Hold a = {};
  set_hold(a, c);
  a.k_out = k_out, a.v_out = v_out, a.k_ld = k_ld, a.v_ld = v_ld;
  a.k_codes = const_cast<void*>(k_codes), a.v_codes = const_cast<void*>(v_codes);
  a.k_scales = static_cast<uint8_t*>(const_cast<void*>(k_scales)), a.v_scales = static_cast<uint8_t*>(const_cast<void*>(v_scales));
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return cache->dtype == DART_BF16 ? launch_hold<kBF16, true>(a, c, st) : launch_hold<kF32, true>(a, c, st);
}

size_t dart_attend_4bit_workspace_bytes(const dart_cache* cache) {
  Cache c;
  AttendPlan p;
  if (make_cache(cache, c, 4) != DART_OK || plan_attend(c, cache->dtype, p, true) != DART_OK) return 0;
  return p.total;
}

dart_status dart_attend_4bit(const dart_cache* cache, const void* q, int64_t q_ld, const void* k_codes, const void* k_scales,
                             const void* v_codes, const void* v_scales, float scale, int32_t causal, void* out, int64_t out_ld, float* lse,
                             void* ws, size_t ws_bytes, int32_t* status, void* stream) {
  Cache c;
  DART_TRY(make_cache(cache, c, 4));
  if (!std::isfinite(scale)) return DART_ERR_SHAPE;
  if (c.T == 0 || c.B == 0) return DART_OK;
  DART_TRY(check_rows(q, q_ld, (int64_t)c.Hq * c.d, cache->dtype));
  DART_TRY(check_rows(out, out_ld, (int64_t)c.Hq * c.d, cache->dtype));
  DART_TRY(check_pool(k_codes, k_scales));
  DART_TRY(check_pool(v_codes, v_scales));
  AttendPlan p;
  DART_TRY(plan_attend(c, cache->dtype, p, true));
  if (!ws || (reinterpret_cast<uintptr_t>(ws) % kAlign) != 0 || ws_bytes < p.total) return DART_ERR_WORKSPACE;
  c.status = status;
  const Attend a = {q, k_codes, v_codes, out, lse, q_ld, out_ld, scale, causal != 0, 1.0 / (c.Hq / c.Hkv)};
  const Scales scales = {static_cast<const uint8_t*>(k_scales), static_cast<const uint8_t*>(v_scales)};
  p.own.part_o = p.pre.part_o = static_cast<float*>(ws);
  p.own.part_ml = p.pre.part_ml = reinterpret_cast<float2*>(static_cast<unsigned char*>(ws) + p.o_ml);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return cache->dtype == DART_BF16 ? launch_all<kBF16>(a, scales, c, p, st) : launch_all<kF32>(a, scales, c, p, st);
}

}  // extern "C"
