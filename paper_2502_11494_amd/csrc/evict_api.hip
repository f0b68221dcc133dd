// Host side of the calls of include/dart.h on gathered attention weights and on eviction: argument checks,
// the choice of variants and kernel launches.  No allocation, no synchronisation.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/dart.h"
#include "cache.hpp"
#include "k_evict.hpp"
#include "k_weights.hpp"

using namespace dart;

namespace {

constexpr long kMaxTiles = 1L << 30;  // blocks of a call, over all its launches

// ---- gathered weights ---------------------------------------------------------------------------
struct GatherPlan {
  Shares own, pre;
  size_t total;
};

int keys_of_tile(int dtype, int d, bool few, bool codes) {
  if (few) return 64 * few_tiles(dtype == DART_BF16 ? kBF16 : kF32, d, codes);
  return dtype == DART_BF16 && d <= 128 ? 256 : 128;
}

// rows: (token, head) pairs of a sequence at most, of a group on average.
dart_status plan_shares(const Cache& c, int dtype, bool codes, long rows, long owners, int max_keys, Shares& s, size_t& bytes) {
  s.few = rows <= 48;
  const int keys = keys_of_tile(dtype, c.d, s.few, codes);
  s.tiles = std::max(1, (int)(((long)max_keys + keys - 1) / keys));
  if (owners * s.tiles > kMaxTiles / c.Hkv) return DART_ERR_SHAPE;
  const long blocks = owners * s.tiles * c.Hkv, row_tiles = (rows + 31) / 32;
  // Parts of the rows until there are sixteen blocks to a unit, of four tiles of rows at least: they even out what blocks whose keys
  // few rows see have less to do (two causal prompts of 9216, 28 + 4 heads, 1024, 2048 and 4096 blocks: 987, 866 and 834 us;
  // 637 causal tokens of 32 heads in 32 bits, parts of 8 tiles 53 us, of 4 37, of 2 46).  The keys are counted by the caller's bound:
  // with bounds of 8192 and 131 072 for those 637 keys 53 and 59 us, 33 with 637; those two prompts 730 us with 16 384, 1735 with 131 072
  // (one part), 705 with 9216.
  s.parts = s.few ? 1 : (int)std::max(1L, std::min((4096 + blocks - 1) / blocks, row_tiles / 4));
  bytes = std::max(bytes, s.parts > 1 ? (size_t)s.parts * blocks * keys * 4 : 0);
  return DART_OK;
}

dart_status plan_gather(const Cache& c, int dtype, bool codes, GatherPlan& p) {
  const long r = c.Hq / c.Hkv;
  if (c.T * r > kMaxRows) return DART_ERR_SHAPE;
  p = {};
  size_t bytes = 0;
  DART_TRY(plan_shares(c, dtype, codes, c.max_q * r, std::max(c.B, 1), c.max_kv, p.own, bytes));
  if (c.groups > 0) {
    p.pre.prefix = 1;
    const long rows = std::min((long)c.T, (long)c.max_q * c.B) * r;
    DART_TRY(plan_shares(c, dtype, codes, (rows + c.groups - 1) / c.groups, c.groups, c.max_prefix, p.pre, bytes));
  }
  p.total = kAlign + (bytes + kAlign - 1) / kAlign * kAlign;
  return DART_OK;
}

template <int DT, int DP, class HELD>
dart_status launch_gather(const Gather& a, const Cache& c, const Shares& sp, hipStream_t st) {
  typedef GatherShape<DT, DP> S;
  static_assert(S::kKeys == (DT == kBF16 && DP <= 128 ? 256 : 128), "keys_of_tile");
  const long blocks = (sp.prefix ? c.groups : c.B) * (long)sp.tiles * c.Hkv;
  for (long first = 0; first < blocks * sp.parts; first += kMaxBlocks) {
    const unsigned n = (unsigned)std::min(kMaxBlocks, blocks * sp.parts - first);
    if (sp.few) k_gather_weights_few<DT, DP, HELD><<<dim3(n), dim3(256), 0, st>>>(a, c, sp, (unsigned)first);
    else k_gather_weights<DT, DP, HELD><<<dim3(n), dim3(256), S::kLds, st>>>(a, c, sp, (unsigned)first);
    DART_TRY(launched());
  }
  if (sp.parts == 1) return DART_OK;
  k_join_weights<<<dim3((unsigned)blocks), dim3(256), 0, st>>>(a, c, sp, S::kKeys);
  return launched();
}

template <int DT, class HELD>
dart_status launch_gather_width(const Gather& a, const Cache& c, const Shares& sp, hipStream_t st) {
  return c.d <= 64    ? launch_gather<DT, 64, HELD>(a, c, sp, st)
         : c.d <= 128 ? launch_gather<DT, 128, HELD>(a, c, sp, st)
                      : launch_gather<DT, 256, HELD>(a, c, sp, st);
}

dart_status launch_gather_kind(const Gather& a, const Cache& c, int dtype, const Shares& sp, hipStream_t st) {
  if (a.k_scales)
    return dtype == DART_BF16 ? launch_gather_width<kBF16, In4Bits>(a, c, sp, st) : launch_gather_width<kF32, In4Bits>(a, c, sp, st);
  return dtype == DART_BF16 ? launch_gather_width<kBF16, AsRows>(a, c, sp, st) : launch_gather_width<kF32, AsRows>(a, c, sp, st);
}

// ---- eviction -------------------------------------------------------------------------------------
struct EvictPlan {
  int most;
  size_t left, total;  // bytes: where the sequences' lengths lie behind the kept keys, all
};

dart_status plan_evict(const Cache& c, const dart_eviction* e, EvictPlan& p) {
  if (!e) return DART_ERR_NULL;
  if (e->first < 0 || e->recent < 0 || e->first > kMaxKeys || e->recent > kMaxKeys || e->budget < 0) return DART_ERR_SHAPE;
  if (e->budget == 0 && (e->ratio_den < 1 || e->ratio_num < 0 || e->ratio_num > e->ratio_den)) return DART_ERR_BUDGET;
  p.most = keys_kept(e->budget, e->ratio_num, e->ratio_den, e->first, e->recent, c.max_kv);
  const size_t pairs = (size_t)c.B * c.Hkv;
  if (pairs * (size_t)std::max(p.most, 1) > (size_t)1 << 40) return DART_ERR_SHAPE;
  p.left = (pairs * p.most * 4 + kAlign - 1) / kAlign * kAlign;
  p.total = p.left + ((size_t)c.B * sizeof(int2) + kAlign - 1) / kAlign * kAlign + kAlign;
  return DART_OK;
}

// Arrays of which every address is a multiple of four bytes move by words.
int unit_of(const Column& col, int bytes) {
  const uintptr_t any = reinterpret_cast<uintptr_t>(col.from) | reinterpret_cast<uintptr_t>(col.to) | (uintptr_t)col.page_ld |
                        (uintptr_t)col.head_ld | (uintptr_t)col.row_ld | (uintptr_t)bytes;
  return any % 4 == 0 ? 4 : 1;
}

void add_rows(Moves& m, int x, const Column& col, int bytes, int unit, int most_lanes) {
  m.col[x] = col;
  m.kind[x] = unit;
  m.units[x] = bytes / unit;
  m.lanes_shift[x] = 0;
  while ((1 << m.lanes_shift[x]) < m.units[x] && (1 << m.lanes_shift[x]) < most_lanes) ++m.lanes_shift[x];
  const int lanes = 1 << m.lanes_shift[x];
  m.end[x] = (x ? m.end[x - 1] : 0) + (m.units[x] + lanes - 1) / lanes;
}

}  // namespace

extern "C" {

size_t dart_attend_weights_workspace_bytes(const dart_cache* cache, int32_t four_bit) {
  Cache c;
  GatherPlan p;
  if (make_cache(cache, c, four_bit ? 4 : 0) != DART_OK || plan_gather(c, cache->dtype, four_bit != 0, p) != DART_OK) return 0;
  return p.total;
}

dart_status dart_attend_weights(const dart_cache* cache, const void* q, int64_t q_ld, const void* k_pool, const void* k_scales,
                                const float* lse, float scale, int32_t causal, float carry, float* weights, void* ws, size_t ws_bytes,
                                int32_t* status, void* stream) {
  Cache c;
  DART_TRY(make_cache(cache, c, k_scales ? 4 : 0));
  if (!std::isfinite(scale) || !std::isfinite(carry)) return DART_ERR_SHAPE;
  if (c.T == 0 || c.B == 0) return DART_OK;
  DART_TRY(check_rows(q, q_ld, (int64_t)c.Hq * c.d, cache->dtype));
  if (!k_pool || !lse || !weights) return DART_ERR_NULL;
  if (off16(k_pool)) return DART_ERR_ALIGN;
  GatherPlan p;
  DART_TRY(plan_gather(c, cache->dtype, k_scales != nullptr, p));
  if (!ws || (reinterpret_cast<uintptr_t>(ws) % kAlign) != 0 || ws_bytes < p.total) return DART_ERR_WORKSPACE;
  c.status = status;
  const Gather a = {q, k_pool, static_cast<const uint8_t*>(k_scales), lse, weights, q_ld, scale, carry, causal != 0, 1.0 / (c.Hq / c.Hkv)};
  p.own.sums = p.pre.sums = static_cast<float*>(ws);  // (one launch after the other)
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (c.groups > 0) DART_TRY(launch_gather_kind(a, c, cache->dtype, p.pre, st));
  return launch_gather_kind(a, c, cache->dtype, p.own, st);
}

int32_t dart_evict_most(const dart_cache* cache, const dart_eviction* eviction, int32_t four_bit) {
  Cache c;
  EvictPlan p;
  if (make_cache(cache, c, four_bit ? 4 : 0) != DART_OK || plan_evict(c, eviction, p) != DART_OK) return -1;
  return p.most;
}

size_t dart_evict_workspace_bytes(const dart_cache* cache, const dart_eviction* eviction, int32_t four_bit) {
  Cache c;
  EvictPlan p;
  if (make_cache(cache, c, four_bit ? 4 : 0) != DART_OK || plan_evict(c, eviction, p) != DART_OK) return 0;
  return p.total;
}

dart_status dart_evict(const dart_cache* cache, const dart_eviction* eviction, void* k_pool, void* k_scales, void* v_pool, void* v_scales,
                       const float* weights, float* weights_out, int32_t* kept, int64_t kept_ld, int32_t* kv_len_out, void* ws,
                       size_t ws_bytes, int32_t* status, void* stream) {
  Cache c;
  EvictPlan p;
  if ((k_scales == nullptr) != (v_scales == nullptr)) return DART_ERR_NULL;
  const bool codes = k_scales != nullptr;
  DART_TRY(make_cache(cache, c, codes ? 4 : 0));
  DART_TRY(plan_evict(c, eviction, p));
  if (c.B == 0) return DART_OK;
  if (!k_pool || !v_pool || !weights || !kv_len_out) return DART_ERR_NULL;
  if (off16(k_pool) || off16(v_pool)) return DART_ERR_ALIGN;
  if (kept && (kept_ld < p.most || kept_ld > (int64_t)1 << 33)) return DART_ERR_SHAPE;
  if (!ws || (reinterpret_cast<uintptr_t>(ws) % kAlign) != 0 || ws_bytes < p.total) return DART_ERR_WORKSPACE;
  c.status = status;
  Evict a = {eviction->budget, eviction->ratio_num, std::max(eviction->ratio_den, 1), eviction->first, eviction->recent, weights,
             weights_out, kept ? kept : static_cast<int*>(ws), kept ? (long)kept_ld : (long)p.most,
             reinterpret_cast<int2*>(static_cast<unsigned char*>(ws) + p.left), kv_len_out};
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const long pairs = (long)c.B * c.Hkv;
  const dim3 heads((unsigned)std::min(pairs, 1L << 20));
  if (c.max_kv <= 1024) k_evict_select<4, 4><<<heads, dim3(256), 0, st>>>(a, c);
  else if (c.max_kv <= 4096) k_evict_select<16, 4><<<heads, dim3(1024), 0, st>>>(a, c);
  else k_evict_select<16, 16><<<heads, dim3(1024), 0, st>>>(a, c);
  DART_TRY(launched());

  Moves m = {};
  auto column = [&](const void* from, void* to, long div, long mul) {
    return Column{static_cast<unsigned char*>(const_cast<void*>(from)), static_cast<unsigned char*>(to), c.page_ld * mul / div,
                  c.head_ld * mul / div, c.row_ld * mul / div};
  };
  const int blocks = (c.d + 31) / 32, e = codes ? 1 : elem(cache->dtype);
  const long div = codes ? 2 : 1;
  const int row_bytes = codes ? blocks * 16 : c.d * e;
  add_rows(m, 0, column(k_pool, k_pool, div, e), row_bytes, 16, 8);
  add_rows(m, 1, column(v_pool, v_pool, div, e), row_bytes, 16, 8);
  const Column ks = column(k_scales, k_scales, 32, 1), vs = column(v_scales, v_scales, 32, 1);
  add_rows(m, 2, ks, codes ? blocks : 0, codes ? unit_of(ks, blocks) : 1, 8);
  add_rows(m, 3, vs, codes ? blocks : 0, codes ? unit_of(vs, blocks) : 1, 8);
  const long page = 1L << c.page_shift;
  const Column w = {reinterpret_cast<unsigned char*>(const_cast<float*>(weights)), reinterpret_cast<unsigned char*>(weights_out), 4 * page * c.Hkv,
                    4 * page, 4};
  add_rows(m, 4, w, weights_out ? 4 : 0, 4, 1);
  const long work = pairs * m.end[4];
  k_evict_move<<<dim3((unsigned)std::min(work, 1L << 20)), dim3(p.most <= 256 ? 256 : 1024), 0, st>>>(a, c, m);
  return launched();
}

}  // extern "C"
