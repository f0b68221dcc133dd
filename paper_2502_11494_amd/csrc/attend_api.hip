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

constexpr size_t kAlign = 256;
constexpr int64_t kMaxLd = int64_t(1) << 24;       // row strides of q, k, v and outputs, elements
constexpr int64_t kMaxPoolLd = int64_t(1) << 33;   // strides inside the pools, elements: 16-byte units fit 32 bits
constexpr int kMaxSequences = 1 << 20, kMaxTokens = 1 << 24, kMaxKeys = 1 << 27, kMaxPage = 1 << 20;
constexpr int kMaxHeads = 1024, kMaxHead = 256;
constexpr long kJoinSets = 1L << 15;  // sets of lanes of a join that fill the chip
constexpr long kMaxJoined = 1L << 24;  // (token, query head) pairs whose parts are joined
constexpr long kMaxRows = 1L << 28, kMaxBlocks = (1L << 23) - 1;  // (token, head) pairs of a key head; blocks of a launch

inline bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
inline int elem(int dtype) { return dtype == DART_BF16 ? 2 : 4; }

#define DART_TRY(expr)                    \
  do {                                    \
    dart_status _s = (expr);              \
    if (_s != DART_OK) return _s;         \
  } while (0)

dart_status launched() { return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP; }

dart_status check_heads(int Hq, int Hkv, int d, int dtype) {
  if (dtype != DART_F32 && dtype != DART_BF16) return DART_ERR_DTYPE;
  if (Hkv < 1 || Hq < Hkv || Hq > kMaxHeads || Hq % Hkv || d < 8 || d > kMaxHead || d % 8) return DART_ERR_SHAPE;
  return DART_OK;
}

// A tensor of rows of `width` elements.
dart_status check_rows(const void* p, int64_t ld, int64_t width, int dtype) {
  if (!p) return DART_ERR_NULL;
  if (ld < width || ld > kMaxLd) return DART_ERR_SHAPE;
  if (off16(p) || ld * elem(dtype) % 16) return DART_ERR_ALIGN;
  return DART_OK;
}

dart_status make_cache(const dart_cache* u, Cache& c) {
  if (!u) return DART_ERR_NULL;
  DART_TRY(check_heads(u->Hq, u->Hkv, u->d, u->dtype));
  if (u->B < 0 || u->B > kMaxSequences || u->T < 0 || u->T > kMaxTokens || u->max_q < 0 || u->max_kv < 0 ||
      u->max_kv > kMaxKeys || u->pages_ld < 1 || u->pages_n < 0 || u->n_pages < 1)
    return DART_ERR_SHAPE;
  if (u->page_size < 1 || u->page_size > kMaxPage || (u->page_size & (u->page_size - 1))) return DART_ERR_SHAPE;
  if (u->row_ld < u->d || u->row_ld > kMaxPoolLd || u->head_ld < 0 || u->head_ld > kMaxPoolLd || u->page_ld < 0 ||
      u->page_ld > kMaxPoolLd)
    return DART_ERR_SHAPE;
  if (u->groups < 0 || u->groups > u->B) return DART_ERR_SHAPE;
  if (!u->cu_q && u->T != u->B) return DART_ERR_SHAPE;
  const int64_t a16 = 16 / elem(u->dtype);
  if (u->row_ld % a16 || u->head_ld % a16 || u->page_ld % a16) return DART_ERR_ALIGN;
  c = {};
  c.B = u->B;
  c.Hq = u->Hq;
  c.Hkv = u->Hkv;
  c.d = u->d;
  c.T = u->T;
  c.max_q = u->cu_q ? std::min(u->max_q, u->T) : 1;
  c.max_kv = u->max_kv;
  c.cu = u->cu_q;
  c.kv_len = u->kv_len;
  c.pages = u->pages;
  c.pages_ld = u->pages_ld;
  c.pages_n = u->pages_n ? u->pages_n : u->pages_ld;
  c.n_pages = u->n_pages;
  c.page_shift = __builtin_ctz((unsigned)u->page_size);
  c.page_ld = u->page_ld;
  c.head_ld = u->head_ld;
  c.row_ld = u->row_ld;
  c.page_16 = (uint32_t)(u->page_ld / a16);
  c.row_16 = (uint32_t)(u->row_ld / a16);
  c.groups = u->groups;
  if (u->groups > 0) {
    if (u->max_prefix < 0 || u->max_prefix > kMaxKeys || u->prefix_ld < 1 || u->prefix_n < 0) return DART_ERR_SHAPE;
    if (!u->group_cu || !u->prefix_pages || !u->prefix_len) return DART_ERR_NULL;
    c.max_prefix = u->max_prefix;
    c.prefix_ld = u->prefix_ld;
    c.prefix_n = u->prefix_n ? u->prefix_n : u->prefix_ld;
    c.group_cu = u->group_cu;
    c.prefix_pages = u->prefix_pages;
    c.prefix_len = u->prefix_len;
  }
  if (u->B > 0 && (!u->kv_len || !u->pages)) return DART_ERR_NULL;
  return DART_OK;
}

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

// ---- attention: which tiles, how many parts ---------------------------------------------------
enum Kind { kFew, kMany, kWide };  // 16 rows, the keys dealt to four waves; four waves of rows; eight

struct AttendPlan {
  Kind own_kind, pre_kind;
  Parting own, pre;
  bool both;  // one launch takes the prefixes and the own keys
  int parts;
  size_t o_ml, total;
};

int rows_of(Kind k, int dtype, int d) { return k == kFew ? 16 : k == kWide ? 256 : 4 * many_columns(dtype == DART_BF16 ? kBF16 : kF32, d); }
long blocks_of(const Cache& c, const Parting& p) { return p.slots * c.Hkv * p.chunks; }

// rows: (token, head) pairs of a sequence at most, of a group on average (nothing on the host says how many sequences the
// largest has); owners: how many of them.  Uneven groups read their prefix in smaller tiles than they could: 64 answers of 32 heads
// over four prefixes of 2880 53 us with 16 sequences to each, 65 with 61, 1, 1 and 1.  max_keys: the caller's bound, which
// divides the keys, whatever the lengths are: one token over 2000 keys, 28 + 4 heads, 12.4 us, 27 with a bound of 131 072; 32 of
// them 28 and 44.
Kind plan_parting(const Cache& c, int dtype, bool prefix, long rows, int owners, int max_keys, Parting& p) {
  const int r = c.Hq / c.Hkv;
  // 256-row tiles take the least from LDS and caches per row, but each has a compute unit to itself, so that nothing
  // hides its start and end: they pay from 1024 keys and 1.5 tiles to a unit on.  28 + 4 heads, causal, 128- and
  // 256-row tiles: two sequences of 9216 1347 and 1258 us, one of 4096 159 and 136, one of 3600 124 and 116, one of 2048
  // 58 and 66; 24 of 1000 291 and 283, 16 of 600 91 and 95.
  const bool wide = dtype == DART_BF16 && c.d <= 128 && rows > 128 && max_keys >= 1024 && (long)c.T * r / 256 * c.Hkv >= 384;
  // 16-row tiles with the keys dealt to four waves end sooner while the chip is not full (256 units of 384 keys):
  // one sequence of 9 tokens over 300 keys, 28 + 4 heads, 11.7 us and 14.1 in 128-row tiles, over 3000 keys 13.4 and 16.2;
  // 32 such sequences 89 and 63.  Up to 16 rows nothing is gained by reading for more.
  const long few = std::min((long)c.T * r / 16 + owners, (long)owners * ((rows + 15) / 16)) * c.Hkv;
  Kind kind = rows <= 16 || (rows <= 64 && few * max_keys <= 256 * 384) ? kFew : wide ? kWide : kMany;
  if (dtype == DART_F32 && c.d > 128) kind = kMany;
  const int bm = rows_of(kind, dtype, c.d);
  p = {};
  p.prefix = prefix;
  p.few = kind == kFew;
  if (!prefix && !c.cu) {
    p.per_owner = (r + bm - 1) / bm;
    p.slots = (long)owners * p.per_owner;
  } else {
    p.slots = (long)c.T * r / bm + owners;
  }
  const long blocks = std::max(1L, std::min(p.slots, (long)owners * ((rows + bm - 1) / bm)) * c.Hkv);
  // Parts until every compute unit has a block, of 256 keys at least; more cost their start (7 us a round) and the
  // join: 64 rows of 28 + 4 heads over 8000 keys 197 us in one part, 40 in 128 blocks, 31 in 256, 33 in 512, 46 in
  // 1024; 64 answers over one prefix of 9216 229, 43, 34, 42 and 48.  32-bit tiles of four waves are bound by the
  // matrix cores' latency and want company: 637 causal tokens of 32 heads 69 us in 320 blocks, 58 in 960.
  const long want = std::max(1L, (dtype == DART_F32 && kind == kMany ? 1024 : 256) / blocks);
  const long chunk = std::max(256L, ((max_keys + want - 1) / want + 255) / 256 * 256);
  p.chunk = (int)chunk;
  p.chunks = std::max(1, (int)((max_keys + chunk - 1) / chunk));
  return kind;
}

dart_status plan_attend(const Cache& c, int dtype, AttendPlan& p) {
  const int r = c.Hq / c.Hkv;
  if ((long)c.T * r > kMaxRows) return DART_ERR_SHAPE;
  p = {};
  p.own_kind = plan_parting(c, dtype, false, (long)c.max_q * r, c.B, c.max_kv, p.own);
  p.parts = p.own.chunks;
  if (c.groups > 0) {
    const long rows = std::min((long)c.T, (long)c.max_q * c.B) * r;
    p.pre_kind = plan_parting(c, dtype, true, std::max(1L, (rows + c.groups - 1) / c.groups), c.groups, c.max_prefix, p.pre);
    p.parts += p.pre.chunks;
    p.own.first_part = p.pre.chunks;
    // One launch for both: 64 answers over a prefix of 9216 keys, 28 + 4 heads, 33 us and 44 in two, 32 prompts over four of 2880
    // 126 and 143.  With 32-bit rows it takes the registers of two blocks, which costs more than a launch where there are
    // blocks enough: 16 answers over two prefixes of 3000, 64 + 8 heads (320 blocks), 50 and 69; those 64 answers (1264) 149 and 129.
    p.both = p.own_kind != kWide && p.pre_kind != kWide && blocks_of(c, p.own) + blocks_of(c, p.pre) <= kMaxBlocks &&
             (dtype == DART_BF16 || (c.d <= 128 && blocks_of(c, p.own) + blocks_of(c, p.pre) <= 1024));
  }
  if (p.parts > 1 && (long)c.T * c.Hq > kMaxJoined) return DART_ERR_SHAPE;
  p.own.parts = p.pre.parts = p.parts;
  auto up = [](size_t v) { return (v + kAlign - 1) / kAlign * kAlign; };
  const size_t rows = (size_t)c.T * c.Hq;
  p.total = kAlign;
  if (p.parts > 1) {
    p.o_ml = up((size_t)p.parts * rows * c.d * 4);
    p.total = p.o_ml + up((size_t)p.parts * rows * 8);
  }
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
  int lanes_shift = 0, split_shift = 0;
  while ((4 << lanes_shift) < c.d) ++lanes_shift;
  // many parts of few rows are shared by up to a block's sets of lanes, four parts at least to each
  while (split_shift < 8 - lanes_shift && (4 << split_shift) < p.parts && ((long)c.T * c.Hq << split_shift) < kJoinSets) ++split_shift;
  const int rows_shift = 8 - lanes_shift - split_shift;
  const long blocks = (((long)c.T * c.Hq - 1) >> rows_shift) + 1;
  if (bf16)
    k_attend_join<kBF16><<<dim3((unsigned)blocks), dim3(256), 0, st>>>(a, c, p.pre.chunk, p.pre.chunks, p.own.chunk, part_o, part_ml,
                                                                      lanes_shift, split_shift);
  else
    k_attend_join<kF32><<<dim3((unsigned)blocks), dim3(256), 0, st>>>(a, c, p.pre.chunk, p.pre.chunks, p.own.chunk, part_o, part_ml,
                                                                     lanes_shift, split_shift);
  return launched();
}

}  // extern "C"
