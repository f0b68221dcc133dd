// The paged cache as kernels see it, and the checks every one of them makes the same way.
#pragma once

#include <algorithm>

#include "../../include/dart.h"
#include "common.hpp"

namespace dart {

enum { kBadSequence = 1, kBadPage = 2 };  // bits of the caller's status word

struct Cache {
  int B, Hq, Hkv, d, T, max_q, max_kv;
  const int *cu, *kv_len, *pages;
  int pages_ld, pages_n, n_pages, page_shift;  // pages_n: entries of a row of the table
  long page_ld, head_ld, row_ld;  // elements
  uint32_t page_16, row_16;       // the same strides in units of 16 bytes
  int groups, max_prefix, prefix_ld, prefix_n;
  const int *group_cu, *prefix_pages, *prefix_len;
  int* status;
};

__device__ __forceinline__ void flag(const Cache& c, int bit) {
  if (c.status != nullptr) atomicOr(c.status, bit);
}

// The last of count offsets that is at most v, 0 if none is: last_at_most for offsets that nothing has
// checked yet (any index it gives is one of theirs).
__device__ __forceinline__ int owner_of(const int* offset, int count, int v) {
  const int lane = threadIdx.x & 63;
  int from = 0, left = count;
  while (true) {
    const int stride = (left + kWave - 1) / kWave, d = lane * stride;
    const unsigned long long low = __ballot(d < left && offset[from + (d < left ? d : 0)] <= v);
    const int skip = (low ? 63 - __builtin_clzll(low) : 0) * stride;
    from += skip;
    if (stride == 1) return __builtin_amdgcn_readfirstlane(from);
    left = left - skip < stride ? left - skip : stride;
  }
}

// The tokens and keys of one sequence; valid: its offsets and lengths are as they have to be.  Of a
// sequence that is not, [tok0, tok0 + n) are those of its tokens that are tokens of the call.
struct Seq {
  int tok0, n, kv;
  bool valid;
};

__device__ __forceinline__ Seq make_sequence(const Cache& c, int lo, int hi, int kv) {
  Seq s;
  s.valid = lo >= 0 && hi >= lo && hi <= c.T && hi - lo <= c.max_q;
  s.tok0 = lo < 0 ? 0 : lo < c.T ? lo : c.T;
  const int end = hi < 0 ? 0 : hi < c.T ? hi : c.T;
  s.n = end > s.tok0 ? end - s.tok0 : 0;
  s.kv = kv;
  if (kv < 0 || kv > c.max_kv || (long)kv > ((long)c.pages_n << c.page_shift)) s.valid = false;
  if (!s.valid) s.kv = 0;
  return s;
}

__device__ __forceinline__ Seq sequence_of(const Cache& c, int b) {
  const bool one = c.cu == nullptr;  // a token each
  return make_sequence(c, one ? b : c.cu[b], one ? b + 1 : c.cu[b + 1], c.kv_len[b]);
}

// Keys of a group's prefix; -1 if its length or its sequences are not as they have to be.
__device__ __forceinline__ int make_prefix(const Cache& c, int b0, int b1, int n) {
  if (n < 0 || n > c.max_prefix || (long)n > ((long)c.prefix_n << c.page_shift) || b0 < 0 || b1 < b0 || b1 > c.B)
    return -1;
  return n;
}

__device__ __forceinline__ int prefix_of(const Cache& c, int g) {
  return make_prefix(c, c.group_cu[g], c.group_cu[g + 1], c.prefix_len[g]);
}

// The offset of row `key` of a page table's keys, in elements; of page 0 if its page is none.
__device__ __forceinline__ long key_offset(const Cache& c, const int* table, int key, bool& bad) {
  const int page = table[key >> c.page_shift];
  bad = (unsigned)page >= (unsigned)c.n_pages;
  return (bad ? 0L : (long)page * c.page_ld) + (long)(key & ((1 << c.page_shift) - 1)) * c.row_ld;
}

// ---- host: limits and checks of descriptors and tensors ------------------------------------
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

inline dart_status launched() { return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP; }

inline dart_status check_heads(int Hq, int Hkv, int d, int dtype) {
  if (dtype != DART_F32 && dtype != DART_BF16) return DART_ERR_DTYPE;
  if (Hkv < 1 || Hq < Hkv || Hq > kMaxHeads || Hq % Hkv || d < 8 || d > kMaxHead || d % 8) return DART_ERR_SHAPE;
  return DART_OK;
}

// A tensor of rows of `width` elements.
inline dart_status check_rows(const void* p, int64_t ld, int64_t width, int dtype) {
  if (!p) return DART_ERR_NULL;
  if (ld < width || ld > kMaxLd) return DART_ERR_SHAPE;
  if (off16(p) || ld * elem(dtype) % 16) return DART_ERR_ALIGN;
  return DART_OK;
}

// bits: 4 where the pools are held in 4 bits, in whole blocks of 32 values; otherwise their rows are of u->dtype.
inline dart_status make_cache(const dart_cache* u, Cache& c, int bits = 0) {
  if (!u) return DART_ERR_NULL;
  DART_TRY(check_heads(u->Hq, u->Hkv, u->d, u->dtype));
  if (u->B < 0 || u->B > kMaxSequences || u->T < 0 || u->T > kMaxTokens || u->max_q < 0 || u->max_kv < 0 ||
      u->max_kv > kMaxKeys || u->pages_ld < 1 || u->pages_n < 0 || u->n_pages < 1)
    return DART_ERR_SHAPE;
  if (u->page_size < 1 || u->page_size > kMaxPage || (u->page_size & (u->page_size - 1))) return DART_ERR_SHAPE;
  if (u->row_ld < (bits == 4 ? (u->d + 31) / 32 * 32 : u->d) || u->row_ld > kMaxPoolLd || u->head_ld < 0 || u->head_ld > kMaxPoolLd || u->page_ld < 0 ||
      u->page_ld > kMaxPoolLd)
    return DART_ERR_SHAPE;
  if (u->groups < 0 || u->groups > u->B) return DART_ERR_SHAPE;
  if (!u->cu_q && u->T != u->B) return DART_ERR_SHAPE;
  const int64_t a16 = bits == 4 ? 32 : 16 / elem(u->dtype);
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

}  // namespace dart
