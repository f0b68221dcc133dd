// The paged cache as kernels see it, and the checks every one of them makes the same way.
#pragma once

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

}  // namespace dart
