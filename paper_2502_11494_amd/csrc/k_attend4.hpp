// Attention over pages held in 4 bits.
#pragma once

#include "fourbit.hpp"
#include "k_attend.hpp"

namespace dart {

// The tiles of attention over rows, keys and values brought to the rows' type on their way to LDS, or of few rows the keys on their way to
// the products.  Many rows are bound by what is not a product, as over rows (2304 tokens after 6912, two sequences, 28 + 4 heads: 506 us,
// 1.03 PF/s); single tokens by memory (32 over 8000 keys each 36 us with the join, 4.8 TB/s at most, ragged ones 4.0).
template <int DT, int DP, int QW, int WM, int WK, int KT, class HELD>
__global__ __launch_bounds__(64 * WM * WK, HELD::kPages && DT == kBF16 ? 3 : DP <= 128 && (DT == kBF16 || WK == 1) ? 2 : 1) void k_attend_4bit(Attend a, Scales scales, Cache c, Parting sp) {
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ AttendShared sh;
  long slot;
  int head, part;
  attend_place(c, sp, blockIdx.x, slot, head, part);
  if (HELD::kPages && sp.share != 0) {  // (the parts that no sequence has come last)
    const unsigned rows = (unsigned)sp.slots * (unsigned)c.Hkv, rest = blockIdx.x % rows;
    part = (int)(blockIdx.x / rows);
    head = (int)(rest % (unsigned)c.Hkv);
    slot = (long)(rest / (unsigned)c.Hkv);
  }
  attend_tile<DT, DP, QW, WM, WK, KT, HELD>(a, c, sp, lds, sh, slot, head, part, scales);
}

// Prefixes and own keys in one launch (64 answers over one prefix of 9216, 28 + 4 heads: 24 us and 7 for the join, the steps of a
// block one after the other).
template <int DT, int DP, int KT>
__global__ __launch_bounds__(256, DT == kBF16 && DP <= 128 ? 2 : 1) void k_attend_4bit_both(Attend a, Scales scales, Cache c, Parting pre, Parting own,
                                                                                            unsigned pre_blocks) {
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ AttendShared sh;
  const bool first = blockIdx.x < pre_blocks;
  const Parting sp = first ? pre : own;
  long slot;
  int head, part;
  attend_place(c, sp, first ? blockIdx.x : blockIdx.x - pre_blocks, slot, head, part);
  if (sp.few) attend_tile<DT, DP, 16, 1, 4, 32, In4Bits>(a, c, sp, lds, sh, slot, head, part, scales);
  else attend_tile<DT, DP, many_columns(DT, DP), 4, 1, KT, In4Bits>(a, c, sp, lds, sh, slot, head, part, scales);
}

}  // namespace dart
