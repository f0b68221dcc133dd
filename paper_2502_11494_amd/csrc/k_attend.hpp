// Attention over the paged cache: tiles of query rows against tiles of keys on the matrix cores.
#pragma once

#include "cache.hpp"
#include "k_rotate.hpp"

namespace dart {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
// The running maximum before any score: finite, so that a hidden score's -infinity less it is -infinity
// and no NaN, and no larger than any score.
constexpr float kLowest = -3.402823466e38f;
// References from here on are coarse: their spacing is 2^-9 and more.  A score's fused distance from one carries the
// reference's own rounding, the same for all keys of a row, which the sum of weights takes out again as long as it is small: a
// largest score of 2^32 could weigh anything from 2^-128 to 2^128.  Products rounded like the reference itself do not.
constexpr float kCoarse = 0x1p14f;

struct Attend {
  const void *q, *k_pool, *v_pool;
  void* out;
  float* lse;  // or nullptr
  long q_ld, out_ld;
  float scale;
  int causal;
  double per_token;  // 1 / (rows of a token: query heads of a key head)
};

// row / rows of a token, exactly: rows are below 2^28.
__device__ __forceinline__ int token_in(const Attend& a, int row) { return (int)(((double)row + 0.5) * a.per_token); }

// How the keys of a launch are divided, and where its results go.  A row's results are joined from
// `parts` partial ones (running sum, maximum and weighted values of some of its keys each), or written
// at once where there is one.
struct Parting {
  int prefix;      // the keys are the groups' shared prefixes (else each sequence's own)
  int few;         // tiles of 16 rows, the keys dealt to four waves (else four waves of rows)
  int chunk;       // keys of a part
  int chunks;
  int first_part;  // part number of the first chunk
  int parts;
  int per_owner;   // tiles of a sequence where each has one token; 0: see slot_owner
  long slots;      // row tiles
  float* part_o;   // [parts][T*Hq][d]
  float2* part_ml; // [parts][T*Hq]: maximum (of scores times log2 e), sum
};

// ---- the arithmetic of a wave ----------------------------------------------------------------
// QW queries (32, or 16 where a block has no more) lie in the columns of a matrix tile, lane % QW, and its
// keys in the rows, so that each of the kGroups groups of QW lanes holds, of every query, one run of four
// keys in 4 * kGroups.  The maximum and the sum of a query are then within a lane but for an exchange
// between the groups; the weights are, rounded, the right operand of the second product as they
// stand (its sum over keys does not mind their order, as long as the values are read in the same one),
// and its result has the queries in the columns again, so that rescaling it is a product by a number
// of the lane's own.
template <int QW>
struct Acc { typedef f32x16 type; };
template <>
struct Acc<16> { typedef f32x4v type; };

template <int DT, int QW>
struct Math {
  typedef typename Acc<QW>::type acc;
  static constexpr int kVec = DT == kBF16 ? 8 : 4;           // elements of a 16-byte piece
  static constexpr int kGroups = 64 / QW, kRegs = QW * QW / 64;
  static constexpr int kScores = QW / 2;                     // of a lane, for 32 keys
  static constexpr int kTiles = 32 / QW;                     // of 32 keys
  static constexpr int kRun = 4 * kGroups;
  // what score (or row of a result tile) number u of a lane of group g is of
  __device__ static __forceinline__ constexpr int place(int u, int g) { return kRun * (u / 4) + 4 * g + u % 4; }
  // key and query pieces of step s: number kGroups * s + g of the row
  template <int DP>
  static constexpr int steps() { return DP / (kVec * kGroups); }
  __device__ static __forceinline__ acc qk(const u32x4& k, const u32x4& q, acc c) {
    if constexpr (DT == kBF16) {
      const bf16x8 x = __builtin_bit_cast(bf16x8, k), y = __builtin_bit_cast(bf16x8, q);
      if constexpr (QW == 32) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
      else c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) c = av(__uint_as_float(k[j]), __uint_as_float(q[j]), c);
    }
    return c;
  }
  // (32-bit rows, 16 columns) one key of each group by one weight of each group
  __device__ static __forceinline__ acc av(float v, float p, acc c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(v, p, c, 0, 0, 0); }
  __device__ static __forceinline__ acc pv(const u32x4& v, const u32x4& p, acc c) { return qk(v, p, c); }
};

// Rows of a tile in LDS lie at multiples of their length, their 16-byte pieces permuted by the row
// so that neither 16 rows read at one piece (keys) nor 4 rows read at four (values) meet in the
// banks.
template <int RB>
__device__ __forceinline__ int mix(int row) {
  return RB == 128 ? (((row >> 1) & 1) << 2) | ((row >> 2) & 3) : ((row & 3) << 2) | ((row >> 2) & 3);
}

// Over the lanes that hold the same query.
template <int QW>
__device__ __forceinline__ float groups_max(float x) {
  if constexpr (QW == 16) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <int QW>
__device__ __forceinline__ float groups_sum(float x) {
  if constexpr (QW == 16) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Between the lanes' stores to their wave's tiles and its reads of them, and between those and the next stores: LDS takes a
// wave's accesses in order, so that only the compiler has to be held to it.
__device__ __forceinline__ void tiles_handed_over() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
}

// Rounded by itself, not fused with a sum it is in.
__device__ __forceinline__ float product(float x, float y) {
#pragma clang fp contract(off)
  return x * y;
}

// Puts 0 in the place of infinities and NaN; not 0 if there were any.  (An exponent of ones carries into
// the bit above it.)
template <int DT>
__device__ __forceinline__ uint32_t drop_infinities(u32x4& v) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t hi = ((v[i] & 0x7f800000u) + 0x00800000u) >> 31;
    const uint32_t lo = DT == kBF16 ? ((v[i] & 0x7f80u) + 0x80u) >> 15 : 0u;
    any |= hi | lo;
    v[i] &= DT == kBF16 ? ~((0u - hi) << 16 | ((0u - lo) >> 16)) : ~(0u - hi);
  }
  return any;
}

__device__ __forceinline__ int token_of(const Cache& c, int b) {
  if (c.cu == nullptr) return b < c.B ? b : c.B;
  const int t = c.cu[b];
  return t < 0 ? 0 : t < c.T ? t : c.T;
}

// Tile slot -> sequence (or group).  Sequence i of `count` owns the slots from floor(first token * r /
// BM) + i on: at least as many as it has tiles, whatever its length, and found without a sum over the
// sequences before it.
template <int BM>
__device__ __forceinline__ int slot_owner(const Cache& c, const int* group_cu, int count, int r, long slot) {
  if (count == 1) return 0;
  const int lane = threadIdx.x & 63;
  int from = 0, left = count;
  while (true) {
    const int stride = (left + kWave - 1) / kWave, d = lane * stride;
    const int i = from + (d < left ? d : 0);
    const int b = group_cu ? group_cu[i] : i;
    const long start = (long)token_of(c, b < 0 ? 0 : b < c.B ? b : c.B) * r / BM + i;
    const unsigned long long low = __ballot(d < left && start <= slot);
    const int skip = (low ? 63 - __builtin_clzll(low) : 0) * stride;
    from += skip;
    if (stride == 1) return __builtin_amdgcn_readfirstlane(from);
    left = left - skip < stride ? left - skip : stride;
  }
}

// WM waves along the rows, QW each, by WK along the keys; a step takes KT keys per key group.
template <int DT, int DP, int QW, int WM, int WK, int KT>
struct AttendShape {
  static constexpr int kEsz = DT == kBF16 ? 2 : 4;
  static constexpr int kRowBytes = DP * kEsz;
  static constexpr int kPieces = kRowBytes / 16;
  static constexpr int kThreads = 64 * WM * WK;
  static constexpr int kGroup = 64 * WM;                 // threads that stage a key group's tiles
  static constexpr int kLoads = KT * kPieces / kGroup;   // pieces of keys (and of values) per thread
  static constexpr int kApart = kGroup / kPieces;        // rows between a thread's pieces
  static constexpr int kBuffers = WM > 1 ? 2 : 1;
  static constexpr int kTileBytes = KT * kRowBytes;
  static constexpr int kBM = QW * WM;
  static constexpr int kLds = WK * kBuffers * 2 * kTileBytes;
  static_assert(kGroup % kPieces == 0 && KT * kPieces % kGroup == 0 && KT % 32 == 0, "");
  static_assert(WK == 1 || WM == 1, "");
  static_assert(WK == 1 || QW * DP * 4 <= kBuffers * 2 * kTileBytes, "joined in the tiles' place");
};

// Columns of a wave's tile where four waves take the rows: 32 halve what LDS has to deliver per product, but with
// 32-bit rows the matrix cores are what counts, and with heads over 128 the registers are.
constexpr int many_columns(int dt, int d) { return dt == kBF16 && d <= 128 ? 32 : 16; }

// What a block keeps in LDS beside the tiles.
struct AttendShared {
  int odd_values[4];
  float2 joined[5][32];
};

// out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m) with s = scale * K q, in one pass over the keys: a step takes a tile
// of keys, S^T = K Q^T, moves the running maximum m if it has to (out and sum rescaled), and adds exp(S^T - m) and
// V^T exp(S^T - m).  Exponentials are powers of 2; scores, maximum, sum and result are in 32 bits, the weights of bf16
// rows are rounded to bf16 for their product.  A thread's share of the next step's keys and values is on its way in
// registers while this one's lies in LDS; with four or eight waves of rows LDS holds two steps, so that one barrier a
// step is enough; where the waves share out the keys each has its own tiles and there is none.
// What bounds it: many rows, the instructions of a step that are not matrix products (two causal sequences of 9216,
// 28 + 4 heads of 128, 1.26 ms, 0.97 PF/s of the 1.37 of a large product: the matrix cores are busy 44 % of the time, the
// vector units 52 %, and the two overlap little; no bank conflicts; 64 queries to a wave spill, two waves half a step apart
// or other orders of a step gain nothing); one token each, memory (32 answers over 1024 to 16 384 keys: 122 us, 4.66 TB/s
// where a large copy moves 4.79); a few rows over a few keys, latency (131 keys: 8 us, of which 1.3 for each step of 128);
// 32-bit rows, the matrix cores' rate (637 causal tokens of 32 heads 55 us with the join's 8,
// the matrix cores busy for 22; 4096 tokens of 28 + 4 heads 1.07 ms, 112 TFLOP/s of the 153 of a large product).
// One block: row tile `slot` against chunk `part` of the keys of head `head`.
template <int DT, int DP, int QW, int WM, int WK, int KT>
__device__ __forceinline__ void attend_tile(const Attend& a, const Cache& c, const Parting& sp, unsigned char* lds, AttendShared& sh,
                                            long slot, int head, int part) {
  typedef AttendShape<DT, DP, QW, WM, WK, KT> S;
  typedef Math<DT, QW> M;
  typedef typename M::acc acc;
  constexpr int kSteps = M::template steps<DP>(), kDT = DP / QW, kSub = KT / 32, RB = S::kRowBytes;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave % WM, wk = wave / WM;
  const int grp = lane / QW, col = lane % QW;
  const int r = c.Hq / c.Hkv;

  // ---- whose rows (token-major pairs of a token and a head of the key head's group), which keys
  int tok0, n, kv, tile;
  const int* table;
  if (sp.prefix) {
    const int g = slot_owner<S::kBM>(c, c.group_cu, c.groups, r, slot);
    const int b0 = c.group_cu[g], b1 = c.group_cu[g + 1];
    const int keys = prefix_of(c, g);
    if (keys < 0 && threadIdx.x == 0) flag(c, kBadSequence);
    tok0 = token_of(c, b0 < 0 ? 0 : b0 < c.B ? b0 : c.B);
    n = keys >= 0 ? token_of(c, b1) - tok0 : 0;
    kv = keys >= 0 ? keys : 0;
    table = c.prefix_pages + (long)g * c.prefix_ld;
    tile = (int)(slot - ((long)tok0 * r / S::kBM + g));
  } else {
    int b;
    Seq s;
    if (sp.per_owner) {
      b = (int)slot / sp.per_owner;
      s = sequence_of(c, b);
    } else if (c.B <= kWave) {  // (all sequences in one look: the loads do not wait for one another)
      const int i = lane < c.B ? lane : c.B - 1, lo = c.cu[i], hi = c.cu[i + 1], keys = c.kv_len[i];
      const unsigned long long low =
          __ballot(lane < c.B && (long)(lo < 0 ? 0 : lo < c.T ? lo : c.T) * r / S::kBM + lane <= slot);
      b = low ? 63 - __builtin_clzll(low) : 0;
      s = make_sequence(c, __builtin_amdgcn_readlane(lo, b), __builtin_amdgcn_readlane(hi, b), __builtin_amdgcn_readlane(keys, b));
    } else {
      b = slot_owner<S::kBM>(c, nullptr, c.B, r, slot);
      s = sequence_of(c, b);
    }
    if (!s.valid && threadIdx.x == 0) flag(c, kBadSequence);
    tok0 = s.tok0;
    n = s.n;
    kv = s.kv;
    table = c.pages + (long)b * c.pages_ld;
    tile = sp.per_owner ? (int)slot % sp.per_owner : (int)(slot - ((long)tok0 * r / S::kBM + b));
  }
  const int rows = n > 0 ? n * r : 0, row0 = tile * S::kBM;
  if (tile < 0 || row0 >= rows) return;
  const bool causal = a.causal && !sp.prefix;
  int k1 = kv;
  if (causal) k1 = min(kv, kv - n + token_in(a, min(row0 + S::kBM, rows) - 1) + 1);
  const int k0 = part * sp.chunk;
  k1 = min(k1, k0 + sp.chunk);
  if (k1 <= k0 && (sp.parts > 1 || part > 0)) return;

  // ---- staging: pieces of keys and values, through registers into LDS.  Loads are unconditional: what lies
  // past the keys (or the head) is read again from the last of them, and put right as it goes to LDS.
  const int gt = threadIdx.x - wk * S::kGroup;
  const int my_row = gt / S::kPieces, my_piece = gt % S::kPieces;
  const bool my_on = my_piece * M::kVec < c.d;
  const long piece_at = ((long)head * c.head_ld + (my_on ? my_piece * M::kVec : 0)) * S::kEsz;
  const unsigned char* kp = static_cast<const unsigned char*>(a.k_pool) + piece_at;
  const unsigned char* vp = static_cast<const unsigned char*>(a.v_pool) + piece_at;
  unsigned char* const my_lds = lds + wk * (S::kBuffers * 2 * S::kTileBytes);
  const int row_mask = (1 << c.page_shift) - 1, last_key = k1 - 1;
  u32x4 kr[S::kLoads], vr[S::kLoads];
  int pg[S::kLoads];
  bool bad_page = false;
  auto load_pages = [&](int kb) {
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) pg[i] = table[min(kb + my_row + i * S::kApart, last_key) >> c.page_shift];
  };
  // (page offsets by 32-bit products: the wider ones cost as much as a fifth of a step's exponentials)
  auto place_of = [&](int i, int kb) {
    int page = pg[i];
    if ((unsigned)page >= (unsigned)c.n_pages) page = 0, bad_page = true;
    const uint32_t row = min(kb + my_row + i * S::kApart, last_key) & row_mask;
    return ((uint64_t)(uint32_t)page * c.page_16 + (uint64_t)row * c.row_16) << 4;
  };
  auto load_tile = [&](int kb) {
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const uint64_t off = place_of(i, kb);
      kr[i] = *reinterpret_cast<const u32x4*>(kp + off);
      vr[i] = *reinterpret_cast<const u32x4*>(vp + off);
    }
  };
  const int steps = (k1 - k0 + KT * WK - 1) / (KT * WK);
  const int kstep = KT * WK, kfirst = k0 + wk * KT;
  if (steps > 0) load_pages(kfirst);

  // ---- this lane's query: the last key it sees, and its pieces
  const int my = row0 + wm * QW + col;
  const bool in = my < rows;
  const int mine = in ? my : rows - 1, my_tok = token_in(a, mine);
  const int qh = head * r + mine - my_tok * r;
  const int lim = causal ? min(kv - n + my_tok, last_key) : last_key;
  const uint32_t flip = a.scale < 0.f ? (DT == kBF16 ? 0x80008000u : 0x80000000u) : 0u;  // (scores then scale by |scale|)
  const unsigned char* q_at =
      static_cast<const unsigned char*>(a.q) + ((long)(tok0 + my_tok) * a.q_ld + (long)qh * c.d) * S::kEsz;
  u32x4 q[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int e = (M::kGroups * s + grp) * M::kVec;
    u32x4 v = *reinterpret_cast<const u32x4*>(q_at + (e < c.d ? e : 0) * S::kEsz);
    // (scale 0: queries of zeros, so that a hidden score stays -infinity)
    v = e < c.d && a.scale != 0.f ? v ^ flip : u32x4{0, 0, 0, 0};
    q[s] = v;
  }
  const float scale2 = a.scale != 0.f ? fabsf(a.scale) * kLog2e : 1.f;
  const int lim_first = __builtin_amdgcn_readfirstlane(lim);                              // of the wave's rows
  const int lim_last = row0 + wm * QW < rows ? __builtin_amdgcn_readlane(lim, 63) : -1;   // (none: no key)
  const int lim_block = causal ? min(kv - n + token_in(a, row0), last_key) : last_key;    // of the block's

  auto store_keys = [&](unsigned char* to) {
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const int row = my_row + i * S::kApart;
      *reinterpret_cast<u32x4*>(to + row * RB + ((my_piece ^ mix<RB>(row)) << 4)) = my_on ? kr[i] : u32x4{0, 0, 0, 0};
    }
  };
  auto store_values = [&](unsigned char* to, int kb) {
    if (kb + KT > k1) {
      // What lies behind the keys may be anything; its weight is 0, and 0 times NaN is NaN.
#pragma unroll
      for (int i = 0; i < S::kLoads; ++i)
        if (kb + my_row + i * S::kApart >= k1) vr[i] = u32x4{0, 0, 0, 0};
    }
    if (kb + KT - 1 > lim_block && causal) {
      // Some row does not see some of these keys.  Their weight is 0 there, but its product with a value
      // that is no number would be none either: such values are left out here and added at the end.
      uint32_t odd = 0;
#pragma unroll
      for (int i = 0; i < S::kLoads; ++i) odd |= drop_infinities<DT>(vr[i]);
      if (odd) sh.odd_values[wk] = 1;
    }
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const int row = my_row + i * S::kApart;
      *reinterpret_cast<u32x4*>(to + row * RB + ((my_piece ^ mix<RB>(row)) << 4)) = vr[i];
    }
  };

  // This lane's share of its query's result, four elements of the head at a time: quad number x is elements
  // quad_at(x) .. + 3.
  acc o[kDT];
  constexpr int kQuads = kDT * M::kRegs / 4;
  auto quad_at = [&](int x) {
    if (DT == kBF16) return x / (M::kRegs / 4) * QW + M::place(4 * (x % (M::kRegs / 4)), grp);
    return 4 * (x / M::kRegs * QW + M::place(x % M::kRegs, grp));
  };
  auto quad = [&](int x) {
    f32x4v v;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      v[k] = DT == kBF16 ? o[x / (M::kRegs / 4)][4 * (x % (M::kRegs / 4)) + k] : o[(4 * (x / M::kRegs) + k) % kDT][x % M::kRegs];
    return v;
  };
  float m = kLowest, l = 0.f;
  // The weights are 2^(score * scale2 - less).  A row whose maximum is over `above` goes through the branch that moves its
  // reference m; one whose reference is coarse does at every step, and has its scores replaced by their distances from m there.
  float above = kLowest, less = kLowest;
  const float back = 1.f / scale2;
#pragma unroll
  for (int i = 0; i < kDT; ++i) o[i] = acc{};
  // (all of a wave's lanes, without a branch: kernels short of registers park some in accumulation registers about here, and the
  // compiler puts those copies in front of the end of a short branch, where only the lanes that took it make them)
  sh.odd_values[wk] = 0;

  // ---- the three parts of a step: scores of its keys, 32 at a time in sc[sub]; their weights; the weighted values
  float sc[kSub][M::kScores];
  auto scores = [&](const unsigned char* kl) {
#pragma unroll
    for (int t = 0; t < kSub * M::kTiles; ++t) {
      const int krow = t * QW + col;
      acc x = acc{};
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        x = M::qk(*reinterpret_cast<const u32x4*>(kl + krow * RB + (((M::kGroups * s + grp) ^ mix<RB>(krow)) << 4)), q[s], x);
#pragma unroll
      for (int i = 0; i < M::kRegs; ++i) sc[t / M::kTiles][t % M::kTiles * M::kRegs + i] = x[i];
    }
    if constexpr (DT == kBF16) {
      // Three reads of keys on their way before the first product.  (Left to itself the compiler, short of registers, waits for
      // each read right before its product: 64 answers over a prefix of 9216 35 us instead of 33.)
      constexpr int kAll = kSub * M::kTiles * kSteps, kLead = 3;
      __builtin_amdgcn_sched_group_barrier(0x100, kLead, 0);
#pragma unroll
      for (int i = 0; i < kAll - kLead; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x8, kLead, 0);
    }
  };
  auto reference = [&](int kb) {
    if (kb + KT - 1 > lim_first) {
#pragma unroll
      for (int sub = 0; sub < kSub; ++sub)
#pragma unroll
        for (int u = 0; u < M::kScores; ++u) sc[sub][u] = kb + sub * 32 + M::place(u, grp) <= lim ? sc[sub][u] : -INFINITY;
    }
    float top = sc[0][0];
#pragma unroll
    for (int sub = 0; sub < kSub; ++sub)
#pragma unroll
      for (int u = 0; u < M::kScores; ++u) top = fmaxf(top, sc[sub][u]);
    top = groups_max<QW>(top) * scale2;
    // The reference of the exponentials follows the maximum only where it has grown by more than a factor
    // of 2^6: until then the weights are at most 64, and nothing is rescaled.
    if (__any(top > above)) {
      const float now = fmaxf(m, top);
      const float keep = __builtin_amdgcn_exp2f(m - now);
      m = now;
      l *= keep;
#pragma unroll
      for (int i = 0; i < kDT; ++i) o[i] *= keep;
      const bool coarse = fabsf(m) >= kCoarse && m > kLowest;
      above = coarse ? -INFINITY : m + 6.f;
      less = coarse ? 0.f : m;
      if (__any(coarse)) {
#pragma unroll
        for (int sub = 0; sub < kSub; ++sub)
#pragma unroll
          for (int u = 0; u < M::kScores; ++u) sc[sub][u] = coarse ? (product(sc[sub][u], scale2) - m) * back : sc[sub][u];
      }
    }
  };
  auto weights = [&](int sub) {
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < M::kScores; ++u) {
      sc[sub][u] = __builtin_amdgcn_exp2f(fmaf(sc[sub][u], scale2, -less));
      sum += sc[sub][u];
    }
    l += sum;
  };
  // bf16 (the matrix cores take the weights in no more bits; products for what the rounding leaves would double those with
  // the values): the right operand of product s of a sub-step, and the product with the values: four keys at a lane's column
  // of 16 by the transposing read of 16 lanes
  auto packed = [&](int sub, int s) {
    u32x4 p;
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = bf16_pair(sc[sub][8 * s + 2 * i], sc[sub][8 * s + 2 * i + 1]);
    return p;
  };
  auto values_bf16 = [&](const unsigned char* vl, int sub, int s, const u32x4& p) {
    const int vrow = 4 * grp + ((lane & 15) >> 2);
#pragma unroll
    for (int i = 0; i < kDT; ++i) {
      uint2 two[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int row = sub * 32 + M::kRun * (2 * s + j) + vrow;
        const int piece = i * (QW / 8) + (QW == 32 ? 2 * ((lane >> 4) & 1) : 0) + ((lane >> 1) & 1);
        const int at = row * RB + ((piece ^ mix<RB>(row)) << 4) + 8 * (lane & 1);
        two[j] = __builtin_bit_cast(
            uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(vl + at)));
      }
      o[i] = M::pv(u32x4{two[0].x, two[0].y, two[1].x, two[1].y}, p, o[i]);
    }
  };
  // (32-bit rows: a lane's 16 bytes feed four result tiles, whose rows are therefore every fourth element of the head)
  auto values_f32 = [&](const unsigned char* vl, int sub) {
#pragma unroll
    for (int u = 0; u < M::kScores; ++u) {
      const int row = sub * 32 + M::place(u, grp);
#pragma unroll
      for (int i = 0; i < kDT / 4; ++i) {
        const f32x4v v = *reinterpret_cast<const f32x4v*>(vl + row * RB + (((i * QW + col) ^ mix<RB>(row)) << 4));
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if constexpr (DT == kF32) o[4 * i + k] = M::av(v[k], sc[sub][u], o[4 * i + k]);
      }
    }
  };

  if (steps > 0) {
    load_tile(kfirst);
    load_pages(kfirst + kstep);
  }
  __syncthreads();
  for (int it = 0; it < steps; ++it) {
    const int kb = kfirst + it * kstep;
    unsigned char* kl = my_lds + (S::kBuffers > 1 ? (it & 1) * 2 * S::kTileBytes : 0);
    unsigned char* vl = kl + S::kTileBytes;
    if (S::kBuffers == 1) tiles_handed_over();
    store_keys(kl);
    store_values(vl, kb);
    load_tile(kb + kstep);
    load_pages(kb + 2 * kstep);
    if (WM > 1) __syncthreads();
    else tiles_handed_over();
    if (kb > lim_last) continue;  // (none of this wave's rows sees a key of the step)
    scores(kl);
    reference(kb);
#pragma unroll
    for (int sub = 0; sub < kSub; ++sub) {
      weights(sub);
      if constexpr (DT == kBF16) {
#pragma unroll
        for (int s = 0; s < M::kScores / 8; ++s) values_bf16(vl, sub, s, packed(sub, s));
      } else {
        values_f32(vl, sub);
      }
    }
  }
  if (bad_page) flag(c, kBadPage);
  if (causal) {
    if (WM > 1) __syncthreads();
    if (*(volatile int*)&sh.odd_values[wk] != 0) {
      // Values that are no numbers, key by key, for the rows that see them.
#pragma unroll 1
      for (int it = 0; it < steps * KT; ++it) {
        const int kb = kfirst + it / KT * kstep, key = kb + it % KT;
        if (kb + KT - 1 <= lim_block || key >= k1) continue;
        bool bad;
        const long at = key_offset(c, table, key, bad) + (long)head * c.head_ld;
        float w = 0.f;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const int e = (M::kGroups * s + grp) * M::kVec;
          Piece<DT, M::kVec> kf = {}, qf;
          if (e < c.d) kf = load_piece<DT, M::kVec>(a.k_pool, at + e);
          __builtin_memcpy(&qf, &q[s], 16);
#pragma unroll
          for (int j = 0; j < M::kVec; ++j) w = fmaf(qf.get(j), kf.get(j), w);
        }
        w = groups_sum<QW>(w);
        w = __builtin_amdgcn_exp2f(fabsf(m) >= kCoarse ? product(w, scale2) - m : fmaf(w, scale2, -m));
        if (key > lim) continue;
#pragma unroll
        for (int x = 0; x < kQuads; ++x) {
          const Piece<DT, 4> v = load_piece<DT, 4>(a.v_pool, at + min(quad_at(x), c.d - 4));  // (past the head: not stored)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (fabsf(v.get(k)) < INFINITY) continue;
            if constexpr (DT == kBF16) o[x / (M::kRegs / 4)][4 * (x % (M::kRegs / 4)) + k] += w * v.get(k);
            else o[4 * (x / M::kRegs) + k][x % M::kRegs] += w * v.get(k);
          }
        }
      }
    }
  }
  l = groups_sum<QW>(l);

  const long all = (long)c.T * c.Hq;
  if constexpr (WK == 1) {
    if (!in) return;
    const long id = (long)(tok0 + my_tok) * c.Hq + qh;
    if (sp.parts > 1) {
      const long at = (sp.first_part + part) * all + id;
      if (grp == 0) sp.part_ml[at] = make_float2(m, l);
#pragma unroll
      for (int x = 0; x < kQuads; ++x)
        if (quad_at(x) < c.d) *reinterpret_cast<f32x4v*>(sp.part_o + at * c.d + quad_at(x)) = quad(x);
      return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (a.lse != nullptr && grp == 0) a.lse[id] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
    const long at = (long)(tok0 + my_tok) * a.out_ld + (long)qh * c.d;
#pragma unroll
    for (int x = 0; x < kQuads; ++x) {
      if (quad_at(x) >= c.d) continue;
      const f32x4v v = quad(x) * inv;
      const float y[4] = {v[0], v[1], v[2], v[3]};
      store_piece<DT, 4>(a.out, at + quad_at(x), round_piece<DT, 4>(y));
    }
  } else {
    // The key groups' results are joined in LDS, in the tiles' place.
    if (grp == 0) sh.joined[wk][col] = make_float2(m, l);
    __syncthreads();
    float top = kLowest, total = 0.f;
#pragma unroll
    for (int w = 0; w < WK; ++w) top = fmaxf(top, sh.joined[w][col].x);
#pragma unroll
    for (int w = 0; w < WK; ++w) total += sh.joined[w][col].y * __builtin_amdgcn_exp2f(sh.joined[w][col].x - top);
    const float keep = __builtin_amdgcn_exp2f(m - top);
    float* mat = reinterpret_cast<float*>(my_lds);
#pragma unroll
    for (int x = 0; x < kQuads; ++x)
      *reinterpret_cast<f32x4v*>(mat + col * DP + ((quad_at(x) / 4 ^ (col & 7)) << 2)) = quad(x) * keep;
    if (wk == 0 && grp == 0) sh.joined[4][col] = make_float2(top, total);
    __syncthreads();
    constexpr int kRow = DP / 4;
    for (int e = threadIdx.x; e < QW * kRow; e += S::kThreads) {
      const int rr = e / kRow, piece = e % kRow, row = row0 + rr;
      if (row >= rows || piece * 4 >= c.d) continue;
      f32x4v x = {};
#pragma unroll
      for (int w = 0; w < WK; ++w)
        x += *reinterpret_cast<const f32x4v*>(reinterpret_cast<const float*>(lds + w * (S::kBuffers * 2 * S::kTileBytes)) + rr * DP +
                                              ((piece ^ (rr & 7)) << 2));
      const int i = token_in(a, row), h = head * r + row - i * r;
      const long id = (long)(tok0 + i) * c.Hq + h;
      const float2 ml = sh.joined[4][rr];
      if (sp.parts > 1) {
        const long at = (sp.first_part + part) * all + id;
        if (piece == 0) sp.part_ml[at] = ml;
        *reinterpret_cast<f32x4v*>(sp.part_o + at * c.d + piece * 4) = x;
        continue;
      }
      const float inv = ml.y == 0.f ? 0.f : 1.f / ml.y;
      if (a.lse != nullptr && piece == 0) a.lse[id] = ml.y == 0.f ? -INFINITY : (ml.x + log2f(ml.y)) * kLn2;
      const float y[4] = {x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
      store_piece<DT, 4>(a.out, (long)(tok0 + i) * a.out_ld + (long)h * c.d + piece * 4, round_piece<DT, 4>(y));
    }
  }
}

// Block number -> (row tile, head, part): the pairs of a head and a part fastest, so that the blocks that
// read the same keys lie on the same die wherever the pairs are a multiple of eight; the tiles that see
// most keys first.
__device__ __forceinline__ void attend_place(const Cache& c, const Parting& sp, unsigned id, long& slot, int& head, int& part) {
  const unsigned pairs = (unsigned)c.Hkv * (unsigned)sp.chunks, s = id / pairs, p = id - s * pairs;
  part = (int)(p / (unsigned)c.Hkv);
  head = (int)(p - (unsigned)part * (unsigned)c.Hkv);
  slot = sp.slots - 1 - (long)s;
}

template <int DT, int DP, int QW, int WM, int WK, int KT>
__global__ __launch_bounds__(64 * WM * WK, DP <= 128 && (DT == kBF16 || WK == 1) ? 2 : 1) void k_attend(Attend a, Cache c, Parting sp) {
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ AttendShared sh;
  long slot;
  int head, part;
  attend_place(c, sp, blockIdx.x, slot, head, part);
  attend_tile<DT, DP, QW, WM, WK, KT>(a, c, sp, lds, sh, slot, head, part);
}

// Prefixes and own keys in one launch: the first blocks take the prefixes, the rest fill in beside them (64 answers over
// one prefix of 9216 keys, 28 + 4 heads: 33 us, 5 of them the join, where a copy of the keys' bytes would take 11;
// 32 prompts of 9 to 71 tokens over four prefixes of 2880, 32 heads: 129 us, 0.49 PF/s, bound by units that have two
// tiles where others have one).
template <int DT, int DP, int KT>
__global__ __launch_bounds__(256, DT == kBF16 && DP <= 128 ? 2 : 1) void k_attend_both(Attend a, Cache c, Parting pre, Parting own,
                                                                                       unsigned pre_blocks) {
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ AttendShared sh;
  const bool first = blockIdx.x < pre_blocks;
  const Parting sp = first ? pre : own;
  long slot;
  int head, part;
  attend_place(c, sp, first ? blockIdx.x : blockIdx.x - pre_blocks, slot, head, part);
  if (sp.few) attend_tile<DT, DP, 16, 1, 4, 32>(a, c, sp, lds, sh, slot, head, part);
  else attend_tile<DT, DP, many_columns(DT, DP), 4, 1, KT>(a, c, sp, lds, sh, slot, head, part);
}

// Joins a row's parts.  2^lanes_shift lanes hold a row, four elements each; 2^split_shift such sets of a block
// share one row's parts where there are many, and join through LDS (8 rows of 16 000 keys in 63 parts: 48 us with a set to
// a row, 16 with sixteen, attention included).  Bound by latency: what a row's sequence is, its parts, its result, one after
// the other; with many rows by memory (42 000 rows of two parts 15 us, of which a copy would need 11 for their 55 MB).  Two
// parts are asked for at once: eight, of which those past the last are read in vain, take 2 us more there and gain nothing
// with 63 parts.
template <int DT>
__global__ __launch_bounds__(256) void k_attend_join(Attend a, Cache c, int pre_chunk, int pre_parts, int own_chunk, const float* part_o,
                                                     const float2* part_ml, int lanes_shift, int split_shift) {
  __shared__ f32x4v set_x[256];
  __shared__ float2 set_ml[256];
  const int all = c.T * c.Hq;  // (2^24 at most)
  const int lane = threadIdx.x & 63, set = threadIdx.x >> lanes_shift, sub = set & ((1 << split_shift) - 1);
  const int rows_shift = 8 - lanes_shift - split_shift;  // rows of a block
  const int first = (int)blockIdx.x << rows_shift, id = first + (set >> split_shift);
  bool row = id < all;
  const int t = row ? id / c.Hq : 0, h = row ? id - t * c.Hq : 0;
  Seq s = {};
  int prefix = 0;
  if (c.B <= kWave && c.groups <= kWave) {
    // All sequences and groups in one look: seven dependent loads less in a block's life, which is little else.
    const int i = min(lane, c.B - 1), lo = c.cu ? c.cu[i] : i, hi = c.cu ? c.cu[i + 1] : i + 1, keys = c.kv_len[i];
    int from = 0, to = 0, front = 0;
    if (c.groups > 0) {
      const int g = min(lane, c.groups - 1);
      from = c.group_cu[g], to = c.group_cu[g + 1], front = c.prefix_len[g];
    }
    for (int k = 0; k < kWave >> lanes_shift; ++k) {  // the wave's rows
      const int tk = __builtin_amdgcn_readlane(t, k << lanes_shift);
      const unsigned long long low = __ballot(lane < c.B && lo <= tk);
      const int b = low ? 63 - __builtin_clzll(low) : 0;
      const Seq sk = make_sequence(c, __builtin_amdgcn_readlane(lo, b), __builtin_amdgcn_readlane(hi, b), __builtin_amdgcn_readlane(keys, b));
      int pk = 0;
      if (c.groups > 0) {
        const unsigned long long before = __ballot(lane < c.groups && from <= b);
        const int g = before ? 63 - __builtin_clzll(before) : 0;
        const int b0 = __builtin_amdgcn_readlane(from, g), b1 = __builtin_amdgcn_readlane(to, g);
        pk = b < b0 || b >= b1 ? -1 : make_prefix(c, b0, b1, __builtin_amdgcn_readlane(front, g));
      }
      if (lane >> lanes_shift == k) s = sk, prefix = pk;
    }
  } else {
    int b = t;
    if (c.cu != nullptr) {
      b = owner_of(c.cu, c.B, first / c.Hq);
      while (b + 1 < c.B && c.cu[b + 1] <= t) ++b;  // (a block's rows are a few tokens')
    }
    s = sequence_of(c, b);
    if (c.groups > 0) {
      int g = 0, end = c.groups;
      while (end - g > 1) {
        const int mid = (g + end) / 2;
        if (c.group_cu[mid] <= b) g = mid; else end = mid;
      }
      prefix = b < c.group_cu[g] || b >= c.group_cu[g + 1] ? -1 : prefix_of(c, g);
    }
  }
  int own = s.kv;
  if (a.causal && s.kv - s.n + (t - s.tok0) + 1 < own) own = s.kv - s.n + (t - s.tok0) + 1;
  row = row && t >= s.tok0 && t < s.tok0 + s.n;  // (else no sequence's token)
  if (prefix < 0) {
    flag(c, kBadSequence);
    prefix = own = 0;
  }
  if (!s.valid || !row) prefix = own = 0;
  const int np = prefix > 0 ? (prefix + pre_chunk - 1) / pre_chunk : 0;
  const int n = np + (own > 0 ? (own + own_chunk - 1) / own_chunk : 0);
  const int e = (lane & ((1 << lanes_shift) - 1)) * 4;
  const bool in = e < c.d;
  float top = kLowest, l = 0.f;
  f32x4v x = {};
  constexpr int kAtOnce = 2;
  for (int i0 = sub; i0 < n; i0 += kAtOnce << split_shift) {
    float2 ml[kAtOnce];
    f32x4v y[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const int i = min(i0 + (j << split_shift), n - 1);  // (past the last: the last again, with no weight)
      const long at = (long)(i < np ? i : pre_parts + i - np) * all + id;
      ml[j] = part_ml[at];
      y[j] = *reinterpret_cast<const f32x4v*>(part_o + at * c.d + (in ? e : 0));
    }
    float now = top;
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) now = fmaxf(now, ml[j].x);
    const float f = __builtin_amdgcn_exp2f(top - now);
    top = now;
    l *= f;
    x *= f;
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      if (i0 + (j << split_shift) >= n) break;
      const float w = __builtin_amdgcn_exp2f(ml[j].x - now);
      l += ml[j].y * w;
      x += y[j] * w;
    }
  }
  if (split_shift > 0) {
    set_x[threadIdx.x] = x;
    set_ml[threadIdx.x] = make_float2(top, l);
    __syncthreads();
    if (sub != 0) return;
    const float mine = top;
    for (int i = 1; i < 1 << split_shift; ++i) top = fmaxf(top, set_ml[threadIdx.x + (i << lanes_shift)].x);
    const float f = __builtin_amdgcn_exp2f(mine - top);
    l *= f;
    x *= f;
    for (int i = 1; i < 1 << split_shift; ++i) {
      const float2 ml = set_ml[threadIdx.x + (i << lanes_shift)];
      const float w = __builtin_amdgcn_exp2f(ml.x - top);
      l += ml.y * w;
      x += set_x[threadIdx.x + (i << lanes_shift)] * w;
    }
  }
  if (!row) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (a.lse != nullptr && e == 0) a.lse[id] = l == 0.f ? -INFINITY : (top + log2f(l)) * kLn2;
  if (!in) return;
  const float y[4] = {x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
  store_piece<DT, 4>(a.out, (long)t * a.out_ld + (long)h * c.d + e, round_piece<DT, 4>(y));
}

}  // namespace dart
