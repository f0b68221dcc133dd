// The attention weight that each key of a cache gathers from the queries of a call.
#pragma once

#include "fourbit.hpp"
#include "k_attend.hpp"

namespace dart {

struct Gather {
  const void *q, *k_pool;
  const uint8_t* k_scales;  // (keys held in 4 bits)
  const float* lse;
  float* weights;
  long q_ld;
  float scale, carry;
  int causal;
  double per_token;  // 1 / (rows of a token: query heads of a key head)
};

// How a launch is divided: block -> (sequence or group, part of its rows, tile of its keys, key head), heads fastest.
struct Shares {
  int prefix;  // the keys are the groups' shared prefixes (else each sequence's own)
  int tiles;   // of keys, of the longest
  int few;     // the kernel for few rows
  int parts;   // of the rows
  float* sums; // [parts][blocks of a part][keys of a tile], where there is more than one part
};

// 32 rows by 32 keys: a lane holds of its key the products with rows 8 (u / 4) + 4 (lane / 32) + u % 4, so that what a key
// gathers is added up within the lane.
template <int DT>
struct Tile32 {
  static constexpr int kVec = DT == kBF16 ? 8 : 4;
  __device__ static __forceinline__ f32x16 product(const u32x4& q, const u32x4& k, f32x16 c) {
    if constexpr (DT == kBF16) {
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, q), __builtin_bit_cast(bf16x8, k), c, 0, 0, 0);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(q[j]), __uint_as_float(k[j]), c, 0, 0, 0);
      return c;
    }
  }
};

// KW times 32 keys to a wave, four waves.
template <int DT, int DP>
struct GatherShape {
  static constexpr int KW = DT == kBF16 && DP <= 128 ? 2 : 1;
  static constexpr int kKeys = 128 * KW;
  static constexpr int kRowBytes = DP * (DT == kBF16 ? 2 : 4);
  static constexpr int kPieces = kRowBytes / 16;
  static constexpr int kRows = kRowBytes <= 512 ? 64 : 32;  // of a stage: what the block brings to LDS between two barriers
  static constexpr int kLoads = kRows * kPieces / 256;
  static constexpr int kStage = kRows * kRowBytes;
  static constexpr int kLds = 2 * kStage;
};

// Whose rows and keys a block has.  n < 0: there is nothing to do for it.
struct Share {
  int tok0, n, kv, fresh;  // fresh: the first key that belongs to the call's tokens
  const int* table;
  bool valid;
};

__device__ __forceinline__ Share share_of(const Cache& c, bool prefix, int owner) {
  Share s;
  if (!prefix) {
    const Seq q = sequence_of(c, owner);
    s.valid = q.valid;
    s.tok0 = q.tok0, s.n = q.n, s.kv = q.kv;
    s.fresh = q.kv - q.n;
    s.table = c.pages + (long)owner * c.pages_ld;
  } else {
    const int b0 = c.group_cu[owner], b1 = c.group_cu[owner + 1], keys = prefix_of(c, owner);
    bool good = keys >= 0;
    if (good)  // (every sequence of the group has to be as it should: their tokens are then the group's)
      for (int b = b0 + (int)(threadIdx.x & 63); __any(b < b1); b += kWave)
        if (__any(b < b1 && !sequence_of(c, b < b1 ? b : b0).valid)) good = false;
    s.valid = good;
    s.tok0 = good ? token_of(c, b0) : 0;
    s.n = good ? token_of(c, b1) - s.tok0 : 0;
    s.kv = s.fresh = good ? keys : 0;
    s.table = c.prefix_pages + (long)owner * c.prefix_ld;
  }
  return s;
}

// A key's weight; of one in a page that is none (flagged where its key was asked for) another's, not to be written.
__device__ __forceinline__ float* weight_at(const Gather& a, const Cache& c, int head, int key, int page) {
  const bool none = (unsigned)page >= (unsigned)c.n_pages;
  return a.weights + (((none ? 0L : (long)page) * c.Hkv + head) << c.page_shift) + (key & ((1 << c.page_shift) - 1));
}
__device__ __forceinline__ float kept_weight(const Gather& a, const Share& s, int key, float old, float sum) {
  return a.carry == 0.f || key >= s.fresh ? sum : fmaf(a.carry, old, sum);
}

__device__ __forceinline__ void put_weight(const Gather& a, const Cache& c, const Share& s, int head, int key, float sum) {
  const int page = s.table[key >> c.page_shift];
  if ((unsigned)page >= (unsigned)c.n_pages) return;
  float* at = weight_at(a, c, head, key, page);
  *at = kept_weight(a, s, key, a.carry != 0.f ? *at : 0.f, sum);
}

// w_j <- carry * w_j + sum over the rows that see key j of exp(scale <q, k_j> - lse).  A wave holds its keys in registers
// and goes through the rows 32 at a time, which the block brings to LDS while it works on those before.  Sums in 32 bits, those
// of 16 stages of rows by themselves (up to 1024 rows).
// Bound by exponentials and products, which overlap little: two causal prompts of 9216, 28 + 4 heads of 128 in bf16, 705 us where the
// products alone would take 446 (the matrix cores are busy 37 % of the time, the vector units 50 %); 637 causal tokens of 32 heads in 32 bits
// 31 with the join, by keys and rows of short blocks one after the other.
template <int DT, int DP, class HELD>
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void k_gather_weights(Gather a, Cache c, Shares sp, unsigned first) {
  typedef GatherShape<DT, DP> S;
  typedef Tile32<DT> M;
  constexpr int KW = S::KW, RB = S::kRowBytes, kSteps = DP / (2 * M::kVec);
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ long row_at[2][64];
  __shared__ f32x4v less_of[3][16];  // four rows' lse times log2 e
  __shared__ int lim_of[3][64];      // the last key that a row sees
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, grp = lane >> 5, col = lane & 31;
  const int r = c.Hq / c.Hkv;

  unsigned id = first + blockIdx.x;
  const int head = (int)(id % (unsigned)c.Hkv);
  id /= (unsigned)c.Hkv;
  const int tile = (int)(id % (unsigned)sp.tiles);
  id /= (unsigned)sp.tiles;
  const int part = (int)(id % (unsigned)sp.parts), owner = (int)(id / (unsigned)sp.parts);
  const Share s = share_of(c, sp.prefix != 0, owner);
  if (!s.valid && threadIdx.x == 0 && tile == 0) flag(c, kBadSequence);
  const int k0 = tile * S::kKeys, last_key = s.kv - 1;
  if (!s.valid || s.n <= 0 || k0 >= s.kv) return;
  const bool causal = a.causal && !sp.prefix;
  const int rows = s.n * r;
  // Stages of rows, dealt to the parts alike for all tiles (so that tiles that are worked on side by side read the same rows, which
  // then come from the die's cache), from the first on that has a row that sees the first key of the tile.
  const int stages = (rows + S::kRows - 1) / S::kRows, seen_from = causal ? max(0, k0 - s.fresh) * r / S::kRows : 0;
  const int t0 = max(seen_from, (int)((long)stages * part / sp.parts)), t1 = (int)((long)stages * (part + 1) / sp.parts);

  // ---- this lane's keys: of key `col` of 32 the pieces piece(s)
  auto piece = [&](int st) { return HELD::kCodes ? grp * kSteps + st : 2 * st + grp; };
  u32x4 k[KW][kSteps];
#pragma unroll
  for (int w = 0; w < KW; ++w) {
    const int key = min(k0 + (wave * KW + w) * 32 + col, last_key);
    bool bad;
    const long at = key_offset(c, s.table, key, bad) + (long)head * c.head_ld;
    if (bad) flag(c, kBadPage);
    if constexpr (HELD::kCodes) {
      constexpr int kBlocks = DP / 64 > 0 ? DP / 64 : 1, kPer = kSteps / kBlocks;  // blocks of a lane, pieces of a block
      Codes<4> x[kBlocks];
      uint32_t e[kBlocks];
#pragma unroll
      for (int j = 0; j < kBlocks; ++j) {
        const int v = (grp * kBlocks + j) * 32;
        x[j] = Codes<4>{}, e[j] = 0;
        if (v < c.d) {
          __builtin_memcpy(&x[j], __builtin_assume_aligned(static_cast<const unsigned char*>(a.k_pool) + (at + v) / 2, 16), 16);
          e[j] = a.k_scales[(at + v) / 32];
        }
      }
#pragma unroll
      for (int st = 0; st < kSteps; ++st)
        k[w][st] = HELD::template piece<DT>(x[st / kPer].v[st % kPer * M::kVec / 8], e[st / kPer], st % kPer * M::kVec / 4 % 2);
    } else {
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        const int e = piece(st) * M::kVec;
        k[w][st] = u32x4{0, 0, 0, 0};
        if (e < c.d) k[w][st] = *reinterpret_cast<const u32x4*>(static_cast<const unsigned char*>(a.k_pool) + (at + e) * (16 / M::kVec));
      }
    }
  }

  // ---- rows to LDS.  Where the rows of a stage lie is found three stages before, by a thread each (by all threads for themselves it
  // costs as much as a third of the exponentials).
  const int my_piece = threadIdx.x % S::kPieces, my_row = threadIdx.x / S::kPieces;
  constexpr int kApart = 256 / S::kPieces;
  const bool in_head = my_piece * M::kVec < c.d && a.scale != 0.f;  // (else zeros, from the start on)
  const unsigned char* q_at = static_cast<const unsigned char*>(a.q) + ((long)s.tok0 * a.q_ld + (long)head * r * c.d + (in_head ? my_piece * M::kVec : 0)) * (16 / M::kVec);
  const float* lse_at = a.lse + (long)s.tok0 * c.Hq + head * r;
  const bool finds = (int)threadIdx.x < S::kRows;
  float lse = 0.f;
  int tok = 0, lim = 0;
  long at = 0;
  auto find_rows = [&](int t) {
    if (!finds) return;
    const int row = t * S::kRows + (int)threadIdx.x, have = min(row, rows - 1);  // (past the last: the last again)
    tok = (int)(((double)have + 0.5) * a.per_token);
    const int h = have - tok * r;
    lse = lse_at[(long)tok * c.Hq + h];
    lim = row >= rows ? -1 : causal ? min(s.fresh + tok, last_key) : last_key;
    at = ((long)tok * a.q_ld + (long)h * c.d) * (16 / M::kVec);
  };
  auto tell_rows = [&](int t) {
    if (!finds) return;
    // (a row past the last, or one that saw nothing, gives nothing to any key)
    row_at[t & 1][threadIdx.x] = at;
    reinterpret_cast<float*>(less_of[t % 3])[threadIdx.x] = lse * kLog2e;
    lim_of[t % 3][threadIdx.x] = lse == -INFINITY ? -1 : lim;
  };
  u32x4 qr[S::kLoads];
  auto load_rows = [&](int t) {
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) qr[i] = *reinterpret_cast<const u32x4*>(q_at + row_at[t & 1][my_row + i * kApart]);
  };
  auto store_rows = [&](int t) {
    unsigned char* to = lds + (t & 1) * S::kStage;
    if (!in_head) return;
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const int row = my_row + i * kApart;
      *reinterpret_cast<u32x4*>(to + row * RB + ((my_piece ^ mix<RB>(row)) << 4)) = qr[i];
    }
  };
  if (!in_head) {
#pragma unroll
    for (int i = 0; i < 2 * S::kLoads; ++i) {
      const int row = my_row + i * kApart;
      *reinterpret_cast<u32x4*>(lds + row * RB + ((my_piece ^ mix<RB>(row)) << 4)) = u32x4{0, 0, 0, 0};
    }
  }

  const float scale2 = a.scale * kLog2e;
  const int my_k0 = k0 + wave * KW * 32, my_end = my_k0 + KW * 32 - 1;
  // (added up by 32 rows, then by 16 stages, then all: long sums in one go would lose digits)
  float sum[KW], total[KW];
#pragma unroll
  for (int w = 0; w < KW; ++w) sum[w] = total[w] = 0.f;
  if (t0 < t1) {
    find_rows(t0);
    tell_rows(t0);
    find_rows(t0 + 1);
    tell_rows(t0 + 1);
    find_rows(t0 + 2);
    __syncthreads();
    load_rows(t0);
  }
  for (int t = t0; t < t1; ++t) {
    store_rows(t);
    __syncthreads();
    if (t + 1 < t1) {
      load_rows(t + 1);
      tell_rows(t + 2);
      find_rows(t + 3);
    }
    const bool all_seen = !__any(lim_of[t % 3][lane & (S::kRows - 1)] < my_end);
#pragma unroll
    for (int half = 0; half < S::kRows / 32; ++half) {
      const unsigned char* from = lds + (t & 1) * S::kStage + half * 32 * RB;
      f32x4v less[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) less[i] = less_of[t % 3][half * 8 + 2 * i + grp];
      auto read_row = [&](int st) { return *reinterpret_cast<const u32x4*>(from + col * RB + ((piece(st) ^ mix<RB>(col)) << 4)); };
      u32x4 q[kSteps];  // (for several tiles of keys; one takes them as they come)
      if (KW > 1) {
#pragma unroll
        for (int st = 0; st < kSteps; ++st) q[st] = read_row(st);
      }
      if (all_seen) {
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          f32x16 x = f32x16{};
#pragma unroll
          for (int st = 0; st < kSteps; ++st) x = M::product(KW > 1 ? q[st] : read_row(st), k[w][st], x);
          float y = 0.f;
#pragma unroll
          for (int u = 0; u < 16; ++u) y += __builtin_amdgcn_exp2f(fmaf(x[u], scale2, -less[u / 4][u % 4]));
          sum[w] += y;
        }
      } else {
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          f32x16 x = f32x16{};
#pragma unroll
          for (int st = 0; st < kSteps; ++st) x = M::product(KW > 1 ? q[st] : read_row(st), k[w][st], x);
          float y = 0.f;
#pragma unroll
          for (int u = 0; u < 16; ++u) {
            const float e = __builtin_amdgcn_exp2f(fmaf(x[u], scale2, -less[u / 4][u % 4]));
            y += my_k0 + w * 32 + col <= lim_of[t % 3][half * 32 + 8 * (u / 4) + 4 * grp + u % 4] ? e : 0.f;
          }
          sum[w] += y;
        }
      }
    }
    if ((t - t0) % 16 == 15) {
#pragma unroll
      for (int w = 0; w < KW; ++w) total[w] += sum[w], sum[w] = 0.f;
    }
  }

  __syncthreads();
  float* out = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int w = 0; w < KW; ++w) {
    float y = total[w] + sum[w];
    y += __shfl_xor(y, 32);
    if (grp == 0) out[(wave * KW + w) * 32 + col] = y;
  }
  __syncthreads();
  const int key = k0 + (int)threadIdx.x;
  if ((int)threadIdx.x >= S::kKeys) return;
  if (sp.parts > 1) {
    const long block = ((long)owner * sp.tiles + tile) * c.Hkv + head, blocks = (long)(sp.prefix ? c.groups : c.B) * sp.tiles * c.Hkv;
    sp.sums[(part * blocks + block) * S::kKeys + threadIdx.x] = out[threadIdx.x];
  } else if (key < s.kv) {
    put_weight(a, c, s, head, key, out[threadIdx.x]);
  }
}

// Two numbers of every lane, added over pairs of lane groups LANES apart: the lower group gets the sum of the first numbers, the
// upper that of the second ones.
template <int LANES>
__device__ __forceinline__ float pairs_sum(float x, float y) {
  if constexpr (LANES == 16) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  } else {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
}

// A few rows: a wave takes tiles of 16 keys against 16 rows at a time and leaves LDS alone.  All its keys are asked for at once, the rows
// before them, so that a call of single tokens is bound by memory and, over codes, by instructions.  NT: tiles of a wave (32 tokens over
// 8000 keys, 28 + 4 heads: in 4 bits 17.4 us with eight, 19.0 with four; in rows 54 with either, of 32 bits 212 and 111; with
// 16 + 4 heads of 256 in 4 bits 36 and 33, of 32-bit queries 94 and 101).
constexpr int few_tiles(int dt, int d, bool codes) { return codes && (dt == kF32 || d <= 128) ? 8 : 4; }
template <int DT, int DP, bool CODES>
struct GatherFewShape {
  static constexpr int NT = few_tiles(DT, DP, CODES);
  static constexpr int kKeys = 4 * 16 * NT;
};

template <int DT, int DP, class HELD>
__global__ __launch_bounds__(256, DT == kF32 && DP == 256 ? 1 : 2) void k_gather_weights_few(Gather a, Cache c, Shares sp, unsigned first) {
  typedef GatherFewShape<DT, DP, HELD::kCodes> S;
  typedef Math<DT, 16> M;
  constexpr int NT = S::NT, kSteps = M::template steps<DP>(), kMine = DP / 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, grp = lane >> 4, col = lane & 15;
  const int r = c.Hq / c.Hkv;

  unsigned id = first + blockIdx.x;
  const int head = (int)(id % (unsigned)c.Hkv);
  id /= (unsigned)c.Hkv;
  const int tile = (int)(id % (unsigned)sp.tiles), owner = (int)(id / (unsigned)sp.tiles);
  const Share s = share_of(c, sp.prefix != 0, owner);
  if (!s.valid && threadIdx.x == 0 && tile == 0) flag(c, kBadSequence);
  const int k0 = tile * S::kKeys + wave * 16 * NT, last_key = s.kv - 1;
  if (!s.valid || s.n <= 0 || k0 >= s.kv) return;
  const bool causal = a.causal && !sp.prefix;
  const int rows = s.n * r, row_first = causal ? max(0, k0 - s.fresh) * r : 0, mask = (1 << c.page_shift) - 1;

  // ---- rows.  The first are asked for before the keys: after them they would come a look into memory later.
  auto piece = [&](int st) { return HELD::kCodes ? grp * kSteps + st : 4 * st + grp; };
  float lse;
  int lim;
  u32x4 q[kSteps];
  auto load_rows = [&](int row0) {
    const int row = row0 + col, have = min(row, rows - 1), tok = (int)(((double)have + 0.5) * a.per_token), qh = head * r + have - tok * r;
    lse = a.lse[(long)(s.tok0 + tok) * c.Hq + qh];
    lim = row >= rows ? -1 : causal ? min(s.fresh + tok, last_key) : last_key;
    const unsigned char* q_at = static_cast<const unsigned char*>(a.q) + ((long)(s.tok0 + tok) * a.q_ld + (long)qh * c.d) * (16 / M::kVec);
#pragma unroll
    for (int st = 0; st < kSteps; ++st) q[st] = *reinterpret_cast<const u32x4*>(q_at + (piece(st) * M::kVec < c.d ? piece(st) * 16 : 0));
  };
  load_rows(row_first);

  // ---- keys: of key `col` of a tile the lane group's pieces of the row, every fourth, or one run of codes
  int page[NT], page_out[NT / 4];
#pragma unroll
  for (int t = 0; t < NT; ++t) page[t] = s.table[min(k0 + t * 16 + col, last_key) >> c.page_shift];
  // (a lane writes key `col` of tile 4 x + grp)
  auto key_out = [&](int x) { return k0 + (4 * x + grp) * 16 + col; };
#pragma unroll
  for (int x = 0; x < NT / 4; ++x) page_out[x] = s.table[min(key_out(x), last_key) >> c.page_shift];
  bool bad = false;
  constexpr int kBlocks = kMine > 32 ? kMine / 32 : 1;
  typedef Codes<(kMine < 32 ? kMine : 32) / 8> Run;
  u32x4 kr[NT][HELD::kCodes ? 1 : kSteps];
  Run kc[NT][kBlocks];
  uint32_t ke[NT][kBlocks];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    bool none = (unsigned)page[t] >= (unsigned)c.n_pages;
    bad = bad || none;
    const long at = (none ? 0L : (long)page[t] * c.page_ld) + (long)(min(k0 + t * 16 + col, last_key) & mask) * c.row_ld + (long)head * c.head_ld;
    if constexpr (HELD::kCodes) {
#pragma unroll
      for (int j = 0; j < kBlocks; ++j) {
        const int v = grp * kMine + j * 32 < c.d ? grp * kMine + j * 32 : 0;  // (past the head: what is there, by queries of zeros)
        __builtin_memcpy(&kc[t][j], __builtin_assume_aligned(static_cast<const unsigned char*>(a.k_pool) + (at + v) / 2, sizeof(Run)), sizeof(Run));
        ke[t][j] = a.k_scales[(at + v) / 32];
      }
    } else {
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        const int e = piece(st) * M::kVec;
        kr[t][st] = u32x4{0, 0, 0, 0};
        if (e < c.d) kr[t][st] = *reinterpret_cast<const u32x4*>(static_cast<const unsigned char*>(a.k_pool) + (at + e) * (16 / M::kVec));
      }
    }
  }
  if (bad) flag(c, kBadPage);
  // What the keys had, asked for beside their codes (of a key that is not there, some place's; a branch would wait for it).
  float old[NT / 4];
  float* put[NT / 4];
  bool there[NT / 4];
#pragma unroll
  for (int x = 0; x < NT / 4; ++x) {
    const int key = key_out(x);
    there[x] = (unsigned)page_out[x] < (unsigned)c.n_pages && key <= last_key;
    put[x] = weight_at(a, c, head, key, page_out[x]);
    old[x] = 0.f;
    if (a.carry != 0.f) old[x] = *put[x];
  }

  const float scale2 = a.scale * kLog2e;
  float sum[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) sum[t] = 0.f;
  for (int row0 = row_first; row0 < rows; row0 += 16) {
    if (row0 > row_first) load_rows(row0);
    // (keys lie in the columns of the product, this lane group's four rows in its registers)
    float less[4];
    int lims[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) less[u] = __shfl(lse * kLog2e, 4 * grp + u), lims[u] = __shfl(lse == -INFINITY ? -1 : lim, 4 * grp + u);
#pragma unroll
    for (int st = 0; st < kSteps; ++st)
      if (piece(st) * M::kVec >= c.d || a.scale == 0.f) q[st] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if constexpr (HELD::kCodes) {
#pragma unroll
        for (int j = 0; j < kBlocks; ++j) made_here(ke[t][j]);
      }
      f32x4v x = {};
#pragma unroll
      for (int st = 0; st < kSteps; ++st) {
        u32x4 k;
        if constexpr (HELD::kCodes) {
          constexpr int kPer = kMine < 32 ? kSteps : 32 / M::kVec;
          k = HELD::template piece<DT>(kc[t][st / kPer].v[st % kPer * M::kVec / 8], ke[t][st / kPer], st * M::kVec / 4 % 2);
        } else {
          k = kr[t][st];
        }
        x = M::qk(q[st], k, x);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float y = __builtin_amdgcn_exp2f(fmaf(x[u], scale2, -less[u]));
        sum[t] += k0 + t * 16 + col <= lims[u] ? y : 0.f;
      }
    }
  }
  // ---- over the lane groups; each then has the sums of a tile of its own
#pragma unroll
  for (int x = 0; x < NT / 4; ++x) {
    const float mine = pairs_sum<16>(pairs_sum<32>(sum[4 * x], sum[4 * x + 2]), pairs_sum<32>(sum[4 * x + 1], sum[4 * x + 3]));
    if (there[x]) *put[x] = kept_weight(a, s, key_out(x), old[x], mine);
  }
}

// The parts of a key's sum, in order; a block for each tile and head.
__global__ __launch_bounds__(256) void k_join_weights(Gather a, Cache c, Shares sp, int keys) {
  unsigned id = blockIdx.x;
  const int head = (int)(id % (unsigned)c.Hkv);
  id /= (unsigned)c.Hkv;
  const int tile = (int)(id % (unsigned)sp.tiles), owner = (int)(id / (unsigned)sp.tiles);
  const Share s = share_of(c, sp.prefix != 0, owner);
  const int key = tile * keys + (int)threadIdx.x;
  if (!s.valid || s.n <= 0 || key >= s.kv || (int)threadIdx.x >= keys) return;
  const long blocks = (long)(sp.prefix ? c.groups : c.B) * sp.tiles * c.Hkv;
  const int page = s.table[key >> c.page_shift];
  float sum = 0.f, old = 0.f;
  float* at = nullptr;
  for (int p0 = 0; p0 < sp.parts; p0 += 8) {  // (eight on their way together: 637 causal tokens of 32 heads in 32 bits 33.2 us, one by one 34.2)
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = sp.sums[(min(p0 + i, sp.parts - 1) * blocks + blockIdx.x) * keys + threadIdx.x];
    if (p0 == 0) {
      at = weight_at(a, c, head, key, page);
      if (a.carry != 0.f) old = *at;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += p0 + i < sp.parts ? v[i] : 0.f;
  }
  if ((unsigned)page < (unsigned)c.n_pages) *at = kept_weight(a, s, key, old, sum);
}

}  // namespace dart
