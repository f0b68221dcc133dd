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
  int parts;   // of the rows
  float* sums; // [parts][blocks of a part][keys of a tile], where there is more than one part
};

// 32 keys by 32 queries: keys in the rows of the product, queries in its columns.
template <int DT>
struct Tile32 {
  static constexpr int kVec = DT == kBF16 ? 8 : 4;
  __device__ static __forceinline__ f32x16 product(const u32x4& k, const u32x4& q, f32x16 c) {
    if constexpr (DT == kBF16) {
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q), c, 0, 0, 0);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[j]), __uint_as_float(q[j]), c, 0, 0, 0);
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
  static constexpr int kLoads = 32 * kPieces / 256 > 0 ? 32 * kPieces / 256 : 1;
  static constexpr int kTile = 32 * kRowBytes;
  static constexpr int kLds = 2 * kTile;
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

__device__ __forceinline__ void put_weight(const Gather& a, const Cache& c, const Share& s, int head, int key, float sum) {
  const int page = s.table[key >> c.page_shift];
  if ((unsigned)page >= (unsigned)c.n_pages) return;  // (flagged where its key was asked for)
  float* at = a.weights + (((long)page * c.Hkv + head) << c.page_shift) + (key & ((1 << c.page_shift) - 1));
  *at = a.carry == 0.f || key >= s.fresh ? sum : fmaf(a.carry, *at, sum);
}

// w_j <- carry * w_j + sum over the rows that see key j of exp(scale <q, k_j> - lse).  A wave holds its keys in registers
// and goes through the rows 32 at a time, which the block brings to LDS while it works on those before.  Sums in 32 bits, those
// of 16 tiles of rows by themselves.
template <int DT, int DP, class HELD>
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void k_gather_weights(Gather a, Cache c, Shares sp, unsigned first) {
  typedef GatherShape<DT, DP> S;
  typedef Tile32<DT> M;
  constexpr int KW = S::KW, RB = S::kRowBytes, kSteps = DP / (2 * M::kVec);
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ float2 row_of[2][32];  // a row's lse times log2 e, and the last key that it sees
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
  // the rows from the first on that sees the first key of the tile, 32 at a time, dealt to the parts
  const int row_first = causal ? max(0, k0 - s.fresh) * r : 0;
  const int all = (rows - row_first + 31) / 32;
  const int t0 = (int)((long)all * part / sp.parts), t1 = (int)((long)all * (part + 1) / sp.parts);

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

  // ---- rows to LDS
  const int my_piece = threadIdx.x % S::kPieces, my_row = threadIdx.x / S::kPieces;
  constexpr int kApart = 256 / S::kPieces;
  u32x4 qr[S::kLoads];
  float2 mine;
  auto load_rows = [&](int t) {
    const int row0 = row_first + t * 32;
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const int row = min(row0 + my_row + i * kApart, rows - 1), tok = (int)(((double)row + 0.5) * a.per_token);
      const long at = (long)(s.tok0 + tok) * a.q_ld + (long)(head * r + row - tok * r) * c.d + my_piece * M::kVec;
      qr[i] = u32x4{0, 0, 0, 0};
      if (my_piece * M::kVec < c.d && a.scale != 0.f && my_row < 32)
        qr[i] = *reinterpret_cast<const u32x4*>(static_cast<const unsigned char*>(a.q) + at * (16 / M::kVec));
    }
    if (threadIdx.x < 32) {
      const int row = row0 + (int)threadIdx.x, have = min(row, rows - 1), tok = (int)(((double)have + 0.5) * a.per_token);
      const float lse = a.lse[(long)(s.tok0 + tok) * c.Hq + head * r + have - tok * r];
      // (a row past the last, or one that saw nothing, gives nothing to any key)
      const int lim = row >= rows || lse == -INFINITY ? -1 : causal ? min(s.fresh + tok, last_key) : last_key;
      mine = make_float2(lse * kLog2e, __int_as_float(lim));
    }
  };
  auto store_rows = [&](int t) {
    unsigned char* to = lds + (t & 1) * S::kTile;
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const int row = my_row + i * kApart;
      if (row < 32) *reinterpret_cast<u32x4*>(to + row * RB + ((my_piece ^ mix<RB>(row)) << 4)) = qr[i];
    }
    if (threadIdx.x < 32) row_of[t & 1][threadIdx.x] = mine;
  };

  const float scale2 = a.scale * kLog2e;
  const int my_k0 = k0 + wave * KW * 32, my_end = my_k0 + KW * 32 - 1;
  f32x16 sum[KW], total[KW];
#pragma unroll
  for (int w = 0; w < KW; ++w) sum[w] = total[w] = f32x16{};
  if (t0 < t1) load_rows(t0);
  for (int t = t0; t < t1; ++t) {
    store_rows(t);
    __syncthreads();
    if (t + 1 < t1) load_rows(t + 1);
    const unsigned char* from = lds + (t & 1) * S::kTile;
    f32x16 x[KW];
#pragma unroll
    for (int w = 0; w < KW; ++w) x[w] = f32x16{};
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
      const u32x4 q = *reinterpret_cast<const u32x4*>(from + col * RB + ((piece(st) ^ mix<RB>(col)) << 4));
#pragma unroll
      for (int w = 0; w < KW; ++w) x[w] = M::product(k[w][st], q, x[w]);
    }
    const float2 row = row_of[t & 1][col];
    const int lim = __float_as_int(row.y);
    if (__any(lim < my_end)) {
#pragma unroll
      for (int w = 0; w < KW; ++w)
#pragma unroll
        for (int u = 0; u < 16; ++u) {
          const int key = my_k0 + w * 32 + 8 * (u / 4) + 4 * grp + u % 4;
          const float y = __builtin_amdgcn_exp2f(fmaf(x[w][u], scale2, -row.x));
          sum[w][u] += key <= lim ? y : 0.f;
        }
    } else {
#pragma unroll
      for (int w = 0; w < KW; ++w)
#pragma unroll
        for (int u = 0; u < 16; ++u) sum[w][u] += __builtin_amdgcn_exp2f(fmaf(x[w][u], scale2, -row.x));
    }
    if ((t - t0) % 16 == 15) {
#pragma unroll
      for (int w = 0; w < KW; ++w) total[w] += sum[w], sum[w] = f32x16{};
    }
  }

  // ---- over the 32 columns: half the values go to the partner lane each time
  __syncthreads();
  float* out = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int w = 0; w < KW; ++w) {
    float v[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) v[u] = total[w][u] + sum[w][u];
#pragma unroll
    for (int half = 8; half >= 1; half /= 2) {
      const bool high = (col & half) != 0;
#pragma unroll
      for (int u = 0; u < half; ++u) {
        const float give = high ? v[u] : v[u + half], keep = high ? v[u + half] : v[u];
        v[u] = keep + __shfl_xor(give, half);
      }
    }
    v[0] += __shfl_xor(v[0], 16);
    const int u = col & 15;
    if (col < 16) out[wave * KW * 32 + w * 32 + 8 * (u / 4) + 4 * grp + u % 4] = v[0];
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
  float sum = 0.f;
  for (int p = 0; p < sp.parts; ++p) sum += sp.sums[(p * blocks + blockIdx.x) * keys + threadIdx.x];
  put_weight(a, c, s, head, key, sum);
}

}  // namespace dart
