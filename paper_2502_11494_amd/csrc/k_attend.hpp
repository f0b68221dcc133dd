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

struct Attend {
  const void *q, *k_pool, *v_pool;
  void* out;
  float* lse;  // or nullptr
  long q_ld, out_ld;
  float scale;
  int causal;
};

// How a launch divides its keys, and where its results go.  A row's results are joined from `parts`
// partial ones (running sum, maximum and weighted values of some of its keys each), or written at
// once where there is one.
struct Parting {
  int prefix;      // the keys are the groups' shared prefixes (else each sequence's own)
  int chunk;       // keys of a part
  int first_part;  // part number of the launch's first chunk
  int parts;
  float* part_o;   // [parts][T*Hq][d]
  float2* part_ml; // [parts][T*Hq]: maximum (of scores times log2 e), sum
};

// ---- the arithmetic of a wave ----------------------------------------------------------------
// 32 queries lie in the columns of a 32x32 tile (lane % 32), 32 keys in its rows: a lane holds of
// its query the 16 keys 8*(i/4) + 4*(lane/32) + i%4.  So the maximum and the sum of a query are within
// a lane but for one exchange with lane ^ 32; the weights are, rounded, the right operand of the
// second product as they stand (its sum over keys does not mind their order, as long as the
// values are read in the same one), and its result has the queries in the columns again, so that
// rescaling it is a product by a number of the lane's own.
template <int DT>
struct Math;

template <>
struct Math<kBF16> {
  static constexpr int kVec = 8;                       // elements of a 16-byte piece
  typedef bf16x8 QFrag;
  template <int DP>
  static constexpr int steps() { return DP / 16; }     // of the first product
  // 8 elements from 16*s + 8*half of query or key `row`
  __device__ static __forceinline__ int piece(int s, int half) { return 2 * s + half; }
  __device__ static __forceinline__ f32x16 qk(const QFrag& k, const QFrag& q, f32x16 acc) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q, acc, 0, 0, 0);
  }
};

template <>
struct Math<kF32> {
  static constexpr int kVec = 4;
  typedef f32x4v QFrag;
  template <int DP>
  static constexpr int steps() { return DP / 8; }
  __device__ static __forceinline__ int piece(int s, int half) { return 2 * s + half; }
  // (four products of two elements each: element j of both halves' pieces)
  __device__ static __forceinline__ f32x16 qk(const QFrag& k, const QFrag& q, f32x16 acc) {
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(k[j], q[j], acc, 0, 0, 0);
    return acc;
  }
};

// Rows of a tile in LDS lie at multiples of their length, their 16-byte pieces permuted by the row
// so that neither 16 rows read at one piece (keys) nor 4 rows read at four (values) meet in the
// banks.
template <int RB>
__device__ __forceinline__ int mix(int row) {
  return RB == 128 ? (((row >> 1) & 1) << 2) | ((row >> 2) & 3) : ((row & 3) << 2) | ((row >> 2) & 3);
}

__device__ __forceinline__ float other_half_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float other_half_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <int DT>
__device__ __forceinline__ bool finite_piece(const u32x4& v) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (DT == kBF16) bad |= (v[i] & 0x7f80u) == 0x7f80u || (v[i] & 0x7f800000u) == 0x7f800000u;
    else bad |= (v[i] & 0x7f800000u) == 0x7f800000u;
  }
  return !bad;
}
// The rows of one block, and the keys they are taken against.
struct Tile {
  int tok0;          // first token of the sequence (or group)
  int rows;          // (token, head of the key head's group) pairs of it: token-major
  int n, kv;         // tokens; keys
  int shift;         // causal: token i sees keys up to kv - n + i; else unused
  const int* table;  // pages
};

__device__ __forceinline__ int token_of(const Cache& c, int b) {
  if (c.cu == nullptr) return b < c.B ? b : c.B;
  const int t = c.cu[b];
  return t < 0 ? 0 : t < c.T ? t : c.T;
}

// Tile slot -> (sequence or group, tile).  Sequence i of `count` owns the slots from start(i) =
// floor(first token * r / bm) + i on: at least as many as it has tiles, whatever its length, and found
// without a sum over the sequences before it.
template <int BM>
__device__ __forceinline__ int slot_owner(const Cache& c, const int* group_cu, int count, int r, long slot) {
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

// WM waves along the rows (QT tiles of 32 each) by WK along the keys; a step takes KT keys per key group.
template <int DT, int DP, int WM, int WK, int QT, int KT>
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
  static constexpr int kBM = 32 * WM * QT;
  static constexpr int kLds = WK * kBuffers * 2 * kTileBytes;
  static_assert(kGroup % kPieces == 0 && KT * kPieces % kGroup == 0 && KT % 32 == 0, "");
  static_assert(WK == 1 || (QT == 1 && WM == 1), "");
  static_assert(WK == 1 || 32 * DP * 4 <= kBuffers * 2 * kTileBytes, "joined in the tiles' place");
};

template <int DT, int DP, int WM, int WK, int QT, int KT>
__global__ __launch_bounds__(64 * WM * WK) void k_attend(Attend a, Cache c, Parting sp) {
  typedef AttendShape<DT, DP, WM, WK, QT, KT> S;
  typedef Math<DT> M;
  typedef typename M::QFrag QFrag;
  constexpr int kSteps = M::template steps<DP>(), kDT = DP / 32, kSub = KT / 32, RB = S::kRowBytes;
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ int odd_values[4];
  __shared__ float2 joined[WK + 1][32];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave % WM, wk = wave / WM;
  const int half = lane >> 5, col = lane & 31;
  const int r = c.Hq / c.Hkv, head = blockIdx.y;

  // ---- whose rows, which keys
  Tile tl;
  int tile;
  {
    const long slot = (long)gridDim.x - 1 - blockIdx.x;  // the tiles that see most keys first
    if (sp.prefix) {
      const int g = slot_owner<S::kBM>(c, c.group_cu, c.groups, r, slot);
      const int b0 = c.group_cu[g], b1 = c.group_cu[g + 1];
      const int n = prefix_of(c, g);
      const bool ok = n >= 0;
      if (!ok && threadIdx.x == 0) flag(c, kBadSequence);
      tl.tok0 = token_of(c, b0 < 0 ? 0 : b0 < c.B ? b0 : c.B);
      tl.n = ok ? token_of(c, b1) - tl.tok0 : 0;
      tl.kv = ok ? n : 0;
      tl.table = c.prefix_pages + (long)g * c.prefix_ld;
      tile = (int)(slot - ((long)tl.tok0 * r / S::kBM + g));
    } else {
      const int b = slot_owner<S::kBM>(c, nullptr, c.B, r, slot);
      const Seq s = sequence_of(c, b);
      if (!s.valid && threadIdx.x == 0) flag(c, kBadSequence);
      tl.tok0 = s.tok0;
      tl.n = s.n;
      tl.kv = s.kv;
      tl.table = c.pages + (long)b * c.pages_ld;
      tile = (int)(slot - ((long)s.tok0 * r / S::kBM + b));
    }
    tl.rows = tl.n > 0 ? tl.n * r : 0;
  }
  const int row0 = tile * S::kBM;
  if (tile < 0 || row0 >= tl.rows) return;
  const bool causal = a.causal && !sp.prefix;
  const int last_tok = ((row0 + S::kBM < tl.rows ? row0 + S::kBM : tl.rows) - 1) / r;
  int k1 = causal && tl.kv - tl.n + last_tok + 1 < tl.kv ? tl.kv - tl.n + last_tok + 1 : tl.kv;
  const int k0 = blockIdx.z * sp.chunk;
  if (k1 - k0 > sp.chunk) k1 = k0 + sp.chunk;
  if (k1 <= k0 && (sp.parts > 1 || blockIdx.z > 0)) return;

  // ---- this wave's queries: the last key each of them sees, and their pieces
  QFrag q[QT][kSteps];
  int lim[QT], tok[QT], qh[QT];
  const uint32_t flip = a.scale < 0.f ? (DT == kBF16 ? 0x80008000u : 0x80000000u) : 0u;  // (scores then scale by |scale|)
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int row = row0 + (wm * QT + t) * 32 + col;
    const bool in = row < tl.rows;
    const int i = (in ? row : tl.rows - 1) / r;
    tok[t] = in ? tl.tok0 + i : -1;
    qh[t] = head * r + (in ? row : tl.rows - 1) - i * r;
    lim[t] = causal ? tl.kv - tl.n + i : tl.kv - 1;
    if (lim[t] > k1 - 1) lim[t] = k1 - 1;
    const long at = (long)(tl.tok0 + i) * a.q_ld + (long)qh[t] * c.d;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int e = M::piece(s, half) * M::kVec;
      u32x4 v = {0, 0, 0, 0};
      if (e < c.d && a.scale != 0.f) {
        v = *reinterpret_cast<const u32x4*>(static_cast<const unsigned char*>(a.q) + (at + e) * S::kEsz);
        v ^= flip;
      }
      q[t][s] = __builtin_bit_cast(QFrag, v);
    }
  }
  // (scale 0: queries of zeros, so that a hidden score stays -infinity)
  const float scale2 = a.scale != 0.f ? fabsf(a.scale) * kLog2e : 1.f;
  const int lim_first = __builtin_amdgcn_readfirstlane(lim[0]);                 // of the wave's rows
  const int lim_block = causal ? min(tl.kv - tl.n + row0 / r, k1 - 1) : k1 - 1;  // of the block's

  // ---- staging: pieces of keys and values, through registers into LDS
  const int gt = threadIdx.x - wk * S::kGroup;
  const int my_row = gt / S::kPieces, my_piece = gt % S::kPieces;
  const bool my_on = my_piece * M::kVec < c.d;
  const unsigned char* kp = static_cast<const unsigned char*>(a.k_pool) + ((long)head * c.head_ld + my_piece * M::kVec) * S::kEsz;
  const unsigned char* vp = static_cast<const unsigned char*>(a.v_pool) + ((long)head * c.head_ld + my_piece * M::kVec) * S::kEsz;
  unsigned char* const my_lds = lds + wk * (S::kBuffers * 2 * S::kTileBytes);
  const int row_mask = (1 << c.page_shift) - 1;
  u32x4 kr[S::kLoads], vr[S::kLoads];
  int pg[S::kLoads];
  bool bad_page = false;
  auto load_pages = [&](int kb) {
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const int key = kb + my_row + i * S::kApart;
      pg[i] = key < k1 ? tl.table[key >> c.page_shift] : 0;
    }
  };
  auto load_tile = [&](int kb) {
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const int key = kb + my_row + i * S::kApart;
      kr[i] = u32x4{0, 0, 0, 0};
      vr[i] = u32x4{0, 0, 0, 0};  // (what lies behind the keys may be anything; its weight is 0, and 0 times NaN is NaN)
      int page = pg[i];
      if ((unsigned)page >= (unsigned)c.n_pages) page = 0, bad_page = true;
      const long off = ((long)page * c.page_ld + (long)(key & row_mask) * c.row_ld) * S::kEsz;
      if (key < k1 && my_on) {
        kr[i] = *reinterpret_cast<const u32x4*>(kp + off);
        vr[i] = *reinterpret_cast<const u32x4*>(vp + off);
      }
    }
  };
  auto store_tile = [&](unsigned char* buf, int kb, int it) {
    if (causal && kb + KT - 1 > lim_block) {
      // Some row does not see some of these keys.  Their weight is 0 there, but its product with a value
      // that is no number would be none either: such a tile is taken key by key (below).
      bool fine = true;
#pragma unroll
      for (int i = 0; i < S::kLoads; ++i) fine = fine && finite_piece<DT>(vr[i]);
      if (!fine) odd_values[(WM > 1 ? it : wk) & 3] = 1;
    }
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const int row = my_row + i * S::kApart;
      const int at = row * RB + ((my_piece ^ mix<RB>(row)) << 4);
      *reinterpret_cast<u32x4*>(buf + at) = kr[i];
      *reinterpret_cast<u32x4*>(buf + S::kTileBytes + at) = vr[i];
    }
  };

  f32x16 o[QT][kDT];
  float m[QT], l[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = kLowest;
    l[t] = 0.f;
#pragma unroll
    for (int i = 0; i < kDT; ++i) o[t][i] = f32x16{};
  }

  if (threadIdx.x < 4) odd_values[threadIdx.x] = 0;
  const int steps = (k1 - k0 + KT * WK - 1) / (KT * WK);
  const int kstep = KT * WK, kfirst = k0 + wk * KT;
  load_pages(kfirst);
  load_tile(kfirst);
  load_pages(kfirst + kstep);
  __syncthreads();

  for (int it = 0; it < steps; ++it) {
    const int kb = kfirst + it * kstep;
    unsigned char* buf = my_lds + (S::kBuffers > 1 ? (it & 1) * 2 * S::kTileBytes : 0);
    if (S::kBuffers == 1) __builtin_amdgcn_wave_barrier();
    store_tile(buf, kb, it);
    load_tile(kb + kstep);
    load_pages(kb + 2 * kstep);
    if (WM > 1) {
      __syncthreads();
      if (causal && threadIdx.x == 0) odd_values[(it + 3) & 3] = 0;  // the last step's, used again three steps on
    } else {
      __builtin_amdgcn_wave_barrier();
    }
    const bool odd = causal && kb + KT - 1 > lim_block && *(volatile int*)&odd_values[(WM > 1 ? it : wk) & 3] != 0;
    const unsigned char* kl = buf;
    const unsigned char* vl = buf + S::kTileBytes;
#pragma unroll
    for (int sub = 0; sub < kSub; ++sub) {
      f32x16 sc[QT];
#pragma unroll
      for (int t = 0; t < QT; ++t) sc[t] = f32x16{};
      const int krow = sub * 32 + col;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int at = krow * RB + ((M::piece(s, half) ^ mix<RB>(krow)) << 4);
        const QFrag kf = *reinterpret_cast<const QFrag*>(kl + at);
#pragma unroll
        for (int t = 0; t < QT; ++t) sc[t] = M::qk(kf, q[t][s], sc[t]);
      }
      const int first = kb + sub * 32;
      if (first + 31 > lim_first) {
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = first + 8 * (i / 4) + 4 * half + i % 4;
            sc[t][i] = key <= lim[t] ? sc[t][i] : -INFINITY;
          }
      }
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        float top = sc[t][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, sc[t][i]);
        top = other_half_max(top) * scale2;
        // The reference of the exponentials follows the maximum only where it has grown by more than a factor
        // of 2^6: until then the weights are at most 64, and nothing is rescaled.
        if (__any(top > m[t] + 6.f)) {
          const float now = fmaxf(m[t], top);
          const float keep = __builtin_amdgcn_exp2f(m[t] - now);
          m[t] = now;
          l[t] *= keep;
#pragma unroll
          for (int i = 0; i < kDT; ++i) o[t][i] *= keep;
        }
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          sc[t][i] = __builtin_amdgcn_exp2f(fmaf(sc[t][i], scale2, -m[t]));
          sum += sc[t][i];
        }
        l[t] += sum;
      }
      if (__builtin_expect(odd, 0)) {
#pragma unroll 1
        for (int kk = 0; kk < 32; ++kk) {
          const int row = sub * 32 + kk;
#pragma unroll
          for (int t = 0; t < QT; ++t) {
            float w = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) w = 8 * (i / 4) + i % 4 == (kk & ~4) ? sc[t][i] : w;
            w = __shfl(w, col + 32 * ((kk >> 2) & 1));
            if (DT == kBF16) w = bf16_lo(bf16_pair(w, 0.f));
            const bool seen = first + kk <= lim[t];
#pragma unroll
            for (int i = 0; i < kDT; ++i)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const int e = i * 32 + 8 * j + 4 * half;
                const int at = row * RB + (((e / M::kVec) ^ mix<RB>(row)) << 4) + (e % M::kVec) * S::kEsz;
                Piece<DT, 4> v;
                __builtin_memcpy(&v, __builtin_assume_aligned(vl + at, sizeof v), sizeof v);
#pragma unroll
                for (int k = 0; k < 4; ++k) o[t][i][4 * j + k] = seen ? fmaf(w, v.get(k), o[t][i][4 * j + k]) : o[t][i][4 * j + k];
              }
          }
        }
        continue;
      }
      if constexpr (DT == kBF16) {
        bf16x8 p[QT][2];
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = bf16_pair(sc[t][8 * s + 2 * i], sc[t][8 * s + 2 * i + 1]);
            p[t][s] = __builtin_bit_cast(bf16x8, w);
          }
        // values: four keys at a lane's column of 32, by the transposing read of 16 lanes
        const int vrow = 4 * half + ((lane & 15) >> 2);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < kDT; ++i) {
            bf16x8 vf;
            i16x4 part[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const int row = sub * 32 + 16 * s + 8 * j + vrow;
              const int piece = i * 4 + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
              const int at = row * RB + ((piece ^ mix<RB>(row)) << 4) + 8 * (lane & 1);
              part[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                  (__attribute__((address_space(3))) i16x4*)(vl + at));
            }
            const u32x4 both = {__builtin_bit_cast(uint2, part[0]).x, __builtin_bit_cast(uint2, part[0]).y,
                                __builtin_bit_cast(uint2, part[1]).x, __builtin_bit_cast(uint2, part[1]).y};
            vf = __builtin_bit_cast(bf16x8, both);
#pragma unroll
            for (int t = 0; t < QT; ++t) o[t][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, p[t][s], o[t][i], 0, 0, 0);
          }
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int row = sub * 32 + 8 * (j / 4) + 4 * half + j % 4;
#pragma unroll
          for (int i = 0; i < kDT; ++i) {
            const int at = row * RB + (((i * 8 + (col >> 2)) ^ mix<RB>(row)) << 4) + 4 * (col & 3);
            const float vf = *reinterpret_cast<const float*>(vl + at);
#pragma unroll
            for (int t = 0; t < QT; ++t) o[t][i] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, sc[t][j], o[t][i], 0, 0, 0);
          }
        }
      }
    }
  }
  if (bad_page) flag(c, kBadPage);
#pragma unroll
  for (int t = 0; t < QT; ++t) l[t] = other_half_sum(l[t]);

  const long all = (long)c.T * c.Hq;
  if constexpr (WK == 1) {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      if (tok[t] < 0) continue;
      const long id = (long)tok[t] * c.Hq + qh[t];
      if (sp.parts > 1) {
        const long at = (sp.first_part + blockIdx.z) * all + id;
        if (half == 0) sp.part_ml[at] = make_float2(m[t], l[t]);
#pragma unroll
        for (int i = 0; i < kDT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int e = i * 32 + 8 * j + 4 * half;
            if (e < c.d)
              *reinterpret_cast<f32x4v*>(sp.part_o + at * c.d + e) =
                  f32x4v{o[t][i][4 * j], o[t][i][4 * j + 1], o[t][i][4 * j + 2], o[t][i][4 * j + 3]};
          }
        continue;
      }
      const float inv = l[t] == 0.f ? 0.f : 1.f / l[t];
      if (a.lse != nullptr && half == 0) a.lse[id] = l[t] == 0.f ? -INFINITY : (m[t] + log2f(l[t])) * kLn2;
      const long at = (long)tok[t] * a.out_ld + (long)qh[t] * c.d;
#pragma unroll
      for (int i = 0; i < kDT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int e = i * 32 + 8 * j + 4 * half;
          if (e >= c.d) continue;
          float x[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) x[k] = o[t][i][4 * j + k] * inv;
          store_piece<DT, 4>(a.out, at + e, round_piece<DT, 4>(x));
        }
    }
  } else {
    // The key groups' results are joined in LDS, in the tiles' place.
    if (half == 0) joined[wk][col] = make_float2(m[0], l[0]);
    __syncthreads();
    float top = kLowest, total = 0.f;
#pragma unroll
    for (int w = 0; w < WK; ++w) top = fmaxf(top, joined[w][col].x);
#pragma unroll
    for (int w = 0; w < WK; ++w) total += joined[w][col].y * __builtin_amdgcn_exp2f(joined[w][col].x - top);
    const float mine = __builtin_amdgcn_exp2f(m[0] - top);
    float* mat = reinterpret_cast<float*>(my_lds);
#pragma unroll
    for (int i = 0; i < kDT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int piece = i * 8 + 2 * j + half;  // (of four elements)
        *reinterpret_cast<f32x4v*>(mat + col * DP + ((piece ^ (col & 7)) << 2)) =
            f32x4v{o[0][i][4 * j] * mine, o[0][i][4 * j + 1] * mine, o[0][i][4 * j + 2] * mine, o[0][i][4 * j + 3] * mine};
      }
    if (wk == 0 && half == 0) joined[WK][col] = make_float2(top, total);
    __syncthreads();
    constexpr int kQuads = DP / 4;
    for (int e = threadIdx.x; e < 32 * kQuads; e += S::kThreads) {
      const int rr = e / kQuads, piece = e % kQuads, row = row0 + rr;
      if (row >= tl.rows || piece * 4 >= c.d) continue;
      f32x4v x = {};
#pragma unroll
      for (int w = 0; w < WK; ++w)
        x += *reinterpret_cast<const f32x4v*>(reinterpret_cast<const float*>(lds + w * (S::kBuffers * 2 * S::kTileBytes)) + rr * DP +
                                              ((piece ^ (rr & 7)) << 2));
      const int i = row / r, h = head * r + row - i * r;
      const long id = (long)(tl.tok0 + i) * c.Hq + h;
      const float2 ml = joined[WK][rr];
      if (sp.parts > 1) {
        const long at = (sp.first_part + blockIdx.z) * all + id;
        if (piece == 0) sp.part_ml[at] = ml;
        *reinterpret_cast<f32x4v*>(sp.part_o + at * c.d + piece * 4) = x;
        continue;
      }
      const float inv = ml.y == 0.f ? 0.f : 1.f / ml.y;
      if (a.lse != nullptr && piece == 0) a.lse[id] = ml.y == 0.f ? -INFINITY : (ml.x + log2f(ml.y)) * kLn2;
      const float y[4] = {x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
      store_piece<DT, 4>(a.out, (long)(tl.tok0 + i) * a.out_ld + (long)h * c.d + piece * 4, round_piece<DT, 4>(y));
    }
  }
}

// Joins a row's parts: 2^lanes_shift lanes per row, four elements each.
template <int DT>
__global__ __launch_bounds__(256) void k_attend_join(Attend a, Cache c, int pre_chunk, int pre_parts, int own_chunk, const float* part_o,
                                                     const float2* part_ml, int lanes_shift) {
  const long all = (long)c.T * c.Hq;
  const int lane = threadIdx.x & 63;
  const long first = ((long)blockIdx.x * 4 + (threadIdx.x >> 6)) << (6 - lanes_shift);
  const long id = first + (lane >> lanes_shift);
  const int t0 = (int)(first / c.Hq);
  int b0 = 0;
  if (c.cu != nullptr && first < all) b0 = owner_of(c.cu, c.B, t0);
  if (id >= all) return;
  const int t = (int)(id / c.Hq), h = (int)(id - (long)t * c.Hq);
  int b = c.cu == nullptr ? t : b0;
  if (c.cu != nullptr)
    while (b + 1 < c.B && c.cu[b + 1] <= t) ++b;  // (a wave's rows are a few tokens')
  const Seq s = sequence_of(c, b);
  int own = s.kv;
  if (a.causal && s.kv - s.n + (t - s.tok0) + 1 < own) own = s.kv - s.n + (t - s.tok0) + 1;
  if (t < s.tok0 || t >= s.tok0 + s.n) return;  // no sequence's token
  int prefix = 0;
  if (c.groups > 0) {
    int g = 0, end = c.groups;
    while (end - g > 1) {
      const int mid = (g + end) / 2;
      if (c.group_cu[mid] <= b) g = mid; else end = mid;
    }
    prefix = prefix_of(c, g);
    if (prefix < 0 || b < c.group_cu[g] || b >= c.group_cu[g + 1]) {
      flag(c, kBadSequence);
      prefix = own = 0;
    }
  }
  if (!s.valid) prefix = own = 0;
  const int np = prefix > 0 ? (prefix + pre_chunk - 1) / pre_chunk : 0;
  const int no = own > 0 ? (own + own_chunk - 1) / own_chunk : 0;
  const int e = (lane & ((1 << lanes_shift) - 1)) * 4;
  const bool in = e < c.d;
  float top = kLowest, l = 0.f;
  f32x4v x = {};
  for (int i = 0; i < np + no; ++i) {
    const long at = (i < np ? i : pre_parts + i - np) * all + id;
    const float2 ml = part_ml[at];
    const f32x4v y = in ? *reinterpret_cast<const f32x4v*>(part_o + at * c.d + e) : f32x4v{};
    const float now = fmaxf(top, ml.x);
    const float f = __builtin_amdgcn_exp2f(top - now), w = __builtin_amdgcn_exp2f(ml.x - now);
    top = now;
    l = l * f + ml.y * w;
    x = x * f + y * w;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (a.lse != nullptr && e == 0) a.lse[id] = l == 0.f ? -INFINITY : (top + log2f(l)) * kLn2;
  if (!in) return;
  const float y[4] = {x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
  store_piece<DT, 4>(a.out, (long)t * a.out_ld + (long)h * c.d + e, round_piece<DT, 4>(y));
}

}  // namespace dart
