// Eviction: the keys of a cache that are kept, and the move of their rows to the front of their pages.
#pragma once

#include "cache.hpp"

namespace dart {

struct Evict {
  int budget, num, den, first, recent;
  const float* weights;
  float* weights_out;     // or nullptr
  int* kept;              // [B][Hkv], kept_ld apart
  long kept_ld;
  int2* left;             // [B]: keys kept, or ~keys of a sequence that stays as it is; keys it then has
  int* kv_len_out;
};

// Keys that a sequence of kv keeps.
__host__ __device__ inline int keys_kept(int budget, int num, int den, int first, int recent, int kv) {
  const long k = budget > 0 ? (long)budget : (long)kv * num / den;
  const long least = (long)first + recent;
  const long keep = k < least ? least : k;
  return keep < kv ? (int)keep : kv;
}

// A weight as a number whose order is the weights'; NaN is the least, and zeros are alike.
__device__ __forceinline__ uint32_t order_of(float w) {
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
  return w != w ? 0u : u >> 31 ? ~u : u | 0x80000000u;
}

constexpr int kBuckets = 2048, kListed = 128;

// What a block of W waves keeps in LDS.
template <int W>
struct SelectShared {
  int bucket[kBuckets];
  uint32_t low[W], high[W];
  int wave_sum[W];
  int found, before, inside, bad, listed, last;
  uint32_t border;
  unsigned long long list[kListed];  // weights about the border, and below them places from the last on
};

// Over the lanes up to this one.
__device__ __forceinline__ int lanes_sum(int x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// Chooses the keys of one key head of one sequence: `first` and `recent` ones, and of those between the ones of largest weight,
// of equals the first.  The border is the last key taken, by (weight, place).  It is found from the top: the range of the weights that
// are left, as whole numbers of their order, is cut in 2048 buckets, and the one that the border falls in is the next range,
// until so few weights are left that each is compared with all others, or all that are left are alike.  Then the keys up to the
// border are counted to their places in order.  A block of W waves, a wave H times 64 keys in a row; so many keys (H * W * 64)
// are read once and held in registers, longer sequences are read again by every step.  Bound by latency, a few looks into memory and
// LDS one after the other: 637 keys of 32 heads 7 us; 32 sequences of 1024 to 16 384 keys, 4 heads (128 blocks), 25 us, 5 each in the range,
// two cuts and the places.
template <int W, int H>
__global__ __launch_bounds__(W * kWave) void k_evict_select(Evict a, Cache c) {
  __shared__ SelectShared<W> sh;
  constexpr int kThreads = W * kWave, kHeld = kThreads * H;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long pairs = (long)c.B * c.Hkv;
  for (long id = blockIdx.x; id < pairs; id += gridDim.x) {
    const int b = (int)(id / c.Hkv), h = (int)(id - (long)b * c.Hkv);
    const int kv = c.kv_len[b];
    const bool valid = kv >= 0 && kv <= c.max_kv && (long)kv <= ((long)c.pages_n << c.page_shift);
    const int keep = valid ? keys_kept(a.budget, a.num, a.den, a.first, a.recent, kv) : -1;
    if (tid == 0 && h == 0) {
      a.left[b] = make_int2(!valid ? ~0 : keep == kv ? ~keep : keep, valid ? keep : kv);
      if (!valid) flag(c, kBadSequence);
    }
    if (!valid) continue;
    int* kept = a.kept + id * a.kept_ld;
    const int* table = c.pages + (long)b * c.pages_ld;
    // The pages of all keys, by the first head's block for all heads: the choice looks at some keys only, the move at those kept.
    bool missing = false;
    if (h == 0)
      for (int p = tid; p <= (kv - 1) >> c.page_shift; p += kThreads) missing |= (unsigned)table[p] >= (unsigned)c.n_pages;
    if (keep == kv) {
      if (missing) flag(c, kBadPage);
      for (int j = tid; j < kv; j += kThreads) kept[j] = j;
      continue;
    }
    // candidates first .. first + n - 1, of which `want` are taken
    const int n = kv - a.recent - a.first, want = keep - a.recent - a.first;
    for (int j = tid; j < a.first; j += kThreads) kept[j] = j;
    for (int j = tid; j < a.recent; j += kThreads) kept[a.first + want + j] = kv - a.recent + j;
    const int groups = (n + kHeld - 1) / kHeld;
    uint32_t u[H];
    auto place = [&](int g, int i) { return g * kHeld + (wave * H + i) * kWave + lane; };
    auto load = [&](int g) {
      int page[H];
#pragma unroll
      for (int i = 0; i < H; ++i) page[i] = table[(a.first + min(place(g, i), n - 1)) >> c.page_shift];
#pragma unroll
      for (int i = 0; i < H; ++i) {
        const bool none = (unsigned)page[i] >= (unsigned)c.n_pages;
        const int row = (a.first + min(place(g, i), n - 1)) & ((1 << c.page_shift) - 1);
        const float w = a.weights[(((long)(none ? 0 : page[i]) * c.Hkv + h) << c.page_shift) + row];
        u[i] = none ? 0u : order_of(w);
      }
    };

    // ---- the range of the weights (past the last the last again)
    uint32_t lo = 0xffffffffu, hi = 0;
    for (int g = 0; g < groups; ++g) {
      load(g);
#pragma unroll
      for (int i = 0; i < H; ++i) lo = u[i] < lo ? u[i] : lo, hi = u[i] > hi ? u[i] : hi;
    }
    for (int x = tid; x < kBuckets; x += kThreads) sh.bucket[x] = 0;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const uint32_t l = __shfl_xor(lo, o), m = __shfl_xor(hi, o);
      lo = l < lo ? l : lo, hi = m > hi ? m : hi;
    }
    if (lane == 0) sh.low[wave] = lo, sh.high[wave] = hi;
    if (tid == 0) sh.bad = 0, sh.listed = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) {
      lo = sh.low[w] < lo ? sh.low[w] : lo;
      hi = sh.high[w] > hi ? sh.high[w] : hi;
    }
    if (missing) sh.bad = 1;

    // ---- the border: [lo, lo + 2^bits) holds it; `need` of the weights in it are taken, all above are
    int bits = hi == lo ? 0 : 32 - __builtin_clz(hi - lo), need = want, inside = n;
    while (bits > 0 && need > 0 && inside > kListed) {
      const int shift = bits > 11 ? bits - 11 : 0;
      const uint32_t used = 1u << (bits - shift);  // buckets
      for (int g = 0; g < groups; ++g) {
        if (groups > 1) load(g);
#pragma unroll
        for (int i = 0; i < H; ++i) {
          const uint32_t x = (u[i] - lo) >> shift;  // (weights below lo are far above)
          if (place(g, i) < n && x < used) atomicAdd(&sh.bucket[x], 1);
        }
      }
      __syncthreads();
      // a thread's run of buckets, from the top; weights above it, from the sums of the lanes and the waves above
      constexpr int kRun = kBuckets / kThreads;
      int mine[kRun], all = 0;
      const int top = kBuckets - 1 - kRun * tid;
#pragma unroll
      for (int i = 0; i < kRun; ++i) mine[i] = sh.bucket[top - i], all += mine[i], sh.bucket[top - i] = 0;
      const int upto = lanes_sum(all);
      if (lane == kWave - 1) sh.wave_sum[wave] = upto;
      __syncthreads();
      int over = upto - all;
#pragma unroll
      for (int w = 0; w < W; ++w) over += w < wave ? sh.wave_sum[w] : 0;
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        if (over < need && need <= over + mine[i]) sh.found = top - i, sh.before = over, sh.inside = mine[i];
        over += mine[i];
      }
      __syncthreads();
      lo += (uint32_t)sh.found << shift;
      need -= sh.before;
      inside = sh.inside;
      bits = shift;
    }
    const uint32_t span = bits >= 32 ? 0xffffffffu : (1u << bits) - 1u;
    if (tid == 0) sh.border = 0xffffffffu, sh.last = -1;  // (nothing wanted)
    if (need > 0 && inside <= kListed) {
      for (int g = 0; g < groups; ++g) {
        if (groups > 1) load(g);
        uint32_t in = 0;
        int all = 0, at = 0;
#pragma unroll
        for (int i = 0; i < H; ++i) {
          const bool x = place(g, i) < n && u[i] - lo <= span;
          in |= (x ? 1u : 0u) << i;
          all += __popcll(__ballot(x));
        }
        if (lane == 0 && all > 0) at = atomicAdd(&sh.listed, all);  // (in any order)
        at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
        for (int i = 0; i < H; ++i) {
          const unsigned long long m = __ballot(in >> i & 1);
          if (in >> i & 1) sh.list[at + __popcll(m & ((1ull << lane) - 1ull))] = (unsigned long long)u[i] << 32 | ~(uint32_t)place(g, i);
          at += __popcll(m);
        }
      }
      __syncthreads();
      // a wave compares its entries with all of them, which its lanes hold
      constexpr int kPer = kListed / kWave;
      unsigned long long all[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) all[i] = i * kWave + lane < inside ? sh.list[i * kWave + lane] : 0ull;
      for (int x = wave; x < inside; x += W) {
        const unsigned long long mine = sh.list[x];
        int before = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) before += __popcll(__ballot(all[i] > mine));
        if (before == need - 1 && lane == 0) sh.border = (uint32_t)(mine >> 32), sh.last = (int)~(uint32_t)mine;
      }
    } else if (need > 0) {  // all alike: the need-th of them in order
      int done = 0;
      for (int g = 0; g < groups; ++g) {
        if (groups > 1) load(g);
        int all = 0;
#pragma unroll
        for (int i = 0; i < H; ++i) all += __popcll(__ballot(place(g, i) < n && u[i] == lo));
        if (lane == 0) sh.wave_sum[wave] = all;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) done += w < wave ? sh.wave_sum[w] : 0;
#pragma unroll
        for (int i = 0; i < H; ++i) {
          const bool same = place(g, i) < n && u[i] == lo;
          const unsigned long long e = __ballot(same);
          if (same && done + __popcll(e & ((1ull << lane) - 1ull)) == need - 1) sh.border = lo, sh.last = place(g, i);
          done += __popcll(e);
        }
#pragma unroll
        for (int w = 0; w < W; ++w) done += w > wave ? sh.wave_sum[w] : 0;
        __syncthreads();
      }
    }
    __syncthreads();
    const uint32_t border = sh.border;
    const int last = sh.last;

    // ---- places, by wave, round and lane
    int done = 0;
    for (int g = 0; g < groups; ++g) {
      if (groups > 1) load(g);
      uint32_t taken = 0;
      int all = 0;
#pragma unroll
      for (int i = 0; i < H; ++i) {
        const bool t = place(g, i) < n && (u[i] > border || (u[i] == border && place(g, i) <= last));
        taken |= (t ? 1u : 0u) << i;
        all += __popcll(__ballot(t));
      }
      if (lane == 0) sh.wave_sum[wave] = all;
      __syncthreads();
      int to = done;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const int x = sh.wave_sum[w];
        done += x;
        to += w < wave ? x : 0;
      }
#pragma unroll
      for (int i = 0; i < H; ++i) {
        const unsigned long long m = __ballot(taken >> i & 1);
        if (taken >> i & 1) kept[a.first + to + __popcll(m & ((1ull << lane) - 1ull))] = a.first + place(g, i);
        to += __popcll(m);
      }
      __syncthreads();
    }
    if (tid == 0 && sh.bad) flag(c, kBadPage);
    __syncthreads();
  }
}

// Row i of a key head takes row kept[i] >= i.  A block has one column of one array of one key head of one sequence and goes through
// its rows from the front, a chunk at a time: a chunk's rows are read, then written.  What it writes has been read, by itself or
// before: row i is the source of no row after i.  So no copy of the rows is needed, and blocks do not wait for one another.  Bound by
// memory: 64 sequences of 2100 keys to 2048 in bf16 4.8 TB/s, choice included; those 32 to 11.1 %, 127 MB, 36 us, 27 where the call before
// left some of the rows in the last cache.
struct Column {
  unsigned char* from;
  unsigned char* to;
  long page_ld, head_ld, row_ld;  // bytes
};

template <class T, int ROWS>
__device__ __forceinline__ void move_rows(const Cache& c, const Column& col, const int* table, const int* kept, int keep, int h,
                                          int lanes_shift, bool on, long at) {
  const int tid = threadIdx.x, row = tid >> lanes_shift, per = (int)blockDim.x >> lanes_shift;
  const int mask = (1 << c.page_shift) - 1;
  for (int i0 = 0; i0 < keep; i0 += per * ROWS) {
    T v[ROWS];
    int src[ROWS];
    bool go[ROWS];
#pragma unroll
    for (int x = 0; x < ROWS; ++x) {
      const int i = i0 + x * per + row;
      src[x] = i < keep ? kept[i] : 0;
      go[x] = on && i < keep && (src[x] != i || col.from != col.to);
    }
    int page[ROWS], page_to[ROWS];
#pragma unroll
    for (int x = 0; x < ROWS; ++x) {
      const int i = i0 + x * per + row;
      page[x] = table[src[x] >> c.page_shift];
      page_to[x] = table[(i < keep ? i : 0) >> c.page_shift];
    }
#pragma unroll
    for (int x = 0; x < ROWS; ++x) {
      go[x] = go[x] && (unsigned)page[x] < (unsigned)c.n_pages && (unsigned)page_to[x] < (unsigned)c.n_pages;
      if (go[x]) v[x] = *reinterpret_cast<const T*>(col.from + (long)page[x] * col.page_ld + (long)h * col.head_ld + (long)(src[x] & mask) * col.row_ld + at);
    }
    stores_done();  // (every load of the wave has come back)
    __syncthreads();
#pragma unroll
    for (int x = 0; x < ROWS; ++x) {
      const int i = i0 + x * per + row;
      if (go[x]) *reinterpret_cast<T*>(col.to + (long)page_to[x] * col.page_ld + (long)h * col.head_ld + (long)(i & mask) * col.row_ld + at) = v[x];
    }
  }
}

// The arrays that move: rows of keys and values in columns of up to 128 bytes, their scales, weights.
struct Moves {
  Column col[5];
  int kind[5];         // bytes that a lane takes: 16, 4 or 1
  int units[5];        // of them in a row; 0: there is no such array
  int lanes_shift[5];  // 2^lanes_shift lanes to a row of a column
  int end[5];          // columns up to the end of this array
};

__global__ __launch_bounds__(1024) void k_evict_move(Evict a, Cache c, Moves m) {
  const int columns = m.end[4];
  const long all = (long)c.B * c.Hkv * columns;
  for (long id = blockIdx.x; id < all; id += gridDim.x) {
    const long pair = id / columns;
    const int column = (int)(id - pair * columns), b = (int)(pair / c.Hkv), h = (int)(pair - (long)b * c.Hkv);
    const int2 left = a.left[b];
    if (column == 0 && h == 0 && threadIdx.x == 0) a.kv_len_out[b] = left.y;
    int x = 0;
    while (column >= m.end[x]) ++x;
    const int keep = left.x < 0 ? ~left.x : left.x;
    if (left.x < 0 && m.col[x].from == m.col[x].to) continue;
    const int shift = m.lanes_shift[x], unit = ((column - (x ? m.end[x - 1] : 0)) << shift) + ((int)threadIdx.x & ((1 << shift) - 1));
    const bool on = unit < m.units[x];
    const int* table = c.pages + (long)b * c.pages_ld;
    const int* kept = a.kept + pair * a.kept_ld;
    if (m.kind[x] == 16) move_rows<u32x4, 8>(c, m.col[x], table, kept, keep, h, shift, on, (long)unit * 16);
    else if (m.kind[x] == 4) move_rows<uint32_t, 8>(c, m.col[x], table, kept, keep, h, shift, on, (long)unit * 4);
    else move_rows<uint8_t, 8>(c, m.col[x], table, kept, keep, h, shift, on, (long)unit);
  }
}

}  // namespace dart
