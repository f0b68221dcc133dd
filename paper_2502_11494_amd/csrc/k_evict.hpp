// Eviction: the keys of a cache that are kept, and the move of their rows to the front of their pages.
#pragma once

#include "cache.hpp"

namespace dart {

struct Evict {
  int budget, num, den, first, recent;
  int most;               // keys that any sequence keeps, at most
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

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / kWave;
constexpr int kSelectHeld = 16;  // keys of a thread that it holds
constexpr int kBuckets = 2048;

struct SelectShared {
  int bucket[kBuckets];
  uint32_t low[kSelectWaves], high[kSelectWaves];
  int wave_sum[kSelectWaves];
  int found, before, inside, bad;
  int above[kSelectHeld * kSelectWaves], equal[kSelectHeld * kSelectWaves];
};

// Chooses the keys of one key head of one sequence: `first` and `recent` ones, and of those between the ones of largest weight,
// of equals the first.  The border is found from the top: the range of the weights that are left, as whole numbers of their
// order, is cut in 2048 buckets, and the one that the border falls in is the next range.  Then the keys are counted up to their
// places in order.  A block of 16 waves; up to 16 384 keys are read once and held in registers.
__global__ __launch_bounds__(kSelectThreads) void k_evict_select(Evict a, Cache c) {
  __shared__ SelectShared sh;
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
    if (keep == kv) {
      for (int j = tid; j < kv; j += kSelectThreads) kept[j] = j;
      continue;
    }
    const int* table = c.pages + (long)b * c.pages_ld;
    // candidates first .. first + n - 1, of which `want` are taken
    const int n = kv - a.recent - a.first, want = keep - a.recent - a.first;
    for (int j = tid; j < a.first; j += kSelectThreads) kept[j] = j;
    for (int j = tid; j < a.recent; j += kSelectThreads) kept[a.first + want + j] = kv - a.recent + j;
    const int groups = (n + kSelectHeld * kSelectThreads - 1) / (kSelectHeld * kSelectThreads);
    uint32_t u[kSelectHeld];
    bool bad = false;
    auto load = [&](int g) {
      int page[kSelectHeld];
#pragma unroll
      for (int i = 0; i < kSelectHeld; ++i) {
        const int x = (g * kSelectHeld + i) * kSelectThreads + tid;
        page[i] = table[(a.first + (x < n ? x : n - 1)) >> c.page_shift];
      }
#pragma unroll
      for (int i = 0; i < kSelectHeld; ++i) {
        const int x = (g * kSelectHeld + i) * kSelectThreads + tid;
        const bool none = (unsigned)page[i] >= (unsigned)c.n_pages;
        const int row = (a.first + (x < n ? x : n - 1)) & ((1 << c.page_shift) - 1);
        const float w = a.weights[(((long)(none ? 0 : page[i]) * c.Hkv + h) << c.page_shift) + row];
        u[i] = none ? 0u : order_of(w);
        bad = bad || none;
      }
    };
    auto counts = [&](int g, int i) { return (g * kSelectHeld + i) * kSelectThreads + tid < n; };

    // ---- the range of the weights
    uint32_t lo = 0xffffffffu, hi = 0;
    for (int g = 0; g < groups; ++g) {
      load(g);
#pragma unroll
      for (int i = 0; i < kSelectHeld; ++i)
        if (counts(g, i)) lo = u[i] < lo ? u[i] : lo, hi = u[i] > hi ? u[i] : hi;
    }
    for (int o = 1; o < kWave; o <<= 1) {
      const uint32_t l = __shfl_xor(lo, o), m = __shfl_xor(hi, o);
      lo = l < lo ? l : lo, hi = m > hi ? m : hi;
    }
    __syncthreads();  // (of the block's work before)
    if (lane == 0) sh.low[wave] = lo, sh.high[wave] = hi;
    if (tid == 0) sh.bad = 0;
    __syncthreads();
    for (int w = 0; w < kSelectWaves; ++w) {
      lo = sh.low[w] < lo ? sh.low[w] : lo;
      hi = sh.high[w] > hi ? sh.high[w] : hi;
    }
    if (bad) sh.bad = 1;

    // ---- the border: [lo, lo + 2^bits) holds it; `need` of the weights in it are taken, all above are
    int bits = hi == lo ? 0 : 32 - __builtin_clz(hi - lo), need = want;
    while (bits > 0 && need > 0) {
      const int shift = bits > 11 ? bits - 11 : 0;
      const uint32_t used = 1u << (bits - shift);  // buckets
      for (int x = tid; x < kBuckets; x += kSelectThreads) sh.bucket[x] = 0;
      __syncthreads();
      for (int g = 0; g < groups; ++g) {
        if (groups > 1) load(g);
#pragma unroll
        for (int i = 0; i < kSelectHeld; ++i) {
          const uint32_t x = (u[i] - lo) >> shift;
          if (counts(g, i) && u[i] >= lo && x < used) atomicAdd(&sh.bucket[x], 1);
        }
      }
      __syncthreads();
      // weights in buckets above one's own two, from the sums of the waves above and of the lanes above
      const int top = kBuckets - 1 - 2 * tid, c0 = sh.bucket[top], c1 = sh.bucket[top - 1];
      int upto = c0 + c1;
      for (int o = 1; o < kWave; o <<= 1) {
        const int y = __shfl_up(upto, o);
        if (lane >= o) upto += y;
      }
      if (lane == kWave - 1) sh.wave_sum[wave] = upto;
      __syncthreads();
      int over = upto - c0 - c1;
      for (int w = 0; w < wave; ++w) over += sh.wave_sum[w];
      if (over < need && need <= over + c0) sh.found = top, sh.before = over, sh.inside = c0;
      else if (over + c0 < need && need <= over + c0 + c1) sh.found = top - 1, sh.before = over + c0, sh.inside = c1;
      __syncthreads();
      lo += (uint32_t)sh.found << shift;
      need -= sh.before;
      bits = shift;
      const bool all = need == sh.inside;
      __syncthreads();
      if (all) break;
    }
    const uint32_t span = bits >= 32 ? 0xffffffffu : (1u << bits) - 1u;
    // (nothing wanted: the border lies above all; a range that ends at the top of the order has nothing above it)
    auto is_above = [&](uint32_t x) { return want > 0 && x > lo && x - lo > span; };
    auto is_equal = [&](uint32_t x) { return want > 0 && x >= lo && x - lo <= span; };

    // ---- places: of the keys above the border and of those at it, counted by wave and round
    int done_above = 0, done_equal = 0;
    for (int g = 0; g < groups; ++g) {
      if (groups > 1) load(g);
#pragma unroll
      for (int i = 0; i < kSelectHeld; ++i) {
        const unsigned long long m = __ballot(counts(g, i) && is_above(u[i])), e = __ballot(counts(g, i) && is_equal(u[i]));
        if (lane == 0) sh.above[i * kSelectWaves + wave] = __popcll(m), sh.equal[i * kSelectWaves + wave] = __popcll(e);
      }
      __syncthreads();
      if (tid < kSelectHeld * kSelectWaves) {
        int m = sh.above[tid], e = sh.equal[tid];
        const int m0 = m, e0 = e;
        for (int o = 1; o < kWave; o <<= 1) {
          const int x = __shfl_up(m, o), y = __shfl_up(e, o);
          if (lane >= o) m += x, e += y;
        }
        if (lane == kWave - 1) sh.wave_sum[wave] = m, sh.wave_sum[kSelectHeld * kSelectWaves / kWave + wave] = e;
        sh.above[tid] = m - m0, sh.equal[tid] = e - e0;
      }
      __syncthreads();
      constexpr int kFour = kSelectHeld * kSelectWaves / kWave;
#pragma unroll
      for (int i = 0; i < kSelectHeld; ++i) {
        const bool m = counts(g, i) && is_above(u[i]), e = counts(g, i) && is_equal(u[i]);
        const unsigned long long mm = __ballot(m), ee = __ballot(e), mine = (1ull << lane) - 1ull;
        const int place = i * kSelectWaves + wave;
        int na = done_above + sh.above[place] + __popcll(mm & mine), ne = done_equal + sh.equal[place] + __popcll(ee & mine);
        for (int w = 0; w < place / kWave; ++w) na += sh.wave_sum[w], ne += sh.wave_sum[kFour + w];
        // (the keys at the border before this one that are taken: `need` of them at most)
        const int x = (g * kSelectHeld + i) * kSelectThreads + tid;
        if (m || (e && ne < need)) kept[a.first + na + (ne < need ? ne : need)] = a.first + x;
      }
      for (int w = 0; w < kFour; ++w) done_above += sh.wave_sum[w], done_equal += sh.wave_sum[kFour + w];
      __syncthreads();
    }
    if (tid == 0 && sh.bad) flag(c, kBadPage);
    __syncthreads();
  }
}

// Row i of a key head takes row kept[i] >= i.  A block has one column of one array of one key head of one sequence and goes through
// its rows from the front, a chunk at a time: a chunk's rows are read, then written.  What it writes has been read, by itself or
// before: row i is the source of no row after i.  So no copy of the rows is needed, and blocks do not wait for one another.
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
