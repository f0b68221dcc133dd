/* Host-side sweep of the rotation, paged-cache and attention calls under AddressSanitizer and
 * UndefinedBehaviorSanitizer, linked against a build of the library whose host code carries the
 * same sanitizers.  Every call returns on the host before anything is enqueued (arguments it
 * refuses, or a workspace that is too small), so no GPU is needed; what runs is the checks and
 * the plan of the launch, with the extremes of every integer field.  Prints "sanitize ok". */
#include <limits.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "dart.h"

static uint64_t state = 0x13198A2E03707344ull;
static uint32_t rnd(void) { /* splitmix64, upper half */
  uint64_t z = (state += 0x9E3779B97F4A7C15ull);
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return (uint32_t)((z ^ (z >> 31)) >> 32);
}

static const int32_t sizes[] = {INT_MIN, -1, 0, 1, 2, 3, 4, 7, 8, 16, 28, 32, 64, 65, 80, 128, 256, 264, 577, 2880,
                                16384, 65536, 1 << 20, (1 << 20) + 1, 1 << 24, (1 << 24) + 1, 1 << 28, INT_MAX};
static const int64_t strides[] = {INT64_MIN, -1, 0, 4, 8, 128, 4096, 1ll << 24, 1ll << 33, (1ll << 33) + 8, 1ll << 40, INT64_MAX};
enum { NS = sizeof sizes / sizeof sizes[0], NL = sizeof strides / sizeof strides[0] };
static int32_t any(void) { return sizes[rnd() % NS]; }
static int64_t stride(int64_t plausible) { return rnd() % 4 ? plausible : strides[rnd() % NL]; }
/* mostly a plausible value, sometimes an extreme one */
static int32_t likely(int32_t plausible) { return rnd() % 6 ? plausible : any(); }

int main(void) {
  void* fake = (void*)(uintptr_t)0x10000;
  long planned = 0;
  for (int it = 0; it < 60000; ++it) {
    static const int32_t heads[] = {1, 2, 4, 7, 28, 32}, widths[] = {8, 40, 64, 128, 256}, lens[] = {1, 2, 9, 300, 9216, 16384};
    dart_cache c;
    memset(&c, 0, sizeof c);
    c.dtype = rnd() % 8 ? (int32_t)(rnd() % 2) : any();
    c.Hkv = likely(heads[rnd() % 6]);
    c.Hq = likely(c.Hkv > 0 && c.Hkv < 100 ? c.Hkv * (int32_t)(1 + rnd() % 8) : 8);
    c.d = likely(widths[rnd() % 5]);
    c.B = likely(lens[rnd() % 4]);
    c.max_q = likely(lens[rnd() % 6]);
    c.T = likely(c.B > 0 && c.B < 400 && c.max_q > 0 && c.max_q < 20000 ? c.B * c.max_q : 64);
    c.max_kv = likely(lens[rnd() % 6]);
    c.page_size = likely(1 << (rnd() % 9));
    c.n_pages = likely(1000);
    c.pages_ld = likely(16384);
    c.row_ld = stride(c.d > 0 && c.d < 1000 ? c.d : 64);
    c.head_ld = stride(1 << 16);
    c.page_ld = stride(1 << 20);
    if (rnd() % 3) c.cu_q = (const int32_t*)fake;
    if (rnd() % 8) c.kv_len = (const int32_t*)fake;
    if (rnd() % 8) c.pages = (const int32_t*)fake;
    if (rnd() % 2) {
      c.groups = likely(c.B > 0 && c.B < 1000 ? 1 + (int32_t)(rnd() % (uint32_t)c.B) : 1);
      c.max_prefix = likely(lens[rnd() % 6]);
      c.prefix_ld = likely(16384);
      if (rnd() % 8) c.group_cu = (const int32_t*)fake;
      if (rnd() % 8) c.prefix_pages = (const int32_t*)fake;
      if (rnd() % 8) c.prefix_len = (const int32_t*)fake;
    }
    const size_t need = dart_attend_workspace_bytes(&c);
    if (need > 0) ++planned;
    const int64_t ld = stride(c.Hq > 0 && c.Hq < 1000 && c.d > 0 && c.d < 1000 ? (int64_t)c.Hq * c.d : 64);
    if (c.T != 0 && c.B != 0) {
      if (dart_attend(&c, fake, ld, fake, fake, 0.1f, (int32_t)(rnd() % 2), fake, ld, NULL, fake, need ? need - 1 : 0, fake, NULL) == DART_OK)
        return printf("a workspace too small was taken\n"), 1;
      if (dart_attend(&c, NULL, ld, fake, fake, 0.1f, 1, fake, ld, NULL, fake, need, fake, NULL) == DART_OK)
        return printf("no queries were taken\n"), 1;
    }
    dart_rotation t;
    memset(&t, 0, sizeof t);
    t.Hq = likely(c.Hq);
    t.Hkv = likely(c.Hkv);
    t.d = likely(c.d);
    t.dtype = c.dtype;
    t.rot = likely(t.d);
    t.interleaved = (int32_t)(rnd() % 2);
    t.planes = likely(1 + (int32_t)(rnd() % 3));
    for (int p = 0; p < 4; ++p) t.sections[p] = likely(16);
    t.inv_freq = rnd() % 8 ? (const float*)fake : NULL;
    t.q_weight = rnd() % 2 ? fake : NULL;
    t.eps = rnd() % 4 ? 1e-6f : -1.f;
    t.scale = 1.f;
    const int64_t plane = stride(c.T > 0 ? c.T : 1);
    /* one required tensor is missing: refused before anything is enqueued */
    if (c.T != 0 && dart_norm_rotate(&t, c.T, NULL, ld, fake, ld, (const int64_t*)fake, plane, fake, ld, fake, ld, NULL, NULL) == DART_OK)
      return printf("no rows were taken\n"), 1;
    if (c.T != 0 && c.B != 0 &&
        dart_norm_rotate_append(&t, &c, fake, ld, NULL, ld, fake, ld, (const int64_t*)fake, plane, fake, ld, NULL, 0, NULL, fake, fake,
                                fake, NULL) == DART_OK)
      return printf("no keys were taken\n"), 1;
  }
  if (planned < 3000) return printf("only %ld plausible caches\n", planned), 1;
  printf("sanitize ok: %ld of 60000 planned\n", planned);
  return 0;
}
