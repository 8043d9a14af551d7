/* Host-only check of the entry points on packed rows and of the eviction, compiled as C99 and linked with the library's host layer
 * built under AddressSanitizer and UndefinedBehaviorSanitizer.  As in cache_check.c, it runs only where no GPU is present and its device
 * pointers are fake addresses: every call is rejected, has nothing to do, or passes validation and must report the failed
 * launch as CRISP_EHIP.  Exit status 0 iff every expectation held. */
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "crisp.h"

static int failures;
static int checks;

#define EXPECT(cond)                                                                    \
  do {                                                                                  \
    ++checks;                                                                           \
    if (!(cond)) {                                                                      \
      ++failures;                                                                       \
      fprintf(stderr, "FAIL line %d [last error: %s]\n", __LINE__, crisp_last_error()); \
    }                                                                                   \
  } while (0)

static void* const P = (void*)(uintptr_t)0x7f0000100000ull; /* 256-byte aligned */

static const int32_t ints[] = {INT32_MIN, INT32_MIN + 1, -129, -128, -1, 0, 1, 2, 3, 16, 63, 64, 65, 127, 128, 129, 4095, 4096,
                               65535, 65536, 1 << 20, 1 << 24, (1 << 24) + 1, 1 << 30, INT32_MAX - 127, INT32_MAX};
static const int64_t strides[] = {INT64_MIN, INT64_MIN + 7, -128, -8, 0, 8, 120, 128, 129, 136, 256, 1 << 20, 1 << 23, (int64_t)1 << 40,
                                  INT64_MAX - 7, INT64_MAX};
static const double reals[] = {-INFINITY, -1.0, -0.0, 0.0, 1e-300, 0.5, 1.0, 1.0000001, 2.0, 32.0, 8192.0, 1e30, 1e308, INFINITY, NAN};
#define N(x) ((int)(sizeof(x) / sizeof((x)[0])))

static int known(crisp_status s) { return s == CRISP_OK || s == CRISP_EINVAL || s == CRISP_EUNSUPPORTED || s == CRISP_EHIP; }

static crisp_status rope(const crisp_packed_shape* p, const crisp_rope_table* t, int64_t head, int64_t row) {
  return crisp_rope(p, t, P, P, P, head, row, P, head, row, P, head, row, P, head, row, NULL);
}
static crisp_status attn(const crisp_packed_shape* p, float scale, int64_t head, int64_t row) {
  return crisp_packed_attn(p, scale, P, P, head, row, P, head, row, P, head, row, P, head, row, NULL);
}
static crisp_status weights(const crisp_cache_shape* c, const crisp_cache_batch* b, int32_t hq, int64_t head, int64_t row, int32_t width,
                            size_t ws) {
  return crisp_cache_weights(c, b, hq, 0.f, P, P, P, P, P, P, head, row, P, P, width, P, P, ws, NULL);
}

int main(void) {
  const crisp_packed_shape packed = {2, 300, 4, 2, 128};
  const crisp_cache_shape cache = {8, 2, 128, 64, CRISP_CACHE_E4M3};
  const crisp_cache_batch batch = {2, 4, 3};
  const crisp_rope_params params = {64, CRISP_ROPE_HALF, CRISP_ROPE_RAMP, 10000.0, 8.0, 4096.0, 1.0, 32.0};
  crisp_rope_table table;
  size_t bytes = 0;
  int i, j, k;
  EXPECT(crisp_rope_init(&params, &table) == CRISP_OK && table.rotary_dim == 64);
  EXPECT(rope(&packed, &table, 300 * 128, 128) == CRISP_EHIP);
  EXPECT(attn(&packed, 0.f, 300 * 128, 128) == CRISP_EHIP);
  EXPECT(crisp_cache_weights_workspace_size(&cache, &batch, 4, &bytes) == CRISP_OK && bytes > 0);
  EXPECT(weights(&cache, &batch, 4, 384, 128, 256, bytes) == CRISP_EHIP);
  EXPECT(weights(&cache, &batch, 4, 384, 128, 256, bytes - 1) == CRISP_EINVAL);
  EXPECT(crisp_cache_keep(2, 2, 256, P, P, P, P, 4, 8, 64, P, P, NULL, NULL, 0, NULL) == CRISP_EHIP);
  EXPECT(crisp_cache_gather(&cache, &batch, P, P, P, P, 64, P, P, 1, NULL) == CRISP_EHIP);

  /* every field over the ends of its type */
  for (i = 0; i < N(ints); ++i) {
    for (j = 0; j < 5; ++j) {
      crisp_packed_shape s = packed;
      *(j == 0 ? &s.n_seqs : j == 1 ? &s.n_rows : j == 2 ? &s.n_q_heads : j == 3 ? &s.n_kv_heads : &s.head_dim) = ints[i];
      for (k = 0; k < N(strides); ++k) {
        EXPECT(known(rope(&s, &table, strides[k], 128)) && known(rope(&s, &table, 1 << 20, strides[k])));
        EXPECT(known(attn(&s, 0.f, strides[k], 128)) && known(attn(&s, 0.f, 1 << 20, strides[k])));
      }
    }
    for (j = 0; j < 3; ++j) {
      crisp_rope_params p = params;
      crisp_rope_table t = table;
      *(j == 0 ? &p.rotary_dim : j == 1 ? &p.layout : &p.scaling) = ints[i];
      EXPECT(known(crisp_rope_init(&p, &t)));
      if (j < 2) {
        t = table;
        *(j == 0 ? &t.rotary_dim : &t.layout) = ints[i];
        EXPECT(known(rope(&packed, &t, 300 * 128, 128)));
      }
    }
    for (j = 0; j < N(ints); ++j) {
      crisp_cache_batch b = batch;
      crisp_status s;
      b.n_seqs = ints[i];
      b.n_rows = ints[j];
      s = crisp_cache_weights_workspace_size(&cache, &b, 4, &bytes);
      EXPECT(known(s) && s != CRISP_EHIP);
      EXPECT(known(weights(&cache, &b, 4, (int64_t)1 << 33, 128, 256, SIZE_MAX)));
      b = batch;
      b.max_pages = ints[i];
      EXPECT(known(weights(&cache, &b, ints[j], 384, 128, 256, SIZE_MAX)) && known(weights(&cache, &batch, 4, 384, 128, ints[i], SIZE_MAX)));
      EXPECT(known(crisp_cache_gather(&cache, &b, P, P, P, P, 64, P, P, ints[j], NULL)));
      EXPECT(known(crisp_cache_gather(&cache, &batch, P, P, P, P, ints[i], P, P, ints[j], NULL)));
      EXPECT(known(crisp_cache_keep(ints[i], ints[j], 256, P, P, P, P, 4, 8, 64, P, P, P, P, SIZE_MAX, NULL)));
      EXPECT(known(crisp_cache_keep(2, 2, ints[i], P, P, P, P, ints[j], ints[i], ints[j], P, P, P, P, SIZE_MAX, NULL)));
      s = crisp_cache_keep_workspace_size(ints[i], 2, ints[j], i & 1, &bytes);
      EXPECT(known(s) && s != CRISP_EHIP);
    }
  }
  for (i = 0; i < N(reals); ++i)
    for (j = 0; j < 5; ++j)
      for (k = 0; k <= CRISP_ROPE_RAMP; ++k) {
        crisp_rope_params p = params;
        crisp_rope_table t;
        crisp_status s;
        p.scaling = k;
        *(j == 0 ? &p.base : j == 1 ? &p.factor : j == 2 ? &p.original_len : j == 3 ? &p.low : &p.high) = reals[i];
        s = crisp_rope_init(&p, &t);
        EXPECT(s == CRISP_OK || s == CRISP_EINVAL);
        if (s == CRISP_OK) {
          int x;
          for (x = 0; x < 32; ++x) EXPECT(isfinite(t.turns[x]) && t.turns[x] >= 0.0 && t.turns[x] <= 0.16);
        }
      }
  printf("%d checks, %d failures\n", checks, failures);
  return failures != 0;
}
