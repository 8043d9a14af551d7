/* Host-only check of the K/V cache's entry points, compiled as C99 and linked with the library's host layer
 * built under AddressSanitizer and UndefinedBehaviorSanitizer.  As in abi_check.c, it runs only where no GPU
 * is present and its device pointers are fake addresses: every call is rejected, has nothing to do, or
 * passes validation and must report the failed launch as CRISP_EHIP.
 * Exit status 0 iff every expectation held. */
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

static const int32_t ints[] = {INT32_MIN, INT32_MIN + 1, -129, -128, -1, 0, 1, 2, 3, 63, 64, 65, 127, 128, 129, 4095, 4096, 4097,
                               65535, 65536, 1 << 24, (1 << 24) + 1, 1 << 30, INT32_MAX - 127, INT32_MAX};
static const int64_t strides[] = {INT64_MIN, INT64_MIN + 7, -128, -8, 0, 8, 120, 128, 129, 136, 256, 1 << 20, (int64_t)1 << 40,
                                  INT64_MAX - 7, INT64_MAX};
#define N(x) ((int)(sizeof(x) / sizeof((x)[0])))

static int known(crisp_status s) { return s == CRISP_OK || s == CRISP_EINVAL || s == CRISP_EUNSUPPORTED || s == CRISP_EHIP; }

static crisp_status append(const crisp_cache_shape* c, const crisp_cache_batch* b, int64_t head, int64_t row) {
  return crisp_cache_append(c, b, P, P, P, P, P, P, head, row, P, head, row, NULL);
}

static crisp_status attn(const crisp_cache_shape* c, const crisp_cache_batch* b, int32_t hq, float scale, int64_t head, int64_t row,
                         size_t ws) {
  return crisp_cache_attn(c, b, hq, scale, P, P, P, P, P, P, head, row, P, head, row, P, ws, NULL);
}

int main(void) {
  const crisp_cache_shape good = {8, 2, 128, 64, CRISP_CACHE_E4M3};
  const crisp_cache_batch batch = {2, 4, 3};
  size_t a = 0, b = 0;
  int i, j, k;
  EXPECT(crisp_cache_bytes(&good, &a, &b) == CRISP_OK && a == (size_t)8 * 2 * 2 * 8192 && b == 8 * 2 * 2 * 4);
  EXPECT(crisp_cache_bytes(NULL, &a, &b) == CRISP_EINVAL && crisp_cache_bytes(&good, NULL, &b) == CRISP_EINVAL);

  /* every field over the ends of its type */
  for (i = 0; i < N(ints); ++i)
    for (j = 0; j < 5; ++j) {
      crisp_cache_shape s = good;
      crisp_status st;
      *(j == 0 ? &s.n_pages : j == 1 ? &s.n_kv_heads : j == 2 ? &s.head_dim : j == 3 ? &s.block : &s.format) = ints[i];
      st = crisp_cache_bytes(&s, &a, &b);
      EXPECT(known(st) && st != CRISP_EHIP);
      if (st != CRISP_OK) {
        EXPECT(append(&s, &batch, 384, 128) == st);
        EXPECT(attn(&s, &batch, 4, 0.f, 384, 128, (size_t)1 << 40) == st);
        EXPECT(crisp_cache_copy(&s, P, P, P, 1, NULL, NULL) == st);
      }
    }
  for (i = 0; i < N(ints); ++i)
    for (j = 0; j < N(ints); ++j)
      for (k = 0; k < 3; ++k) {
        crisp_cache_batch x = batch;
        size_t bytes = 0;
        crisp_status st;
        *(k == 0 ? &x.n_seqs : &x.max_pages) = ints[i];
        *(k == 1 ? &x.n_seqs : &x.n_rows) = ints[j];
        st = crisp_cache_attn_workspace_size(&good, &x, 4, &bytes);
        EXPECT(known(st) && st != CRISP_EHIP && bytes < (size_t)1 << 31);
        st = attn(&good, &x, 4, 0.f, (int64_t)1 << 40, 128, bytes);
        EXPECT(known(st));
        st = attn(&good, &x, ints[i], 0.f, (int64_t)1 << 40, 128, 0);
        EXPECT(known(st) && st != CRISP_EHIP);
        EXPECT(known(append(&good, &x, 384, 128)));
      }
  for (i = 0; i < N(strides); ++i)
    for (j = 0; j < N(strides); ++j) {
      EXPECT(known(append(&good, &batch, strides[i], strides[j])));
      EXPECT(known(attn(&good, &batch, 4, 0.f, strides[i], strides[j], (size_t)1 << 40)));
    }
  EXPECT(attn(&good, &batch, 4, NAN, 384, 128, (size_t)1 << 40) == CRISP_EINVAL);
  EXPECT(attn(&good, &batch, 4, -1.f, 384, 128, (size_t)1 << 40) == CRISP_EINVAL);
  EXPECT(attn(&good, &batch, 4, 0.f, 384, 128, 255) == CRISP_EINVAL);

  /* bookkeeping */
  for (i = 0; i < N(ints); ++i) {
    const int64_t words = crisp_pool_words(ints[i]);
    EXPECT(ints[i] >= 1 && ints[i] <= 1 << 24 ? words == (int64_t)ints[i] + ((int64_t)ints[i] + 31) / 32 : words == -1);
    EXPECT(known(crisp_pool_init(ints[i], P, NULL)));
    EXPECT(known(crisp_cache_copy(&good, P, P, P, ints[i], NULL, NULL)));
    for (j = 0; j < N(ints); ++j) {
      EXPECT(known(crisp_pool_reserve(ints[i], 64, ints[j], 4, P, P, P, P, P, NULL)));
      EXPECT(known(crisp_pool_reserve(100, ints[i], 4, ints[j], P, P, P, P, P, NULL)));
      EXPECT(known(crisp_pool_fork(100, 128, ints[i], 4, P, P, P, P, P, ints[j], P, NULL)));
      EXPECT(known(crisp_pool_free(100, ints[i], 4, P, P, P, P, ints[j], NULL)));
      EXPECT(known(crisp_pool_compact(100, ints[i], ints[j], P, P, P, P, NULL)));
    }
  }

  /* nothing to do; and what passes the checks reaches a launch, which fails here */
  {
    const crisp_cache_batch none = {0, 4, 3}, empty = {2, 4, 0};
    EXPECT(crisp_cache_append(&good, &none, NULL, NULL, NULL, NULL, NULL, NULL, 0, 0, NULL, 0, 0, NULL) == CRISP_OK);
    EXPECT(crisp_cache_append(&good, &empty, NULL, NULL, NULL, NULL, NULL, NULL, 0, 0, NULL, 0, 0, NULL) == CRISP_OK);
  }
  EXPECT(append(&good, &batch, 384, 128) == CRISP_EHIP);
  EXPECT(attn(&good, &batch, 4, 0.f, 384, 128, (size_t)1 << 40) == CRISP_EHIP);
  EXPECT(crisp_cache_copy(&good, P, P, P, 1, NULL, NULL) == CRISP_EHIP);
  EXPECT(crisp_pool_init(100, P, NULL) == CRISP_EHIP);

  printf("%d checks, %d failures\n", checks, failures);
  return failures != 0;
}
