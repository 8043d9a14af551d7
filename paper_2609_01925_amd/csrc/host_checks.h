// Argument checks of the host layers behind the crisp_cache_*, crisp_pool_* and packed-row entry points (cache_api.cpp,
// packed_api.cpp, evict_api.cpp).  They touch no device state.
#pragma once

#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <hip/hip_runtime.h>

#include "cache_internal.h"
#include "crisp.h"

namespace crisp {

namespace {  // a copy in each host layer, which uses some of them

constexpr int kMaxPages = 1 << 24;
constexpr int kMaxRows = 1 << 24;         // with all query heads: rows of a sequence x G stays in int32
constexpr int kMaxSeqs = 1 << 24;         // of a call on a cache: each workgroup of the attention looks them all over
constexpr int64_t kMaxTokens = 1 << 30;   // of one sequence's table

crisp_status fail(crisp_status s, const char* fmt, ...) {
  char msg[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(msg, sizeof(msg), fmt, ap);
  va_end(ap);
  set_error(msg);
  return s;
}

#define CHECK(expr)                       \
  do {                                    \
    crisp_status s_ = (expr);             \
    if (s_ != CRISP_OK) return s_;        \
  } while (0)

crisp_status hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return CRISP_OK;
  return fail(CRISP_EHIP, "%s: %s", what, hipGetErrorString(e));
}

crisp_status check_ptr(const void* p, size_t align, const char* name) {
  if (!p) return fail(CRISP_EINVAL, "%s is null", name);
  if ((uintptr_t)p % align) return fail(CRISP_EINVAL, "%s is not %zu-byte aligned", name, align);
  return CRISP_OK;
}

crisp_status check_cache(const crisp_cache_shape* s, CacheDims* d) {
  if (!s) return fail(CRISP_EINVAL, "cache shape is null");
  if (s->n_pages < 1 || s->n_kv_heads < 1)
    return fail(CRISP_EINVAL, "bad cache shape: n_pages=%d n_kv_heads=%d", s->n_pages, s->n_kv_heads);
  if (s->head_dim != kHeadDim) return fail(CRISP_EUNSUPPORTED, "head_dim %d unsupported (only 128)", s->head_dim);
  if (s->block != 64 && s->block != 128) return fail(CRISP_EUNSUPPORTED, "block %d unsupported (64 or 128)", s->block);
  if (s->format != CRISP_CACHE_E4M3 && s->format != CRISP_CACHE_INT8)
    return fail(CRISP_EINVAL, "cache format %d unknown", s->format);
  if (s->n_pages > kMaxPages) return fail(CRISP_EUNSUPPORTED, "n_pages %d above the supported %d", s->n_pages, kMaxPages);
  if (s->n_kv_heads > 65535) return fail(CRISP_EUNSUPPORTED, "n_kv_heads %d above the supported 65535", s->n_kv_heads);
  *d = CacheDims{s->n_pages, s->n_kv_heads, s->block, s->block / kTile, s->format};
  return CRISP_OK;
}

crisp_status check_table(int block, int n_seqs, int max_pages) {
  if (n_seqs < 0 || max_pages < 0) return fail(CRISP_EINVAL, "bad table: n_seqs=%d max_pages=%d", n_seqs, max_pages);
  if ((int64_t)max_pages * block > kMaxTokens)
    return fail(CRISP_EUNSUPPORTED, "max_pages %d of %d tokens above the supported 2^30 tokens", max_pages, block);
  if ((int64_t)n_seqs * max_pages > INT32_MAX)
    return fail(CRISP_EUNSUPPORTED, "a table of %d x %d entries is above the supported 2^31 - 1", n_seqs, max_pages);
  return CRISP_OK;
}

crisp_status check_batch(const crisp_cache_batch* b, const CacheDims& c, BatchDims* d) {
  if (!b) return fail(CRISP_EINVAL, "batch is null");
  if (b->n_rows < 0) return fail(CRISP_EINVAL, "bad batch: n_rows=%d", b->n_rows);
  CHECK(check_table(c.B, b->n_seqs, b->max_pages));
  if (b->n_rows > kMaxRows) return fail(CRISP_EUNSUPPORTED, "n_rows %d above the supported %d", b->n_rows, kMaxRows);
  if (b->n_seqs > kMaxSeqs) return fail(CRISP_EUNSUPPORTED, "n_seqs %d above the supported %d", b->n_seqs, kMaxSeqs);
  *d = BatchDims{b->n_seqs, b->max_pages, b->n_rows};
  return CRISP_OK;
}

bool empty(const BatchDims& b) { return b.n_seqs == 0 || b.n_rows == 0; }

crisp_status check_seqs(const BatchDims& b, const int32_t* table, const int32_t* seq_len, const int32_t* row_ptr) {
  if (b.max_pages > 0) CHECK(check_ptr(table, 4, "table"));
  CHECK(check_ptr(seq_len, 4, "seq_len"));
  return check_ptr(row_ptr, 4, "row_ptr");
}

// An input may repeat a head or a row (stride 0); an output's heads lie behind one another or between its rows.
crisp_status check_strides(int64_t head, int64_t row, bool output, int heads, int rows, const char* name) {
  if (head < 0 || row < 0 || head % 8 || row % 8)
    return fail(CRISP_EINVAL, "%s: strides (%lld, %lld) must be multiples of 8 elements and >= 0", name,
                (long long)head, (long long)row);
  const auto apart = [](int64_t stride, int64_t n, int64_t inner) {  // stride >= inner's n pieces and the last one's 128
    return n < 1 || (stride >= kHeadDim && (stride - kHeadDim) / n >= inner);
  };
  if (output && !(heads > 1 ? rows > 1 ? (row >= kHeadDim && apart(head, rows - 1, row)) || (head >= kHeadDim && apart(row, heads - 1, head))
                                       : head >= kHeadDim
                            : rows <= 1 || row >= kHeadDim))
    return fail(CRISP_EINVAL, "%s: strides (%lld, %lld) overlap its rows", name, (long long)head, (long long)row);
  return CRISP_OK;
}

crisp_status check_pages(const uint8_t* pages, const float* scales) {
  CHECK(check_ptr(pages, 16, "pages"));
  return check_ptr(scales, 4, "scales");
}

crisp_status check_heads(const CacheDims& c, const BatchDims& b, int n_q_heads) {
  if (n_q_heads < 0 || n_q_heads % c.hkv)
    return fail(CRISP_EINVAL, "n_q_heads (%d) is not a multiple of n_kv_heads (%d)", n_q_heads, c.hkv);
  if ((int64_t)b.n_rows * (n_q_heads / c.hkv) > (1 << 30))
    return fail(CRISP_EUNSUPPORTED, "n_rows %d of %d query heads a KV head above the supported 2^30 rows", b.n_rows,
                n_q_heads / c.hkv);
  return CRISP_OK;
}

}  // namespace

}  // namespace crisp
