// Host layer of the 8-bit paged K/V cache: argument validation and launches behind the
// crisp_cache_* and crisp_pool_* entry points of include/crisp.h.  As in api.cpp, validation touches
// no device state, so every argument error is reported before anything is queued.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <hip/hip_runtime.h>

#include "cache_internal.h"
#include "crisp.h"

namespace crisp {

namespace {

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

crisp_status check_pool(int32_t n_pages, const int32_t* pool) {
  if (n_pages < 1) return fail(CRISP_EINVAL, "bad pool: n_pages=%d", n_pages);
  if (n_pages > kMaxPages) return fail(CRISP_EUNSUPPORTED, "n_pages %d above the supported %d", n_pages, kMaxPages);
  return check_ptr(pool, 4, "pool");
}

crisp_status check_pool_table(int32_t n_pages, int32_t block, int32_t n_seqs, int32_t max_pages, const int32_t* pool,
                              const int32_t* table) {
  CHECK(check_pool(n_pages, pool));
  if (block != 64 && block != 128) return fail(CRISP_EUNSUPPORTED, "block %d unsupported (64 or 128)", block);
  CHECK(check_table(block, n_seqs, max_pages));
  if (n_seqs > 0 && max_pages > 0) CHECK(check_ptr(table, 4, "table"));
  return CRISP_OK;
}

}  // namespace

}  // namespace crisp

using namespace crisp;

extern "C" {

crisp_status crisp_cache_bytes(const crisp_cache_shape* cache, size_t* page_bytes, size_t* scale_bytes) {
  CacheDims c;
  CHECK(check_cache(cache, &c));
  if (!page_bytes || !scale_bytes) return fail(CRISP_EINVAL, "page_bytes or scale_bytes is null");
  *page_bytes = (size_t)c.n_pages * c.hkv * 2 * c.B * kHeadDim;
  *scale_bytes = (size_t)c.n_pages * c.hkv * 2 * sizeof(float);
  return CRISP_OK;
}

crisp_status crisp_cache_append(const crisp_cache_shape* cache, const crisp_cache_batch* batch, uint8_t* pages,
                                float* scales, const int32_t* table, const int32_t* seq_len, const int32_t* row_ptr,
                                const crisp_bf16* k, int64_t k_head_stride, int64_t k_row_stride, const crisp_bf16* v,
                                int64_t v_head_stride, int64_t v_row_stride, crisp_stream stream) {
  CacheDims c;
  BatchDims b;
  CHECK(check_cache(cache, &c));
  CHECK(check_batch(batch, c, &b));
  CHECK(check_strides(k_head_stride, k_row_stride, false, c.hkv, b.n_rows, "k"));
  CHECK(check_strides(v_head_stride, v_row_stride, false, c.hkv, b.n_rows, "v"));
  if (empty(b) || b.max_pages == 0) return CRISP_OK;
  CHECK(check_pages(pages, scales));
  CHECK(check_seqs(b, table, seq_len, row_ptr));
  CHECK(check_ptr(k, 16, "k"));
  CHECK(check_ptr(v, 16, "v"));
  return hip_status(launch_cache_append(c, b, Seqs{table, seq_len, row_ptr}, k, Strides{k_head_stride, k_row_stride}, v,
                                        Strides{v_head_stride, v_row_stride}, pages, scales, (hipStream_t)stream),
                    "crisp_cache_append launch");
}

crisp_status crisp_cache_attn_workspace_size(const crisp_cache_shape* cache, const crisp_cache_batch* batch,
                                             int32_t n_q_heads, size_t* bytes) {
  CacheDims c;
  BatchDims b;
  CHECK(check_cache(cache, &c));
  CHECK(check_batch(batch, c, &b));
  CHECK(check_heads(c, b, n_q_heads));
  if (!bytes) return fail(CRISP_EINVAL, "bytes is null");
  *bytes = cache_attn_plan(c, b, n_q_heads).bytes;
  return CRISP_OK;
}

crisp_status crisp_cache_attn(const crisp_cache_shape* cache, const crisp_cache_batch* batch, int32_t n_q_heads,
                              float softmax_scale, const uint8_t* pages, const float* scales, const int32_t* table,
                              const int32_t* seq_len, const int32_t* row_ptr, const crisp_bf16* q,
                              int64_t q_head_stride, int64_t q_row_stride, crisp_bf16* o, int64_t o_head_stride,
                              int64_t o_row_stride, void* workspace, size_t workspace_bytes, crisp_stream stream) {
  CacheDims c;
  BatchDims b;
  CHECK(check_cache(cache, &c));
  CHECK(check_batch(batch, c, &b));
  CHECK(check_heads(c, b, n_q_heads));
  if (!(softmax_scale >= 0.f) || !isfinite(softmax_scale))
    return fail(CRISP_EINVAL, "softmax_scale must be finite and >= 0");
  CHECK(check_strides(q_head_stride, q_row_stride, false, n_q_heads, b.n_rows, "q"));
  CHECK(check_strides(o_head_stride, o_row_stride, true, n_q_heads, b.n_rows, "o"));
  if (empty(b) || n_q_heads == 0) return CRISP_OK;
  CHECK(check_pages(pages, scales));
  CHECK(check_seqs(b, table, seq_len, row_ptr));
  CHECK(check_ptr(q, 16, "q"));
  CHECK(check_ptr(o, 16, "o"));
  CHECK(check_ptr(workspace, 256, "workspace"));
  const size_t need = cache_attn_plan(c, b, n_q_heads).bytes;
  if (workspace_bytes < need) return fail(CRISP_EINVAL, "workspace too small: %zu < %zu", workspace_bytes, need);
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)kHeadDim);
  return hip_status(launch_cache_attn(c, b, Seqs{table, seq_len, row_ptr}, n_q_heads, scale, q,
                                      Strides{q_head_stride, q_row_stride}, pages, scales, o,
                                      Strides{o_head_stride, o_row_stride}, workspace, (hipStream_t)stream),
                    "crisp_cache_attn launch");
}

crisp_status crisp_cache_copy(const crisp_cache_shape* cache, uint8_t* pages, float* scales, const int32_t* pairs,
                              int32_t n_pairs, const int32_t* count_or_null, crisp_stream stream) {
  CacheDims c;
  CHECK(check_cache(cache, &c));
  if (n_pairs < 0) return fail(CRISP_EINVAL, "n_pairs must be >= 0");
  if (n_pairs == 0) return CRISP_OK;
  CHECK(check_pages(pages, scales));
  CHECK(check_ptr(pairs, 4, "pairs"));
  if (count_or_null) CHECK(check_ptr(count_or_null, 4, "count"));
  return hip_status(launch_cache_copy(c, pairs, n_pairs, count_or_null, pages, scales, (hipStream_t)stream),
                    "crisp_cache_copy launch");
}

int64_t crisp_pool_words(int32_t n_pages) {
  if (n_pages < 1 || n_pages > kMaxPages) {
    fail(CRISP_EINVAL, "n_pages %d outside [1, %d]", n_pages, kMaxPages);
    return -1;
  }
  return pool_words(n_pages);
}

crisp_status crisp_pool_init(int32_t n_pages, int32_t* pool, crisp_stream stream) {
  CHECK(check_pool(n_pages, pool));
  return hip_status(launch_pool_init(n_pages, pool, (hipStream_t)stream), "crisp_pool_init launch");
}

crisp_status crisp_pool_reserve(int32_t n_pages, int32_t block, int32_t n_seqs, int32_t max_pages, int32_t* pool,
                                int32_t* table, const int32_t* seq_len, const int32_t* counts, int32_t* granted,
                                crisp_stream stream) {
  CHECK(check_pool_table(n_pages, block, n_seqs, max_pages, pool, table));
  if (n_seqs > kPoolMaxSeqs) return fail(CRISP_EUNSUPPORTED, "n_seqs %d above the supported %d", n_seqs, kPoolMaxSeqs);
  if (n_seqs == 0) return CRISP_OK;
  CHECK(check_ptr(seq_len, 4, "seq_len"));
  CHECK(check_ptr(counts, 4, "counts"));
  CHECK(check_ptr(granted, 4, "granted"));
  return hip_status(launch_pool_reserve(n_pages, block, n_seqs, max_pages, pool, table, seq_len, counts, granted,
                                        (hipStream_t)stream),
                    "crisp_pool_reserve launch");
}

crisp_status crisp_pool_fork(int32_t n_pages, int32_t block, int32_t n_seqs, int32_t max_pages, int32_t* pool,
                             int32_t* table, int32_t* seq_len, const int32_t* src, const int32_t* dst, int32_t n,
                             int32_t* copies, crisp_stream stream) {
  CHECK(check_pool_table(n_pages, block, n_seqs, max_pages, pool, table));
  if (n < 0) return fail(CRISP_EINVAL, "n must be >= 0");
  if (n_seqs > kPoolMaxSeqs || n > kPoolMaxSeqs)
    return fail(CRISP_EUNSUPPORTED, "n_seqs %d or n %d above the supported %d", n_seqs, n, kPoolMaxSeqs);
  if (n == 0) return CRISP_OK;
  if (n_seqs > 0) CHECK(check_ptr(seq_len, 4, "seq_len"));
  CHECK(check_ptr(src, 4, "src"));
  CHECK(check_ptr(dst, 4, "dst"));
  CHECK(check_ptr(copies, 4, "copies"));
  return hip_status(launch_pool_fork(n_pages, block, n_seqs, max_pages, pool, table, seq_len, src, dst, n, copies,
                                     (hipStream_t)stream),
                    "crisp_pool_fork launch");
}

crisp_status crisp_pool_free(int32_t n_pages, int32_t n_seqs, int32_t max_pages, int32_t* pool, int32_t* table,
                             int32_t* seq_len, const int32_t* ids, int32_t n, crisp_stream stream) {
  CHECK(check_pool_table(n_pages, 64, n_seqs, max_pages, pool, table));
  if (n < 0) return fail(CRISP_EINVAL, "n must be >= 0");
  if (n == 0 || n_seqs == 0) return CRISP_OK;
  CHECK(check_ptr(seq_len, 4, "seq_len"));
  CHECK(check_ptr(ids, 4, "ids"));
  return hip_status(launch_pool_free(n_pages, n_seqs, max_pages, pool, table, seq_len, ids, n, (hipStream_t)stream),
                    "crisp_pool_free launch");
}

crisp_status crisp_pool_compact(int32_t n_pages, int32_t n_seqs, int32_t max_pages, int32_t* pool, int32_t* table,
                                int32_t* moves, int32_t* count, crisp_stream stream) {
  CHECK(check_pool_table(n_pages, 64, n_seqs, max_pages, pool, table));
  CHECK(check_ptr(moves, 4, "moves"));
  CHECK(check_ptr(count, 4, "count"));
  return hip_status(launch_pool_compact(n_pages, n_seqs, max_pages, pool, table, moves, count, (hipStream_t)stream),
                    "crisp_pool_compact launch");
}

}  // extern "C"
