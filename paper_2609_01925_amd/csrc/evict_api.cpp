// Host layer of the eviction from the 8-bit paged K/V cache: argument validation and launches behind crisp_cache_weights,
// crisp_cache_keep and crisp_cache_gather of include/crisp.h.
#include "host_checks.h"

namespace crisp {

namespace {

constexpr int64_t kMaxHeads = (int64_t)1 << 20;  // sequences x KV heads, some workgroups each
constexpr int kMaxWidth = 1 << 28;               // of the weights and lists: their chunks are a launch's second dimension
constexpr int64_t kMaxWeights = (int64_t)1 << 34;  // all heads' widths: workgroups of 1024 threads and 8192 tokens, fewer than 2^32 threads

crisp_status check_seq_heads(int64_t n_seqs, int64_t heads) {
  if (n_seqs * heads > kMaxHeads)
    return fail(CRISP_EUNSUPPORTED, "%lld sequences of %lld KV heads are above the supported 2^20", (long long)n_seqs, (long long)heads);
  return CRISP_OK;
}

crisp_status check_width(int width, const char* name) {
  if (width < 1) return fail(CRISP_EINVAL, "%s must be >= 1", name);
  if (width > kMaxWidth) return fail(CRISP_EUNSUPPORTED, "%s %d above the supported 2^28", name, width);
  return CRISP_OK;
}

crisp_status check_keep(int n_seqs, int heads, int width) {
  if (n_seqs < 0 || heads < 1) return fail(CRISP_EINVAL, "bad sizes: n_seqs=%d n_kv_heads=%d", n_seqs, heads);
  if (heads > 65535) return fail(CRISP_EUNSUPPORTED, "n_kv_heads %d above the supported 65535", heads);
  CHECK(check_seq_heads(n_seqs, heads));
  CHECK(check_width(width, "width"));
  if ((int64_t)n_seqs * heads * width > kMaxWeights)
    return fail(CRISP_EUNSUPPORTED, "%d sequences of %d KV heads and width %d are above the supported 2^34 weights", n_seqs, heads, width);
  return CRISP_OK;
}

}  // namespace

}  // namespace crisp

using namespace crisp;

extern "C" {

crisp_status crisp_cache_weights_workspace_size(const crisp_cache_shape* cache, const crisp_cache_batch* batch,
                                                int32_t n_q_heads, size_t* bytes) {
  CacheDims c;
  BatchDims b;
  CHECK(check_cache(cache, &c));
  CHECK(check_batch(batch, c, &b));
  CHECK(check_heads(c, b, n_q_heads));
  CHECK(check_seq_heads(b.n_seqs, c.hkv));
  if (!bytes) return fail(CRISP_EINVAL, "bytes is null");
  *bytes = cache_weights_bytes(c, b, n_q_heads);
  return CRISP_OK;
}

crisp_status crisp_cache_weights(const crisp_cache_shape* cache, const crisp_cache_batch* batch, int32_t n_q_heads,
                                 float softmax_scale, const uint8_t* pages, const float* scales, const int32_t* table,
                                 const int32_t* seq_len, const int32_t* row_ptr, const crisp_bf16* q,
                                 int64_t q_head_stride, int64_t q_row_stride, const float* weights, float* out,
                                 int32_t width, const int32_t* held, void* workspace, size_t workspace_bytes,
                                 crisp_stream stream) {
  CacheDims c;
  BatchDims b;
  CHECK(check_cache(cache, &c));
  CHECK(check_batch(batch, c, &b));
  CHECK(check_heads(c, b, n_q_heads));
  CHECK(check_seq_heads(b.n_seqs, c.hkv));
  CHECK(check_width(width, "width"));
  if (!(softmax_scale >= 0.f) || !isfinite(softmax_scale))
    return fail(CRISP_EINVAL, "softmax_scale must be finite and >= 0");
  CHECK(check_strides(q_head_stride, q_row_stride, false, n_q_heads, b.n_rows, "q"));
  if (b.n_seqs == 0) return CRISP_OK;  // (without rows the weights that are held still go to out)
  CHECK(check_pages(pages, scales));
  CHECK(check_seqs(b, table, seq_len, row_ptr));
  if (b.n_rows > 0 && n_q_heads > 0) CHECK(check_ptr(q, 16, "q"));
  CHECK(check_ptr(weights, 4, "weights"));
  CHECK(check_ptr(out, 4, "out"));
  CHECK(check_ptr(held, 4, "held"));
  const size_t need = cache_weights_bytes(c, b, n_q_heads);
  if (need > 0) CHECK(check_ptr(workspace, 256, "workspace"));
  if (workspace_bytes < need) return fail(CRISP_EINVAL, "workspace too small: %zu < %zu", workspace_bytes, need);
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)kHeadDim);
  return hip_status(launch_cache_weights(c, b, Seqs{table, seq_len, row_ptr}, n_q_heads, scale, q,
                                         Strides{q_head_stride, q_row_stride}, pages, scales, weights, out, width, held,
                                         workspace, (hipStream_t)stream),
                    "crisp_cache_weights launch");
}

crisp_status crisp_cache_keep_workspace_size(int32_t n_seqs, int32_t n_kv_heads, int32_t width, int32_t in_place,
                                             size_t* bytes) {
  CHECK(check_keep(n_seqs, n_kv_heads, width));
  if (!bytes) return fail(CRISP_EINVAL, "bytes is null");
  *bytes = cache_keep_bytes((int64_t)n_seqs * n_kv_heads, width, in_place != 0);
  return CRISP_OK;
}

crisp_status crisp_cache_keep(int32_t n_seqs, int32_t n_kv_heads, int32_t width, const float* weights, const int32_t* held,
                              const int32_t* seq_len, const int32_t* keep, int32_t sink, int32_t recent, int32_t cap,
                              int32_t* kept, int32_t* count, float* new_weights_or_null, void* workspace,
                              size_t workspace_bytes, crisp_stream stream) {
  CHECK(check_keep(n_seqs, n_kv_heads, width));
  CHECK(check_width(cap, "cap"));
  if (sink < 0 || recent < 0) return fail(CRISP_EINVAL, "sink %d and recent %d must be >= 0", sink, recent);
  if (n_seqs == 0) return CRISP_OK;
  CHECK(check_ptr(weights, 4, "weights"));
  CHECK(check_ptr(held, 4, "held"));
  CHECK(check_ptr(seq_len, 4, "seq_len"));
  CHECK(check_ptr(keep, 4, "keep"));
  CHECK(check_ptr(kept, 4, "kept"));
  CHECK(check_ptr(count, 4, "count"));
  if (new_weights_or_null) CHECK(check_ptr(new_weights_or_null, 4, "new_weights"));
  const size_t need = cache_keep_bytes((int64_t)n_seqs * n_kv_heads, width, new_weights_or_null == weights);
  if (need > 0) CHECK(check_ptr(workspace, 256, "workspace"));
  if (workspace_bytes < need) return fail(CRISP_EINVAL, "workspace too small: %zu < %zu", workspace_bytes, need);
  return hip_status(launch_cache_keep(KeepArgs{n_seqs, n_kv_heads, width, sink, recent, cap, weights, held, seq_len, keep, kept,
                                               count, new_weights_or_null, (char*)workspace},
                                      (hipStream_t)stream),
                    "crisp_cache_keep launch");
}

crisp_status crisp_cache_gather(const crisp_cache_shape* cache, const crisp_cache_batch* batch, uint8_t* pages,
                                float* scales, const int32_t* table, const int32_t* kept, int32_t cap,
                                const int32_t* count, const int32_t* new_table, int32_t new_pages, crisp_stream stream) {
  CacheDims c;
  BatchDims b;
  CHECK(check_cache(cache, &c));
  CHECK(check_batch(batch, c, &b));
  CHECK(check_seq_heads(b.n_seqs, c.hkv));
  CHECK(check_width(cap, "cap"));
  CHECK(check_table(c.B, b.n_seqs, new_pages));
  if (b.n_seqs == 0 || new_pages == 0) return CRISP_OK;
  CHECK(check_pages(pages, scales));
  if (b.max_pages > 0) CHECK(check_ptr(table, 4, "table"));
  CHECK(check_ptr(kept, 4, "kept"));
  CHECK(check_ptr(count, 4, "count"));
  CHECK(check_ptr(new_table, 4, "new_table"));
  return hip_status(launch_cache_gather(GatherArgs{c, b.n_seqs, b.max_pages, new_pages, cap, pages, scales, table, kept, count,
                                                   new_table},
                                        (hipStream_t)stream),
                    "crisp_cache_gather launch");
}

}  // extern "C"
