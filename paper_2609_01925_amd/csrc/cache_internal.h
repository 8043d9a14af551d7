// Internal interface of the 8-bit paged K/V cache: sizes and launches shared by its C ABI layer
// (cache_api.cpp) and its kernels (cache.hip, cache_attn.hip, pool.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "crisp_internal.h"

namespace crisp {

constexpr int kTile = 64;                       // tokens of a tile
constexpr int kTileBytes = kTile * kHeadDim;    // one tensor's tile of one head, 8-bit codes
constexpr int kChunk = 16;                      // bytes that one lane loads at once
constexpr int kScaleExpMin = -64, kScaleExpMax = 122;  // of a page's scale 2^e
constexpr int kCacheE4M3 = 0, kCacheInt8 = 1;

struct CacheDims {
  int n_pages, hkv, B, tiles, fmt;  // tiles = B / 64 per page and head
};

struct BatchDims {
  int n_seqs, max_pages, n_rows;
};

// Element strides of a [heads][rows][128] tensor; the 128 elements of a row are contiguous.
struct Strides {
  int64_t head, row;
};

// Device arrays that tell which pages and rows a sequence has.
struct Seqs {
  const int32_t* table;    // [n_seqs][max_pages]
  const int32_t* seq_len;  // [n_seqs] tokens held before the call
  const int32_t* row_ptr;  // [n_seqs + 1]
};

hipError_t launch_cache_append(const CacheDims& c, const BatchDims& b, const Seqs& s, const uint16_t* k, Strides ks,
                               const uint16_t* v, Strides vs, uint8_t* pages, float* scales, hipStream_t stream);

hipError_t launch_cache_copy(const CacheDims& c, const int32_t* pairs, int n_pairs, const int32_t* count,
                             uint8_t* pages, float* scales, hipStream_t stream);

// What the attention's launch is cut into: units of so many query rows of one sequence and KV head, and workgroups
// with an equal share of the units' 64-token tiles each.
struct CacheAttnPlan {
  int rows, grain, workgroups;  // grain: tiles that are never cut apart
  bool once;                    // most tiles are read by one workgroup only
  size_t cut_bytes, bytes;      // workspace: what each boundary between shares cuts (0: nothing is cut), and all of it
};
CacheAttnPlan cache_attn_plan(const CacheDims& c, const BatchDims& b, int hq);

hipError_t launch_cache_attn(const CacheDims& c, const BatchDims& b, const Seqs& s, int hq, float scale,
                             const uint16_t* q, Strides qs, const uint8_t* pages, const float* scales, uint16_t* o,
                             Strides os, void* ws, hipStream_t stream);

size_t cache_weights_bytes(const CacheDims& c, const BatchDims& b, int hq);  // of launch_cache_weights's workspace
hipError_t launch_cache_weights(const CacheDims& c, const BatchDims& b, const Seqs& s, int hq, float scale, const uint16_t* q,
                                Strides qs, const uint8_t* pages, const float* scales, const float* weights, float* out,
                                int width, const int32_t* held, void* ws, hipStream_t stream);

struct KeepArgs {
  int n_seqs, hkv, width, sink, recent, cap;
  const float* weights;  // [n_seqs][hkv][width]
  const int32_t* held;
  const int32_t* seq_len;
  const int32_t* keep;
  int32_t* kept;         // [n_seqs][hkv][cap]
  int32_t* count;
  float* new_weights;    // as weights, which it may be; or null
  char* ws;              // cache_keep_bytes
};
size_t cache_keep_bytes(int64_t heads, int width, bool in_place);
hipError_t launch_cache_keep(const KeepArgs& a, hipStream_t stream);

struct GatherArgs {
  CacheDims c;
  int n_seqs, max_pages, new_pages, cap;
  uint8_t* pages;
  float* scales;
  const int32_t* table;      // [n_seqs][max_pages]
  const int32_t* kept;       // [n_seqs][hkv][cap]
  const int32_t* count;
  const int32_t* new_table;  // [n_seqs][new_pages]
};
hipError_t launch_cache_gather(const GatherArgs& a, hipStream_t stream);

// Page bookkeeping: pool = uses of each page [n_pages], then one bit a page in use, lowest first.
constexpr int kPoolMaxSeqs = 4096;  // sequences (reserve) and forks of one call: their sums live in LDS
inline int64_t pool_words(int64_t n_pages) { return n_pages + (n_pages + 31) / 32; }
hipError_t launch_pool_init(int n_pages, int32_t* pool, hipStream_t stream);
hipError_t launch_pool_reserve(int n_pages, int block, int n_seqs, int max_pages, int32_t* pool, int32_t* table,
                               const int32_t* seq_len, const int32_t* counts, int32_t* granted, hipStream_t stream);
hipError_t launch_pool_fork(int n_pages, int block, int n_seqs, int max_pages, int32_t* pool, int32_t* table,
                            int32_t* seq_len, const int32_t* src, const int32_t* dst, int n, int32_t* copies,
                            hipStream_t stream);
hipError_t launch_pool_free(int n_pages, int n_seqs, int max_pages, int32_t* pool, int32_t* table, int32_t* seq_len,
                            const int32_t* ids, int n, hipStream_t stream);
hipError_t launch_pool_compact(int n_pages, int n_seqs, int max_pages, int32_t* pool, int32_t* table, int32_t* moves,
                               int32_t* count, hipStream_t stream);

// The C ABI layer's thread-local message (api.cpp).
void set_error(const char* msg);

}  // namespace crisp
