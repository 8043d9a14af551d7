// Writing the 8-bit paged K/V cache: quantise-and-append, and page copies.
#include "cache_device.h"

namespace crisp {

namespace {

constexpr int kThreads = 256;
// A tile's chunks in LDS, 16 bytes behind every 16 chunks, so that the eight-byte (K) and
// four-byte (V) pieces that 16 lanes store for one token row fall on different banks.
constexpr int kTileLds = kTileBytes + kTileBytes / 256 * 16;
__device__ __forceinline__ int lds_chunk(int c) { return c * kChunk + (c >> 4) * 16; }

struct AppendArgs {
  CacheDims c;
  BatchDims b;
  Seqs s;
  const uint16_t* k;
  const uint16_t* v;
  Strides ks, vs;
  uint8_t* pages;
  float* scales;
};

__device__ __forceinline__ int pages_touched(const SeqRows& r, int B) {
  return r.n == 0 ? 0 : (r.len + r.n - 1) / B - r.len / B + 1;
}

// |x| of eight bf16 as bits, the largest finite one.
__device__ __forceinline__ int amax_bits(u32x4 raw, int m) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int lo = raw[i] & 0x7fff, hi = (raw[i] >> 16) & 0x7fff;
    m = lo < 0x7f80 ? max(m, lo) : m;
    m = hi < 0x7f80 ? max(m, hi) : m;
  }
  return m;
}

template <int FMT>
__device__ __forceinline__ u32x4 rescale(u32x4 x, float f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x4 v = from_codes<FMT>(x[i]);
    x[i] = to_codes<FMT>(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
  }
  return x;
}

// One workgroup writes the call's rows into one page of one KV head: it reads them once, takes
// the scale from their largest magnitude (and from the scale of the tokens that the page holds
// already, which never shrinks), lays the codes out in LDS in the tile's order and stores whole
// chunks.  A chunk of V holds 16 tokens of one element, so one that is only partly new is read,
// merged and written back by its thread; a page whose scale grew has its other codes rounded
// again.  Bound by HBM on long appends (512 bytes read and 256 written a token and head), by
// the chain row table -> page -> scale -> old chunks on single tokens.
template <int FMT, int TILES>
__global__ __launch_bounds__(kThreads) void cache_append(AppendArgs a) {
  constexpr int B = TILES * kTile;
  __shared__ __attribute__((aligned(16))) char stage[2 * TILES * kTileLds];
  __shared__ int wsum[4], at[3], amax[2][4];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  // which page of which sequence: the blockIdx.x-th one that the call writes to
  if (tid == 0) at[0] = -1;
  int before = 0;
  for (int s0 = 0; s0 < a.b.n_seqs; s0 += kThreads) {
    const int s = s0 + tid;
    int cnt = 0;
    if (s < a.b.n_seqs) cnt = pages_touched(seq_rows(a.s, a.b, B, s), B);
    int total;
    __syncthreads();
    const int end = before + block_scan<int, 4>(cnt, wsum, &total);
    if ((int)blockIdx.x >= end - cnt && (int)blockIdx.x < end) {
      at[0] = s;
      at[1] = (int)blockIdx.x - (end - cnt);
    }
    before += total;
    if ((int)blockIdx.x < before) break;  // the same on every thread
  }
  __syncthreads();
  const int s = at[0];
  if (s < 0) return;
  const SeqRows r = seq_rows(a.s, a.b, B, s);
  const int slot = r.len / B + at[1];
  const int first = slot * B;                                      // position of the page's first token
  const int t0 = max(r.len - first, 0), t1 = min(r.len + r.n - first, B);  // the call's tokens in the page
  const int page = slot < a.b.max_pages ? a.s.table[(int64_t)s * a.b.max_pages + slot] : -1;
  if (page < 0 || page >= a.c.n_pages) return;
  const int head = blockIdx.y;
  const int row0 = r.row0 + first - r.len;                         // the call's row of token 0 (before its first, if t0 > 0)
  const uint16_t* src[2] = {a.k + head * a.ks.head, a.v + head * a.vs.head};
  const int64_t rs[2] = {a.ks.row, a.vs.row};
  // thread: tokens 4 (tid / 16) + [0, 4) of each tile, elements 8 (tid % 16) + [0, 8)
  const int tr = 4 * (tid >> 4), d0 = 8 * (tid & 15);
  u32x4 raw[2][TILES][4];
  int m[2] = {0, 0};
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int tl = 0; tl < TILES; ++tl)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = tl * kTile + tr + i;
        raw[x][tl][i] = u32x4{0, 0, 0, 0};
        if (t >= t0 && t < t1) raw[x][tl][i] = *reinterpret_cast<const u32x4*>(src[x] + (row0 + t) * rs[x] + d0);
      }
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int tl = 0; tl < TILES; ++tl)
#pragma unroll
      for (int i = 0; i < 4; ++i) m[x] = amax_bits(raw[x][tl][i], m[x]);
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int v = (int)wave_reduce((uint32_t)m[x], [](uint32_t p, uint32_t q) { return p > q ? p : q; });
    if (lane == 0) amax[x][w] = v;
  }
  float* scale = a.scales + ((int64_t)page * a.c.hkv + head) * 2;
  const float s_old[2] = {scale[0], scale[1]};
  __syncthreads();
  float down[2];  // what old codes are multiplied by; 1: they stay
  float inv[2];
  int e_new[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    int e = scale_exp<FMT>(max(max(amax[x][0], amax[x][1]), max(amax[x][2], amax[x][3])));
    down[x] = 1.f;
    if (t0 > 0) {
      const int old = stored_exp(s_old[x]);
      if (e > old) down[x] = pow2f(max(old - e, -126));
      e = max(e, old);
    }
    e_new[x] = e;
    inv[x] = pow2f(-e);
  }
  // codes into LDS, in the tiles' order
#pragma unroll
  for (int tl = 0; tl < TILES; ++tl) {
    uint32_t c[2][4][2];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x4 q = raw[x][tl][i];
        float f[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f[2 * e] = __uint_as_float(q[e] << 16) * inv[x];
          f[2 * e + 1] = __uint_as_float(q[e] & 0xffff0000u) * inv[x];
        }
        c[x][i][0] = to_codes<FMT>(f[0], f[1], f[2], f[3]);
        c[x][i][1] = to_codes<FMT>(f[4], f[5], f[6], f[7]);
      }
    char* kt = stage + tl * kTileLds;
    char* vt = stage + (TILES + tl) * kTileLds;
    const int q = (tid >> 4) & 3;
    // K: token 16 w + 4 q + i is row r = 4 w + i of score tile q; elements d0.. are half of a chunk
    const int kc = ((q * 2 + ((d0 >> 4) & 1)) * 4 + (d0 >> 5)) * 16 + 4 * w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<u32x2*>(kt + lds_chunk(kc + i) + (d0 & 8)) = u32x2{c[0][i][0], c[0][i][1]};
    // V: four tokens of one element are a quarter of a chunk
    const int vc = ((d0 >> 4) * 4 + w) * 16 + (d0 & 8);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int h = j >> 2, sh = 8 * (j & 3);
      const uint32_t y = ((c[1][0][h] >> sh) & 255u) | ((c[1][1][h] >> sh) & 255u) << 8 |
                         ((c[1][2][h] >> sh) & 255u) << 16 | ((c[1][3][h] >> sh) & 255u) << 24;
      *reinterpret_cast<uint32_t*>(vt + lds_chunk(vc + j) + 4 * q) = y;
    }
  }
  if (tid < 2) scale[tid] = pow2f(e_new[tid]);
  __syncthreads();
  uint8_t* dst = a.pages + ((int64_t)page * a.c.hkv + head) * (2 * B * kHeadDim);
#pragma unroll
  for (int tl = 0; tl < TILES; ++tl)
#pragma unroll
    for (int i = 0; i < kTileBytes / kChunk / kThreads; ++i) {
      const int c = i * kThreads + tid;
      u32x4* kd = reinterpret_cast<u32x4*>(dst + (2 * tl) * kTileBytes) + c;
      u32x4* vd = reinterpret_cast<u32x4*>(dst + (2 * tl + 1) * kTileBytes) + c;
      const int r = c & 15, g = (c >> 4) & 3;
      const int tk = tl * kTile + 16 * (r >> 2) + 4 * (c >> 7) + (r & 3);
      if (tk >= t0 && tk < t1)
        *kd = *reinterpret_cast<const u32x4*>(stage + tl * kTileLds + lds_chunk(c));
      else if (down[0] != 1.f)
        *kd = rescale<FMT>(*kd, down[0]);
      const int tv = tl * kTile + 16 * g;
      const int lo = max(t0 - tv, 0), hi = min(t1 - tv, 16);  // new tokens of this chunk
      u32x4 y = *reinterpret_cast<const u32x4*>(stage + (TILES + tl) * kTileLds + lds_chunk(c));
      if (lo == 0 && hi == 16) {
        *vd = y;
      } else if (hi > lo || down[1] != 1.f) {
        u32x4 old = *vd;
        if (down[1] != 1.f) old = rescale<FMT>(old, down[1]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t take = 0;
#pragma unroll
          for (int z = 0; z < 4; ++z) take |= 4 * e + z >= lo && 4 * e + z < hi ? 255u << (8 * z) : 0u;
          y[e] = (y[e] & take) | (old[e] & ~take);
        }
        *vd = y;
      }
    }
}

// pairs[i] = (from, to): 16 KB pieces (one tile of K and V of one head) over a persistent grid; a
// pair with a page out of range or with from == to moves nothing.  Bound by HBM.
__global__ __launch_bounds__(kThreads) void cache_copy(CacheDims c, const int32_t* pairs, int n_pairs,
                                                       const int32_t* count, uint8_t* pages, float* scales) {
  const int n = count ? min(max(*count, 0), n_pairs) : n_pairs;
  const int pieces = c.hkv * c.tiles;
  const int64_t total = (int64_t)n * pieces;
  for (int64_t u = blockIdx.x; u < total; u += gridDim.x) {
    const int i = (int)(u / pieces), p = (int)(u % pieces);
    const int from = pairs[2 * i], to = pairs[2 * i + 1];
    if (from < 0 || from >= c.n_pages || to < 0 || to >= c.n_pages || from == to) continue;
    const u32x4* s = reinterpret_cast<const u32x4*>(pages + ((int64_t)from * pieces + p) * (2 * kTileBytes)) + threadIdx.x;
    u32x4* d = reinterpret_cast<u32x4*>(pages + ((int64_t)to * pieces + p) * (2 * kTileBytes)) + threadIdx.x;
    u32x4 x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = s[e * kThreads];
#pragma unroll
    for (int e = 0; e < 4; ++e) d[e * kThreads] = x[e];
    if (p == 0)
      for (int e = threadIdx.x; e < 2 * c.hkv; e += kThreads)
        scales[(int64_t)to * 2 * c.hkv + e] = scales[(int64_t)from * 2 * c.hkv + e];
  }
}

}  // namespace

hipError_t launch_cache_append(const CacheDims& c, const BatchDims& b, const Seqs& s, const uint16_t* k, Strides ks,
                               const uint16_t* v, Strides vs, uint8_t* pages, float* scales, hipStream_t stream) {
  // a sequence's n rows touch at most (n - 1) / B + 2 pages, and at most n
  const int64_t with_rows = b.n_seqs < b.n_rows ? b.n_seqs : b.n_rows;
  int64_t items = b.n_rows / c.B + 2 * with_rows;
  if (items > b.n_rows) items = b.n_rows;
  const AppendArgs a{c, b, s, k, v, ks, vs, pages, scales};
  const dim3 grid((unsigned)items, (unsigned)c.hkv);
  if (c.fmt == kCacheE4M3) {
    if (c.tiles == 1) hipLaunchKernelGGL((cache_append<kCacheE4M3, 1>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((cache_append<kCacheE4M3, 2>), grid, dim3(kThreads), 0, stream, a);
  } else {
    if (c.tiles == 1) hipLaunchKernelGGL((cache_append<kCacheInt8, 1>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((cache_append<kCacheInt8, 2>), grid, dim3(kThreads), 0, stream, a);
  }
  return hipGetLastError();
}

hipError_t launch_cache_copy(const CacheDims& c, const int32_t* pairs, int n_pairs, const int32_t* count,
                             uint8_t* pages, float* scales, hipStream_t stream) {
  const int64_t pieces = (int64_t)n_pairs * c.hkv * c.tiles;
  const unsigned grid = (unsigned)(pieces < 2048 ? pieces : 2048);
  hipLaunchKernelGGL(cache_copy, dim3(grid), dim3(kThreads), 0, stream, c, pairs, n_pairs, count, pages, scales);
  return hipGetLastError();
}

}  // namespace crisp
