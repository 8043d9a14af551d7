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

typedef __attribute__((__vector_size__(2 * sizeof(uint16_t)))) uint16_t u16x2;

// The larger of m and |x| of eight bf16 as bits, in each half of a dword.
__device__ __forceinline__ uint32_t amax_bits(u32x4 raw, uint32_t m) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, raw[i] & 0x7fff7fffu)));
  return m;
}
// The same of the finite ones only.
__device__ __forceinline__ uint32_t amax_finite(u32x4 raw, uint32_t m) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = raw[i] & 0x7fffu, hi = raw[i] & 0x7fff0000u;
    raw[i] = (lo < 0x7f80u ? lo : 0u) | (hi < 0x7f800000u ? hi : 0u);
  }
  return amax_bits(raw, m);
}

constexpr int kNonFinite = 0x7f80;

template <int FMT>
__device__ __forceinline__ u32x4 rescale(u32x4 x, float f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x4 v = from_codes<FMT>(x[i]);
    x[i] = to_codes<FMT>(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
  }
  return x;
}

template <int TILES>
struct PageLds {
  __attribute__((aligned(16))) char stage[2 * TILES * kTileLds];
  uint32_t amax[2][2][4 * TILES];
};

// One workgroup, 256 threads a tile, writes the rows r of sequence seq that go into its page `slot`, one KV head: it reads
// them once, takes the scale from their largest magnitude (and from the scale of the tokens that the page
// holds already, which never shrinks), lays the codes out in LDS in the tile's order and stores whole
// chunks.  A chunk of V holds 16 tokens of one element, so one that is only partly new is read,
// merged and written back by its thread; a page whose scale grew has its other codes rounded
// again.  Bound by HBM on long appends (512 bytes read and 256 written a token and head): 32768 rows of 8 heads, int8,
// 128 tokens a page, 36 us, 5.6 TB/s; by the chain lengths -> rows -> scale -> codes on short ones, whose look-up of the
// page runs beside the rows': 24 sequences of up to 700 rows, 4 heads, 9.6 us.
template <int FMT, int TILES>
__device__ __forceinline__ void append_page(const AppendArgs& a, const SeqRows& r, int seq, int slot, int head, PageLds<TILES>& l) {
  constexpr int B = TILES * kTile, kThreads = 256 * TILES, kW = kThreads / kWave;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int first = slot * B;                                              // position of the page's first token
  const int t0 = max(r.len - first, 0), t1 = min(r.len + r.n - first, B);  // the call's tokens in the page
  const int row0 = r.row0 + first - r.len;  // the call's row of token 0 (before its first, if t0 > 0)
  const uint16_t* src[2] = {a.k + head * a.ks.head, a.v + head * a.vs.head};
  const int64_t rs[2] = {a.ks.row, a.vs.row};
  // thread: of tile tid / 256, tokens 4 (tid / 16 % 16) + [0, 4) and elements 8 (tid % 16) + [0, 8)
  const int tl = tid >> 8, tr = tl * kTile + 4 * ((tid >> 4) & 15), d0 = 8 * (tid & 15);
  u32x4 raw[2][4];
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = tr + i;
      raw[x][i] = u32x4{0, 0, 0, 0};
      if (t >= t0 && t < t1) raw[x][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src[x] + (row0 + t) * rs[x] + d0));
    }
  const int page = slot < a.b.max_pages ? a.s.table[(int64_t)seq * a.b.max_pages + slot] : -1;
  if (page < 0 || page >= a.c.n_pages) return;
  float* scale = a.scales + ((int64_t)page * a.c.hkv + head) * 2;
  const float s_old[2] = {scale[0], scale[1]};
  const auto reduce = [&](int turn, const auto& of) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) m = of(raw[x][i], m);
      m = max(m & 0xffffu, m >> 16);
      m = wave_reduce(m, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
      if (lane == 0) l.amax[turn][x][w] = m;
    }
    __syncthreads();
  };
  int top[2];
  const auto tops = [&](int turn) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      uint32_t m = l.amax[turn][x][0];
#pragma unroll
      for (int i = 1; i < kW; ++i) m = max(m, l.amax[turn][x][i]);
      top[x] = (int)m;
    }
  };
  reduce(0, amax_bits);
  tops(0);
  const bool finite = max(top[0], top[1]) < kNonFinite;
  if (!finite) {
    reduce(1, amax_finite);
    tops(1);
  }
  float down[2];  // what old codes are multiplied by; 1: they stay
  int e_new[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    int e = scale_exp<FMT>(top[x]);
    down[x] = 1.f;
    if (t0 > 0) {
      const int old = stored_exp(s_old[x]);
      if (e > old) down[x] = pow2f(max(old - e, -126));
      e = max(e, old);
    }
    e_new[x] = e;
  }
  // codes into LDS, in the tiles' order
  uint32_t c[2][4][2];
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4 q = raw[x][i];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (finite) {
          c[x][i][h] = finite_codes<FMT>(q[2 * h], q[2 * h + 1], e_new[x]);
        } else {
          const float inv = pow2f(-e_new[x]);
          c[x][i][h] = to_codes<FMT>(__uint_as_float(q[2 * h] << 16) * inv, __uint_as_float(q[2 * h] & 0xffff0000u) * inv,
                                     __uint_as_float(q[2 * h + 1] << 16) * inv, __uint_as_float(q[2 * h + 1] & 0xffff0000u) * inv);
        }
      }
    }
  {
    char* kt = l.stage + tl * kTileLds;
    char* vt = l.stage + (TILES + tl) * kTileLds;
    const int q = (tid >> 4) & 3, w4 = w & 3;
    // K: token 16 w4 + 4 q + i is row r = 4 w4 + i of score tile q; elements d0.. are half of a chunk
    const int kc = ((q * 2 + ((d0 >> 4) & 1)) * 4 + (d0 >> 5)) * 16 + 4 * w4;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<u32x2*>(kt + lds_chunk(kc + i) + (d0 & 8)) = u32x2{c[0][i][0], c[0][i][1]};
    // V: four tokens of one element are a quarter of a chunk
    const int vc = ((d0 >> 4) * 4 + w4) * 16 + (d0 & 8);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t y[4];
      transpose4(c[1][0][h], c[1][1][h], c[1][2][h], c[1][3][h], y);
#pragma unroll
      for (int j = 0; j < 4; ++j) *reinterpret_cast<uint32_t*>(vt + lds_chunk(vc + 4 * h + j) + 4 * q) = y[j];
    }
  }
  if (tid < 2) scale[tid] = pow2f(tid == 0 ? e_new[0] : e_new[1]);
  __syncthreads();
  u32x4* dst = reinterpret_cast<u32x4*>(a.pages + ((int64_t)page * a.c.hkv + head) * (2 * B * kHeadDim));
  constexpr int kChunks = kTileBytes / kChunk;  // of a tile and tensor
#pragma unroll
  for (int i = 0; i < kChunks * TILES / kThreads; ++i) {
    const int n = i * kThreads + tid, td = n / kChunks, ch = n % kChunks;
    u32x4* kd = dst + (2 * td) * kChunks + ch;
    u32x4* vd = kd + kChunks;
    const int rr = ch & 15, g = (ch >> 4) & 3;
    const int tk = td * kTile + 16 * (rr >> 2) + 4 * (ch >> 7) + (rr & 3);
    if (tk >= t0 && tk < t1)
      *kd = *reinterpret_cast<const u32x4*>(l.stage + td * kTileLds + lds_chunk(ch));
    else if (down[0] != 1.f)
      *kd = rescale<FMT>(*kd, down[0]);
    const int tv = td * kTile + 16 * g;
    const int lo = max(t0 - tv, 0), hi = min(t1 - tv, 16);  // new tokens of this chunk
    u32x4 y = *reinterpret_cast<const u32x4*>(l.stage + (TILES + td) * kTileLds + lds_chunk(ch));
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

// The page of blockIdx.x: the so-many-th one that the call writes to.  Up to 64 sequences every wave looks them
// over, one a lane; more are counted by the workgroup.
template <int FMT, int TILES>
__global__ __launch_bounds__(256 * TILES) void cache_append(AppendArgs a) {
  constexpr int B = TILES * kTile, kThreads = 256 * TILES, kW = kThreads / kWave;
  __shared__ PageLds<TILES> l;
  __shared__ int wsum[kW], at[2];
  const int tid = threadIdx.x, lane = tid & 63;
  SeqRows r;
  int seq, slot;
  const int item = blockIdx.x;
  if (a.b.n_seqs <= kWave) {
    SeqRows mine = {0, 0, 0};
    if (lane < a.b.n_seqs) mine = seq_rows(a.s, a.b, B, lane);
    const int cnt = pages_touched(mine, B), end = wave_scan(cnt);
    const unsigned long long past = __ballot(item < end);
    if (past == 0) return;
    seq = __builtin_ctzll(past);
    r = SeqRows{__builtin_amdgcn_readlane(mine.len, seq), __builtin_amdgcn_readlane(mine.row0, seq), __builtin_amdgcn_readlane(mine.n, seq)};
    slot = r.len / B + item - __builtin_amdgcn_readlane(end - cnt, seq);
  } else {
    if (tid == 0) at[0] = -1;
    int before = 0;
    for (int s0 = 0; s0 < a.b.n_seqs; s0 += kThreads) {
      const int s = s0 + tid;
      int cnt = 0;
      if (s < a.b.n_seqs) cnt = pages_touched(seq_rows(a.s, a.b, B, s), B);
      int total;
      __syncthreads();
      const int end = before + block_scan<int, kW>(cnt, wsum, &total);
      if (item >= end - cnt && item < end) {
        at[0] = s;
        at[1] = item - (end - cnt);
      }
      before += total;
      if (item < before) break;  // the same on every thread
    }
    __syncthreads();
    seq = __builtin_amdgcn_readfirstlane(at[0]);
    if (seq < 0) return;
    r = seq_rows(a.s, a.b, B, seq);
    slot = r.len / B + at[1];
  }
  append_page<FMT, TILES>(a, r, seq, slot, blockIdx.y, l);
}

// The n <= kFewRows rows from row `row` on that the call writes to a page, its token t0 first, by one wave.  A lane holds two
// elements; codes go out as they are, two bytes of K and a byte each of two of V's chunks, since what lies beside
// them is only touched where a scale grows.  No LDS and no barrier: the page's chain without its waits.
constexpr int kFewRows = 3;
template <int FMT>
__device__ __forceinline__ void append_rows(const AppendArgs& a, int row, int n, int t0, int page, int head) {
  const int lane = threadIdx.x & 63, B = a.c.B;
  const uint16_t* src[2] = {a.k + head * a.ks.head + row * a.ks.row + 2 * lane, a.v + head * a.vs.head + row * a.vs.row + 2 * lane};
  const int64_t rs[2] = {a.ks.row, a.vs.row};
  uint32_t x[2][kFewRows];
#pragma unroll
  for (int j = 0; j < kFewRows; ++j)
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      x[y][j] = 0;
      if (j < n) x[y][j] = *reinterpret_cast<const uint32_t*>(src[y] + j * rs[y]);
    }
  if (page < 0 || page >= a.c.n_pages) return;
  float* scale = a.scales + ((int64_t)page * a.c.hkv + head) * 2;
  uint8_t* dst = a.pages + ((int64_t)page * a.c.hkv + head) * (2 * (int64_t)B * kHeadDim);
  const auto finite = [](uint32_t bits) { return bits < 0x7f80u ? bits : 0u; };
  float inv[2];
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < kFewRows; ++j) m = max(m, max(finite(x[y][j] & 0x7fffu), finite((x[y][j] >> 16) & 0x7fffu)));
    m = wave_reduce(m, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
    int e = scale_exp<FMT>((int)m);
    if (t0 > 0) {
      const int old = stored_exp(scale[y]);
      if (e > old) {  // the page's other codes under the new scale
        const float down = pow2f(max(old - e, -126));
        for (int c = lane; c < a.c.tiles * (kTileBytes / kChunk); c += kWave) {
          u32x4* at = reinterpret_cast<u32x4*>(dst + (c / (kTileBytes / kChunk) * 2 + y) * kTileBytes) + c % (kTileBytes / kChunk);
          *at = rescale<FMT>(*at, down);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the new codes are stored behind these
      }
      e = max(e, old);
    }
    if (lane == 0) scale[y] = pow2f(e);
    inv[y] = pow2f(-e);
  }
  const int e0 = 2 * lane;
#pragma unroll
  for (int j = 0; j < kFewRows; ++j) {
    if (j >= n) break;
    uint32_t c[2];
#pragma unroll
    for (int y = 0; y < 2; ++y)
      c[y] = to_codes<FMT>(__uint_as_float(x[y][j] << 16) * inv[y], __uint_as_float(x[y][j] & 0xffff0000u) * inv[y], 0.f, 0.f);
    const int t = (t0 + j) % kTile;
    uint8_t* tile = dst + (t0 + j) / kTile * (2 * kTileBytes);
    *reinterpret_cast<uint16_t*>(tile + ((t / 4 % 4 * 2 + e0 / 16 % 2) * 64 + e0 / 32 * 16 + t / 16 * 4 + t % 4) * 16 + e0 % 16) = (uint16_t)c[0];
    uint8_t* v = tile + kTileBytes + (e0 / 16 * 64 + t / 16 * 16 + e0 % 16) * 16 + t % 16;
    v[0] = (uint8_t)c[1];
    v[16] = (uint8_t)(c[1] >> 8);
  }
}

// A wave looks at one row: if it is the first that the call writes to its page and few follow there, the wave writes them;
// pages with more are then written by the workgroup, one after the other.  All latency: 64 sequences of one row, 8 heads, 4.1 us.
template <int FMT, int TILES>
__global__ __launch_bounds__(256 * TILES) void cache_append_few(AppendArgs a) {
  constexpr int B = TILES * kTile, kW = 4 * TILES;
  __shared__ PageLds<TILES> l;
  __shared__ int seqs[kW], slots[kW];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = (int)blockIdx.x * kW + w, head = blockIdx.y;
  // the row's sequence: among up to 64 the one that has it, among more the last that begins at or before it,
  // looked for 64 at a time
  int seq = 0;
  SeqRows r{0, 0, 0};
  if (a.b.n_seqs <= kWave) {
    SeqRows x{0, 0, 0};
    if (lane < a.b.n_seqs) x = seq_rows(a.s, a.b, B, lane);
    const unsigned long long found = __ballot(row >= x.row0 && row < x.row0 + x.n);
    if (found != 0) {
      seq = __builtin_ctzll(found);
      r = SeqRows{__builtin_amdgcn_readlane(x.len, seq), __builtin_amdgcn_readlane(x.row0, seq), __builtin_amdgcn_readlane(x.n, seq)};
    }
  } else {
    for (int n = a.b.n_seqs; n > 1;) {
      const int step = (n + kWave - 1) / kWave, probe = lane * step;
      const unsigned long long ok = __ballot(probe < n && a.s.row_ptr[seq + min(probe, n - 1)] <= row);
      const int k = max(__popcll(ok) - 1, 0);
      seq += k * step;
      n = min(step, n - k * step);
    }
    r = seq_rows(a.s, a.b, B, seq);
  }
  const int i = row - r.row0, pos = r.len + i, t0 = pos % B, slot = pos / B;
  const int n = i >= 0 && i < r.n && (i == 0 || t0 == 0) ? min(r.n - i, B - t0) : 0;  // rows of a page that begins here
  if (lane == 0) {
    seqs[w] = n > kFewRows ? seq : -1;
    slots[w] = slot;
  }
  __syncthreads();
  if (n > 0 && n <= kFewRows)
    append_rows<FMT>(a, row, n, t0, slot < a.b.max_pages ? a.s.table[(int64_t)seq * a.b.max_pages + slot] : -1, head);
  for (int x = 0; x < kW; ++x) {
    const int s = __builtin_amdgcn_readfirstlane(seqs[x]);
    if (s >= 0) append_page<FMT, TILES>(a, seq_rows(a.s, a.b, B, s), s, __builtin_amdgcn_readfirstlane(slots[x]), head, l);
  }
}

// pairs[i] = (from, to): 16 KB pieces (one tile of K and V of one head) over a persistent grid; a
// pair with a page out of range or with from == to moves nothing.  Bound by HBM: 986 pages of 8 heads, 64 tokens each (259 MB
// read and written), 48 us, 5.4 TB/s; one page of each of 24 forks 3.1 us.
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
    for (int e = 0; e < 4; ++e) x[e] = __builtin_nontemporal_load(s + e * kThreads);
#pragma unroll
    for (int e = 0; e < 4; ++e) __builtin_nontemporal_store(x[e], d + e * kThreads);
    if (p == 0)
      for (int e = threadIdx.x; e < 2 * c.hkv; e += kThreads)
        scales[(int64_t)to * 2 * c.hkv + e] = scales[(int64_t)from * 2 * c.hkv + e];
  }
}

}  // namespace

hipError_t launch_cache_append(const CacheDims& c, const BatchDims& b, const Seqs& s, const uint16_t* k, Strides ks,
                               const uint16_t* v, Strides vs, uint8_t* pages, float* scales, hipStream_t stream) {
  const AppendArgs a{c, b, s, k, v, ks, vs, pages, scales};
  // Few rows a sequence on average: no list of pages is needed, a wave looks at each row.  8 heads, e4m3, the page kernel / this
  // one, us: 256 sequences of one row 10.6 / 7.6, of 4 13.4 / 13.4, of 8 13.3 / 20.9, 255 of one and one of 512 13.6 / 11.0, one of
  // 2000 7.9 / 14.3; past that the page kernel has to count for long: 1000 of one 38.5 / 11.2, of 4.5 56.1 / 39.7, of 10 62.5 / 62.7;
  // 4000 of one 221 / 29.1, of 5 390 / 145.
  if (b.n_rows <= (b.n_seqs <= 512 ? 3 : 8) * (int64_t)b.n_seqs) {
    const dim3 few((unsigned)((b.n_rows + 4 * c.tiles - 1) / (4 * c.tiles)), (unsigned)c.hkv);
    if (c.fmt == kCacheE4M3) {
      if (c.tiles == 1) hipLaunchKernelGGL((cache_append_few<kCacheE4M3, 1>), few, dim3(256), 0, stream, a);
      else hipLaunchKernelGGL((cache_append_few<kCacheE4M3, 2>), few, dim3(512), 0, stream, a);
    } else {
      if (c.tiles == 1) hipLaunchKernelGGL((cache_append_few<kCacheInt8, 1>), few, dim3(256), 0, stream, a);
      else hipLaunchKernelGGL((cache_append_few<kCacheInt8, 2>), few, dim3(512), 0, stream, a);
    }
    return hipGetLastError();
  }
  // a sequence's n rows touch at most (n - 1) / B + 2 pages, and at most n
  const int64_t with_rows = b.n_seqs < b.n_rows ? b.n_seqs : b.n_rows;
  int64_t items = b.n_rows / c.B + 2 * with_rows;
  if (items > b.n_rows) items = b.n_rows;
  const dim3 grid((unsigned)items, (unsigned)c.hkv);
  if (c.fmt == kCacheE4M3) {
    if (c.tiles == 1) hipLaunchKernelGGL((cache_append<kCacheE4M3, 1>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((cache_append<kCacheE4M3, 2>), grid, dim3(512), 0, stream, a);
  } else {
    if (c.tiles == 1) hipLaunchKernelGGL((cache_append<kCacheInt8, 1>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((cache_append<kCacheInt8, 2>), grid, dim3(512), 0, stream, a);
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
