// Eviction from the 8-bit paged K/V cache: the choice of the tokens that stay, and their move to pages of their own.
#include "cache_device.h"

namespace crisp {

namespace {

constexpr int kKeepThreads = 1024, kKeepWaves = kKeepThreads / kWave;
constexpr int kBins = 2048, kCopies = 8;              // of a digit of 11 bits (the last has 10)
constexpr int kMost = 16;                             // tokens of a thread where one workgroup chooses
constexpr int kPart = 8, kPiece = kPart * kKeepThreads;  // tokens of a thread and a workgroup, at a time, where several do
constexpr int kMostChunks = 128;                      // workgroups of a head there
constexpr int kList = 16384;                          // weights that share the first digit of the limit, if no more do

// An unsigned order of floats: NaN lowest, -0 equal to 0.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return x != x ? 0u : (b >> 31) ? ~b : b | 0x80000000u;
}

// What a sequence and KV head is to keep: the positions below lo and from hi on, and `wanted` of those between.
struct Choice {
  int n, m, held, lo, hi, wanted;
  bool any;
  __device__ __forceinline__ Choice(const KeepArgs& a, int s) : n(a.seq_len[s]), m(a.keep[s]), held(a.held[s]) {
    any = n <= a.width && m > 0 && m < n && m <= a.cap;
    const int recent = min(a.recent, m), sink = min(a.sink, m - recent);
    lo = sink;
    hi = n - recent;
    wanted = m - recent - sink;
  }
  __device__ __forceinline__ bool between(int j) const { return j >= lo && j < hi; }
};

// The limit: all weights above it stay, and `ties` of its equals.  It is found digit by digit, from the top: `prefix` holds the digits
// so far, and `ties` of the weights that share them are still wanted.
struct Limit {
  uint32_t prefix, value;
  int ties, among;  // how many share the digits so far
  static __device__ __forceinline__ int shift(int digit) { return digit == 0 ? 21 : digit == 1 ? 10 : 0; }
  static __device__ __forceinline__ int bits(int digit) { return digit < 2 ? 11 : 10; }
  // Whether they all stay: then all above value - 1 do, and no further digit is needed.
  __device__ __forceinline__ bool all_stay() const { return ties == among && value > 0; }
  __device__ __forceinline__ void close() {
    if (all_stay()) {
      --value;
      ties = 0;
    }
  }
};

// Weights share few exponents, so lanes add to eight copies of the bins.
struct KeepLds {
  __attribute__((aligned(16))) int hist[kBins][kCopies];
  int sums[kKeepWaves], found[3];
};

__device__ __forceinline__ void clear(KeepLds& l) {  // ends with a barrier
  for (int i = threadIdx.x; i < kBins * kCopies / 4; i += kKeepThreads) reinterpret_cast<int4*>(l.hist)[i] = make_int4(0, 0, 0, 0);
  __syncthreads();
}
__device__ __forceinline__ void add(KeepLds& l, int digit, uint32_t prefix, uint32_t o) {
  if ((uint64_t)o >> (Limit::shift(digit) + Limit::bits(digit)) == prefix)
    atomicAdd(&l.hist[o >> Limit::shift(digit) & ((1u << Limit::bits(digit)) - 1)][threadIdx.x & (kCopies - 1)], 1);
}
__device__ __forceinline__ int bin(const KeepLds& l, int d) {
  const int4* h = reinterpret_cast<const int4*>(l.hist[d]);
  const int4 x = h[0], y = h[1];
  return ((x.x + x.y) + (x.z + x.w)) + ((y.x + y.y) + (y.z + y.w));
}
// From the highest digit down, the one in which the count passes the ties that are still wanted; a0 and a1 are the counts of this thread's
// digits 2047 - 2 tid and 2046 - 2 tid.  Barriers before and after what is shared.
__device__ __forceinline__ void next_digit(KeepLds& l, int digit, int a0, int a1, Limit& x) {
  const int d = kBins - 1 - 2 * (int)threadIdx.x;
  int total;
  const int end = block_scan<int, kKeepWaves>(a0 + a1, l.sums, &total), begin = end - a0 - a1;
  if (begin < x.ties && end >= x.ties) {
    const bool first = begin + a0 >= x.ties;
    l.found[0] = first ? d : d - 1;
    l.found[1] = x.ties - (first ? begin : begin + a0);
    l.found[2] = first ? a0 : a1;
  }
  __syncthreads();
  x.prefix = x.prefix << Limit::bits(digit) | (uint32_t)l.found[0];
  x.ties = l.found[1];
  x.among = l.found[2];
  x.value = x.prefix << Limit::shift(digit);
}

// This thread's `mine` <= N neighbouring tokens from `first` on, of weights x: those that stay are written behind `above` and, of the limit's
// equals, min(equal, ties) that stay before them.  All of x is in registers, so the weights may go over those that they
// were read from.  What the workgroup's tokens add to above, and 2^16 times what they add to equal.
template <int N>
__device__ __forceinline__ int write_kept(const Choice& c, const Limit& limit, const float (&x)[N], int first, int mine, int above, int equal,
                                           int* lds, int32_t* kept, float* moved) {
  uint32_t up = 0, same = 0;  // bits of the tokens that stay whatever the equals do, and of those
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < mine) {
      const int j = first + i;
      const uint32_t o = order_of(x[i]);
      const bool sure = !c.between(j) || o > limit.value;
      up |= (j < c.n && sure ? 1u : 0u) << i;
      same |= (j < c.n && !sure && o == limit.value ? 1u : 0u) << i;
    }
  const int own = __popc(up) | __popc(same) << 16;  // of 16384 tokens: the sums stay apart
  int total;
  const int before = block_scan<int, kKeepWaves>(own, lds, &total) - own;
  int e = equal + (before >> 16), to = above + (before & 0xffff) + min(e, limit.ties);
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < mine && ((up | same) >> i & 1) && ((up >> i & 1) || e++ < limit.ties)) {
      kept[to] = first + i;
      if (moved) moved[to] = x[i];
      ++to;
    }
  return total;
}

// One workgroup a sequence and KV head of up to 16384 tokens, whose weights stay in registers: bound by the digits' rounds, each a clear, an addition
// and a scan of the bins.  32 sequences of 700 to 4100 tokens, 8 heads, 12 us; one of 16384 tokens 15 us, 64 of them 50 (the three launches below 22 and 55).
__device__ __forceinline__ void keep_alone(const KeepArgs& a, const Choice& c, KeepLds& l) {
  const int tid = threadIdx.x, mine = (c.n + kKeepThreads - 1) / kKeepThreads, first = tid * mine;
  const float* weights = a.weights + (int64_t)blockIdx.x * a.width;
  float x[kMost];
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    x[i] = 0.f;
    if (i < mine && first + i < min(c.n, c.held)) x[i] = weights[first + i];
  }
  Limit limit{0, 0xffffffffu, c.wanted, -1};
  if (c.wanted > 0) {
#pragma unroll 1
    for (int digit = 0; digit < 3 && !limit.all_stay(); ++digit) {
      clear(l);
#pragma unroll
      for (int i = 0; i < kMost; ++i)
        if (i < mine && c.between(first + i)) add(l, digit, limit.prefix, order_of(x[i]));
      __syncthreads();
      const int d = kBins - 1 - 2 * tid;
      next_digit(l, digit, bin(l, d), bin(l, d - 1), limit);
    }
    limit.close();
    __syncthreads();
  }
  write_kept<kMost>(c, limit, x, first, mine, 0, 0, l.sums, a.kept + (int64_t)blockIdx.x * a.cap,
                    a.new_weights ? a.new_weights + (int64_t)blockIdx.x * a.width : nullptr);
}

// The places behind the last that stays.
__device__ __forceinline__ void fill_rest(const KeepArgs& a, const Choice& c, int part, int parts) {
  int32_t* kept = a.kept + (int64_t)blockIdx.x * a.cap;
  for (int i = (c.any ? c.m : 0) + part * kKeepThreads + (int)threadIdx.x; i < a.cap; i += parts * kKeepThreads) kept[i] = -1;
  if (part == 0 && blockIdx.x % a.hkv == 0 && threadIdx.x == 0) a.count[blockIdx.x / a.hkv] = c.any ? c.m : 0;
}

__global__ __launch_bounds__(kKeepThreads) void cache_keep(KeepArgs a) {
  __shared__ KeepLds l;
  const Choice c(a, blockIdx.x / a.hkv);
  fill_rest(a, c, 0, 1);
  if (c.any) keep_alone(a, c, l);
}

// Where the weights' rows are longer, three launches: each workgroup has a chunk of a sequence and KV head (one of up to 16384 tokens is
// the first launch's alone), a piece of 8192 tokens or, of more than 128 pieces, several, so that what every workgroup does for all chunks
// grows no faster than the tokens.  1: the first digit's bins of each chunk.  2: their sums give the digit; each chunk counts its weights
// above it and lists those that share it.  3: every workgroup finds the other digits from the list, counts what stays in the chunks
// before its own, and writes its own.  Where more than 16384 share the digit every workgroup goes over all weights in place of the list, three
// times: 2^20 equal weights, 4 heads, 1.1 ms; 2^23 of them 8.5 (with a workgroup for each piece 62).
// 100003 tokens, 4 heads: 4.9 + 9.0 + 12.6 us, latency throughout; one workgroup alone, at 20 instructions a weight and digit on one CU, 88 to 111.
__host__ __device__ __forceinline__ int most_chunks(int width) {
  const int pieces = (width + kPiece - 1) / kPiece;
  return pieces < kMostChunks ? pieces : kMostChunks;
}

struct KeepSpace {
  int chunks;
  int* hist;      // [chunks][kBins], a head
  int* above;     // [chunks]
  int* info;      // weights listed, and what 2 has found: digit, ties, among
  uint2* list;    // (weight, chunk)
  float* copy;    // [width]: of the weights, where they are written over
  static size_t bytes(int width, bool in_place) {
    const size_t chunks = most_chunks(width);
    return (chunks * (kBins + 1) * 4 + 16 + (size_t)kList * 8 + (in_place ? (size_t)width * 4 : 0) + 255) & ~(size_t)255;
  }
  __device__ __forceinline__ KeepSpace(const KeepArgs& a, bool in_place) {
    chunks = most_chunks(a.width);
    const size_t each = ((size_t)chunks * (kBins + 1) * 4 + 16 + (size_t)kList * 8 + (in_place ? (size_t)a.width * 4 : 0) + 255) & ~(size_t)255;
    char* p = a.ws + (size_t)blockIdx.x * each;
    list = reinterpret_cast<uint2*>(p);
    info = reinterpret_cast<int*>(list + kList);
    hist = info + 4;
    above = hist + (size_t)chunks * kBins;
    copy = reinterpret_cast<float*>(above + chunks);
  }
};

// Tokens of a chunk, whole pieces, and the chunks of a sequence.
__device__ __forceinline__ int chunk_tokens(const Choice& c) { return ((c.n - 1) / (kPiece * kMostChunks) + 1) * kPiece; }
__device__ __forceinline__ int chunks_of(const Choice& c) { return (c.n - 1) / chunk_tokens(c) + 1; }

// fn(first token) of each piece of a chunk.
template <typename Fn>
__device__ __forceinline__ void each_piece(const Choice& c, int chunk, Fn fn) {
  const int tokens = chunk_tokens(c), end = min((chunk + 1) * tokens, c.n);
#pragma unroll 1
  for (int first = chunk * tokens; first < end; first += kPiece) fn(first);
}

// f(position, weight) for this thread's tokens of the piece from `first` on.
template <typename F>
__device__ __forceinline__ void each_weight(const Choice& c, const float* weights, int first, F f) {
  float x[kPart];
#pragma unroll
  for (int i = 0; i < kPart; ++i) {
    const int j = first + i * kKeepThreads + (int)threadIdx.x;
    x[i] = j < min(c.n, c.held) ? weights[j] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < kPart; ++i) {
    const int j = first + i * kKeepThreads + (int)threadIdx.x;
    if (j < c.n) f(j, x[i]);
  }
}

// The workgroup's sum, on every thread; ends with lds in use.
__device__ __forceinline__ int block_sum(int x, int* lds) {
  int total;
  block_scan<int, kKeepWaves>(x, lds, &total);
  return total;
}

__global__ __launch_bounds__(kKeepThreads) void keep_count(KeepArgs a) {
  __shared__ KeepLds l;
  const Choice c(a, blockIdx.x / a.hkv);
  const int chunk = blockIdx.y, tid = threadIdx.x;
  const bool alone = !c.any || c.n <= kMost * kKeepThreads;
  const int parts = alone ? 1 : chunks_of(c);
  if (chunk >= parts) return;
  fill_rest(a, c, chunk, parts);
  if (!c.any) return;
  if (alone) return keep_alone(a, c, l);
  const bool in_place = a.new_weights == a.weights;
  const KeepSpace w(a, in_place);
  if (chunk == 0 && tid == 0) w.info[0] = 0;
  clear(l);
  each_piece(c, chunk, [&](int first) {
    each_weight(c, a.weights + (int64_t)blockIdx.x * a.width, first, [&](int j, float x) {
      if (in_place) w.copy[j] = x;
      if (c.between(j)) add(l, 0, 0, order_of(x));
    });
  });
  __syncthreads();
  reinterpret_cast<int2*>(w.hist + (size_t)chunk * kBins)[tid] = make_int2(bin(l, 2 * tid), bin(l, 2 * tid + 1));
}

__global__ __launch_bounds__(kKeepThreads) void keep_list(KeepArgs a) {
  __shared__ KeepLds l;
  const Choice c(a, blockIdx.x / a.hkv);
  const int chunk = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  if (!c.any || c.n <= kMost * kKeepThreads || chunk >= chunks_of(c)) return;
  const KeepSpace w(a, a.new_weights == a.weights);
  Limit limit{0, 0xffffffffu, c.wanted, -1};
  if (c.wanted > 0) {
    int2 sum = {0, 0};  // of digits 2046 - 2 tid and 2047 - 2 tid
    const int n = chunks_of(c);
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const int2 x = reinterpret_cast<const int2*>(w.hist + (size_t)i * kBins)[kKeepThreads - 1 - tid];
      sum.x += x.x;
      sum.y += x.y;
    }
    next_digit(l, 0, sum.y, sum.x, limit);
    if (chunk == 0 && tid == 0) {
      w.info[1] = (int)limit.prefix;
      w.info[2] = limit.ties;
      w.info[3] = limit.among;
    }
  }
  const bool open = c.wanted > 0 && !limit.all_stay();  // some of those that share the digit stay, some do not
  limit.close();
  int more = 0;
  each_piece(c, chunk, [&](int first) {
    int hits = 0;
    uint32_t o[kPart];
    each_weight(c, a.weights + (int64_t)blockIdx.x * a.width, first, [&](int j, float x) {
      const uint32_t y = order_of(x);
      const bool shares = open && c.between(j) && y >> Limit::shift(0) == limit.prefix;
      if (shares) {
#pragma unroll
        for (int i = 0; i < kPart; ++i)
          if (i == hits) o[i] = y;
        ++hits;
      } else {
        more += !c.between(j) || y > limit.value;
      }
    });
    if (open && limit.among <= kList) {
      const int end = wave_scan(hits);
      int to = 0;
      if (lane == kWave - 1 && end > 0) to = atomicAdd(&w.info[0], end);
      to = __builtin_amdgcn_readlane(to, kWave - 1) + end - hits;
#pragma unroll
      for (int i = 0; i < kPart; ++i)
        if (i < hits) w.list[to + i] = make_uint2(o[i], chunk);
    }
  });
  __syncthreads();
  more = block_sum(more, l.sums);
  if (tid == 0) w.above[chunk] = more;
}

__global__ __launch_bounds__(kKeepThreads) void keep_write(KeepArgs a) {
  __shared__ KeepLds l;
  const Choice c(a, blockIdx.x / a.hkv);
  const int chunk = blockIdx.y, tid = threadIdx.x;
  if (!c.any || c.n <= kMost * kKeepThreads || chunk >= chunks_of(c)) return;
  const bool in_place = a.new_weights == a.weights;
  const KeepSpace w(a, in_place);
  const float* weights = in_place ? w.copy : a.weights + (int64_t)blockIdx.x * a.width;
  Limit limit{0, 0xffffffffu, c.wanted, -1};
  int above = 0, equal = 0;
  for (int i = tid; i < chunk; i += kKeepThreads) above += w.above[i];
  if (c.wanted > 0) {
    limit.prefix = (uint32_t)w.info[1];
    limit.value = limit.prefix << Limit::shift(0);
    limit.ties = w.info[2];
    limit.among = w.info[3];
    if (!limit.all_stay()) {
      const bool listed = limit.among <= kList;
      const int entries = listed ? limit.among : 0;
      uint2 x[kList / kKeepThreads];
#pragma unroll
      for (int i = 0; i < kList / kKeepThreads; ++i)
        if (i * kKeepThreads + tid < entries) x[i] = w.list[i * kKeepThreads + tid];
      const auto each = [&](int end, auto f) {  // f(order, chunk) for those that share the first digit, of chunks below end
        if (listed) {
#pragma unroll
          for (int i = 0; i < kList / kKeepThreads; ++i)
            if (i * kKeepThreads + tid < entries) f(x[i].x, (int)x[i].y);
        } else {
          for (int i = 0; i < end; ++i)
            each_piece(c, i, [&](int first) {
              each_weight(c, weights, first, [&](int j, float y) {
                const uint32_t o = order_of(y);
                if (c.between(j) && o >> Limit::shift(0) == (uint32_t)w.info[1]) f(o, i);
              });
            });
        }
      };
#pragma unroll 1
      for (int digit = 1; digit < 3 && !limit.all_stay(); ++digit) {
        clear(l);
        each(chunks_of(c), [&](uint32_t o, int) { add(l, digit, limit.prefix, o); });
        __syncthreads();
        const int d = kBins - 1 - 2 * tid;
        next_digit(l, digit, bin(l, d), bin(l, d - 1), limit);
      }
      limit.close();
      each(chunk, [&](uint32_t o, int of) {
        above += of < chunk && o > limit.value;
        equal += of < chunk && o == limit.value;
      });
    } else {
      limit.close();
    }
  }
  __syncthreads();
  above = block_sum(above, l.sums);
  __syncthreads();
  equal = block_sum(equal, l.sums);
  __syncthreads();
  each_piece(c, chunk, [&](int piece) {
    float x[kPart];
    const int first = piece + tid * kPart;
#pragma unroll
    for (int i = 0; i < kPart; ++i) x[i] = first + i < min(c.n, c.held) ? weights[first + i] : 0.f;
    const int total = write_kept<kPart>(c, limit, x, first, kPart, above, equal, l.sums, a.kept + (int64_t)blockIdx.x * a.cap,
                                        a.new_weights ? a.new_weights + (int64_t)blockIdx.x * a.width : nullptr);
    above += total & 0xffff;
    equal += total >> 16;
    __syncthreads();  // the sums are done with
  });
}

// The smallest e >= kScaleExpMin with x 2^8 <= MAX 2^e, from a value of at most eight significant bits.
template <int FMT>
__device__ __forceinline__ int page_exp(float x) {
  const int bits = (int)(__float_as_uint(x) >> 16), man = bits & 127, exp = (bits >> 7) - 127 + 8;
  const int e = FMT == kCacheE4M3 ? exp - 8 + (man > 96) : exp - 6 + (man > 126);
  return e < kScaleExpMin ? kScaleExpMin : e > kScaleExpMax ? kScaleExpMax : e;
}

// Four values times f, |x f| <= MAX, to codes.  int8: x f + 128 is exact in 32 bits wherever its rounding is in question (x
// has eight significant bits), and the conversion to a byte rounds to even.
template <int FMT>
__device__ __forceinline__ uint32_t pack_codes(const float* x, float f) {
  if constexpr (FMT == kCacheE4M3) {
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * f, x[1] * f, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * f, x[3] * f, r, true);
  } else {
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) r = __builtin_amdgcn_cvt_pk_u8_f32(__builtin_fmaf(x[i], f, 128.f), i, r);
    return r ^ 0x80808080u;
  }
}

// One workgroup a page of the new table and KV head, 256 threads a tile.  K comes in the chunks that it will stand in, a token's 16
// elements.  A chunk of V holds 16 tokens of an element, of which some stay: tokens of one chunk that follow one another make a run,
// and a wave takes a run's chunks of 64 elements and deals the bytes that stay out to the new chunks in LDS.  Bound by HBM, which reads the whole
// chunks of V, most of the pages where every third token stays: 32 sequences of 700 to 4100 tokens cut to 1024, 8 heads (186 MB read, 65
// written), 56 us, 4.4 TB/s; 100003 tokens cut to 16384, 4 heads (90 and 17 MB), 22 us, 4.8 TB/s.  Byte by byte from memory 62 and 26 us; 512 threads
// a tile 70 and 27; items in the order of the XCDs 62 to 65; five waves a SIMD spill.  Values are formed as x 2^-8, which keeps the largest
// finite, and become codes under the exponent of the largest.
template <int FMT, int TILES>
__global__ __launch_bounds__(256 * TILES) void cache_gather(GatherArgs a) {
  constexpr int B = TILES * kTile, kThreads = 256 * TILES, kChunks = kTileBytes / kChunk, kMine = TILES * kChunks / kThreads;
  __shared__ int64_t from[B];                                   // the token's first byte of K
  __shared__ __attribute__((aligned(16))) float scale[2][B];    // 2^(e - 8)
  __shared__ __attribute__((aligned(16))) uint8_t there[B];     // 255, or 0: none
  __shared__ int64_t run_at[TILES][kTile];                      // a run's first byte of V
  __shared__ int run_mask[TILES][kTile], run_to[TILES][kTile], runs[TILES];  // its tokens of the 16, place of the first, runs
  __shared__ __attribute__((aligned(16))) uint8_t stage[TILES][kTileBytes];
  __shared__ float tops[2][kThreads / kWave];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t items = (int64_t)a.n_seqs * a.c.hkv * a.new_pages;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int slot = (int)(item % a.new_pages), sh = (int)(item / a.new_pages), s = sh / a.c.hkv, h = sh - s * a.c.hkv;
    // (what the page is to hold is loaded beside the count, which may say that it is not wanted)
    const int at = slot * B + tid, wanted = tid < B && at < a.cap ? a.kept[(int64_t)sh * a.cap + at] : -1;
    const int n = min(a.count[s], a.cap) - slot * B;  // tokens from this page on
    const int page = a.new_table[(int64_t)s * a.new_pages + slot];
    if (n <= 0 || page < 0 || page >= a.c.n_pages) continue;
    const int64_t to = (int64_t)page * a.c.hkv + h;
    __syncthreads();  // the last item's places are done with
    float of[2] = {0.f, 0.f};
    if (w < TILES) {  // a wave a tile, a lane a token
      const int j = tid < n ? wanted : -1;
      const int p = j >= 0 && j < a.max_pages * B ? a.table[(int64_t)s * a.max_pages + j / B] : -1;
      const bool ok = p >= 0 && p < a.c.n_pages;
      const int64_t ph = ok ? (int64_t)p * a.c.hkv + h : to;
      const int t = ok ? j % kTile : 0;
      const int64_t first = (ph * TILES + (ok ? j % B / kTile : 0)) * (2 * kTileBytes);
      from[tid] = first + ((t >> 2 & 3) * 128 + (t >> 4) * 4 + (t & 3)) * kChunk;
      there[tid] = ok ? 255 : 0;
      const int before = __shfl_up(ok ? j : -1, 1);
      const bool begins = ok && (lane == 0 || before < 0 || before / 16 != j / 16 || before >= j);
      const unsigned long long all = __ballot(begins);
      const int run = __popcll(all & ((2ull << lane) - 1)) - 1;
      run_mask[w][lane] = 0;
      if (begins) {
        run_at[w][run] = first + kTileBytes + (t >> 4) * 256;
        run_to[w][run] = lane;
      }
      if (lane == 0) runs[w] = __popcll(all);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (ok) atomicOr(&run_mask[w][run], 1 << (t & 15));
      if (ok) {
        of[0] = a.scales[2 * ph];
        of[1] = a.scales[2 * ph + 1];
      }
    }
    __syncthreads();
    u32x4 c[2][kMine];
#pragma unroll
    for (int y = 0; y < kMine; ++y) {  // K: chunk (t, half, g, r), token 16 (r / 4) + 4 t + r % 4
      const int ch = y * kThreads + tid, tile = ch / kChunks, in = ch % kChunks, g = in >> 4 & 3, r = in & 15;
      const int i = tile * kTile + 16 * (r >> 2) + 4 * (in >> 7) + (r & 3);
      c[0][y] = *reinterpret_cast<const u32x4*>(a.pages + from[i] + ((in >> 6 & 1) * 64 + g * 16) * kChunk);
    }
    {  // V: elements 64 (w % 2) + lane = 16 dt + r of every second run
      const int tile = w >> 2, own = ((w & 1) * 4 + (lane >> 4)) * 64 + (lane & 15);
      const int count = __builtin_amdgcn_readfirstlane(runs[tile]);
      constexpr int kAhead = 8;
      for (int q0 = w >> 1 & 1; q0 < count; q0 += 2 * kAhead) {
        u32x4 x[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
          x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.pages + run_at[tile][min(q0 + 2 * i, count - 1)] + own * kChunk));
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int q = q0 + 2 * i;
          if (q < count) {
            const int mask = __builtin_amdgcn_readfirstlane(run_mask[tile][q]);
            int place = __builtin_amdgcn_readfirstlane(run_to[tile][q]);
            uint8_t* dst = &stage[tile][own * kChunk];
#pragma unroll
            for (int b = 0; b < 16; ++b)
              if (mask >> b & 1) {
                dst[(place >> 4) * 256 + (place & 15)] = (uint8_t)(x[i][b >> 2] >> (8 * (b & 3)));
                ++place;
              }
          }
        }
      }
    }
    if (tid < B) {
#pragma unroll
      for (int x = 0; x < 2; ++x) scale[x][tid] = pow2f(stored_exp(of[x]) - 8);
    }
    __syncthreads();
    // The 16 values of a thread's chunk y, K's and V's.
    const auto values = [&](int y, float (&k)[16], float (&v)[16]) {
      const int ch = y * kThreads + tid, tile = ch / kChunks, in = ch % kChunks, g = in >> 4 & 3, r = in & 15;
      const float f = scale[0][tile * kTile + 16 * (r >> 2) + 4 * (in >> 7) + (r & 3)];
      const f32x4* fv = reinterpret_cast<const f32x4*>(&scale[1][tile * kTile + 16 * g]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4 kc = from_codes<FMT>(c[0][y][e]), vc = from_codes<FMT>(c[1][y][e]);
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          k[4 * e + z] = kc[z] * f;
          v[4 * e + z] = vc[z] * fv[e][z];
        }
      }
    };
    float top[2] = {0.f, 0.f};
#pragma unroll
    for (int y = 0; y < kMine; ++y) {
      const int ch = y * kThreads + tid, tile = ch / kChunks, in = ch % kChunks, g = in >> 4 & 3, r = in & 15;
      const uint32_t mask = there[tile * kTile + 16 * (r >> 2) + 4 * (in >> 7) + (r & 3)] * 0x01010101u;
      // V: chunk (dt, g, r), element 16 dt + r of tokens 16 g + [0, 16)
      c[1][y] = *reinterpret_cast<const u32x4*>(&stage[tile][in * kChunk]);
      const uint32_t* mv = reinterpret_cast<const uint32_t*>(&there[tile * kTile + 16 * g]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c[0][y][e] = without_nan<FMT>(c[0][y][e] & mask);
        c[1][y][e] = without_nan<FMT>(c[1][y][e] & mv[e]);
      }
      float k[16], v[16];
      values(y, k, v);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        top[0] = fmaxf(top[0], fabsf(k[e]));
        top[1] = fmaxf(top[1], fabsf(v[e]));
      }
    }
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      top[z] = wave_max(top[z]);
      if (lane == 0) tops[z][w] = top[z];
    }
    __syncthreads();
    int e_new[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      float t = tops[z][0];
#pragma unroll
      for (int i = 1; i < kThreads / kWave; ++i) t = fmaxf(t, tops[z][i]);
      e_new[z] = page_exp<FMT>(t);
    }
    if (tid < 2) a.scales[2 * to + tid] = pow2f(tid == 0 ? e_new[0] : e_new[1]);
    const float down[2] = {pow2f(8 - e_new[0]), pow2f(8 - e_new[1])};
#pragma unroll
    for (int y = 0; y < kMine; ++y) {
      const int ch = y * kThreads + tid;
      u32x4* dst = reinterpret_cast<u32x4*>(a.pages + (to * TILES + ch / kChunks) * (2 * kTileBytes)) + ch % kChunks;
      float k[16], v[16];
      values(y, k, v);
      u32x4 kq, vq;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        kq[e] = pack_codes<FMT>(&k[4 * e], down[0]);
        vq[e] = pack_codes<FMT>(&v[4 * e], down[1]);
      }
      dst[0] = kq;
      dst[kChunks] = vq;
    }
  }
}

}  // namespace

size_t cache_keep_bytes(int64_t heads, int width, bool in_place) {
  return width <= kMost * kKeepThreads ? 0 : (size_t)heads * KeepSpace::bytes(width, in_place);
}

hipError_t launch_cache_keep(const KeepArgs& a, hipStream_t stream) {
  const unsigned heads = (unsigned)(a.n_seqs * a.hkv);
  if (a.width <= kMost * kKeepThreads) {
    hipLaunchKernelGGL(cache_keep, dim3(heads), dim3(kKeepThreads), 0, stream, a);
  } else {
    const dim3 grid(heads, (unsigned)most_chunks(a.width));
    hipLaunchKernelGGL(keep_count, grid, dim3(kKeepThreads), 0, stream, a);
    hipLaunchKernelGGL(keep_list, grid, dim3(kKeepThreads), 0, stream, a);
    hipLaunchKernelGGL(keep_write, grid, dim3(kKeepThreads), 0, stream, a);
  }
  return hipGetLastError();
}

hipError_t launch_cache_gather(const GatherArgs& a, hipStream_t stream) {
  const int64_t items = (int64_t)a.n_seqs * a.c.hkv * a.new_pages;
  const dim3 grid((unsigned)(items < 65536 ? items : 65536)), threads(256 * a.c.tiles);
  if (a.c.fmt == kCacheE4M3) {
    if (a.c.tiles == 1) hipLaunchKernelGGL((cache_gather<kCacheE4M3, 1>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((cache_gather<kCacheE4M3, 2>), grid, threads, 0, stream, a);
  } else {
    if (a.c.tiles == 1) hipLaunchKernelGGL((cache_gather<kCacheInt8, 1>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((cache_gather<kCacheInt8, 2>), grid, threads, 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace crisp
