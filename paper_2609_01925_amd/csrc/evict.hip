// Eviction from the 8-bit paged K/V cache: the choice of the tokens that stay, and their move to pages of their own.
#include "cache_device.h"

namespace crisp {

namespace {

constexpr int kKeepThreads = 1024, kKeepWaves = kKeepThreads / kWave;
constexpr int kBins = 2048;                            // of a digit of 11 bits (the last has 10)
constexpr int kRow = 16, kSpan = kRow * kKeepThreads;  // tokens of a thread and of the workgroup at a time

// An unsigned order of floats: NaN lowest, -0 equal to 0.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return x != x ? 0u : (b >> 31) ? ~b : b | 0x80000000u;
}

// One workgroup a sequence and KV head.  The k-th largest weight is found by three digits of its bits, from the top, a histogram in LDS
// for each; what is above it stays, and of its equals the first.  Then the tokens go by once more, in order and kSpan at a
// time, each wave counting its own by ballots, so that what stays is written in ascending order and, since a span is
// in registers before any of it is written, also over the weights that it was read from.
__global__ __launch_bounds__(kKeepThreads) void cache_keep(KeepArgs a) {
  __shared__ int hist[kBins];
  __shared__ int sums[kKeepWaves], found[2];
  __shared__ int2 counts[2][kKeepWaves];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int s = blockIdx.x / a.hkv, h = blockIdx.x % a.hkv;
  const int n = a.seq_len[s], m = a.keep[s], held = a.held[s];
  int32_t* kept = a.kept + (int64_t)blockIdx.x * a.cap;
  const bool chosen = n <= a.width && m > 0 && m < n && m <= a.cap;
  if (h == 0 && tid == 0) a.count[s] = chosen ? m : 0;
  for (int i = (chosen ? m : 0) + tid; i < a.cap; i += kKeepThreads) kept[i] = -1;
  if (!chosen) return;
  const float* weights = a.weights + (int64_t)blockIdx.x * a.width;
  float* moved = a.new_weights ? a.new_weights + (int64_t)blockIdx.x * a.width : nullptr;
  const auto weight = [&](int j) { return j < held ? weights[j] : 0.f; };
  const int recent = min(a.recent, m), sink = min(a.sink, m - recent), lo = sink, hi = n - recent;

  uint32_t limit = 0xffffffffu;  // the weight that the k-th largest has: all above it stay, and `ties` of its equals
  int ties = m - recent - sink;
  if (ties > 0) {
    uint32_t prefix = 0;
#pragma unroll
    for (int digit = 0; digit < 3; ++digit) {
      const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit < 2 ? 11 : 10;
      for (int i = tid; i < kBins; i += kKeepThreads) hist[i] = 0;
      __syncthreads();
      for (int j = lo + tid; j < hi; j += kKeepThreads) {
        const uint32_t x = order_of(weight(j));
        if (digit == 0 || x >> (shift + bits) == prefix) atomicAdd(&hist[x >> shift & ((1u << bits) - 1)], 1);
      }
      __syncthreads();
      // from the highest digit down: the one in which the count passes the ties that are still wanted
      const int d = kBins - 1 - 2 * tid, a0 = hist[d], a1 = hist[d - 1];
      int total;
      const int end = block_scan<int, kKeepWaves>(a0 + a1, sums, &total), begin = end - a0 - a1;
      if (begin < ties && end >= ties) {
        const bool first = begin + a0 >= ties;
        found[0] = first ? d : d - 1;
        found[1] = ties - (first ? begin : begin + a0);
      }
      __syncthreads();
      prefix = prefix << bits | (uint32_t)found[0];
      ties = found[1];
    }
    limit = prefix;
  }
  int above = 0, equal = 0;  // of the spans before
  for (int j0 = 0, turn = 0; j0 < n; j0 += kSpan, turn ^= 1) {
    const int at = j0 + w * (kRow * kWave) + lane;
    float x[kRow];
    unsigned long long up[kRow], same[kRow];
    int2 mine = {0, 0};
#pragma unroll
    for (int i = 0; i < kRow; ++i) x[i] = at + i * kWave < n ? weight(at + i * kWave) : 0.f;
#pragma unroll
    for (int i = 0; i < kRow; ++i) {
      const int j = at + i * kWave;
      const bool sure = j < lo || j >= hi;
      const uint32_t o = order_of(x[i]);
      up[i] = __ballot(j < n && (sure || o > limit));
      same[i] = __ballot(j < n && !sure && o == limit);
      mine.x += __popcll(up[i]);
      mine.y += __popcll(same[i]);
    }
    if (lane == 0) counts[turn][w] = mine;
    __syncthreads();
    int2 before = {above, equal};
#pragma unroll
    for (int i = 0; i < kKeepWaves; ++i) {
      const int2 y = counts[turn][i];
      if (i < w) {
        before.x += y.x;
        before.y += y.y;
      }
      above += y.x;
      equal += y.y;
    }
    const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < kRow; ++i) {
      const int e = before.y + __popcll(same[i] & below), to = before.x + __popcll(up[i] & below) + min(e, ties);
      if ((up[i] >> lane & 1) || ((same[i] >> lane & 1) && e < ties)) {
        kept[to] = at + i * kWave;
        if (moved) moved[to] = x[i];
      }
      before.x += __popcll(up[i]);
      before.y += __popcll(same[i]);
    }
  }
}

constexpr int kThreads = 256;

// |code| 2^-8 of four codes' largest, each under its own scale 2^e, given as 2^(e - 8): the 2^-8 keeps the largest finite.
template <int FMT>
__device__ __forceinline__ float largest(uint32_t codes, f32x4 scale, float top) {
  const f32x4 v = from_codes<FMT>(codes);
#pragma unroll
  for (int i = 0; i < 4; ++i) top = fmaxf(top, fabsf(v[i]) * scale[i]);
  return top;
}

// The smallest e >= kScaleExpMin with x 2^8 <= MAX 2^e, from a value of at most eight significant bits.
template <int FMT>
__device__ __forceinline__ int page_exp(float x) {
  const int bits = (int)(__float_as_uint(x) >> 16), man = bits & 127, exp = (bits >> 7) - 127 + 8;
  const int e = FMT == kCacheE4M3 ? exp - 8 + (man > 96) : exp - 6 + (man > 126);
  return e < kScaleExpMin ? kScaleExpMin : e;
}

__device__ __forceinline__ float pow2_held(int e) { return pow2f(e < -126 ? -126 : e > 126 ? 126 : e); }

// One workgroup a page of the new table and KV head: for each of its tokens the place that it comes from, then a thread some
// chunks of 16 bytes, loaded as they will stand: of K a token's 16 elements, of V an element of 16 tokens, byte by byte
// (neighbouring tokens share the lines).  The page's exponent is that of the largest value.
template <int FMT, int TILES>
__global__ __launch_bounds__(kThreads) void cache_gather(GatherArgs a) {
  constexpr int B = TILES * kTile, kChunks = kTileBytes / kChunk, kEach = TILES * kChunks / kThreads;
  __shared__ int64_t from[B];       // byte of the token's tile of K; negative: none
  __shared__ int place[B];          // its place in the tile
  __shared__ int exps[2][B];
  __shared__ float tops[2][kThreads / kWave];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int64_t items = (int64_t)a.n_seqs * a.c.hkv * a.new_pages;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int slot = (int)(item % a.new_pages), sh = (int)(item / a.new_pages), s = sh / a.c.hkv, h = sh - s * a.c.hkv;
    const int n = min(a.count[s], a.cap) - slot * B;  // tokens from this page on
    const int page = a.new_table[(int64_t)s * a.new_pages + slot];
    if (n <= 0 || page < 0 || page >= a.c.n_pages) continue;
    __syncthreads();  // the last item's places are done with
    for (int i = tid; i < B; i += kThreads) {
      const int j = i < n ? a.kept[(int64_t)sh * a.cap + slot * B + i] : -1;
      const int p = j >= 0 && j < a.max_pages * B ? a.table[(int64_t)s * a.max_pages + j / B] : -1;
      const bool ok = p >= 0 && p < a.c.n_pages;
      const int64_t ph = (int64_t)p * a.c.hkv + h;
      from[i] = ok ? (ph * TILES + j % B / kTile) * (2 * kTileBytes) : -1;
      place[i] = j % kTile;
      exps[0][i] = ok ? stored_exp(a.scales[2 * ph]) : 0;
      exps[1][i] = ok ? stored_exp(a.scales[2 * ph + 1]) : 0;
    }
    __syncthreads();
    u32x4 c[2][kEach];
    float top[2] = {0.f, 0.f};
#pragma unroll
    for (int y = 0; y < kEach; ++y) {
      const int ch = y * kThreads + tid, tile = ch / kChunks, in = ch % kChunks, g = in >> 4 & 3, r = in & 15;
      {  // K: chunk (t, half, g, r), token 16 (r / 4) + 4 t + r % 4
        const int i = tile * kTile + 16 * (r >> 2) + 4 * (in >> 7) + (r & 3), t = place[i];
        c[0][y] = u32x4{0, 0, 0, 0};
        if (from[i] >= 0)
          c[0][y] = *reinterpret_cast<const u32x4*>(a.pages + from[i] + ((((t >> 2 & 3) * 2 + (in >> 6 & 1)) * 4 + g) * 16 + (t >> 4) * 4 + (t & 3)) * 16);
        const float f = pow2_held(exps[0][i] - 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          c[0][y][e] = without_nan<FMT>(c[0][y][e]);
          top[0] = largest<FMT>(c[0][y][e], f32x4{f, f, f, f}, top[0]);
        }
      }
      {  // V: chunk (dt, g, r), element 16 dt + r of tokens 16 g + [0, 16)
        const int at = (in >> 6) * 64 + r;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t x = 0;
          f32x4 f;
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const int i = tile * kTile + 16 * g + 4 * e + z, t = place[i];
            uint32_t byte = 0;
            if (from[i] >= 0) byte = a.pages[from[i] + kTileBytes + (at + (t >> 4) * 16) * 16 + (t & 15)];
            x |= byte << (8 * z);
            f[z] = pow2_held(exps[1][i] - 8);
          }
          c[1][y][e] = without_nan<FMT>(x);
          top[1] = largest<FMT>(c[1][y][e], f, top[1]);
        }
      }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      top[x] = wave_max(top[x]);
      if (lane == 0) tops[x][w] = top[x];
    }
    __syncthreads();
    int e_new[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float t = tops[x][0];
#pragma unroll
      for (int i = 1; i < kThreads / kWave; ++i) t = fmaxf(t, tops[x][i]);
      e_new[x] = page_exp<FMT>(t);
    }
    const int64_t to = (int64_t)page * a.c.hkv + h;
    if (tid < 2) a.scales[2 * to + tid] = pow2f(min(e_new[tid], kScaleExpMax));
#pragma unroll
    for (int y = 0; y < kEach; ++y) {
      const int ch = y * kThreads + tid, tile = ch / kChunks, in = ch % kChunks, g = in >> 4 & 3, r = in & 15;
      u32x4* dst = reinterpret_cast<u32x4*>(a.pages + (to * TILES + tile) * (2 * kTileBytes)) + in;
      const int i = tile * kTile + 16 * (r >> 2) + 4 * (in >> 7) + (r & 3);
      const float f = pow2_held(exps[0][i] - e_new[0]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4 k = from_codes<FMT>(c[0][y][e]), v = from_codes<FMT>(c[1][y][e]);
        c[0][y][e] = to_codes<FMT>(k[0] * f, k[1] * f, k[2] * f, k[3] * f);
        float d[4];
#pragma unroll
        for (int z = 0; z < 4; ++z) d[z] = v[z] * pow2_held(exps[1][tile * kTile + 16 * g + 4 * e + z] - e_new[1]);
        c[1][y][e] = to_codes<FMT>(d[0], d[1], d[2], d[3]);
      }
      dst[0] = c[0][y];
      dst[kChunks] = c[1][y];
    }
  }
}

}  // namespace

hipError_t launch_cache_keep(const KeepArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(cache_keep, dim3((unsigned)(a.n_seqs * a.hkv)), dim3(kKeepThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_cache_gather(const GatherArgs& a, hipStream_t stream) {
  const int64_t items = (int64_t)a.n_seqs * a.c.hkv * a.new_pages;
  const dim3 grid((unsigned)(items < 65536 ? items : 65536)), threads(kThreads);
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
