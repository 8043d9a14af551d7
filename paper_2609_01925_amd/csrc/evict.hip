// Eviction from the 8-bit paged K/V cache: the choice of the tokens that stay, and their move to pages of their own.
#include "cache_device.h"

namespace crisp {

namespace {

constexpr int kKeepThreads = 1024, kKeepWaves = kKeepThreads / kWave;
constexpr int kBins = 2048, kCopies = 8;               // of a digit of 11 bits (the last has 10)
constexpr int kEach = 16, kSpan = kEach * kKeepThreads;  // tokens of a thread and of the workgroup at a time
__device__ __forceinline__ int padded(int i) { return i + i / kEach; }  // neighbours of threads that have some each fall on different banks

// An unsigned order of floats: NaN lowest, -0 equal to 0.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return x != x ? 0u : (b >> 31) ? ~b : b | 0x80000000u;
}

// One workgroup a sequence and KV head.  The k-th largest weight is found by three digits of its bits, from the top, a histogram in LDS
// for each; what is above it stays, and of its equals the first.  Up to kSpan tokens are read once and stay in LDS; of more, the
// weights that share the digits so far are listed there as soon as they fit.  Then the tokens go by in order, each wave counting its own
// by ballots, so that what stays is written in ascending order and, since a span is in LDS before any of it is written,
// also over the weights that it was read from.  Weights share few exponents, so lanes add to eight copies of the bins.
__global__ __launch_bounds__(kKeepThreads) void cache_keep(KeepArgs a) {
  __shared__ __attribute__((aligned(16))) int hist[kBins][kCopies];
  __shared__ uint32_t raw[kSpan + kSpan / kEach];
  __shared__ int sums[kKeepWaves], found[3], n_few;
  __shared__ int sums2[2][kKeepWaves];
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
  const int recent = min(a.recent, m), sink = min(a.sink, m - recent), lo = sink, hi = n - recent;
  const bool whole = n <= kSpan;

  // f(j0, x): this thread's weights of each span, positions j0 + 1024 i + tid, read while the span before is worked on.
  const auto read = [&](int j0, float (&x)[kEach]) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) x[i] = weights[min(j0 + i * kKeepThreads + tid, n - 1)];
  };
  const auto spans = [&](auto f) {
    float x[kEach], next[kEach];
    read(0, next);
    for (int j0 = 0; j0 < n; j0 += kSpan) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int j = j0 + i * kKeepThreads + tid;
        x[i] = j < held ? next[i] : 0.f;
      }
      if (j0 + kSpan < n) read(j0 + kSpan, next);
      f(j0, x);
    }
  };
  const auto each = [&](auto f) {  // f(weight) for the ones to choose from
    spans([&](int j0, const float (&x)[kEach]) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int j = j0 + i * kKeepThreads + tid;
        if (j >= lo && j < hi) f(order_of(x[i]));
      }
    });
  };
  const auto store = [&](const float (&x)[kEach]) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) raw[padded(i * kKeepThreads + tid)] = __float_as_uint(x[i]);
  };
  if (whole) spans([&](int, const float (&x)[kEach]) { store(x); });  // a thread's own places, until the next barrier

  uint32_t limit = 0xffffffffu;  // the weight that the k-th largest has: all above it stay, and `ties` of its equals
  int ties = m - recent - sink;
  if (ties > 0) {
    uint32_t prefix = 0;
    int listed = -1;  // weights in the list, once there is one
#pragma unroll 1
    for (int digit = 0; digit < 3; ++digit) {
      const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit < 2 ? 11 : 10;
      const uint64_t mask = (1u << bits) - 1;
      const auto add = [&](uint32_t o) {
        if ((uint64_t)o >> (shift + bits) == prefix) atomicAdd(&hist[o >> shift & mask][lane & (kCopies - 1)], 1);
      };
      for (int i = tid; i < kBins * kCopies / 4; i += kKeepThreads) reinterpret_cast<int4*>(hist)[i] = make_int4(0, 0, 0, 0);
      if (tid == 0) n_few = 0;
      __syncthreads();
      if (listed >= 0) {
        for (int i = tid; i < listed; i += kKeepThreads) add(raw[i]);
      } else if (whole) {
#pragma unroll 4
        for (int j = tid; j < n; j += kKeepThreads)
          if (j >= lo && j < hi) add(order_of(__uint_as_float(raw[padded(j)])));
      } else {
        each(add);
      }
      __syncthreads();
      // from the highest digit down: the one in which the count passes the ties that are still wanted
      const int d = kBins - 1 - 2 * tid;
      int a0 = 0, a1 = 0, total;
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        a0 += hist[d][i];
        a1 += hist[d - 1][i];
      }
      const int end = block_scan<int, kKeepWaves>(a0 + a1, sums, &total), begin = end - a0 - a1;
      if (begin < ties && end >= ties) {
        const bool first = begin + a0 >= ties;
        found[0] = first ? d : d - 1;
        found[1] = ties - (first ? begin : begin + a0);
        found[2] = first ? a0 : a1;
      }
      __syncthreads();
      prefix = prefix << bits | (uint32_t)found[0];
      ties = found[1];
      const int among = found[2];
      limit = prefix << shift;
      if (ties == among && limit > 0) {  // all that share the digits so far stay
        --limit;
        ties = 0;
        break;
      }
      if (digit < 2 && !whole && listed < 0 && among <= kSpan) {
        spans([&](int j0, const float (&x)[kEach]) {
          uint32_t hit = 0;
#pragma unroll
          for (int i = 0; i < kEach; ++i) {
            const int j = j0 + i * kKeepThreads + tid;
            hit |= (j >= lo && j < hi && order_of(x[i]) >> shift == prefix ? 1u : 0u) << i;
          }
          const int end = wave_scan(__popc(hit));
          int to = 0;
          if (lane == kWave - 1) to = atomicAdd(&n_few, end);
          to = __builtin_amdgcn_readlane(to, kWave - 1) + end - __popc(hit);
#pragma unroll
          for (int i = 0; i < kEach; ++i)
            if (hit >> i & 1) raw[to++] = order_of(x[i]);
        });
        listed = among;
        __syncthreads();
      }
    }
  }
  int above = 0, equal = 0, turn = 0;  // of the spans before
  const auto write = [&](int j0) {
    // a thread has `each` neighbouring tokens; bits of `up` stay whatever their equals do, those of `same` are equal to the limit
    const int mine = (min(n - j0, kSpan) + kKeepThreads - 1) / kKeepThreads, first = tid * mine;
    uint32_t up = 0, same = 0;
#pragma unroll 4
    for (int i = 0; i < mine; ++i) {
      const int j = j0 + first + i;
      const uint32_t o = order_of(__uint_as_float(raw[padded(first + i)]));
      const bool sure = j < lo || j >= hi || o > limit;
      up |= (j < n && sure ? 1u : 0u) << i;
      same |= (j < n && !sure && o == limit ? 1u : 0u) << i;
    }
    const int own = __popc(up) | __popc(same) << 16;  // of 16384 tokens: the sums stay apart
    int total;
    const int before = block_scan<int, kKeepWaves>(own, sums2[turn], &total) - own;
    int to = above + (before & 0xffff), e = equal + (before >> 16);
    to += min(e, ties);
    for (uint32_t todo = up | same; todo != 0; todo &= todo - 1) {
      const int i = __ffs(todo) - 1;
      if ((up >> i & 1) || e++ < ties) {
        kept[to] = j0 + first + i;
        if (moved) moved[to] = __uint_as_float(raw[padded(first + i)]);
        ++to;
      }
    }
    above += total & 0xffff;
    equal += total >> 16;
    turn ^= 1;
  };
  if (whole) {
    __syncthreads();
    write(0);
  } else {
    spans([&](int j0, const float (&x)[kEach]) {
      __syncthreads();  // the list, or the span before, is done with
      store(x);
      __syncthreads();
      write(j0);
    });
  }
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
// and a wave takes a run's chunks of 64 elements and deals the bytes that stay out to the new chunks in LDS (byte by byte from memory
// instead: 32 sequences of 700 to 4100 tokens cut to 1024, 8 heads, 62.4 us).  Values are formed as x 2^-8, which keeps the largest
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

hipError_t launch_cache_keep(const KeepArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(cache_keep, dim3((unsigned)(a.n_seqs * a.hkv)), dim3(kKeepThreads), 0, stream, a);
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
