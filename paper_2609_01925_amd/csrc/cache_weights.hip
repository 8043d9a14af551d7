// The attention weight that each cached token gets from new rows, summed over the rows and the query heads of its KV head:
//   w_j = sum_p exp2(x_pj - lse_p),  x_pj = scale log2(e) q_p . k_j,  lse_p = log2 sum_j exp2(x_pj)
// over the pairs p = i G + g of a sequence's rows i and the G query heads of the KV head.  A pair's sum over all keys has to be known
// before any of its weights, so the products are formed twice: weigh_rows leaves each pair's maximum and sum over a chunk of the
// tokens, weigh_join takes them together, and weigh_tokens forms the weights, a wave a tile of 64 tokens, and sums them over the pairs
// in registers, in a fixed order and without atomics.
#include "cache_device.h"

namespace crisp {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kGroup = 16;                  // pairs of one product
constexpr int kGroups = 8;                  // of a pass over the keys in weigh_rows
constexpr int kPairs = kGroup * kGroups;

struct WeightArgs {
  CacheDims c;
  BatchDims b;
  Seqs s;
  const uint16_t* q;
  Strides qs;
  const uint8_t* pages;
  const float* scales;
  const float* weights;
  float* out;
  const int32_t* held;
  int width, hq, G;
  int chunks;      // of a sequence, at most
  int token_wgs;   // workgroups of a sequence and KV head in weigh_tokens
  float c2;        // scale log2(e)
  float2* stats;   // [n_rows][hq][chunks]: maximum, sum
  float* lse;      // [n_rows][hq]
};

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float acc4;

__device__ __forceinline__ acc4 mfma16(bf16x8 a, bf16x8 b, acc4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ int tiles_of(const WeightArgs& a, const SeqRows& r) {
  return (min(r.len + r.n, a.b.max_pages * a.c.B) + kTile - 1) / kTile;
}
__device__ __forceinline__ int chunks_of(const WeightArgs& a, int tiles) { return min(a.chunks, (tiles + kWaves - 1) / kWaves); }

// K of a tile as the products' operands: k[4 t + kk] is 16 tokens t of elements 32 g + 8 kk + [0, 8).  kc takes products with codes
// to the base-2 exponent; false if the tile has no page.
struct KeyTile {
  bf16x8 k[16];
  float kc;
};
template <int FMT>
__device__ __forceinline__ bool load_keys(const WeightArgs& a, int seq, int head, int t, KeyTile& x) {
  const int slot = a.c.tiles == 2 ? t >> 1 : t;
  const int page = slot < a.b.max_pages ? __builtin_amdgcn_readfirstlane(a.s.table[(int64_t)seq * a.b.max_pages + slot]) : -1;
  if (page < 0 || page >= a.c.n_pages) return false;
  const u32x4* src = reinterpret_cast<const u32x4*>(
      a.pages + (((int64_t)page * a.c.hkv + head) * a.c.tiles + (a.c.tiles == 2 ? t & 1 : 0)) * (2 * kTileBytes)) + lane_id();
  u32x4 raw[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) raw[i] = src[i * kWave];
  x.kc = fmaxf(pow2f(stored_exp(a.scales[((int64_t)page * a.c.hkv + head) * 2])) * a.c2, 1.17549435e-38f);  // not 0, which a masked -inf must not meet
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x.k[2 * i] = codes_to_bf16<FMT>(raw[i][0], raw[i][1]);
    x.k[2 * i + 1] = codes_to_bf16<FMT>(raw[i][2], raw[i][3]);
  }
  return true;
}

__device__ __forceinline__ void products(const KeyTile& x, const bf16x8 (&q)[4], acc4 (&s)[4]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) s[t] = acc4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int kk = 0; kk < 4; ++kk)
#pragma unroll
    for (int t = 0; t < 4; ++t) s[t] = mfma16(x.k[4 * t + kk], q[kk], s[t]);
}

// This lane's part of pair p's q: column lane % 16, elements 32 (lane / 16) + 8 kk + [0, 8); 0 past the last pair.
__device__ __forceinline__ void load_pair(const WeightArgs& a, const SeqRows& r, int head, int p, int pairs, bf16x8 (&q)[4]) {
  const int at = min(p, pairs - 1), i = at / a.G, g = at - i * a.G;
  const uint16_t* src = a.q + (int64_t)(head * a.G + g) * a.qs.head + (int64_t)(r.row0 + i) * a.qs.row + 32 * (lane_id() >> 4);
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    u32x4 x = *reinterpret_cast<const u32x4*>(src + 8 * kk);
    if (p >= pairs) x = u32x4{0, 0, 0, 0};
    q[kk] = __builtin_bit_cast(bf16x8, x);
  }
}

// (m, l) of two disjoint sets of keys together.
__device__ __forceinline__ void merge(float& m, float& l, float m2, float l2) {
  const float top = vmax(m, m2);
  const float ref = top == -__builtin_inff() ? 0.f : top;
  l = l * fast_exp2(m - ref) + l2 * fast_exp2(m2 - ref);
  m = top;
}

struct Item {
  int seq, head, i;
};
__device__ __forceinline__ Item item_of(const WeightArgs& a, int each) {
  const int sh = blockIdx.x / each;
  return Item{sh / a.c.hkv, sh % a.c.hkv, (int)blockIdx.x - sh * each};
}

template <int FMT>
__global__ __launch_bounds__(kThreads) void weigh_rows(WeightArgs a) {
  __shared__ bf16x8 qs[kGroups][4][kWave];
  __shared__ float2 part[kWaves][kPairs];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Item it = item_of(a, a.chunks);
  const SeqRows r = seq_rows(a.s, a.b, a.c.B, it.seq);
  const int T = tiles_of(a, r), n = chunks_of(a, T), pairs = r.n * a.G;
  if (pairs == 0 || it.i >= n) return;
  const int t0 = (int)((int64_t)it.i * T / n), t1 = (int)((int64_t)(it.i + 1) * T / n);
  for (int p0 = 0; p0 < pairs; p0 += kPairs) {
    const int groups = min((pairs - p0 + kGroup - 1) / kGroup, kGroups);
    for (int g = w; g < groups; g += kWaves) {
      bf16x8 q[4];
      load_pair(a, r, it.head, p0 + g * kGroup + (lane & 15), pairs, q);
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) qs[g][kk][lane] = q[kk];
    }
    __syncthreads();
    float m[kGroups], l[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      m[g] = -__builtin_inff();
      l[g] = 0.f;
    }
    for (int t = t0 + w; t < t1; t += kWaves) {
      KeyTile x;
      if (!load_keys<FMT>(a, it.seq, it.head, t, x)) continue;
      const int first = t * kTile + 16 * (lane >> 4);  // position of this lane's first token
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        if (g >= groups) break;
        bf16x8 q[4];
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) q[kk] = qs[g][kk][lane];
        acc4 s[4];
        products(x, q, s);
        if (t * kTile + kTile - 1 > r.len + (p0 + g * kGroup) / a.G) {
          const int see = r.len + (p0 + g * kGroup + (lane & 15)) / a.G;
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (first + e > see) s[e >> 2][e & 3] = -__builtin_inff();
        }
        float top = s[0][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) top = vmax(top, s[e >> 2][e & 3]);
        const float now = vmax(m[g], top * x.kc), ref = now == -__builtin_inff() ? 0.f : now;
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) sum += fast_exp2(__builtin_fmaf(s[e >> 2][e & 3], x.kc, -ref));
        l[g] = l[g] * fast_exp2(m[g] - ref) + sum;
        m[g] = now;
      }
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      if (g >= groups) break;
#pragma unroll
      for (int o = 16; o < kWave; o <<= 1) merge(m[g], l[g], __shfl_xor(m[g], o), __shfl_xor(l[g], o));
      if (lane < kGroup) part[w][g * kGroup + lane] = make_float2(m[g], l[g]);
    }
    __syncthreads();
    if (tid < kPairs && p0 + tid < pairs) {
      float2 x = part[0][tid];
#pragma unroll
      for (int i = 1; i < kWaves; ++i) merge(x.x, x.y, part[i][tid].x, part[i][tid].y);
      const int row = (p0 + tid) / a.G, h = it.head * a.G + (p0 + tid) % a.G;
      a.stats[((int64_t)(r.row0 + row) * a.hq + h) * a.chunks + it.i] = x;
    }
    __syncthreads();
  }
}

// Each pair's log2 of the sum over all its chunks (+infinity if it sees no token): a wave a row, 16 lanes a head.
__global__ __launch_bounds__(kThreads) void weigh_join(WeightArgs a) {
  const int lane = threadIdx.x & 63, j = lane & 15;
  for (int row = blockIdx.x * kWaves + (threadIdx.x >> 6); row < a.b.n_rows; row += gridDim.x * kWaves) {
    int s = 0;  // the last sequence that begins at or before the row
    for (int n = a.b.n_seqs; n > 1;) {
      const int step = (n + kWave - 1) / kWave, probe = lane * step;
      const unsigned long long ok = __ballot(probe < n && a.s.row_ptr[s + min(probe, n - 1)] <= row);
      const int k = max(__popcll(ok) - 1, 0);
      s += k * step;
      n = min(step, n - k * step);
    }
    const SeqRows r = seq_rows(a.s, a.b, a.c.B, s);
    if (row < r.row0 || row >= r.row0 + r.n) continue;
    const int n = chunks_of(a, tiles_of(a, r));
    for (int h = lane >> 4; h < a.hq; h += kWave / 16) {
      const float2* src = a.stats + ((int64_t)row * a.hq + h) * a.chunks;
      float m = -__builtin_inff(), l = 0.f;
      for (int i = j; i < n; i += 16) merge(m, l, src[i].x, src[i].y);
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) merge(m, l, __shfl_xor(m, o), __shfl_xor(l, o));
      if (j == 0) a.lse[(int64_t)row * a.hq + h] = l == 0.f ? __builtin_inff() : m + log2f(l);
    }
  }
}

template <int FMT>
__global__ __launch_bounds__(kThreads) void weigh_tokens(WeightArgs a) {
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Item it = item_of(a, a.token_wgs);
  const SeqRows r = seq_rows(a.s, a.b, a.c.B, it.seq);
  // positions up to the width are written, whether or not the table reaches them
  const int end = (int)min((int64_t)r.len + r.n, (int64_t)a.width), T = (end + kTile - 1) / kTile, pairs = r.n * a.G;
  const int held = a.held[it.seq];
  const int64_t row = ((int64_t)it.seq * a.c.hkv + it.head) * a.width;
  for (int t = it.i * kWaves + w; t < T; t += a.token_wgs * kWaves) {
    const int at = t * kTile + lane;
    float old = 0.f;
    if (at < end && at < held) old = a.weights[row + at];
    KeyTile x;
    float acc[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.f;
    if (pairs > 0 && load_keys<FMT>(a, it.seq, it.head, t, x)) {
      const int first = t * kTile + 16 * (lane >> 4);
      for (int p0 = 0; p0 < pairs; p0 += kGroup) {
        const int p = p0 + (lane & 15), i = min(p, pairs - 1) / a.G, g = min(p, pairs - 1) - i * a.G;
        if (t * kTile > r.len + (min(p0 + kGroup, pairs) - 1) / a.G) continue;  // no pair of the group sees the tile
        bf16x8 q[4];
        load_pair(a, r, it.head, p, pairs, q);
        const float lse = p < pairs ? a.lse[(int64_t)(r.row0 + i) * a.hq + it.head * a.G + g] : __builtin_inff();
        acc4 s[4];
        products(x, q, s);
        if (t * kTile + kTile - 1 > r.len + p0 / a.G) {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            acc[e] += first + e > r.len + i ? 0.f : fast_exp2(__builtin_fmaf(s[e >> 2][e & 3], x.kc, -lse));
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[e] += fast_exp2(__builtin_fmaf(s[e >> 2][e & 3], x.kc, -lse));
        }
      }
    }
    // summed over the 16 lanes of a row; lane c of them takes token c
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float y = acc[e];
      y += __uint_as_float(row_move<0x128>(__float_as_uint(y)));
      y += __uint_as_float(row_move<0x124>(__float_as_uint(y)));
      y += __uint_as_float(row_move<0x122>(__float_as_uint(y)));
      y += __uint_as_float(row_move<0x121>(__float_as_uint(y)));
      if ((lane & 15) == e) sum = y;
    }
    if (at < end) a.out[row + at] = old + sum;
  }
}

// Chunks of a sequence's tokens whose statistics are kept apart, and the workspace.
struct Plan {
  int chunks;
  size_t lse, bytes;  // where the pairs' sums over all chunks begin
};
Plan plan_of(const CacheDims& c, const BatchDims& b, int hq) {
  const int64_t heads = (int64_t)b.n_seqs * c.hkv, pairs = (int64_t)b.n_rows * hq;
  if (heads == 0 || pairs == 0) return Plan{1, 0, 0};
  // Enough workgroups for the GPU, and 16 MB of statistics at most but for calls of very many rows.  The space for them
  // does not shrink as rows are added, so that a workspace is enough for fewer rows, too.
  constexpr int64_t kMost = (int64_t)1 << 21;
  const int64_t want = heads < 128 ? (1024 + heads - 1) / heads : 8, fit = kMost / pairs;
  const int64_t chunks = fit < 1 ? 1 : want < fit ? want : fit;
  const int64_t space = pairs > kMost ? pairs : pairs * want < kMost ? pairs * want : kMost;
  const size_t lse = ((size_t)space * sizeof(float2) + 255) & ~(size_t)255;
  return Plan{(int)chunks, lse, lse + (size_t)pairs * sizeof(float)};
}

}  // namespace

size_t cache_weights_bytes(const CacheDims& c, const BatchDims& b, int hq) { return plan_of(c, b, hq).bytes; }

hipError_t launch_cache_weights(const CacheDims& c, const BatchDims& b, const Seqs& s, int hq, float scale, const uint16_t* q,
                                Strides qs, const uint8_t* pages, const float* scales, const float* weights, float* out,
                                int width, const int32_t* held, void* ws, hipStream_t stream) {
  const Plan p = plan_of(c, b, hq);
  const int64_t heads = (int64_t)b.n_seqs * c.hkv;
  int64_t wgs = (4096 + heads - 1) / heads;
  const int64_t most = ((int64_t)width + kTile * kWaves - 1) / (kTile * kWaves);
  wgs = wgs > most ? most : wgs;
  const WeightArgs a{c, b, s, q, qs, pages, scales, weights, out, held, width, hq, hq / c.hkv, p.chunks, (int)wgs, scale * kLog2e,
                     reinterpret_cast<float2*>(ws), reinterpret_cast<float*>(reinterpret_cast<char*>(ws) + p.lse)};
  const int64_t join = (b.n_rows + kWaves - 1) / kWaves;
  const dim3 rows((unsigned)(heads * p.chunks)), tokens((unsigned)(heads * wgs)), threads(kThreads);
  if (c.fmt == kCacheE4M3) hipLaunchKernelGGL((weigh_rows<kCacheE4M3>), rows, threads, 0, stream, a);
  else hipLaunchKernelGGL((weigh_rows<kCacheInt8>), rows, threads, 0, stream, a);
  hipLaunchKernelGGL(weigh_join, dim3((unsigned)(join < 4096 ? join : 4096)), threads, 0, stream, a);
  if (c.fmt == kCacheE4M3) hipLaunchKernelGGL((weigh_tokens<kCacheE4M3>), tokens, threads, 0, stream, a);
  else hipLaunchKernelGGL((weigh_tokens<kCacheInt8>), tokens, threads, 0, stream, a);
  return hipGetLastError();
}

}  // namespace crisp
