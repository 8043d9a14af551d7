// The attention weight that each cached token gets from new rows, summed over the rows and the query heads of its KV head:
//   w_j = sum_p exp2(x_pj - lse_p),  x_pj = scale log2(e) q_p . k_j,  lse_p = log2 sum_j exp2(x_pj)
// over the pairs p = i G + g of a sequence's rows i and the G query heads of the KV head.  A pair's sum over all keys has to be known
// before any of its weights, so the keys are gone over twice: weigh_rows leaves each pair's maximum and sum over a chunk of the
// tokens, and weigh_tokens takes the chunks' together and forms the weights, a wave a tile of 64 tokens, summed over the pairs in a
// fixed order and without atomics.  Where a sequence has few pairs, x itself waits in the workspace, 4 bytes a pair and token where
// the keys are 128; where it has many, the products are formed again and a launch between the two joins the chunks.
//
// Few pairs are bound by the keys' bytes: a row of each of 48 sequences of 300 to 8191 tokens, 32 heads over 8 (179 MB read), 43 us, 4.2 TB/s, and
// 16 us for the scores and weights (32 MB read: launch, lengths, scores, in turn); without waiting scores 36 + 43 us.  Many pairs are bound by
// vector instructions, three for each score and pass beside the conversion of K: 32 rows of 28 heads over 4 and 131000 tokens (30 GFLOP a
// pass) 44 + 5.5 + 42 us, 35 of them for each pass in proportion to the tokens, 10 to begin.  Products of one group in a fixed order beside
// the exponents of the one before, or the next tile read from LDS beside the last group's, change nothing (47 to 51 and 46 to 50 us).
//
// Rows as many as tokens are not what this is made for: chunks are divided by slots and bounded by the space for statistics, and a pass of 256
// pairs goes over tiles behind all of them, too.  Whole prompts, 32 heads over 8: 4096 rows 1.6 ms, 12000 rows 19 (among 64 slots 77), 32768 rows
// 261, 10 to 70 times their attention.  One row over 128000 tokens 40 us, 159 where 63 further slots hold nothing.
#include <type_traits>

#include "cache_device.h"

namespace crisp {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kGroup = 16;                  // pairs of one product
constexpr int kOwn = 4;                     // groups of a wave in calls of many pairs
constexpr int kPairs = kGroup * kWaves * kOwn;  // of a pass over the keys there
constexpr int kScoreSeqs = 1024;            // sequences of a call whose scores may wait: each workgroup adds up those before its own

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
  int waiting;     // pairs of a sequence whose scores may wait, at most (0: none do)
  int64_t slots;   // tiles that there is room for
  float2* stats;   // [n_rows][hq][chunks]: maximum, sum
  float* lse;      // [n_rows][hq]
  float* scores;   // [slots][hkv][waiting][64]: x
};

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float acc4;

__device__ __forceinline__ acc4 mfma16(bf16x8 a, bf16x8 b, acc4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ int tiles_of(const WeightArgs& a, const SeqRows& r) {
  return (min(r.len + r.n, a.b.max_pages * a.c.B) + kTile - 1) / kTile;
}
__device__ __forceinline__ int chunks_of(const WeightArgs& a, int tiles) { return min(a.chunks, (tiles + kWaves - 1) / kWaves); }

// The first slot of a sequence's scores, -1 if they do not wait (or there are none): the tiles of the sequences before it come first.
__device__ __forceinline__ int64_t first_slot(const WeightArgs& a, int seq, int tiles, int pairs) {
  if (pairs > a.waiting || tiles == 0) return -1;
  int64_t sum = 0;
  for (int i = lane_id(); i < seq; i += kWave) sum += tiles_of(a, seq_rows(a.s, a.b, a.c.B, i));
  sum = wave_scan(sum);
  sum = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)sum, 63) |
                  (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(sum >> 32), 63) << 32);
  return sum + tiles <= a.slots ? sum : -1;
}

// Keeps a loaded chunk in its four registers up to here: left to itself the compiler splits what a loop carries into single
// codes, a register each.
__device__ __forceinline__ void keep_whole(u32x4 (&raw)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) asm("" : "+v"(raw[i]));
}

// The tiles t0, t0 + STEP, ... < t1 of one sequence and KV head, K alone.  64 are looked up in one round of loads, one a lane; the codes of
// the next are loaded while those of the present one are worked on.
template <int STEP>
struct KeyTiles {
  const int32_t* row;
  int tb, end, pg;
  float kc;

  __device__ __forceinline__ KeyTiles(const WeightArgs& a, int seq, int t0, int t1)
      : row(a.s.table + (int64_t)seq * a.b.max_pages), tb(t0 - STEP * kWave), end(t1), pg(-1), kc(0.f) {}

  // Tile t, the one after the last that was asked for: its codes, and what takes products with them to the base-2 exponent;
  // false if it has no page.
  // N = 8: a wave takes the whole tile, chunk 64 x + lane its x-th; N = 2: a workgroup, thread's chunks tid and tid + 256.
  template <int N>
  __device__ __forceinline__ bool load(const WeightArgs& a, int head, int t, u32x4 (&raw)[N], float& scale) {
    if (t >= tb + STEP * kWave) {
      tb = t;
      const int mine = t + STEP * lane_id(), slot = a.c.tiles == 2 ? mine >> 1 : mine;
      pg = mine < end && slot < a.b.max_pages ? row[slot] : -1;
      if (pg >= a.c.n_pages) pg = -1;
      // (not 0, which a masked -infinity must not meet)
      if (pg >= 0) kc = fmaxf(pow2f(stored_exp(a.scales[((int64_t)pg * a.c.hkv + head) * 2])) * a.c2, 1.17549435e-38f);
    }
    const int i = (t - tb) / STEP, page = __builtin_amdgcn_readlane(pg, i);
    scale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(kc), i));
    if (page < 0) return false;
    const u32x4* src = reinterpret_cast<const u32x4*>(
        a.pages + (((int64_t)page * a.c.hkv + head) * a.c.tiles + (a.c.tiles == 2 ? t & 1 : 0)) * (2 * kTileBytes)) + (N == 8 ? lane_id() : (int)threadIdx.x);
#pragma unroll
    for (int x = 0; x < N; ++x) raw[x] = src[x * (N == 8 ? kWave : kThreads)];
    return true;
  }
};

// s[t] = the products of 16 tokens and 16 pairs, from the codes: K's operand (t, kk) is elements 32 g + 8 kk + [0, 8) of the tokens.
template <int FMT>
__device__ __forceinline__ void products(const u32x4 (&raw)[8], const bf16x8 (&q)[4], acc4 (&s)[4]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    s[t] = acc4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const u32x4 x = raw[2 * t + half];
      s[t] = mfma16(codes_to_bf16<FMT>(x[0], x[1]), q[2 * half], s[t]);
      s[t] = mfma16(codes_to_bf16<FMT>(x[2], x[3]), q[2 * half + 1], s[t]);
    }
  }
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

// Where pair p's statistics are.
__device__ __forceinline__ int64_t pair_of(const WeightArgs& a, const SeqRows& r, int head, int p) {
  return (int64_t)(r.row0 + p / a.G) * a.hq + head * a.G + p % a.G;
}

// (m, l) of two disjoint sets of keys together.  Of no keys they are (-infinity, 0); of keys whose scores are all -infinity l is positive:
// beside a finite m it counts for nothing, and alone it makes the logarithm -infinity and so the weights NaN, as the softmax is.
__device__ __forceinline__ void merge(float& m, float& l, float m2, float l2) {
  const float top = vmax(m, m2);
  l = l * (m == top ? 1.f : fast_exp2(m - top)) + l2 * (m2 == top ? 1.f : fast_exp2(m2 - top));
  m = top;
}

// To be called of a lane's pair behind its keys, the first of them that have a page being tile `first`'s.
__device__ __forceinline__ void mark_seen(float m, float& l, int first, int last_seen) {
  if (m == -__builtin_inff() && l == 0.f && first <= last_seen / kTile) l = 1.f;
}

// The four lanes of a column together.
__device__ __forceinline__ void column(float& m, float& l) {
#pragma unroll
  for (int o = 16; o < kWave; o <<= 1) merge(m, l, __shfl_xor(m, o), __shfl_xor(l, o));
}

// The last positions that 16 pairs from p0 on see: the first pair's, and this lane's.  (Divided once, not once a tile.)
struct Sight {
  int all, own;
  __device__ __forceinline__ Sight() {}
  __device__ __forceinline__ Sight(const WeightArgs& a, const SeqRows& r, int p0, int pairs)
      : all(r.len + min(p0, pairs - 1) / a.G), own(r.len + min(p0 + (lane_id() & 15), pairs - 1) / a.G) {}
  __device__ __forceinline__ bool whole(int t) const { return t * kTile + kTile - 1 <= all; }
  // Whether this lane's pair does not see its e-th token of tile t.
  __device__ __forceinline__ bool hides(int t, int e) const { return t * kTile + 16 * (lane_id() >> 4) + e > own; }
};

// Scores of a tile that the pairs do not see become -infinity.
__device__ __forceinline__ void mask_tile(const Sight& see, int t, acc4 (&s)[4]) {
  if (see.whole(t)) return;
#pragma unroll
  for (int e = 0; e < 16; ++e)
    if (see.hides(t, e)) s[e >> 2][e & 3] = -__builtin_inff();
}

struct Item {
  int seq, head, i;
};
__device__ __forceinline__ Item item_of(const WeightArgs& a, int each) {
  const int sh = blockIdx.x / each;
  return Item{sh / a.c.hkv, sh % a.c.hkv, (int)blockIdx.x - sh * each};
}

// For each group, a column's reference m and sum l of exp2(x - m) with a tile's 16 of this lane's, x = s kc, -infinity where masked.  The
// sums are 32-bit floats, so the reference need not be the maximum: it is raised to it where a sum passes 2^60 (or is not a
// number) and where there is none yet, and no maximum is looked for otherwise.
template <int NI>
__device__ __forceinline__ void add_tiles(const acc4 (&s)[NI][4], float kc, float (&m)[NI], float (&l)[NI]) {
  const auto sum = [&](int i, float ref) {
    float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e & 3] += fast_exp2(__builtin_fmaf(s[i][e >> 2][e & 3], kc, -ref));
    return (y[0] + y[1]) + (y[2] + y[3]);
  };
  float more[NI];
  bool raise = false;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    more[i] = sum(i, m[i] == -__builtin_inff() ? 0.f : m[i]);
    raise = raise || !(more[i] <= 0x1p60f) || m[i] == -__builtin_inff();
  }
  if (__ballot(raise)) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      float top = s[i][0][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = vmax(top, s[i][e >> 2][e & 3]);
      top = vmax(m[i], top * kc);
      const float ref = top == -__builtin_inff() ? 0.f : top;
      l[i] *= fast_exp2(m[i] - ref);
      m[i] = top;
      more[i] = sum(i, ref);
    }
  }
#pragma unroll
  for (int i = 0; i < NI; ++i) l[i] += more[i];
}

// Calls of few pairs a sequence, 16 at a time: a wave takes every fourth tile of the chunk, with q in registers.
template <int FMT>
__global__ __launch_bounds__(kThreads, 4) void weigh_rows_few(WeightArgs a) {
  __shared__ float2 part[kWaves][kGroup];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Item it = item_of(a, a.chunks);
  const SeqRows r = seq_rows(a.s, a.b, a.c.B, it.seq);
  const int T = tiles_of(a, r), n = chunks_of(a, T), pairs = r.n * a.G;
  if (pairs == 0 || it.i >= n) return;
  const int t0 = (int)((int64_t)it.i * T / n), t1 = (int)((int64_t)(it.i + 1) * T / n);
  int64_t slot = -1;
  for (int p0 = 0; p0 < pairs; p0 += kGroup) {
    KeyTiles<kWaves> tiles(a, it.seq, t0 + w, t1);
    u32x4 raw[8] = {}, next[8] = {};
    float kc = 0.f, kc_next = 0.f;
    bool ok = false, ok_next = false;
    if (t0 + w < t1) ok = tiles.load(a, it.head, t0 + w, raw, kc);
    bf16x8 q[4];
    load_pair(a, r, it.head, p0 + (lane & 15), pairs, q);
    if (p0 == 0) slot = first_slot(a, it.seq, T, pairs);
    const Sight see(a, r, p0, pairs);
    float m[1] = {-__builtin_inff()}, l[1] = {0.f};
    int first = 0x7fffffff;
    for (int t = t0 + w; t < t1; t += kWaves) {
      if (t + kWaves < t1) ok_next = tiles.load(a, it.head, t + kWaves, next, kc_next);
      keep_whole(raw);
      if (ok) {
        first = min(first, t);
        acc4 s1[1][4];
        acc4(&s)[4] = s1[0];
        products<FMT>(raw, q, s);
        if (slot >= 0 && (lane & 15) < pairs) {
          f32x4* dst = reinterpret_cast<f32x4*>(
              a.scores + (((slot + t) * a.c.hkv + it.head) * a.waiting + (lane & 15)) * kTile + 16 * (lane >> 4));
#pragma unroll
          for (int e = 0; e < 4; ++e) dst[e] = s[e] * kc;
        }
        mask_tile(see, t, s);
        add_tiles<1>(s1, kc, m, l);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) raw[i] = next[i];
      kc = kc_next;
      ok = ok_next;
    }
    mark_seen(m[0], l[0], first, see.own);
    column(m[0], l[0]);
    if (lane < kGroup) part[w][lane] = make_float2(m[0], l[0]);
    __syncthreads();
    if (tid < kGroup && p0 + tid < pairs) {
      float2 x = part[0][tid];
#pragma unroll
      for (int i = 1; i < kWaves; ++i) merge(x.x, x.y, part[i][tid].x, part[i][tid].y);
      a.stats[pair_of(a, r, it.head, p0 + tid) * a.chunks + it.i] = x;
    }
    __syncthreads();
  }
}

// Calls of many pairs: the workgroup converts a tile of K once, into LDS, and each wave has NI groups of 16 pairs for all tiles, q and
// what it gathers in registers (group w + 4 i is its i-th).  The next tile's codes are loaded and converted beside the products of this one.
template <int FMT, int NI, typename Work>
__device__ __forceinline__ void over_tiles(const WeightArgs& a, const SeqRows& r, const Item& it, int p0, int pairs, int t0, int t1,
                                           bf16x8 (&kst)[2][16][kWave], Work work) {
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  bf16x8 q[NI][4];
#pragma unroll
  for (int i = 0; i < NI; ++i) load_pair(a, r, it.head, p0 + (w + kWaves * i) * kGroup + (lane & 15), pairs, q[i]);
  KeyTiles<1> tiles(a, it.seq, t0, t1);
  u32x4 raw[2] = {};  // chunks tid and tid + 256 of the tile
  float kc = 0.f;
  const auto stage = [&](int buf) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      asm("" : "+v"(raw[x]));
      kst[buf][2 * (w + kWaves * x)][lane] = codes_to_bf16<FMT>(raw[x][0], raw[x][1]);
      kst[buf][2 * (w + kWaves * x) + 1][lane] = codes_to_bf16<FMT>(raw[x][2], raw[x][3]);
    }
  };
  bool ok = tiles.load(a, it.head, t0, raw, kc);
  stage(0);
  for (int t = t0, buf = 0; t < t1; ++t, buf ^= 1) {
    const float kc_now = kc;
    const bool now = ok;
    ok = t + 1 < t1 && tiles.load(a, it.head, t + 1, raw, kc);
    __syncthreads();  // this tile is staged, and the other buffer free
    work(t, now, kc_now, q, kst[buf]);
    if (t + 1 < t1) stage(buf ^ 1);
  }
  __syncthreads();
}

// A staged tile's products: a lane's rows are 16 consecutive tokens and its column a pair, or (TURNED) its rows are pairs 4 (lane / 16) + [0, 4)
// and its columns the tokens 16 (c / 4) + 4 t + c % 4, c = lane % 16, so that sums over pairs stay within the lane.
template <bool TURNED = false>
__device__ __forceinline__ void products(const bf16x8 (&k)[16][kWave], const bf16x8 (&q)[4], int lane, acc4 (&s)[4]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) s[t] = acc4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int kk = 0; kk < 4; ++kk)
#pragma unroll
    for (int t = 0; t < 4; ++t) s[t] = TURNED ? mfma16(q[kk], k[4 * t + kk][lane], s[t]) : mfma16(k[4 * t + kk][lane], q[kk], s[t]);
}

// fn(std::integral_constant of the groups that a wave has), 1 .. kOwn.
template <typename Fn>
__device__ __forceinline__ void by_groups(int groups, Fn fn) {
  const int own = (groups + kWaves - 1) / kWaves;
  if (own == 1) fn(std::integral_constant<int, 1>{});
  else if (own == 2) fn(std::integral_constant<int, 2>{});
  else if (own == 3) fn(std::integral_constant<int, 3>{});
  else fn(std::integral_constant<int, kOwn>{});
}

template <int FMT>
__global__ __launch_bounds__(kThreads, 2) void weigh_rows(WeightArgs a) {
  __shared__ bf16x8 kst[2][16][kWave];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Item it = item_of(a, a.chunks);
  const SeqRows r = seq_rows(a.s, a.b, a.c.B, it.seq);
  const int T = tiles_of(a, r), n = chunks_of(a, T), pairs = r.n * a.G;
  if (pairs == 0 || it.i >= n) return;
  const int t0 = (int)((int64_t)it.i * T / n), t1 = (int)((int64_t)(it.i + 1) * T / n);
  for (int p0 = 0; p0 < pairs; p0 += kPairs)
    by_groups((min(pairs - p0, kPairs) + kGroup - 1) / kGroup, [&](auto groups) {
      constexpr int NI = decltype(groups)::value;
      float m[NI], l[NI];
      Sight see[NI];
      int first = 0x7fffffff;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        m[i] = -__builtin_inff();
        l[i] = 0.f;
        see[i] = Sight(a, r, p0 + (w + kWaves * i) * kGroup, pairs);
      }
      over_tiles<FMT, NI>(a, r, it, p0, pairs, t0, t1, kst, [&](int t, bool ok, float kc, const bf16x8 (&q)[NI][4], const bf16x8 (&k)[16][kWave]) {
        if (!ok) return;
        first = min(first, t);
        acc4 s[NI][4];
#pragma unroll
        for (int i = 0; i < NI; ++i) products(k, q[i], lane, s[i]);
        if (!see[0].whole(t)) {
#pragma unroll
          for (int i = 0; i < NI; ++i) mask_tile(see[i], t, s[i]);
        }
        add_tiles<NI>(s, kc, m, l);
      });
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        mark_seen(m[i], l[i], first, see[i].own);
        column(m[i], l[i]);
        const int p = p0 + (w + kWaves * i) * kGroup + lane;
        if (lane < kGroup && p < pairs) a.stats[pair_of(a, r, it.head, p) * a.chunks + it.i] = make_float2(m[i], l[i]);
      }
    });
}

// log2 of a pair's sum over all n chunks, by 16 lanes together; +infinity if it sees no token.
__device__ __forceinline__ float joined(const float2* src, int n) {
  float m = -__builtin_inff(), l = 0.f;
  for (int i = lane_id() & 15; i < n; i += 16) merge(m, l, src[i].x, src[i].y);
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) merge(m, l, __shfl_xor(m, o), __shfl_xor(l, o));
  return l == 0.f ? __builtin_inff() : m + log2f(l);
}

// Every pair's, a wave four heads of a row.
__global__ __launch_bounds__(kThreads) void weigh_join(WeightArgs a) {
  const int lane = threadIdx.x & 63, quads = (a.hq + 3) / 4;
  const int64_t items = (int64_t)a.b.n_rows * quads;
  for (int64_t i = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6); i < items; i += (int64_t)gridDim.x * kWaves) {
    const int row = (int)(i / quads), h = (int)(i - (int64_t)row * quads) * 4 + (lane >> 4);
    int s = 0;  // the last sequence that begins at or before the row
    for (int n = a.b.n_seqs; n > 1;) {
      const int step = (n + kWave - 1) / kWave, probe = lane * step;
      const unsigned long long ok = __ballot(probe < n && a.s.row_ptr[s + min(probe, n - 1)] <= row);
      const int k = max((int)__popcll(ok) - 1, 0);  // (its type is unsigned)
      s += k * step;
      n = min(step, n - k * step);
    }
    const SeqRows r = seq_rows(a.s, a.b, a.c.B, s);
    if (row < r.row0 || row >= r.row0 + r.n) continue;
    const int64_t pair = (int64_t)row * a.hq + min(h, a.hq - 1);
    const float x = joined(a.stats + pair * a.chunks, chunks_of(a, tiles_of(a, r)));
    if ((lane & 15) == 0 && h < a.hq) a.lse[pair] = x;
  }
}

// x[g] summed over the four lanes of a column, on the one of group g.
__device__ __forceinline__ float group_sums(const float (&x)[4]) {
  typedef __attribute__((__vector_size__(2 * sizeof(unsigned)))) unsigned u32x2;
  const auto halves = [](float a, float b) {  // (a below and above lane 32 together, b's on the lanes above)
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  };
  const u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(halves(x[0], x[2])), __float_as_uint(halves(x[1], x[3])), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A tile's sums over the lanes of a row of 16; lane c of them takes token c.
__device__ __forceinline__ float row_sums(const float (&acc)[16], int lane) {
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
  return sum;
}

// acc += the weights of a group of 16 pairs: products s, taken to the exponent by kc, each column's logarithm sub.
__device__ __forceinline__ void add_weights(const Sight& see, const acc4 (&s)[4], float kc, float sub, int t, float (&acc)[16]) {
  if (see.whole(t)) {
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] += fast_exp2(__builtin_fmaf(s[e >> 2][e & 3], kc, -sub));
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] += see.hides(t, e) ? 0.f : fast_exp2(__builtin_fmaf(s[e >> 2][e & 3], kc, -sub));
  }
}

// The weights of calls of many pairs, whose sums are in a.lse.  Each wave's part of a tile waits in LDS for the next tile's barrier; pairs past
// kPairs are added to what the ones before have left.
template <int FMT>
__global__ __launch_bounds__(kThreads, 2) void weigh_tokens(WeightArgs a) {
  __shared__ bf16x8 kst[2][16][kWave];
  __shared__ float parts[2][kWaves][kTile];
  __shared__ __attribute__((aligned(16))) int sight[kPairs];  // the last positions that the pass's pairs see
  static_assert(kPairs == kThreads);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Item it = item_of(a, a.token_wgs);
  const SeqRows r = seq_rows(a.s, a.b, a.c.B, it.seq);
  // positions up to the width are written, whether or not the table reaches them
  const int end = (int)min((int64_t)r.len + r.n, (int64_t)a.width), T = (end + kTile - 1) / kTile, pairs = r.n * a.G;
  const int n = min(a.token_wgs, T);
  if (it.i >= n) return;
  const int t0 = (int)((int64_t)it.i * T / n), t1 = (int)((int64_t)(it.i + 1) * T / n);
  const int held = a.held[it.seq];
  const int64_t row = ((int64_t)it.seq * a.c.hkv + it.head) * a.width;
  if (pairs == 0) {
    for (int at = t0 * kTile + tid; at < min(t1 * kTile, end); at += kThreads) a.out[row + at] = at < held ? a.weights[row + at] : 0.f;
    return;
  }
  for (int p0 = 0; p0 < pairs; p0 += kPairs)
    by_groups((min(pairs - p0, kPairs) + kGroup - 1) / kGroup, [&](auto groups) {
      constexpr int NI = decltype(groups)::value;
      sight[tid] = r.len + min(p0 + tid, pairs - 1) / a.G;  // (the pass before has ended with a barrier, its first tile begins with one)
      float sub[NI][4];  // this lane's pairs' logarithms
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int p = p0 + (w + kWaves * i) * kGroup + 4 * (lane >> 4) + e;
          sub[i][e] = p < pairs ? a.lse[pair_of(a, r, it.head, p)] : __builtin_inff();
        }
      const Sight see(a, r, p0 + w * kGroup, pairs);
      float old = 0.f;
      const auto start = [&](int t) {  // of a tile that this wave writes
        const int at = t * kTile + lane;
        if (p0 > 0) old = at < end ? a.out[row + at] : 0.f;
        else old = at < end && at < held ? a.weights[row + at] : 0.f;
      };
      const auto write = [&](int t) {
        const int at = t * kTile + lane, buf = (t - t0) & 1;
        if (at < end) a.out[row + at] = old + ((parts[buf][0][lane] + parts[buf][1][lane]) + (parts[buf][2][lane] + parts[buf][3][lane]));
      };
      over_tiles<FMT, NI>(a, r, it, p0, pairs, t0, t1, kst, [&](int t, bool ok, float kc, const bf16x8 (&q)[NI][4], const bf16x8 (&k)[16][kWave]) {
        if (t > t0 && w == ((t - 1) & 3)) write(t - 1);
        if (w == (t & 3)) start(t);
        float acc[4] = {0.f, 0.f, 0.f, 0.f};  // of the four columns
        if (ok) {
          acc4 s[NI][4];
#pragma unroll
          for (int i = 0; i < NI; ++i) products<true>(k, q[i], lane, s[i]);
          if (see.whole(t)) {  // by the wave's first pairs, so by all: no branch between the groups
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
              for (int e = 0; e < 16; ++e) acc[e >> 2] += fast_exp2(__builtin_fmaf(s[i][e >> 2][e & 3], kc, -sub[i][e & 3]));
          } else {
            const int first = t * kTile + 16 * ((lane & 15) >> 2) + (lane & 3);
#pragma unroll
            for (int i = 0; i < NI; ++i) {
              const int4 x = *reinterpret_cast<const int4*>(&sight[(w + kWaves * i) * kGroup + 4 * (lane >> 4)]);
              const int own[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
              for (int e = 0; e < 16; ++e)
                acc[e >> 2] += first + 4 * (e >> 2) > own[e & 3] ? 0.f : fast_exp2(__builtin_fmaf(s[i][e >> 2][e & 3], kc, -sub[i][e & 3]));
            }
          }
        }
        parts[(t - t0) & 1][w][16 * ((lane & 15) >> 2) + 4 * (lane >> 4) + (lane & 3)] = group_sums(acc);
      });
      if (w == ((t1 - 1) & 3)) write(t1 - 1);
      __syncthreads();
    });
}

// Calls of few pairs a sequence: the workgroup joins the chunks of 16 pairs by itself.  Where scores wait (SCORES: they do for most
// sequences), a lane takes a token: all latency, so registers are held to what lets a CU have eight workgroups, at the cost of
// spills where the products are formed again for the others.
template <int FMT, bool SCORES>
__global__ __launch_bounds__(kThreads, SCORES ? 8 : 4) void weigh_tokens_few(WeightArgs a) {
  __shared__ float lse[kGroup];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Item it = item_of(a, a.token_wgs);
  const SeqRows r = seq_rows(a.s, a.b, a.c.B, it.seq);
  const int end = (int)min((int64_t)r.len + r.n, (int64_t)a.width), T = (end + kTile - 1) / kTile, pairs = r.n * a.G;
  if (it.i * kWaves >= T) return;
  const int held = a.held[it.seq], in_table = tiles_of(a, r), n = chunks_of(a, in_table), step = a.token_wgs * kWaves;
  const int64_t row = ((int64_t)it.seq * a.c.hkv + it.head) * a.width;
  const auto stage_lse = [&](int p0) {
    const int p = p0 + (tid >> 4);
    const float x = p < pairs ? joined(a.stats + pair_of(a, r, it.head, p) * a.chunks, n) : __builtin_inff();
    if ((tid & 15) == 0) lse[tid >> 4] = x;
  };
  const int32_t* pages = a.s.table + (int64_t)it.seq * a.b.max_pages;
  const auto page_of = [&](int t) {
    const int slot = a.c.tiles == 2 ? t >> 1 : t;
    return t < T && slot < a.b.max_pages ? pages[slot] : -1;
  };
  const int64_t slot = SCORES && pairs > 0 ? first_slot(a, it.seq, in_table, pairs) : -1;
  if (SCORES && slot >= 0) {
    // (scores of a tile without a page are whatever the workspace holds, and are not used; of one past the table none are read)
    const auto load = [&](int t, float (&x)[kGroup], float& old, int& page) {
      const float* src = a.scores + ((slot + min(t, in_table - 1)) * a.c.hkv + it.head) * a.waiting * kTile + lane;
      const int at = t * kTile + lane;
      page = page_of(t);
      old = at < end && at < held ? a.weights[row + at] : 0.f;
#pragma unroll
      for (int p = 0; p < kGroup; ++p)
        if (p < pairs) x[p] = src[p * kTile];
    };
    float x[kGroup], next[kGroup], old, old_next = 0.f;
    int page, page_next = -1, t = it.i * kWaves + w;
    load(t, x, old, page);
    stage_lse(0);
    __syncthreads();
    for (; t < T; t += step) {
      if (t + step < T) load(t + step, next, old_next, page_next);
      const int at = t * kTile + lane;
      float sum = 0.f;
      if (page >= 0 && page < a.c.n_pages) {
#pragma unroll
        for (int p = 0; p < kGroup; ++p)
          if (p < pairs) sum += at > r.len + p / a.G ? 0.f : fast_exp2(x[p] - lse[p]);
      }
      if (at < end) a.out[row + at] = old + sum;
#pragma unroll
      for (int p = 0; p < kGroup; ++p) x[p] = next[p];
      old = old_next;
      page = page_next;
    }
    return;
  }
  for (int t0 = it.i * kWaves; t0 < T; t0 += step) {
    const int t = t0 + w, at = t * kTile + lane;
    const float old = at < end && at < held ? a.weights[row + at] : 0.f;
    u32x4 raw[8] = {};
    float kc = 0.f;
    KeyTiles<kWaves> tiles(a, it.seq, t, t + 1);
    const bool ok = t < T && tiles.load(a, it.head, t, raw, kc);
    keep_whole(raw);
    float acc[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.f;
    for (int p0 = 0; p0 < pairs; p0 += kGroup) {
      __syncthreads();  // the pairs before are done with
      stage_lse(p0);
      __syncthreads();
      if (!ok || t * kTile > r.len + (min(p0 + kGroup, pairs) - 1) / a.G) continue;  // (no pair of the group sees the tile)
      bf16x8 q[4];
      load_pair(a, r, it.head, p0 + (lane & 15), pairs, q);
      acc4 s[4];
      keep_whole(raw);
      products<FMT>(raw, q, s);
      add_weights(Sight(a, r, p0, pairs), s, kc, lse[lane & 15], t, acc);
    }
    const float sum = row_sums(acc, lane);
    if (at < end) a.out[row + at] = old + sum;
  }
}

// Whether a call goes by weigh_rows, weigh_join and weigh_tokens, for more than 32 pairs a sequence on average (one sequence: 16), or by
// weigh_rows_few and weigh_tokens_few, which go over the keys once for every 16 pairs.  32 heads over 8, us, few / many: 48 sequences of 300 to 8191
// tokens 136 / 174 with 20 pairs, 144 / 176 with 32, 197 / 177 with 48; eight of them 30 / 40, 32 / 40, 41 / 41; one of 60000 tokens 29 / 37
// with 16 pairs, 42 / 37 with 20.
bool many_pairs(const CacheDims& c, const BatchDims& b, int hq) {
  return (int64_t)b.n_rows * (hq / c.hkv) > (int64_t)(b.n_seqs == 1 ? kGroup : 2 * kGroup) * b.n_seqs;
}

// Chunks of a sequence's tokens whose statistics are kept apart, room for scores, and the workspace.
struct Plan {
  int chunks, waiting;
  int64_t slots;
  size_t lse, scores, bytes;  // where they begin
};
Plan plan_of(const CacheDims& c, const BatchDims& b, int hq) {
  const int64_t heads = (int64_t)b.n_seqs * c.hkv, pairs = (int64_t)b.n_rows * hq, G = hq / c.hkv;
  if (heads == 0 || pairs == 0) return Plan{1, 0, 0, 0, 0, 0};
  // Workgroups enough for the GPU: of many pairs 512 (a window of 32 rows of 28 heads over 128k tokens 45 + 42 us; 1024 and 1536 workgroups 10
  // and 30 % more), of few 1024, and where there are many heads to go over, up to twelve chunks each, so that the longest sequence is not
  // left to the last.  With four / twelve / 24 chunks, the whole call in us: 48 sequences of 300 to 8191 tokens, 8 heads, 75 / 70 / 79; 24 of 500
  // to 16000, 4 heads, 50 / 47 / 45; 100 of 100 to 4000, 8 heads, 73 / 72 / 76; 200 of 100 to 3000, 2 heads, 40 / 42 / 49; 64 of 8000, 8
  // heads, 161 / 145 / 140; 12 of 1000 to 60000, 8 heads, 116 / 112 / 109.  16 MB of statistics at most but for calls of very many rows; the
  // space for them does not shrink as rows are added, so that a workspace is enough for fewer rows, too.
  constexpr int64_t kMost = (int64_t)1 << 21;
  const auto each = [&](int64_t wgs) { return (wgs + heads - 1) / heads; };
  const auto larger = [](int64_t x, int64_t y) { return x > y ? x : y; };
  const auto smaller = [](int64_t x, int64_t y) { return x < y ? x : y; };
  const int64_t few = larger(each(1024), larger(smaller(12, each(4608)), 3)), fit = larger(kMost / pairs, 1);
  const int64_t chunks = smaller(many_pairs(c, b, hq) ? larger(each(512), 3) : few, fit);
  const int64_t space = larger(pairs, smaller(pairs * few, kMost));
  // Scores of sequences of average rows or fewer wait, if that is one product's pairs, for as many tiles as the cache has (forks have
  // more together) or 256 MB hold.
  const int64_t rows = (b.n_rows + b.n_seqs - 1) / b.n_seqs, most = kGroup / G;
  const int waiting = b.n_seqs > kScoreSeqs ? 0 : (int)(G * (rows < most ? rows : most));
  const int64_t tiles = (int64_t)c.n_pages * c.tiles, slot = (int64_t)c.hkv * waiting * kTile * (int64_t)sizeof(float);
  const int64_t room = slot == 0 ? 0 : ((int64_t)256 << 20) / slot, slots = slot == 0 ? 0 : tiles < room ? tiles : room;
  const auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const size_t lse = up((size_t)space * sizeof(float2)), scores = lse + up((size_t)pairs * sizeof(float));
  const size_t area = slot == 0 ? 0 : (size_t)(tiles * slot < ((int64_t)256 << 20) ? tiles * slot : (int64_t)256 << 20);
  return Plan{(int)chunks, rows <= most ? waiting : 0, slots, lse, scores, scores + area};
}

}  // namespace

size_t cache_weights_bytes(const CacheDims& c, const BatchDims& b, int hq) { return plan_of(c, b, hq).bytes; }

hipError_t launch_cache_weights(const CacheDims& c, const BatchDims& b, const Seqs& s, int hq, float scale, const uint16_t* q,
                                Strides qs, const uint8_t* pages, const float* scales, const float* weights, float* out,
                                int width, const int32_t* held, void* ws, hipStream_t stream) {
  const Plan p = plan_of(c, b, hq);
  const int64_t heads = (int64_t)b.n_seqs * c.hkv;
  const bool join = many_pairs(c, b, hq);
  int64_t wgs = ((join ? 512 : 2048) + heads - 1) / heads;
  const int64_t most = ((int64_t)width + kTile * kWaves - 1) / (kTile * kWaves);
  wgs = wgs > most ? most : wgs;
  char* w = reinterpret_cast<char*>(ws);
  const WeightArgs a{c, b, s, q, qs, pages, scales, weights, out, held, width, hq, hq / c.hkv, p.chunks, (int)wgs, scale * kLog2e,
                     p.waiting, p.slots, reinterpret_cast<float2*>(w), reinterpret_cast<float*>(w + p.lse),
                     reinterpret_cast<float*>(w + p.scores)};
  const dim3 rows((unsigned)(heads * p.chunks)), tokens((unsigned)(heads * wgs)), threads(kThreads);
  if (join) {
    const int64_t items = ((int64_t)b.n_rows * ((hq + 3) / 4) + kWaves - 1) / kWaves;
    const dim3 joins((unsigned)(items < 4096 ? items : 4096));
    if (c.fmt == kCacheE4M3) hipLaunchKernelGGL((weigh_rows<kCacheE4M3>), rows, threads, 0, stream, a);
    else hipLaunchKernelGGL((weigh_rows<kCacheInt8>), rows, threads, 0, stream, a);
    hipLaunchKernelGGL(weigh_join, joins, threads, 0, stream, a);
    if (c.fmt == kCacheE4M3) hipLaunchKernelGGL((weigh_tokens<kCacheE4M3>), tokens, threads, 0, stream, a);
    else hipLaunchKernelGGL((weigh_tokens<kCacheInt8>), tokens, threads, 0, stream, a);
  } else {
    if (b.n_rows > 0 && hq > 0) {
      if (c.fmt == kCacheE4M3) hipLaunchKernelGGL((weigh_rows_few<kCacheE4M3>), rows, threads, 0, stream, a);
      else hipLaunchKernelGGL((weigh_rows_few<kCacheInt8>), rows, threads, 0, stream, a);
    }
    if (p.waiting > 0) {
      if (c.fmt == kCacheE4M3) hipLaunchKernelGGL((weigh_tokens_few<kCacheE4M3, true>), tokens, threads, 0, stream, a);
      else hipLaunchKernelGGL((weigh_tokens_few<kCacheInt8, true>), tokens, threads, 0, stream, a);
    } else {
      if (c.fmt == kCacheE4M3) hipLaunchKernelGGL((weigh_tokens_few<kCacheE4M3, false>), tokens, threads, 0, stream, a);
      else hipLaunchKernelGGL((weigh_tokens_few<kCacheInt8, false>), tokens, threads, 0, stream, a);
    }
  }
  return hipGetLastError();
}

}  // namespace crisp
