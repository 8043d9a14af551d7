// Attention of new rows over the 8-bit paged K/V cache.
//
// Row i of sequence s (rows row_ptr[s] .. row_ptr[s + 1] of the packed q) stands at position
// seq_len[s] + i and sees the cached positions up to its own:
//   o = sum_j softmax_j(scale q . k_j) v_j,  k_j = 2^ek ck_j,  v_j = 2^ev cv_j
// with codes c and one exponent a page, KV head and tensor.  The G query heads of a KV head and the
// rows of a sequence are the columns of one product, row i G + g.
#include "cache_device.h"

namespace crisp {

namespace {

constexpr int kFewWaves = 4, kJoinWaves = 4;
// Tiles that are not cut apart: one a wave of cache_attn.  Sequences of 2000 tokens, 32 heads over 8, grains of 4 / 8 / 16, us: one
// sequence 9.3 / 10.3 / 12.0, 4 10.8 / 10.3 / 12.0, 16 20.6 / 17.6 / 19.7, 64 40.5 / 42.5 / 36.2; one of 6000 9.9 / 10.5 / 11.7.
constexpr int kGrain = 4;

// The unit that the boundary behind a workgroup's share cuts: the first workgroup with a piece of it and
// the number of boundaries inside it (0: the boundary cuts none), KV head, first row in
// the order i G + g, number of rows, first row of the sequence.
struct Cut {
  int first, cuts, head, row, rows, row0;
};

struct AttnArgs {
  CacheDims c;
  BatchDims b;
  Seqs s;
  const uint16_t* q;
  Strides qs;
  const uint8_t* pages;
  const float* scales;
  uint16_t* o;
  Strides os;
  int G;
  int grain;    // tiles
  float c2;     // scale log2(e)
  Cut* cut;     // [gridDim.x]; null where no unit has more than one grain
  float* part;  // [2 gridDim.x][rows of a unit x 128, M, L]
};

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float acc4;

__device__ __forceinline__ acc4 mfma16(bf16x8 a, bf16x8 b, acc4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Keeps a loaded chunk in its four registers up to here: left to itself the compiler splits what
// the loop carries into single codes, a register each.
__device__ __forceinline__ void keep_whole(u32x4& x) { asm("" : "+v"(x)); }

// The value of all four lanes that hold a column (lanes l, l ^ 16, l ^ 32, l ^ 48) combined.
template <typename Op>
__device__ __forceinline__ float column(float x, Op op) {
  const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = op(__uint_as_float(h[0]), __uint_as_float(h[1]));
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ int64_t div64(int64_t x, int64_t y) {  // x, y >= 0; both are small but for the longest calls
  return ((x | y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}

// A place's unit: group rt of the rows (-1: the place stands for none) and KV head; the place is the unit's grain u0 of
// `grains` (of none: u0 of so many), of which the first is place `first`.
struct Unit {
  int rt, head, u0, grains;
  int64_t first;
};

// What a sequence's units are: nrt groups of R rows for each KV head, each over its tiles up to the last that a row
// of it sees (one at least, so that rows that see nothing are written too).  Where the work is
// divided, a unit counts in grains of so many tiles, the last perhaps smaller, and is cut between grains only.
//
// In a chunk of many rows the later groups see more tiles than the first.  The i-th group from the end and from
// the front are then a pair, whose sums of grains differ little: each pair has W places, the larger group first, and at
// its end up to three may be empty.  32 heads over 8, groups counted alike / in pairs, us: 8192 rows over no history 778 / 534
// (1029 TFLOP/s), 16384 3147 / 2068, 2048 over 2048 tokens 123.5 / 118.9, 1024 over 15000 277 / 277.  Units of up to 32
// rows end in the same tile or the next.
template <int R>
struct SeqWork {
  static constexpr bool kPairs = R > 32;
  SeqRows r;
  int T, nrt, grains, W;
  __device__ __forceinline__ SeqWork() {}
  __device__ __forceinline__ SeqWork(const AttnArgs& a, SeqRows rows) : r(rows) {
    const int end = min(r.len + r.n, a.b.max_pages * a.c.B);
    T = max((end + kTile - 1) / kTile, 1);
    nrt = (r.n * a.G + R - 1) / R;
    grains = (T + a.grain - 1) / a.grain;
    if constexpr (kPairs) {
      // group i sees up to position x(i) = len + ((i + 1) R - 1) / G: x / span + 1 grains
      const uint32_t sum = 2u * (uint32_t)r.len + (uint32_t)((R - 1) / a.G) + (uint32_t)((nrt * R - 1) / a.G) + 1u;
      W = (int)min(sum / (uint32_t)(a.grain * kTile) + 2u, 2u * (uint32_t)grains);
    }
  }
  // The last position that group rt sees.
  __device__ __forceinline__ int see_last(const AttnArgs& a, int rt) const {
    return r.len + (min(rt * R + R, r.n * a.G) - 1) / a.G;
  }
  __device__ __forceinline__ int unit_grains(const AttnArgs& a, int rt) const {
    return kPairs ? min(see_last(a, rt) / (a.grain * kTile) + 1, grains) : grains;
  }
  __device__ __forceinline__ int64_t of_head(const AttnArgs& a) const {
    if constexpr (kPairs) return (int64_t)(nrt / 2) * W + (nrt % 2 ? unit_grains(a, nrt / 2) : 0);
    return (int64_t)nrt * grains;
  }
  __device__ __forceinline__ int64_t all(const AttnArgs& a) const { return (int64_t)a.c.hkv * of_head(a); }

  // Of place base + off, base being the sequence's first.
  __device__ __forceinline__ Unit unit(const AttnArgs& a, int64_t base, int64_t off) const {
    Unit u;
    if (kPairs && grains > 1) {
      const int64_t each = of_head(a);
      u.head = (int)div64(off, each);
      off -= u.head * each;
      const int i = (int)div64(off, W);  // the last may be the middle group alone
      u.u0 = (int)(off - (int64_t)i * W);
      u.first = base + u.head * each + (int64_t)i * W;
      const int n = unit_grains(a, nrt - 1 - i);
      u.rt = nrt - 1 - i;
      u.grains = n;
      if (u.u0 >= n) {
        u.rt = i;
        u.u0 -= n;
        u.first += n;
        u.grains = unit_grains(a, i);
        if (u.u0 >= u.grains) {
          u.rt = -1;
          u.u0 -= u.grains;
          u.first += u.grains;
          u.grains = W - n - u.grains;
        }
      }
    } else {  // also where a group is one grain
      const int i = (int)div64(off, grains);
      u.u0 = (int)(off - (int64_t)i * grains);
      u.rt = i % nrt;
      u.head = i / nrt;
      u.grains = grains;
      u.first = base + (int64_t)i * grains;
    }
    return u;
  }
};

// The grains of all units in a row, in shares that differ by one at most: workgroup i of n takes the places
// from i total / n on (rounded down), where n is the grid or, if there are fewer, the grains.  Up to 64 sequences every wave looks
// them over by itself, one a lane; more are counted by the workgroup, some a thread.
template <int R, int NW>
struct Places {
  int64_t total;
  int shares;
  int64_t end, own;  // of this lane's sequence (few), of this thread's sequences (many)
  SeqRows mine;
  bool few;
  int per;

  __device__ __forceinline__ void count(const AttnArgs& a, int workgroups, int64_t* lds) {
    few = a.b.n_seqs <= kWave;
    own = 0;
    if (few) {
      const int lane = lane_id();
      mine = SeqRows{0, 0, 0};
      if (lane < a.b.n_seqs) {
        mine = seq_rows(a.s, a.b, a.c.B, lane);
        own = SeqWork<R>(a, mine).all(a);
      }
      end = wave_scan(own);
      total = lane_value(end, kWave - 1);
    } else {
      per = (a.b.n_seqs + NW * kWave - 1) / (NW * kWave);
      for (int i = 0; i < per; ++i) {
        const int s = (int)threadIdx.x * per + i;
        if (s < a.b.n_seqs) own += SeqWork<R>(a, seq_rows(a.s, a.b, a.c.B, s)).all(a);
      }
      end = block_scan<int64_t, NW>(own, lds, &total);
    }
    total = lane_value(total, 0);
    shares = (int)min((int64_t)workgroups, total);
    // One sequence of several row groups: if that leaves most of the workgroups busy, each unit is cut into the same number of
    // shares, so that the groups go over the keys in step and share them in L2.  28 heads over 4, 32k tokens, as they fall / in
    // step, us: 224 rows 43.5 / 31.5, 448 67.7 / 43.6, 672 89.5 / 57.5; 8k: 448 28.9 / 25.3.
    if (R <= 32 && a.b.n_seqs == 1 && total > 0) {
      const SeqWork<R> w = work(a, 0);
      const int units = (int)min((int64_t)a.c.hkv * w.nrt, (int64_t)workgroups + 1), k = workgroups / units;
      if (w.nrt > 1 && k > 0 && k <= w.grains && 8 * units * k >= 7 * workgroups) shares = units * k;
    }
  }

  __device__ __forceinline__ int64_t start(int wg) const { return div64(wg * total, shares); }
  // The workgroup whose share holds a place.
  __device__ __forceinline__ int owner(int64_t pos) const { return (int)div64((pos + 1) * shares - 1, total); }

  static __device__ __forceinline__ int64_t lane_value(int64_t x, int lane) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)x, lane) |
                     (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32);
  }

  // Sequence s's part of the work.
  __device__ __forceinline__ SeqWork<R> work(const AttnArgs& a, int s) const {
    if (!few) return SeqWork<R>(a, seq_rows(a.s, a.b, a.c.B, s));
    return SeqWork<R>(a, SeqRows{__builtin_amdgcn_readlane(mine.len, s), __builtin_amdgcn_readlane(mine.row0, s),
                                 __builtin_amdgcn_readlane(mine.n, s)});
  }

  // The sequence that holds place `pos` < total, and *base, the places before it.
  __device__ __forceinline__ int find(const AttnArgs& a, int64_t pos, int64_t* lds, int64_t* base) const {
    if (few) {
      const int s = __builtin_ctzll(__ballot(pos < end));
      *base = lane_value(end - own, s);
      return s;
    }
    if (pos >= end - own && pos < end) {
      int64_t b = end - own;
      int s = (int)threadIdx.x * per;
      for (int64_t t; (t = SeqWork<R>(a, seq_rows(a.s, a.b, a.c.B, s)).all(a)) + b <= pos; ++s) b += t;  // ends: pos < end
      lds[NW] = b;
      lds[NW + 1] = s;
    }
    __syncthreads();
    *base = lane_value(lds[NW], 0);
    return __builtin_amdgcn_readfirstlane((int)lds[NW + 1]);
  }
};

// The share of this workgroup, or a number of its own from `shares` on if there are fewer.  Workgroup i runs on XCD i % 8, and the
// grid is a multiple of 8: neighbouring shares go to one XCD, whose L2 then serves the row groups that read the same keys,
// and each XCD has an eighth of them, also where the grid, which the host sizes from bounds, has more workgroups than there are
// shares: 32 sequences of 1000 tokens, one row, the idle ones last / so, 18.1 / 13.0 us, 64 29.8 / 23.1.
__device__ __forceinline__ int share_of(int workgroups, int shares) {
  const int xcd = (int)blockIdx.x % kNumXcd, i = (int)blockIdx.x / kNumXcd;
  const int first = xcd * shares / kNumXcd, mine = (xcd + 1) * shares / kNumXcd - first;
  return i < mine ? first + i : shares + xcd * (workgroups / kNumXcd) - first + i - mine;
}

// The cut, if any, that a share leaves behind it: it ends `done` grains into the unit.
template <typename P>
__device__ __forceinline__ Cut cut_of(const P& pl, const Unit& u, int done, int row, int rows, int row0) {
  Cut k{0, 0, u.head, row, rows, row0};
  if (done < u.grains) {
    k.first = pl.owner(u.first);
    k.cuts = pl.owner(u.first + u.grains - 1) - k.first;
  }
  return k;
}

struct TileInfo {
  int t, page, ev;  // tile of the sequence, its page (-1: no tile is left), exponent of V
  float kc;         // scale of K times the softmax's
};

// The mapped tiles among t0, t0 + STEP, ... < end of one sequence and KV head.  64 are looked up in one round
// of loads, one a lane, and then read from their lanes.
template <int STEP>
struct TileList {
  const int32_t* row;
  int tb, end, pg, ev;
  float kc;
  uint64_t todo;

  __device__ __forceinline__ TileList(const AttnArgs& a, int s, int head, int t0, int t_end)
      : row(a.s.table + (int64_t)s * a.b.max_pages), tb(t0 - STEP * kWave), end(t_end), pg(0), ev(0), kc(0.f), todo(0) {}

  __device__ __forceinline__ TileInfo next(const AttnArgs& a, int head) {
    while (todo == 0 && tb + STEP * kWave < end) {
      tb += STEP * kWave;
      const int t = tb + STEP * lane_id(), slot = a.c.tiles == 2 ? t >> 1 : t;
      pg = t < end && slot < a.b.max_pages ? row[slot] : -1;
      const bool ok = pg >= 0 && pg < a.c.n_pages;
      todo = __ballot(ok);
      if (ok) {
        const float* sc = a.scales + ((int64_t)pg * a.c.hkv + head) * 2;
        kc = fmaxf(pow2f(stored_exp(sc[0])) * a.c2, 1.17549435e-38f);  // not 0, which a masked -inf must not meet
        ev = stored_exp(sc[1]);
      }
    }
    if (todo == 0) return TileInfo{0, -1, 0, 0.f};
    const int i = __builtin_ctzll(todo);
    todo &= todo - 1;
    return TileInfo{tb + STEP * i, __builtin_amdgcn_readlane(pg, i), __builtin_amdgcn_readlane(ev, i),
                    __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(kc), i))};
  }

  __device__ __forceinline__ const uint8_t* at(const AttnArgs& a, const TileInfo& x, int head) const {
    return a.pages + (((int64_t)x.page * a.c.hkv + head) * a.c.tiles + (a.c.tiles == 2 ? x.t & 1 : 0)) * (2 * kTileBytes);
  }
};

// Eight probabilities to bf16, and the sum of what they are rounded to.
__device__ __forceinline__ float form_eight(const float (&p)[8], bf16x8& P) {
  const bf16x2 x = pack_bf16(p[0], p[1]), y = pack_bf16(p[2], p[3]), z = pack_bf16(p[4], p[5]), v = pack_bf16(p[6], p[7]);
  P = bf16x8{x[0], x[1], y[0], y[1], z[0], z[1], v[0], v[1]};
  return dot2_bf16_sum(v, dot2_bf16_sum(z, dot2_bf16_sum(y, dot2_bf16_sum(x, 0.f))));
}

// One tile's softmax for C groups of columns: S (raw products, register i of score tile ti is key
// 16 g + 4 ti + i) becomes P, the next product's operands; kc takes S to the base-2 exponent, and P is made as
// 2^ev p, what V's codes are to be multiplied by.  The probabilities are formed against the reference M
// of their column at once, without looking for the tile's maximum; they stand while a lane's sum of them is
// at most 2^8, so that every p is, where its bf16 rounding is that of one below 1 and the 32-bit sums have
// room.  Otherwise, and for a column without a reference, M is raised to the maximum, O and L are
// rescaled, and P is formed again.  L sums the rounded p's, which are what PV adds.
// P is rounded to bf16, as in the prefill: products of 32 bits would take 16 times the matrix cycles, and fp16's range does not hold
// 2^ev p.  A p is off by up to 2^-8 of itself.  Against 64 bits the listed cases' results are off by 0.0022 to 0.0023 of their
// size, with P in 32 bits by 0.0016 to 0.0017 (the rounding of the result).
// A column without a reference is one that has seen no key yet, unless the tile, whose first position is `first`, holds one that it
// sees: then every product of it so far is NaN or -infinity (a query that is not finite), and what it forms, NaN, stands.
template <int C>
__device__ __forceinline__ void softmax_step(const acc4 (&S)[C][4], float kc, int ev, int first, const int (&see)[C],
                                             float (&M)[C], float (&L)[C], acc4 (&O)[C][8], bf16x8 (&P)[C][2]) {
  const float inv_v = pow2f(-ev);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const auto form = [&] {
      const float sub = M[c] - (float)ev;
      float sum = 0.f;
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = fast_exp2(__builtin_fmaf(S[c][2 * st + e / 4][e & 3], kc, -sub));
        sum += form_eight(p, P[c][st]);
      }
      return sum * inv_v;
    };
    float sum = form();
    if (__ballot(!(sum <= 256.f))) {  // also an infinity or NaN, as from M = -inf
      float mx = S[c][0][0];
#pragma unroll
      for (int ti = 0; ti < 4; ++ti)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, S[c][ti][i]);
      mx = column(mx, [](float x, float y) { return fmaxf(x, y); }) * kc;
      const float m = M[c] > mx ? M[c] : mx;  // NaN where every product is
      if (m != M[c]) {
        const float f = fast_exp2(M[c] - m);
        L[c] *= f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i) O[c][dt][i] *= f;
        M[c] = m;
      }
      sum = form();
      if (M[c] == -__builtin_inff() && first > see[c]) {
        sum = 0.f;
        P[c][0] = P[c][1] = bf16x8{};
      }
    }
    L[c] += sum;
  }
}

// One workgroup's share.  Tiles of a unit go round the waves; each wave keeps its own running
// maximum, sum and output, joined through LDS at the unit's end.  A lane's 16-byte loads are
// matrix operands as they stand (cache_device.h): K of the next tile is loaded while the softmax
// and PV of this one run, V while the next scores are made, nothing passes through LDS.  Bound by HBM: one row of each of
// 48 sequences of 0.3k to 8k tokens, 32 heads over 8, e4m3 (462 MB), 78 us, 5.9 TB/s; one sequence of 128k, 28 heads over 4,
// int8 (134 MB), 27 us, 5.0 TB/s; up to six rows of each of 24 (111 MB, which is three grains a workgroup) 29.6 us, 3.7 TB/s.
template <int FMT, int C, bool ONCE>
__global__ __launch_bounds__(kFewWaves* kWave, 2) void cache_attn(AttnArgs a) {
  constexpr int NW = kFewWaves, kRows = 16 * C;
  __shared__ __attribute__((aligned(16))) float xo[NW][C][8][kWave][4];
  __shared__ float xm[NW][kRows], xl[NW][kRows];
  __shared__ int64_t lds[NW + 2];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int wgs = gridDim.x;
  Places<kRows, NW> pl;
  pl.count(a, wgs, lds);
  const int wg = share_of(wgs, pl.shares);
  if (wg >= pl.shares) {
    if (a.cut && tid == 0) a.cut[wg].cuts = 0;
    return;
  }
  int64_t pos = pl.start(wg);
  const int64_t stop = pl.start(wg + 1);
  int64_t base;
  int s = pl.find(a, pos, lds, &base);
  SeqWork<kRows> sw = pl.work(a, s);
  while (pos < stop) {
    while (pos >= base + sw.all(a) && s + 1 < a.b.n_seqs) {
      base += sw.all(a);
      sw = pl.work(a, ++s);
    }
    const Unit u = sw.unit(a, base, pos - base);
    const int rt = u.rt, head = u.head, u0 = u.u0;
    const int part = (int)min((int64_t)(u.grains - u0), stop - pos);
    const int t0 = u0 * a.grain, t1 = min((u0 + part) * a.grain, sw.T);  // the tiles of this piece
    const int rows = sw.r.n * a.G;  // fits: n_rows G is checked on the host
    const int held = min(sw.r.len + sw.r.n, a.b.max_pages * a.c.B);
    // q: lane holds its column's elements 32 g + [0, 32)
    bf16x8 Q[C][4];
    int see[C];  // the last position that this lane's column sees
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int r = rt * kRows + 16 * c + col;
      const int i = r / a.G;
      see[c] = r < rows ? sw.r.len + i : -1;
      const uint16_t* src = a.q + (head * a.G + (r - i * a.G)) * a.qs.head + (sw.r.row0 + i) * a.qs.row + 32 * g;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        Q[c][j] = bf16x8{};
        if (r < rows) Q[c][j] = *reinterpret_cast<const bf16x8*>(src + 8 * j);
      }
    }
    const int see_first = sw.r.len + rt * kRows / a.G;
    const int see_last = sw.see_last(a, rt);
    acc4 O[C][8];
    float M[C], L[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      M[c] = see[c] >= 0 ? -__builtin_inff() : 0.f;  // a column without a row asks for no reference
      L[c] = 0.f;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) O[c][dt] = acc4{0.f, 0.f, 0.f, 0.f};
    }
    TileList<NW> list(a, s, head, t0 + w, min(t1, see_last / kTile + 1));
    const auto load = [&](u32x4* x, const TileInfo& tl, int tensor) {
      const uint8_t* src = list.at(a, tl, head) + tensor * kTileBytes + lane * kChunk;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const u32x4* at = reinterpret_cast<const u32x4*>(src + i * (kWave * kChunk));
        x[i] = ONCE ? __builtin_nontemporal_load(at) : *at;
      }
    };
    u32x4 K[8], V[8];
    TileInfo now = list.next(a, head);
    if (now.page >= 0) {
      load(K, now, 0);
      load(V, now, 1);
    }
    while (now.page >= 0) {
      const TileInfo next = list.next(a, head);
      acc4 S[C][4];
#pragma unroll
      for (int j = 0; j < 4; ++j)  // by steps of d, so that products into one accumulator are apart
#pragma unroll
        for (int ti = 0; ti < 4; ++ti) {
          if (j % 2 == 0) keep_whole(K[2 * ti + j / 2]);
          const u32x4 x = K[2 * ti + j / 2];
          const bf16x8 k = codes_to_bf16<FMT>(x[2 * (j & 1)], x[2 * (j & 1) + 1]);
#pragma unroll
          for (int c = 0; c < C; ++c) S[c][ti] = mfma16(k, Q[c][j], j == 0 ? acc4{0.f, 0.f, 0.f, 0.f} : S[c][ti]);
        }
      __builtin_amdgcn_sched_barrier(0);
      if (next.page >= 0) load(K, next, 0);
      const int key0 = now.t * kTile + 16 * g;
      if (now.t * kTile + kTile - 1 > see_first) {  // some column does not see the whole tile
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int ti = 0; ti < 4; ++ti)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (key0 + 4 * ti + i > see[c]) S[c][ti][i] = -__builtin_inff();
        // codes behind the last token may be anything; so may those of a later row's token that was never
        // appended: a NaN among them would pass a probability of 0
        const int n = held - key0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int bytes = min(max(n - 4 * e, 0), 4);
          const uint32_t keep = bytes == 4 ? ~0u : (1u << (8 * bytes)) - 1u;
#pragma unroll
          for (int i = 0; i < 8; ++i) V[i][e] = without_nan<FMT>(V[i][e] & keep);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      bf16x8 P[C][2];
      softmax_step<C>(S, now.kc, now.ev, now.t * kTile, see, M, L, O, P);
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
          if (st == 0) keep_whole(V[dt]);
          const bf16x8 v = codes_to_bf16<FMT>(V[dt][2 * st], V[dt][2 * st + 1]);
#pragma unroll
          for (int c = 0; c < C; ++c) O[c][dt] = mfma16(v, P[c][st], O[c][dt]);
        }
      __builtin_amdgcn_sched_barrier(0);
      if (next.page >= 0) load(V, next, 1);
      now = next;
    }
    // join the waves: each leaves its output in LDS and sums 8 / NW of the eight 16-element parts of all
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const float l = column(L[c], [](float x, float y) { return x + y; });
      if (g == 0) {
        xm[w][16 * c + col] = M[c];
        xl[w][16 * c + col] = l;
      }
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<acc4*>(xo[w][c][dt][lane]) = O[c][dt];
    }
    __syncthreads();
    const bool whole = part == u.grains;
    float* slot = a.part + (int64_t)(2 * wg + (u0 == 0)) * (kRows * (kHeadDim + 2));
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int r = rt * kRows + 16 * c + col;
      float m = -__builtin_inff(), l = 0.f, f[NW];
#pragma unroll
      for (int i = 0; i < NW; ++i) m = fmaxf(m, xm[i][16 * c + col]);
      const float ms = m == -__builtin_inff() ? 0.f : m;
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        f[i] = fast_exp2(xm[i][16 * c + col] - ms);
        l += f[i] * xl[i][16 * c + col];
      }
      if (r >= rows) continue;
      const float inv = l > 0.f ? 1.f / l : 0.f;
      const int i = r / a.G;
      uint16_t* dst = a.o + (head * a.G + (r - i * a.G)) * a.os.head + (sw.r.row0 + i) * a.os.row + 4 * g;
#pragma unroll
      for (int x = 0; x < 8 / NW; ++x) {
        const int dt = w * (8 / NW) + x;
        acc4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int y = 0; y < NW; ++y) {
          const acc4 z = *reinterpret_cast<const acc4*>(xo[y][c][dt][lane]);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(f[y], z[e], o[e]);
        }
        if (whole) {
          const bf16x2 p = pack_bf16(o[0] * inv, o[1] * inv), q = pack_bf16(o[2] * inv, o[3] * inv);
          *reinterpret_cast<bf16x4*>(dst + 16 * dt) = bf16x4{p[0], p[1], q[0], q[1]};
        } else {
          *reinterpret_cast<acc4*>(slot + (16 * c + col) * kHeadDim + 16 * dt + 4 * g) = o;
        }
      }
      if (!whole && w == 0 && g == 0) {
        slot[kRows * kHeadDim + 16 * c + col] = m;
        slot[kRows * kHeadDim + kRows + 16 * c + col] = l;
      }
    }
    __syncthreads();
    pos += part;
    if (pos >= stop && a.cut && tid == 0)
      a.cut[wg] = cut_of(pl, u, u0 + part, rt * kRows, min(rows - rt * kRows, kRows), sw.r.row0);
  }
}

// Many rows a sequence: a unit is 128 rows, 32 a wave, and all four waves go over the same tiles, whose
// codes come into LDS once a workgroup by direct loads, three tiles deep.  The waves' rows
// are their own, so nothing is joined inside the workgroup.  Two workgroups share a CU: while a wave of one
// forms probabilities, one of the other feeds the matrix unit.
// Bound by the issue of the two: chunks of 75 to 450 rows of three sequences of 15k to 23k tokens, 28 heads over 4, e4m3: matrix unit
// busy on 47% of the cycles, vector unit on 49%, both on 15%; with the join 237 to 258 us from card to card, 0.98 to 1.07 PFLOP/s, once
// the clock has settled (a burst's first milliseconds have up to 330).
//
// The products are v_mfma_f32_32x32x16_bf16 (layouts in crisp_device.h): beside these the other wave's vector
// instructions run 1.45 times as long as alone, beside the 16 x 16 ones 1.9 times.  The tile's chunks serve them as
// well, each lane reading from LDS the ones it needs (a quarter of a wave reads 256 bytes in a row).
// With h = l / 32:
//   K: score tile T (32 keys), step (g, m): lane l takes chunk (t = 2 T + l % 32 / 16, half = h, g, r = l % 16), bytes
//      8 m ..: key of row l % 32, elements 32 g + 16 h + 8 m + [0, 8).  The result's register i of a lane is key
//      16 (2 q + h) + 4 (2 T + i / 8) + i % 4 with q = i / 4 % 2: 16 keys in a row for each q.
//      int8 codes become fp16, cheaper than bf16 (codes_to_half): 8192 rows over no history 681 / 657, 1024 over 15000 tokens
//      341 / 331, 2048 over 2048 150 / 143.6 (us, as below).
//      e4m3 codes need no conversion: v_mfma_f32_32x32x64_f8f6f4 takes them as they are, 64 elements and so the chunks of two g
//      at a time, and q comes as a sum of two e4m3 (split_row), which costs as many matrix cycles as bf16.  32 heads
//      over 8, codes to bf16 / as they are, us: 8192 rows over no history 536 / 471 (1168 TFLOP/s), 16384 2070 / 1793, 1024
//      over 15000 tokens 277 / 247, 2048 over 2048 119.5 / 107.7.
//   V: output rows 32 D .., step (q, s): chunk (dt = 2 D + l % 32 / 16, g = 2 q + h, r = l % 16), bytes 8 s ..: those
//      keys' 8 s + [0, 8), so that P again stays in its lane.
constexpr int kRowWaves = 4, kRowUnit = 32 * kRowWaves;

#if defined(__HIP_DEVICE_COMPILE__)
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
__device__ __forceinline__ u32x4 lds_chunk_at(int addr) { return *(const lds_u32x4*)(uint32_t)addr; }
#endif

typedef __attribute__((__vector_size__(8 * sizeof(int)))) int i32x8;

// 32 x 32 products over 64 elements, e4m3 codes as they are; the second factor times 2^-5 if `second`.
template <bool second>
__device__ __forceinline__ f32x16 mfma32_codes(i32x8 a, i32x8 b, f32x16 c) {
  return second ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 127, 0, 122)
                : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
}

// The bits of a row's largest |q|, of which a lane holds half: 16 elements in Q[g].
__device__ __forceinline__ uint32_t row_top(const bf16x8 (&Q)[4][2]) {
  uint32_t m = 0;
#pragma unroll
  for (int g = 0; g < 4; ++g)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const u32x4 q = __builtin_bit_cast(u32x4, Q[g][x]);
#pragma unroll
      for (int i = 0; i < 4; ++i) m = max(m, max(q[i] & 0x7fffu, (q[i] >> 16) & 0x7fffu));
    }
  const auto r = __builtin_amdgcn_permlane32_swap(m, m, false, false);
  return max(r[0], r[1]);
}

// The exponent e that takes the largest |q| to [2^top, 2^(top + 1)) 2^e; the least is that of q's own subnormals.
__device__ __forceinline__ int row_exp(uint32_t m, int top) { return max((int)(m >> 7) - 127 - top, -120); }

// Elements 4 i .. 4 i + 3 of Q[g], times inv.
__device__ __forceinline__ f32x4 four_of(const bf16x8 (&Q)[4][2], int g, int i, float inv) {
  const u32x4 q = __builtin_bit_cast(u32x4, Q[g][i / 2]);
  const uint32_t x = q[2 * (i & 1)], y = q[2 * (i & 1) + 1];
  return f32x4{__uint_as_float(x << 16) * inv, __uint_as_float(x & 0xffff0000u) * inv, __uint_as_float(y << 16) * inv,
               __uint_as_float(y & 0xffff0000u) * inv};
}

// A row of q as two rows of e4m3, q = 2^e (a + 2^-5 b), its largest element in [2^7, 2^8) 2^e.  a is q rounded to four
// bits and b the rest, which has no more than four: nothing of a bf16's eight is lost down to 2^-14 of the
// row's largest, below it no more than 2^-22 of that.  A row that is not finite becomes NaN.  Returns 2^e.
__device__ __forceinline__ float split_row(const bf16x8 (&Q)[4][2], i32x8 (&A)[2], i32x8 (&B)[2]) {
  const uint32_t m = row_top(Q);
  const int e = row_exp(m, 7);
#pragma unroll
  for (int g = 0; g < 4; ++g)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 v = four_of(Q, g, i, pow2f(-e));
      int a = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
      a = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], a, true);
      const f32x4 w = from_codes<kCacheE4M3>((uint32_t)a);
      int b = __builtin_amdgcn_cvt_pk_fp8_f32(32.f * (v[0] - w[0]), 32.f * (v[1] - w[1]), 0, false);
      b = __builtin_amdgcn_cvt_pk_fp8_f32(32.f * (v[2] - w[2]), 32.f * (v[3] - w[3]), b, true);
      A[g / 2][4 * (g & 1) + i] = m < 0x7f80u ? a : 0x7f7f7f7f;
      B[g / 2][4 * (g & 1) + i] = m < 0x7f80u ? b : 0;
    }
  return pow2f(e);
}

typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;

// A row of q in fp16, its largest element in [2^14, 2^15) 2^e: nothing is lost down to 2^-31 of that.  A row that is not
// finite becomes NaN.  Returns 2^e.
__device__ __forceinline__ float half_row(const bf16x8 (&Q)[4][2], f16x8 (&H)[4][2]) {
  const uint32_t m = row_top(Q);
  const int e = row_exp(m, 14);
#pragma unroll
  for (int g = 0; g < 4; ++g)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 v = four_of(Q, g, i, pow2f(-e));
#pragma unroll
      for (int x = 0; x < 4; ++x) H[g][i / 2][4 * (i & 1) + x] = m < 0x7f80u ? (_Float16)v[x] : (_Float16)__builtin_nanf("");
    }
  return pow2f(e);
}

// Eight int8 codes to fp16: 1024 + (c + 128), which is a byte set beside the exponent, and 1152 taken off, exactly.
__device__ __forceinline__ f16x8 codes_to_half(uint32_t lo, uint32_t hi) {
  const auto two = [](uint32_t x, uint32_t sel) {
    const f16x2 off = {(_Float16)-1152.f, (_Float16)-1152.f};
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, x, sel)) + off);
  };
  lo ^= 0x80808080u;
  hi ^= 0x80808080u;
  const u32x4 r = {two(lo, 0x04010400u), two(lo, 0x04030402u), two(hi, 0x04010400u), two(hi, 0x04030402u)};
  return __builtin_bit_cast(f16x8, r);
}

template <int FMT>
__global__ __launch_bounds__(kRowWaves* kWave, 2) void cache_attn_rows(AttnArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int NW = kRowWaves, kRows = kRowUnit, kStages = 3;
  constexpr int kStage = 2 * kTileBytes;
  constexpr bool kCodes = FMT == kCacheE4M3;
  __shared__ __attribute__((aligned(1024))) char ring[kStages * kStage];
  __shared__ int64_t lds[NW + 2];
  const int ring0 = __builtin_amdgcn_readfirstlane((int)(size_t)ring);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, h = lane >> 5;
  const int wgs = gridDim.x;
  Places<kRows, NW> pl;
  pl.count(a, wgs, lds);
  const int wg = share_of(wgs, pl.shares);
  if (wg >= pl.shares) {
    if (a.cut && tid == 0) a.cut[wg].cuts = 0;
    return;
  }
  int64_t pos = pl.start(wg);
  const int64_t stop = pl.start(wg + 1);
  int64_t base;
  int s = pl.find(a, pos, lds, &base);
  SeqWork<kRows> sw = pl.work(a, s);
  const int k_at = ring0 + (col >> 4) * 2048 + h * 1024 + (col & 15) * kChunk;              // + T 4096 + g 256
  const int v_at = ring0 + kTileBytes + (col >> 4) * 1024 + h * 256 + (col & 15) * kChunk;  // + D 2048 + q 512
  while (pos < stop) {
    while (pos >= base + sw.all(a) && s + 1 < a.b.n_seqs) {
      base += sw.all(a);
      sw = pl.work(a, ++s);
    }
    const Unit u = sw.unit(a, base, pos - base);
    const int rt = u.rt, head = u.head, u0 = u.u0;
    const int part = (int)min((int64_t)(u.grains - u0), stop - pos);
    if (rt < 0) {
      pos += part;
      if (pos >= stop && a.cut && tid == 0) a.cut[wg].cuts = 0;
      continue;
    }
    const int t0 = u0 * a.grain, t1 = min((u0 + part) * a.grain, sw.T);  // the tiles of this piece
    const int rows = sw.r.n * a.G;
    const int held = min(sw.r.len + sw.r.n, a.b.max_pages * a.c.B);
    const int r0 = rt * kRows + w * 32;  // the wave's first row
    const bool live = r0 < rows;
    const int r = r0 + col, row_i = r / a.G;
    const int see = r < rows ? sw.r.len + row_i : -1;  // the last position that this lane's column sees
    const int64_t q_at = (head * a.G + (r - row_i * a.G)) * a.qs.head + (sw.r.row0 + row_i) * a.qs.row;
    bf16x8 Q[4][2];  // step (g, m)
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        Q[g][m] = bf16x8{};
        if (r < rows) Q[g][m] = *reinterpret_cast<const bf16x8*>(a.q + q_at + 32 * g + 16 * h + 8 * m);
      }
    i32x8 QA[2], QB[2];
    f16x8 QH[4][2];
    float q_scale;
    if constexpr (kCodes) q_scale = split_row(Q, QA, QB);
    else q_scale = half_row(Q, QH);
    const int see_first = sw.r.len + r0 / a.G;
    const int see_last = sw.see_last(a, rt);
    f32x16 O[4];
#pragma unroll
    for (int D = 0; D < 4; ++D) O[D] = zero16();
    float M = see >= 0 ? -__builtin_inff() : 0.f, L = 0.f;  // a column without a row asks for no reference
    TileList<1> list(a, s, head, t0, min(t1, see_last / kTile + 1));
    // a wave copies a quarter of the tile: its chunks 256 w ..
    const auto fetch = [&](const TileInfo& tl, int stage) {
      const uint8_t* src = list.at(a, tl, head);
      const unsigned long long p = (unsigned long long)src;
      const i32x4 rsrc = {__builtin_amdgcn_readfirstlane((int)(unsigned)p), __builtin_amdgcn_readfirstlane((int)(unsigned)(p >> 32)),
                          kStage, 0x00020000};
#pragma unroll
      for (int j = 0; j < kStage / (NW * kWave * kChunk); ++j)
        dma16(rsrc, lane * kChunk, (w * 4 + j) * (kWave * kChunk), ring0 + stage * kStage + (w * 4 + j) * (kWave * kChunk));
    };
    TileInfo now = list.next(a, head), next{0, -1, 0, 0.f};
    if (now.page >= 0) {
      fetch(now, 0);
      next = list.next(a, head);
      if (next.page >= 0) fetch(next, 1);
    }
    int stage = 0;
    while (now.page >= 0) {
      if (next.page >= 0) wait_dma_but4();
      else wait_dma();
      __syncthreads();  // this tile is there for all waves, and all are done with the one before it
      const TileInfo then = next.page >= 0 ? list.next(a, head) : TileInfo{0, -1, 0, 0.f};
      if (then.page >= 0) fetch(then, stage == 0 ? 2 : stage - 1);
      if (live) {
        u32x4 x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = lds_chunk_at(k_at + stage * kStage + (i & 1) * 4096 + (i >> 1) * 256);
        f32x16 S[2] = {zero16(), zero16()};
        if constexpr (kCodes) {
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int T = 0; T < 2; ++T) {
              const u32x4 u = x[4 * m + T], v = x[4 * m + 2 + T];
              const i32x8 k = {(int)u[0], (int)u[1], (int)u[2], (int)u[3], (int)v[0], (int)v[1], (int)v[2], (int)v[3]};
              S[T] = mfma32_codes<false>(k, QA[m], S[T]);
              S[T] = mfma32_codes<true>(k, QB[m], S[T]);
            }
        } else {
#pragma unroll
          for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
              for (int T = 0; T < 2; ++T)
                S[T] = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes_to_half(x[2 * g + T][2 * m], x[2 * g + T][2 * m + 1]), QH[g][m], S[T], 0, 0, 0);
        }
        const float kc = fmaxf(now.kc * q_scale, 1.17549435e-38f);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = lds_chunk_at(v_at + stage * kStage + (i >> 1) * 2048 + (i & 1) * 512);
        if (now.t * kTile + kTile - 1 > see_first) {  // some column does not see the whole tile
#pragma unroll
          for (int T = 0; T < 2; ++T)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (now.t * kTile + 16 * (2 * (i / 4 % 2) + h) + 4 * (2 * T + i / 8) + i % 4 > see) S[T][i] = -__builtin_inff();
#pragma unroll
          for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int bytes = min(max(held - now.t * kTile - 16 * (2 * q + h) - 4 * e, 0), 4);
              const uint32_t keep = bytes == 4 ? ~0u : (1u << (8 * bytes)) - 1u;
#pragma unroll
              for (int D = 0; D < 4; ++D) x[2 * D + q][e] = without_nan<FMT>(x[2 * D + q][e] & keep);
            }
        }
        bf16x8 P[2][2];  // (q, s)
        const float inv_v = pow2f(-now.ev);
        const auto form = [&] {
          const float sub = M - (float)now.ev;
          float sum = 0.f;
#pragma unroll
          for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int st = 0; st < 2; ++st) {
              float p[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) p[j] = fast_exp2(__builtin_fmaf(S[st][4 * (j / 4 * 2 + q) + j % 4], kc, -sub));
              sum += form_eight(p, P[q][st]);
            }
          return sum * inv_v;
        };
        __builtin_amdgcn_s_setprio(1);
        float sum = form();
        if (__ballot(!(sum <= 256.f))) {  // as in softmax_step
          float mx = S[0][0];
#pragma unroll
          for (int T = 0; T < 2; ++T)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, S[T][i]);
          mx = half_max(mx) * kc;
          const float top = M > mx ? M : mx;
          if (top != M) {
            const float f = fast_exp2(M - top);
            L *= f;
#pragma unroll
            for (int D = 0; D < 4; ++D)
#pragma unroll
              for (int i = 0; i < 16; ++i) O[D][i] *= f;
            M = top;
          }
          sum = form();
          if (M == -__builtin_inff() && now.t * kTile > see) {
            sum = 0.f;
            P[0][0] = P[0][1] = P[1][0] = P[1][1] = bf16x8{};
          }
        }
        L += sum;
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
          for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int D = 0; D < 4; ++D)
              O[D] = mfma32(codes_to_bf16<FMT>(x[2 * D + q][2 * st], x[2 * D + q][2 * st + 1]), P[q][st], O[D]);
      }
      now = next;
      next = then;
      stage = stage == 2 ? 0 : stage + 1;
    }
    const bool whole = part == u.grains;
    const float l = half_sum(L);
    if (r < rows) {  // register i of O[D] is element 32 D + 8 (i / 4) + 4 h + i % 4
      if (whole) {
        const float inv = l > 0.f ? 1.f / l : 0.f;
        uint16_t* dst = a.o + (head * a.G + (r - row_i * a.G)) * a.os.head + (sw.r.row0 + row_i) * a.os.row + 4 * h;
#pragma unroll
        for (int D = 0; D < 4; ++D)
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const bf16x2 p = pack_bf16(O[D][i] * inv, O[D][i + 1] * inv), q = pack_bf16(O[D][i + 2] * inv, O[D][i + 3] * inv);
            *reinterpret_cast<bf16x4*>(dst + 32 * D + 2 * i) = bf16x4{p[0], p[1], q[0], q[1]};
          }
      } else {
        float* slot = a.part + (int64_t)(2 * wg + (u0 == 0)) * (kRows * (kHeadDim + 2));
        const int x = r - rt * kRows;
#pragma unroll
        for (int D = 0; D < 4; ++D)
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<acc4*>(slot + x * kHeadDim + 32 * D + 2 * i + 4 * h) = acc4{O[D][i], O[D][i + 1], O[D][i + 2], O[D][i + 3]};
        if (h == 0) {
          slot[kRows * kHeadDim + x] = M;
          slot[kRows * kHeadDim + kRows + x] = l;
        }
      }
    }
    pos += part;
    if (pos >= stop && a.cut && tid == 0)
      a.cut[wg] = cut_of(pl, u, u0 + part, rt * kRows, min(rows - rt * kRows, kRows), sw.r.row0);
    __syncthreads();  // all waves are done with the ring before the next unit fills it
  }
#endif
}

// Pieces p = from, from + step, ... <= last of one row, added up by 32 lanes of four elements each: the common
// reference m, the sum l and the output o under it.  N pieces are loaded at once; past the last it is that
// one again, with the weight 0.
template <int N, typename Slot>
__device__ __forceinline__ void add_pieces(const Slot& slot, int rows, int r, int d, int from, int step, int last, float& m,
                                           float& l, acc4& o) {
  m = -__builtin_inff();
  l = 0.f;
  o = acc4{0.f, 0.f, 0.f, 0.f};
  for (int p0 = from; p0 <= last; p0 += N * step) {
    float pm[N], pl[N];
    acc4 x[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float* src = slot(min(p0 + k * step, last));
      pm[k] = src[rows * kHeadDim + r];
      pl[k] = src[rows * kHeadDim + rows + r];
      x[k] = *reinterpret_cast<const acc4*>(src + r * kHeadDim + d);
    }
    float top = m;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (p0 + k * step > last) pm[k] = -__builtin_inff();
      top = fmaxf(top, pm[k]);
    }
    const float ts = top == -__builtin_inff() ? 0.f : top, f = fast_exp2(m - ts);
    l *= f;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float w = fast_exp2(pm[k] - ts);
      l = __builtin_fmaf(w, pl[k], l);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(w, x[k][e], o[e]);
    }
    m = top;
  }
}

// Joins the pieces of the units that share boundaries cut.  Workgroup b stands at the boundary between
// shares b and b + 1; the boundaries inside one unit take its rows in turn.  A piece that begins
// its unit lies in the second slot of its workgroup, any other in the first.  Pieces are added in
// a fixed order.  All latency, the record, the pieces, the result: 4.6 us; 128 rows a unit, 133 KB at each boundary, 10.8.
template <int kRows>
__global__ __launch_bounds__(kJoinWaves* kWave) void cache_attn_join(AttnArgs a) {
  constexpr int64_t kSlot = kRows * (kHeadDim + 2);
  constexpr int kGroups = kJoinWaves * 2;  // of 32 lanes, each lane four elements
  __shared__ float ms[kGroups], ls[kGroups], acc[kGroups][kHeadDim];
  const int tid = threadIdx.x;
  const Cut k = a.cut[blockIdx.x];
  if (k.cuts == 0) return;
  const int first = k.first, cuts = k.cuts, mine = (int)blockIdx.x - first, rows = k.rows;
  const int grp = tid >> 5, d = 4 * (tid & 31);
  const auto slot = [&](int p) { return a.part + (int64_t)(2 * (first + p) + (p == 0)) * kSlot; };
  const auto write = [&](int r, float l, acc4 o) {
    const float f = l > 0.f ? 1.f / l : 0.f;
    const int i = (k.row + r) / a.G;
    uint16_t* dst = a.o + (k.head * a.G + (k.row + r - i * a.G)) * a.os.head + (k.row0 + i) * a.os.row + d;
    const bf16x2 x = pack_bf16(o[0] * f, o[1] * f), y = pack_bf16(o[2] * f, o[3] * f);
    *reinterpret_cast<bf16x4*>(dst) = bf16x4{x[0], x[1], y[0], y[1]};
  };
  float m, l;
  acc4 o;
  if (cuts < rows) {  // some rows a workgroup: one a group
    for (int r = mine + cuts * (grp + kGroups * (int)blockIdx.y); r < rows; r += cuts * kGroups * (int)gridDim.y) {
      add_pieces<4>(slot, kRows, r, d, 0, 1, cuts, m, l, o);
      write(r, l, o);
    }
    return;
  }
  if (mine >= rows || blockIdx.y > 0) return;
  // at most one: each group takes every eighth piece, and the first joins the groups
  add_pieces<8>(slot, kRows, mine, d, grp, kGroups, cuts, m, l, o);
  if ((tid & 31) == 0) {
    ms[grp] = m;
    ls[grp] = l;
  }
  *reinterpret_cast<acc4*>(&acc[grp][d]) = o;
  __syncthreads();
  if (grp > 0) return;
  float top = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < kGroups; ++i) top = fmaxf(top, ms[i]);
  if (top == -__builtin_inff()) top = 0.f;
  l = 0.f;
  o = acc4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    const float w = fast_exp2(ms[i] - top);
    l = __builtin_fmaf(w, ls[i], l);
    const acc4 x = *reinterpret_cast<const acc4*>(&acc[i][d]);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(w, x[e], o[e]);
  }
  write(mine, l, o);
}

template <int FMT>
hipError_t launch(const AttnArgs& a, const CacheAttnPlan& p, hipStream_t stream) {
  const dim3 grid(p.workgroups), joins(p.workgroups - 1, p.rows <= 32 ? 1 : 4);
  if (p.rows == kRowUnit) hipLaunchKernelGGL((cache_attn_rows<FMT>), grid, dim3(kRowWaves * kWave), 0, stream, a);
  else if (p.rows == 16) hipLaunchKernelGGL((cache_attn<FMT, 1, true>), grid, dim3(kFewWaves * kWave), 0, stream, a);
  else if (p.once) hipLaunchKernelGGL((cache_attn<FMT, 2, true>), grid, dim3(kFewWaves * kWave), 0, stream, a);
  else hipLaunchKernelGGL((cache_attn<FMT, 2, false>), grid, dim3(kFewWaves * kWave), 0, stream, a);
  if (joins.x > 0 && a.cut) {
    if (p.rows == 16) hipLaunchKernelGGL((cache_attn_join<16>), joins, dim3(kJoinWaves * kWave), 0, stream, a);
    else if (p.rows == 32) hipLaunchKernelGGL((cache_attn_join<32>), joins, dim3(kJoinWaves * kWave), 0, stream, a);
    else hipLaunchKernelGGL((cache_attn_join<kRowUnit>), joins, dim3(kJoinWaves * kWave), 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace

CacheAttnPlan cache_attn_plan(const CacheDims& c, const BatchDims& b, int hq) {
  CacheAttnPlan p{16, kGrain, 0, false, 0, 0};
  if (b.n_seqs == 0 || b.n_rows == 0 || hq == 0) return p;
  const int64_t G = hq / c.hkv;
  // Rows of a unit: 16, 32 or 128.  By the rows of an average sequence and KV head; sequences of 4k to 8k tokens, 16 / 32 / 128 rows a
  // unit, us: 32 of 10 rows 77.5 / 77.3 / 113, of 18 103 / 81.6 / 115, of 27 122 / 105 / 135; 64 of 4 rows, 2k tokens, 57.5 / 58.5 / 89.4, of
  // 16 each 22.6 / 24.3 / 26.8.
  // Between 8 and 16 rows on average it depends on how they are spread, which only the device knows.  A step of as many tokens for each
  // sequence (drafts of one length) has n_rows a multiple of n_seqs, so that is taken for one.  32 heads over 8, three tokens each / one
  // to five / one or nine, units of 16 and of 32, us: 32 sequences of 4k to 8k tokens 71.8 and 76.3 / 79.6 and 77.2 / 96.3 and 91.5, 64 of 1k
  // to 3k 54.4 and 58.3 / 59.2 and 59.4 / 68.9 and 69.1: gained where the guess holds, 0 to 5% lost where it does not.
  const int64_t rows = (int64_t)b.n_rows * G, seqs = b.n_seqs;
  const bool even16 = b.n_rows % seqs == 0 && rows <= 16 * seqs;
  p.rows = rows <= 8 * seqs || even16 ? 16 : 32;
  // units, and tiles of one, that the table has room for: upper bounds of what the lengths say on the device
  const int64_t room = (int64_t)b.max_pages * c.tiles > 1 ? (int64_t)b.max_pages * c.tiles : 1;
  // Short tables: units are not cut, which saves the second launch.  One row a sequence, 32 heads over 8, cut / not, us:
  // 1 sequence of 1000 tokens (16 tiles) 11.0 / 9.5, 16 12.5 / 10.9, 64 25.2 / 23.1, 256 88.5 / 86.6; 1 of 2000 (alone on the GPU) 9.3 / 12.3.
  const bool whole = room <= 16;
  if (whole) p.grain = (int)room;
  const auto units = [&](int r) { return (rows / r + seqs) * c.hkv; };
  const auto work = [&](int r) { return (double)units(r) * (double)((room + p.grain - 1) / p.grain); };
  constexpr int kMost = 512;  // what the GPU holds at once: two a CU, of four waves with up to 256 registers
  // 128 rows halve the work of a product, but its fewer units are cut into more pieces, each with 128 rows of partial sums: from six
  // grains a workgroup on.  32 heads over 8, 32 / 128 rows a unit, us, one sequence of 8k tokens: 128 rows 21.9 / 31.0, 512 33.2 / 38.1,
  // 1024 (4.6 grains) 51.1 / 53.8, 1600 (6.7) 74.6 / 74.0; of 32k: 128 32.6 / 40.1, 256 (5.9) 46.4 / 48.7, 512 (9.8) 77.4 / 73.8, 1600 312 /
  // 199.  Up to 64 rows half of its waves or more would have none (int8, whose codes cost more in each wave, 96), which gains little
  // where it gains and costs much where sequences are short in a wide table: 32 sequences of 2k tokens, 40 rows 59.5 / 53.7, 80
  // 71.3 / 63.5, 112 107 / 70.1; int8 80 79.5 / 79.8, 112 107 / 86.5; 2 of 3k, 64 rows 18.2 / 26.1.
  if (rows > (c.fmt == kCacheE4M3 ? 64 : 96) * seqs && work(kRowUnit) > 6 * kMost) p.rows = kRowUnit;
  // About one unit a sequence and KV head: tiles are not read again, and the loads say so.  Plain / such loads, us: 48 rows
  // over 0.3k to 8k tokens 93.6 / 83.6, one over 128k 37.5 / 33.5; in units of 32 rows, 32 sequences of 18 rows 96.6 / 83.6, of
  // 27 109 / 106, of 38 44.3 / 46.8, of 54 73.3 / 84.2.
  p.once = rows <= 32 * seqs;
  const auto workgroups = [&](int r) {
    const double w = work(r);
    // Whole units of 32 rows and more take a workgroup each; of 16, whose work is much the same, 512 workgroups take them in turn,
    // us: 256 sequences of 500 tokens, one row, 51.7 / 45.6, of 200 37.8 / 28.7; 32 sequences of 500, 40 rows, 36.7 / 39.0 (int8 37.6 / 43.5).
    const int most = whole && r > 16 ? 4096 : kMost;
    const int64_t wgs = (int64_t)(w < most ? w : most);
    return (size_t)((wgs + kNumXcd - 1) / kNumXcd * kNumXcd);
  };
  const auto cut_bytes = [&](int r) { return (workgroups(r) * sizeof(Cut) + 255) / 256 * 256; };
  p.workgroups = (int)workgroups(p.rows);
  if (whole) {
    p.bytes = 256;
  } else {
    p.cut_bytes = cut_bytes(p.rows);
    // even16 counts as units of 32 here: so a workspace is enough for fewer rows of the same sequences too
    const int r = even16 && rows > 8 * seqs ? 32 : p.rows;
    p.bytes = cut_bytes(r) + workgroups(r) * 2 * r * (kHeadDim + 2) * sizeof(float);
  }
  return p;
}

hipError_t launch_cache_attn(const CacheDims& c, const BatchDims& b, const Seqs& s, int hq, float scale,
                             const uint16_t* q, Strides qs, const uint8_t* pages, const float* scales, uint16_t* o,
                             Strides os, void* ws, hipStream_t stream) {
  const CacheAttnPlan p = cache_attn_plan(c, b, hq);
  const AttnArgs a{c, b, s, q, qs, pages, scales, o, os, hq / c.hkv, p.grain, scale * kLog2e,
                   p.cut_bytes ? (Cut*)ws : nullptr, (float*)((char*)ws + p.cut_bytes)};
  return c.fmt == kCacheE4M3 ? launch<kCacheE4M3>(a, p, stream) : launch<kCacheInt8>(a, p, stream);
}

}  // namespace crisp
