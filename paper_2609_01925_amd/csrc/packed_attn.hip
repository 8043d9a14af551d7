// Causal attention of whole prompts of different lengths, packed behind one another.
//
// A workgroup takes 128 rows of the packed tensor and one query head, whatever sequences the rows are of, so the grid follows from
// the sizes that the host knows, and neighbouring short prompts share a block.  Row r of a sequence that begins at lo sees the keys
// [lo, r].  With q0 the block's first row and lo its sequence's begin, the keys come in tiles of 64 from lo on:
//   whole tiles   [lo, kd), kd = lo + (q0 - lo) / 64 * 64: every row of that first sequence sees all of them.  Rows of
//                 sequences that begin within the block are carried along, and what they gather is dropped behind;
//   edge tiles    [kd, last row], three at most: a lane masks the keys outside [lo, r] of its own row.
// Scores are transposed (S^T = K Q^T, a lane owns one query), P goes from one product to the other in registers and V's operands
// come from LDS through the transposing read, as in the sparse prefill.
#include <type_traits>

#include "packed_device.h"
#include "packed_internal.h"

namespace crisp {

namespace {

constexpr int kRows = 128, kWaves = 4, kThreads = kWaves * kWave;

struct PackedArgs {
  PackedDims d;
  const int32_t* row_ptr;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* o;
  Strides qs, ks, vs, os;
  int G, blocks;
  float c;       // scale log2(e)
  int per_xcd;   // KV groups of an XCD (H_kv a multiple of 8), 0: see rep
  int rep;       // XCDs of a KV group (8 a multiple of H_kv), 0: workgroups in natural order
};

// Workgroup -> query head and block of rows.  The heads of a KV group go to one XCD (or to its share of them), whose L2
// then serves the group's keys to all; later blocks, which see more keys, come first.
__device__ __forceinline__ bool unit_of(const PackedArgs& a, int wg, int& h, int& qb) {
  const int xcd = wg % kNumXcd, u = wg / kNumXcd;
  if (a.per_xcd > 0) {
    const int each = a.per_xcd * a.G, i = u % each;
    qb = a.blocks - 1 - u / each;
    h = (xcd + kNumXcd * (i / a.G)) * a.G + i % a.G;
    return qb >= 0;
  }
  if (a.rep > 0) {
    qb = a.blocks - 1 - (u / a.G * a.rep + xcd / a.d.hkv);
    h = xcd % a.d.hkv * a.G + u % a.G;
    return qb >= 0;
  }
  qb = a.blocks - 1 - wg / a.d.hq;
  h = wg % a.d.hq;
  return qb >= 0;
}

#if defined(__HIP_DEVICE_COMPILE__)

constexpr int kKeys = 64;                    // of a tile
constexpr int kStage = kKeys * 256;          // bytes of a K or V tile; two rings of two stages
constexpr int kSubs = kKeys / 32;            // 32-key parts of a tile
constexpr float kSumLimit = 256.0f;          // a lane's tile sum of P above this raises the reference

typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
__device__ __forceinline__ bf16x8 lds_chunk(int at) { return *(const lds_bf16x8*)(uint32_t)at; }
__device__ __forceinline__ bf16x4 lds_turned(int at) {
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(uint32_t)at));
}

// A lane's byte offsets in a tile: K's operand of element step kk, V's two transposing reads of 32 elements db.
struct Operands {
  int k[8], v[4][2];
  __device__ __forceinline__ explicit Operands(int l) {
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) k[kk] = lds_off(l & 31, 16 * kk + 8 * (l >> 5));
    const int row = 4 * (l >> 5) + ((l & 15) >> 2), col = 16 * ((l >> 4) & 1) + 4 * (l & 3);
#pragma unroll
    for (int db = 0; db < 4; ++db) {
      v[db][0] = lds_off(row, 32 * db + col);
      v[db][1] = lds_off(row + 8, 32 * db + col);
    }
  }
  __device__ __forceinline__ bf16x8 key(int tile, int kk, int sub) const { return lds_chunk(tile + 32 * 256 * sub + k[kk]); }
  // Operand x = 8 sub + 4 half + db of a V tile: 16 keys of 32 elements.
  __device__ __forceinline__ bf16x8 value(int tile, int x) const {
    const int at = tile + (32 * (x >> 3) + 16 * ((x >> 2) & 1)) * 256;
    return cat(lds_turned(at + v[x & 3][0]), lds_turned(at + v[x & 3][1]));
  }
};

// One KV head's rows of a tensor, which tiles are taken from.  The range of a tile's descriptor ends with the last row: keys behind read as 0.
struct Source {
  const uint16_t* base;
  int64_t stride;  // elements
  int n, voff;     // rows; this lane's byte offset in 16 keys
  __device__ __forceinline__ Source(const uint16_t* p, Strides s, int head, int rows, int w, int l)
      : base(p + head * s.head), stride(s.row), n(rows) {
    const int r = 4 * w + (l >> 4);
    voff = r * (int)(2 * s.row) + (((l & 15) ^ swz(r)) << 4);
  }
  __device__ __forceinline__ void fetch(int key0, int stage, int w) const {
    const unsigned long long p = (unsigned long long)(base + key0 * stride);
    const int64_t bytes = (n - 1 - key0) * stride * 2 + 256;
    const i32x4 rsrc = {(int)(unsigned)p, (int)(unsigned)(p >> 32), (int)(bytes < 0x7fffffff ? bytes : 0x7fffffff), 0x00020000};
#pragma unroll
    for (int i = 0; i < kKeys / 16; ++i) dma16(rsrc, voff, i * (int)(32 * stride), stage + (16 * i + 4 * w) * 256);
  }
};

typedef bf16x8 Probs[kSubs][2];

__device__ __forceinline__ void score_tile(int tile, const bf16x8 (&qf)[8], const Operands& at, f32x16 (&s)[kSubs],
                                           const bf16x8 (&first)[kSubs]) {
#pragma unroll
  for (int sub = 0; sub < kSubs; ++sub) s[sub] = zero16();
#pragma unroll
  for (int kk = 0; kk < 8; ++kk)
#pragma unroll
    for (int sub = 0; sub < kSubs; ++sub) s[sub] = mfma32(kk == 0 ? first[sub] : at.key(tile, kk, sub), qf[kk], s[sub]);
}

__device__ __forceinline__ float tile_max(const f32x16 (&s)[kSubs]) {
  float m = vmax(s[0][0], s[0][1]);
#pragma unroll
  for (int sub = 0; sub < kSubs; ++sub)
#pragma unroll
    for (int i = sub == 0 ? 2 : 0; i < 16; i += 2) m = vmax(vmax(m, s[sub][i]), s[sub][i + 1]);
  return half_max(m);
}

// P = exp2(s c - mc), rounded to bf16, and the lane's sum of the rounded ones.
__device__ __forceinline__ float form_tile(const f32x16 (&s)[kSubs], float c, float mc, Probs& p) {
  float part[2] = {0.f, 0.f};
#pragma unroll
  for (int sub = 0; sub < kSubs; ++sub)
#pragma unroll
    for (int hh = 0; hh < 2; ++hh)
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const bf16x2 pr = pack_bf16(fast_exp2(__builtin_fmaf(s[sub][8 * hh + e], c, -mc)),
                                    fast_exp2(__builtin_fmaf(s[sub][8 * hh + e + 1], c, -mc)));
        p[sub][hh][e] = pr[0];
        p[sub][hh][e + 1] = pr[1];
        part[hh] = dot2_bf16_sum(pr, part[hh]);
      }
  return part[0] + part[1];
}

__device__ __forceinline__ void add_values(int tile, const Operands& at, const Probs& p, f32x16 (&o)[4]) {
#pragma unroll
  for (int x = 0; x < 8 * kSubs; ++x) o[x & 3] = mfma32(at.value(tile, x), p[x >> 3][(x >> 2) & 1], o[x & 3]);
}

// form_tile of this tile beside add_values of the one before, in a fixed order: three pairs of probabilities ahead, then one
// pair under each product and the sums under the last ones, V's operands read two products ahead.
__device__ __forceinline__ float form_beside_values(const f32x16 (&s)[kSubs], float c, float mc, Probs& pn, int tile,
                                                    const Operands& at, const Probs& pp, f32x16 (&o)[4]) {
  constexpr int M = 8 * kSubs, kPre = 3, kAhead = 2, kBeside = M - kPre;
  float e0[M], e1[M], part[2] = {0.f, 0.f};
  const auto expo = [&](int x) {
    const int sub = x >> 3, i = 2 * (x & 7);
    e0[x] = fast_exp2(__builtin_fmaf(s[sub][i], c, -mc));
    e1[x] = fast_exp2(__builtin_fmaf(s[sub][i + 1], c, -mc));
    asm volatile("" : "+v"(e0[x]), "+v"(e1[x]));  // formed here
  };
  const auto pack = [&](int x) {
    uint32_t u = __builtin_bit_cast(uint32_t, pack_bf16(e0[x], e1[x]));
    asm volatile("" : "+v"(u));
    const bf16x2 pr = __builtin_bit_cast(bf16x2, u);
    pn[x >> 3][(x >> 2) & 1][2 * (x & 3)] = pr[0];
    pn[x >> 3][(x >> 2) & 1][2 * (x & 3) + 1] = pr[1];
  };
  const auto dot = [&](int i) {
    const int hh = i & 1, e = 2 * ((i >> 1) & 3);
    bf16x2 pr;
    pr[0] = pn[i >> 3][hh][e];
    pr[1] = pn[i >> 3][hh][e + 1];
    part[hh] = dot2_bf16_sum(pr, part[hh]);
    asm volatile("" : "+v"(part[hh]));
  };
  bf16x8 av[M];
#pragma unroll
  for (int x = 0; x < kAhead; ++x) av[x] = at.value(tile, x);
#pragma unroll
  for (int x = 0; x < kPre; ++x) {
    expo(x);
    if (x > 0) pack(x - 1);
  }
#pragma unroll
  for (int x = 0; x < M; ++x) {
    __builtin_amdgcn_sched_barrier(0);
    o[x & 3] = mfma32(av[x], pp[x >> 3][(x >> 2) & 1], o[x & 3]);
    if (x + kAhead < M) av[x + kAhead] = at.value(tile, x + kAhead);
    if (x < kBeside) {
      pack(kPre + x - 1);
      expo(kPre + x);
    } else {
      if (x == kBeside) pack(M - 1);
#pragma unroll
      for (int i = 0; i < M; ++i)
        if (i * kPre / M == x - kBeside) dot(i);
    }
  }
  __builtin_amdgcn_sched_barrier(0);
  return part[0] + part[1];
}

// The key of register i of a score tile's part `sub`.
__device__ __forceinline__ int key_of(int key0, int sub, int i, int l) {
  return key0 + 32 * sub + 8 * (i >> 2) + 4 * (l >> 5) + (i & 3);
}

// add_values for an edge tile in which some value is not finite: a masked one, whose p is 0, must not reach the row.  The finite ones
// are summed as ever; a row gets an infinity of each sign that it sees in an element, NaN counting as both.
__device__ __forceinline__ void add_mixed_values(int tile, const Operands& at, const Probs& p, int key0, int lo, int row, int l,
                                                 f32x16 (&o)[4]) {
#pragma unroll
  for (int db = 0; db < 4; ++db) {
    f32x16 up = zero16(), down = zero16();
#pragma unroll
    for (int y = 0; y < 2 * kSubs; ++y) {
      bf16x8 seen;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = key_of(key0, y >> 1, 8 * (y & 1) + e, l);
        seen[e] = (__bf16)(key >= lo && key <= row ? 1.f : 0.f);
      }
      u32x4 raw = __builtin_bit_cast(u32x4, at.value(tile, 4 * y + db)), pos, neg;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t keep = 0, plus = 0, minus = 0;
#pragma unroll
        for (int z = 0; z < 32; z += 16) {
          const uint32_t x = (raw[i] >> z) & 0xffffu;
          const bool fin = (x & 0x7f80u) != 0x7f80u;
          if (fin) keep |= x << z;
          if (!fin && x != 0xff80u) plus |= 0x3f80u << z;
          if (!fin && x != 0x7f80u) minus |= 0x3f80u << z;
        }
        raw[i] = keep;
        pos[i] = plus;
        neg[i] = minus;
      }
      o[db] = mfma32(__builtin_bit_cast(bf16x8, raw), p[y >> 1][y & 1], o[db]);
      up = mfma32(__builtin_bit_cast(bf16x8, pos), seen, up);
      down = mfma32(__builtin_bit_cast(bf16x8, neg), seen, down);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
      o[db][i] += (up[i] > 0.f ? __builtin_inff() : 0.f) - (down[i] > 0.f ? __builtin_inff() : 0.f);
  }
}

// Whether this wave's part of a tile, the rows that it fetched itself, holds a value that is not finite.
__device__ __forceinline__ bool odd_values(int tile, int w, int l) {
  typedef __attribute__((__vector_size__(2 * sizeof(uint16_t)))) uint16_t u16x2;
  asm volatile("" ::: "memory");  // behind the wait for the loads
  u16x2 top = {0, 0};
#pragma unroll
  for (int i = 0; i < kKeys / 16; ++i) {
    const u32x4 x = __builtin_bit_cast(u32x4, lds_chunk(tile + (16 * i + 4 * w) * 256 + 16 * l));
#pragma unroll
    for (int e = 0; e < 4; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, x[e] & 0x7fff7fffu));
  }
  return __ballot(top[0] >= 0x7f80 || top[1] >= 0x7f80) != 0;
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

#endif  // __HIP_DEVICE_COMPILE__

__global__ __launch_bounds__(kThreads, 2) void packed_attn(PackedArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[4 * kStage + kWaves * sizeof(int)];
  int* odd_wave = reinterpret_cast<int*>(smem + 4 * kStage);
  const int lds0 = uniform((int)(size_t)smem);
  const auto kst = [&](int i) { return lds0 + i * kStage; };
  const auto vst = [&](int i) { return lds0 + (2 + i) * kStage; };
  const int tid = threadIdx.x, l = tid & 63, w = uniform(tid >> 6);
  int head, qb;
  if (!unit_of(a, blockIdx.x, head, qb)) return;
  const int q0 = qb * kRows, row = q0 + 32 * w + (l & 31);

  // The begin of the first row's sequence, then of this lane's: the last begin at or before its row.
  const int n_seqs = a.d.n_seqs;
  const int s0 = uniform(seq_of_row(a.row_ptr, n_seqs, q0));
  const int end = min(uniform(a.row_ptr[n_seqs]), a.d.n_rows), q_end = min(q0 + kRows, end);
  if (s0 >= n_seqs || q_end <= q0) return;
  const int head_lo = s0 < 0 ? q0 : min(max(uniform(a.row_ptr[s0]), 0), q0);
  int lo = s0 < 0 ? 0x7fffffff : head_lo;
  for (int from = s0 + 1; from < n_seqs; from += kWave) {
    const int begin = from + l < n_seqs ? a.row_ptr[from + l] : 0x7fffffff;
    const bool near = begin < q_end;
    for (unsigned long long todo = __ballot(near); todo != 0; todo &= todo - 1) {
      const int b = __builtin_amdgcn_readlane(begin, __builtin_ctzll(todo));
      if (b <= row) lo = b;
    }
    if (~__ballot(near) != 0) break;
  }
  lo = max(lo, 0);
  const bool covered = row < q_end && lo <= row;

  const int g = head / a.G;
  const Operands at(l);
  const Source K(a.k, a.ks, g, a.d.n_rows, w, l), V(a.v, a.vs, g, a.d.n_rows, w, l);
  bf16x8 qf[8];
  {
    const uint16_t* src = a.q + head * a.qs.head + (int64_t)min(row, a.d.n_rows - 1) * a.qs.row + 8 * (l >> 5);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(src + 16 * kk);
  }
  f32x16 o[4];
#pragma unroll
  for (int db = 0; db < 4; ++db) o[db] = zero16();
  float m = -__builtin_inff(), sum = 0.f;
  f32x16 s[kSubs];

  const int T = (q0 - head_lo) / kKeys, kd = head_lo + T * kKeys;
  if (T > 0) {
    // Step j: K(j+1) and V(j-1) have landed; K(j+2) and V(j) go into the stages that step j-1 has done with.  P(j) is formed from
    // the scores in registers, against the standing reference, beside V(j-1) P(j-1); then the scores of j+1.
    const auto step = [&](int j, auto parity, auto first, const Probs& pp, Probs& pn) {
      constexpr int P = decltype(parity)::value;
      wait_dma();
      __syncthreads();
      if (j + 2 < T) K.fetch(head_lo + (j + 2) * kKeys, kst(P), w);
      V.fetch(head_lo + j * kKeys, vst(P), w);
      bf16x8 k0[kSubs];
#pragma unroll
      for (int sub = 0; sub < kSubs; ++sub) k0[sub] = at.key(kst(1 - P), 0, sub);
      __builtin_amdgcn_s_setprio(1);
      const float mc = m == -__builtin_inff() ? 0.f : m * a.c;
      float ts;
      if constexpr (decltype(first)::value) ts = form_tile(s, a.c, mc, pn);
      else ts = form_beside_values(s, a.c, mc, pn, vst(1 - P), at, pp, o);
#pragma unroll
      for (int sub = 0; sub < kSubs; ++sub) asm volatile("" ::"v"(pn[sub][0]), "v"(pn[sub][1]));
      asm volatile("" ::"v"(ts));
      const bool raise = !(ts <= kSumLimit) || m == -__builtin_inff();
      if (__ballot(raise)) {  // of the rows that need it, so that a row's result is its own whatever its neighbours hold
        const float top = half_max(raise ? 1.f : 0.f) > 0.f ? vmax(m, tile_max(s)) : m;
        const float alpha = m == -__builtin_inff() ? 0.f : fast_exp2((m - top) * a.c);
        sum *= alpha;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
        m = top;
        ts = form_tile(s, a.c, top == -__builtin_inff() ? 0.f : top * a.c, pn);
      }
      sum += ts;
      __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int sub = 0; sub < kSubs; ++sub) asm volatile("" ::"v"(k0[sub]));
      __builtin_amdgcn_iglp_opt(0);
      score_tile(kst(1 - P), qf, at, s, k0);  // of the last step: a stage that no load goes to, and never used
    };
    using Even = std::integral_constant<int, 0>;
    using Odd = std::integral_constant<int, 1>;
    K.fetch(head_lo, kst(0), w);
    if (T > 1) K.fetch(head_lo + kKeys, kst(1), w);
    wait_dma();
    __syncthreads();
    {
      bf16x8 k0[kSubs];
#pragma unroll
      for (int sub = 0; sub < kSubs; ++sub) k0[sub] = at.key(kst(0), 0, sub);
      score_tile(kst(0), qf, at, s, k0);
    }
    Probs pa, pz;
    step(0, Even{}, std::true_type{}, pz, pa);
    int j = 1;
    for (; j + 1 < T; j += 2) {
      step(j, Odd{}, std::false_type{}, pa, pz);
      step(j + 1, Even{}, std::false_type{}, pz, pa);
    }
    if (j < T) {
      step(j, Odd{}, std::false_type{}, pa, pz);
      wait_dma();
      __syncthreads();
      add_values(vst(1), at, pz, o);
    } else {
      wait_dma();
      __syncthreads();
      add_values(vst(0), at, pa, o);
    }
    __syncthreads();  // the rings are free
    if (lo != head_lo) {  // a row of another sequence starts anew
      m = -__builtin_inff();
      sum = 0.f;
    }
  }

  const int edges = (q_end - kd + kKeys - 1) / kKeys;
  for (int t = 0; t < edges; ++t) {
    if (t == 0 || t == 2) {  // two tiles at a time
      if (t == 2) __syncthreads();
      for (int x = t; x < t + 2 && x < edges; ++x) {
        K.fetch(kd + x * kKeys, kst(x & 1), w);
        V.fetch(kd + x * kKeys, vst(x & 1), w);
      }
      wait_dma();
      const bool odd = odd_values(vst(0), w, l) || (t + 1 < edges && odd_values(vst(1), w, l));
      if (l == 0) odd_wave[w] = odd;
      __syncthreads();
    }
    const int key0 = kd + t * kKeys;
    if (__ballot(covered && lo < key0 + kKeys && row >= key0) == 0) continue;  // no row of this wave sees the tile
    {
      bf16x8 k0[kSubs];
#pragma unroll
      for (int sub = 0; sub < kSubs; ++sub) k0[sub] = at.key(kst(t & 1), 0, sub);
      score_tile(kst(t & 1), qf, at, s, k0);
    }
#pragma unroll
    for (int sub = 0; sub < kSubs; ++sub)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = key_of(key0, sub, i, l);
        if (key < lo || key > row) s[sub][i] = -__builtin_inff();
      }
    const float top = vmax(m, tile_max(s));
    const bool fresh = m == -__builtin_inff();
    const float alpha = fresh ? 0.f : fast_exp2((m - top) * a.c);
    m = top;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = fresh ? 0.f : o[db][i] * alpha;  // (fresh: of rows not its own, perhaps NaN)
    Probs p;
    sum = sum * alpha + form_tile(s, a.c, top == -__builtin_inff() ? 0.f : top * a.c, p);
    if (uniform(odd_wave[0] | odd_wave[1] | odd_wave[2] | odd_wave[3]) == 0) add_values(vst(t & 1), at, p, o);
    else add_mixed_values(vst(t & 1), at, p, key0, lo, row, l, o);
  }

  // A row sees itself, so its sum is 0 only where all its scores are -infinity: then 0 / 0 is NaN, as the softmax is.
  const float inv = 1.f / half_sum(sum);
  if (covered) {
    uint16_t* dst = a.o + head * a.os.head + (int64_t)row * a.os.row + 4 * (l >> 5);
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16x2 x = pack_bf16(o[db][4 * i] * inv, o[db][4 * i + 1] * inv);
        const bf16x2 y = pack_bf16(o[db][4 * i + 2] * inv, o[db][4 * i + 3] * inv);
        *reinterpret_cast<bf16x4*>(dst + 32 * db + 8 * i) = bf16x4{x[0], x[1], y[0], y[1]};
      }
  }
#endif  // __HIP_DEVICE_COMPILE__
}

}  // namespace

hipError_t launch_packed_attn(const PackedDims& d, float scale, const int32_t* row_ptr, const uint16_t* q, Strides qs,
                              const uint16_t* k, Strides ks, const uint16_t* v, Strides vs, uint16_t* o, Strides os,
                              hipStream_t stream) {
  PackedArgs a{d, row_ptr, q, k, v, o, qs, ks, vs, os, d.hq / d.hkv, (d.n_rows + kRows - 1) / kRows, scale * kLog2e, 0, 0};
  int64_t grid = (int64_t)a.blocks * d.hq;
  if (d.hkv % kNumXcd == 0) {
    a.per_xcd = d.hkv / kNumXcd;
  } else if (kNumXcd % d.hkv == 0) {
    a.rep = kNumXcd / d.hkv;
    grid = (int64_t)kNumXcd * a.G * ((a.blocks + a.rep - 1) / a.rep);
  }
  hipLaunchKernelGGL(packed_attn, dim3((unsigned)grid), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace crisp
