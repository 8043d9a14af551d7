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
//
// Bound by the matrix units and, beside them, the softmax's vector instructions: three prompts of 5000 to 12000 tokens, 32 heads over 8
// (2982 GFLOP), 2.53 to 2.64 ms, 1128 to 1178 TFLOP/s at a clock of 1.7 GHz, MFMA 64% of cycles, VALU 45%, both 21%.  Short prompts are bound by their
// edges: 16 of 40 to 2500 tokens, 28 heads over 4 (252 GFLOP), 322 to 338 us, MFMA 40%; without the edge tiles' work 282 of 333, without the whole tiles
// 131, without either 102.  A wave all of whose rows begin anew in the block still takes part in the whole tiles' products (458 of that case's 8308
// tiles of a wave).  A dozen of 1 to 90 tokens 14 us, the chain of one block: begins, keys, scores, values.
// Two query heads a workgroup, with the next one's q and keys under way, took 381 where one took 360 (four 464, 48 for the short ones).
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
// then serves the group's keys to all (16 prompts of 40 to 2500 tokens 352 us, in natural order 359; the long ones the same); later
// blocks, which see more keys, come first.
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

// P = exp2(s c - mc), rounded to bf16, which the products with V take, and the lane's sum of the rounded ones, so that a row's weights still
// add up to 1.  It puts a result 0.0020 from the 64-bit one, relative to all of them, where the result's own rounding alone is 0.0016.
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

// A masked value that is not finite must not reach a row whose p it meets is 0.  In an edge tile, which rows see in part, a wave
// makes such values of the rows that it fetched itself 0; whether there were any.
__device__ __forceinline__ bool only_finite(int tile, int w, int l) {
  typedef __attribute__((__vector_size__(2 * sizeof(uint16_t)))) uint16_t u16x2;
  typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
  asm volatile("" ::: "memory");  // behind the wait for the loads
  u32x4 x[kKeys / 16];
  u16x2 top = {0, 0};
#pragma unroll
  for (int i = 0; i < kKeys / 16; ++i) {
    x[i] = __builtin_bit_cast(u32x4, lds_chunk(tile + (16 * i + 4 * w) * 256 + 16 * l));
#pragma unroll
    for (int e = 0; e < 4; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, x[i][e] & 0x7fff7fffu));
  }
  if (__ballot(top[0] >= 0x7f80 || top[1] >= 0x7f80) == 0) return true;
#pragma unroll
  for (int i = 0; i < kKeys / 16; ++i) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if ((x[i][e] & 0x7f80u) == 0x7f80u) x[i][e] &= 0xffff0000u;
      if ((x[i][e] & 0x7f800000u) == 0x7f800000u) x[i][e] &= 0xffffu;
    }
    *(lds_u32x4*)(uint32_t)(tile + (16 * i + 4 * w) * 256 + 16 * l) = x[i];
  }
  return false;
}

// What only_finite left out of the wave's 32 rows, from row0 on and stored already: an element becomes an infinity for each sign that the row
// sees among keys [kd, row] of V, NaN counting as both.  A lane has two elements and goes over the keys once, with the rows.
__device__ __forceinline__ void add_infinities(const PackedArgs& a, int head, int kd, int row0, int lo, bool covered, int l) {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");  // the rows as other lanes have stored them
  const uint16_t* v = a.v + head / a.G * a.vs.head + 2 * l;
  const unsigned long long rows = __ballot(covered);
  int from = -1, key = 0;
  float up[2] = {0.f, 0.f}, down[2] = {0.f, 0.f};
  for (int r = 0; r < 32; ++r) {
    if ((rows >> r & 1) == 0) continue;
    const int begin = __builtin_amdgcn_readlane(lo, r);
    if (begin != from) {
      from = begin;
      key = max(kd, begin);
      up[0] = up[1] = down[0] = down[1] = 0.f;
    }
    for (; key <= row0 + r; ++key) {
      const uint32_t x = *reinterpret_cast<const uint32_t*>(v + key * a.vs.row);
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const uint32_t y = z == 0 ? x & 0xffffu : x >> 16;
        if ((y & 0x7f80u) == 0x7f80u) {
          if (y != 0xff80u) up[z] = __builtin_inff();
          if (y != 0x7f80u) down[z] = __builtin_inff();
        }
      }
    }
    if (__ballot(up[0] + up[1] + down[0] + down[1] != 0.f)) {
      uint32_t* dst = reinterpret_cast<uint32_t*>(a.o + head * a.os.head + (int64_t)(row0 + r) * a.os.row + 2 * l);
      const uint32_t x = *dst;
      const bf16x2 y = pack_bf16(__uint_as_float(x << 16) + up[0] - down[0], __uint_as_float(x & 0xffff0000u) + up[1] - down[1]);
      *dst = __builtin_bit_cast(uint32_t, y);
    }
  }
}

// Waits until at most N loads of this wave are under way; kLoads make a tile.
template <int N>
__device__ __forceinline__ void wait_but() {
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4 | 15 << 8);
}
constexpr int kLoads = kKeys / 16;

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

#endif  // __HIP_DEVICE_COMPILE__

__global__ __launch_bounds__(kThreads, 2) void packed_attn(PackedArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[4 * kStage + kWaves * sizeof(int)];
  int* odd_wave = reinterpret_cast<int*>(smem + 4 * kStage);  // whether a wave has met values that are not finite
  const int lds0 = uniform((int)(size_t)smem);
  const auto kst = [&](int i) { return lds0 + i * kStage; };
  const auto vst = [&](int i) { return lds0 + (2 + i) * kStage; };
  const int tid = threadIdx.x, l = tid & 63, w = uniform(tid >> 6);
  int head, qb;
  if (!unit_of(a, blockIdx.x, head, qb)) return;
  const int q0 = qb * kRows, row = q0 + 32 * w + (l & 31);

  const int g = head / a.G;
  const Operands at(l);
  const Source K(a.k, a.ks, g, a.d.n_rows, w, l), V(a.v, a.vs, g, a.d.n_rows, w, l);
  bf16x8 qf[8];
  {
    const uint16_t* src = a.q + head * a.qs.head + (int64_t)min(row, a.d.n_rows - 1) * a.qs.row + 8 * (l >> 5);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(src + 16 * kk);
  }

  // The begin of the first row's sequence, then of this lane's: the last begin at or before its row.  Up to 64 sequences all
  // of it comes from one round of loads, a begin a lane.
  const int n_seqs = a.d.n_seqs, end = uniform(a.row_ptr[n_seqs]);
  const bool few = n_seqs <= kWave;
  const int mine = few ? a.row_ptr[min(l, n_seqs - 1)] : 0;
  int s0, head_lo;
  if (few) {
    s0 = __popcll(__ballot(l < n_seqs && mine <= q0)) - 1;
    head_lo = __builtin_amdgcn_readlane(mine, max(s0, 0));
  } else {
    s0 = uniform(seq_of_row(a.row_ptr, n_seqs, q0));
    head_lo = uniform(a.row_ptr[max(s0, 0)]);
  }
  const int q_end = min(q0 + kRows, min(end, a.d.n_rows));
  if (s0 >= n_seqs || q_end <= q0) return;
  head_lo = s0 < 0 ? q0 : min(max(head_lo, 0), q0);
  int lo = s0 < 0 ? 0x7fffffff : head_lo;
  for (int from = few ? 0 : s0 + 1; from < n_seqs; from += kWave) {
    const int begin = few ? mine : from + l < n_seqs ? a.row_ptr[from + l] : 0x7fffffff;
    const bool near = begin < q_end && from + l < n_seqs;
    for (unsigned long long todo = __ballot(near && from + l > s0); todo != 0; todo &= todo - 1) {
      const int b = __builtin_amdgcn_readlane(begin, __builtin_ctzll(todo));
      if (b <= row) lo = b;
    }
    if (~__ballot(near) != 0) break;
  }
  lo = max(lo, 0);
  const bool covered = row < q_end && lo <= row;

  f32x16 o[4];
#pragma unroll
  for (int db = 0; db < 4; ++db) o[db] = zero16();
  float m = -__builtin_inff(), sum = 0.f;
  f32x16 s[kSubs];

  // Tiles of 64 keys from head_lo on: T whole ones, then the edge tiles, the last ending at q_end.
  const int T = (q0 - head_lo) / kKeys, total = (q_end - head_lo + kKeys - 1) / kKeys;
  const auto key0_of = [&](int j) { return head_lo + j * kKeys; };
  const auto score = [&](int tile) {
    bf16x8 k0[kSubs];
#pragma unroll
    for (int sub = 0; sub < kSubs; ++sub) k0[sub] = at.key(tile, 0, sub);
    score_tile(tile, qf, at, s, k0);
  };
  // The reference of the rows that need it goes up to their maximum, and o and sum with it; P anew.  A row's result is its own
  // whatever its neighbours hold.  (A row without a reference has gathered nothing of its own: o may be NaN.)
  const auto raise_to_max = [&](bool raise, Probs& p) {
    const float top = half_max(raise ? 1.f : 0.f) > 0.f ? vmax(m, tile_max(s)) : m;
    const bool fresh = m == -__builtin_inff();
    const float alpha = fresh ? 0.f : fast_exp2((m - top) * a.c);
    sum *= alpha;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] = fresh ? 0.f : o[db][i] * alpha;
    m = top;
    return form_tile(s, a.c, top == -__builtin_inff() ? 0.f : top * a.c, p);
  };
  K.fetch(key0_of(0), kst(0), w);
  if (total > 1) K.fetch(key0_of(1), kst(1), w);
  if (T == 0) {
    V.fetch(key0_of(0), vst(0), w);
    if (total > 1) V.fetch(key0_of(1), vst(1), w);
  }
  // (only the first tile's keys are needed yet)
  if (T > 0) wait_but<kLoads>();
  else if (total > 1) wait_but<3 * kLoads>();
  else wait_but<kLoads>();
  __syncthreads();
  score(kst(0));
  if (T > 0) {
    // Step j: K(j+1) and V(j-1) have landed; K(j+2) and V(j) go into the stages that step j-1 has done with.  P(j) is formed from
    // the scores in registers, against the standing reference, beside V(j-1) P(j-1); then the scores of j+1.
    const auto step = [&](int j, auto parity, auto first, const Probs& pp, Probs& pn) {
      constexpr int P = decltype(parity)::value;
      wait_dma();
      __syncthreads();
      if (j + 2 < total) K.fetch(key0_of(j + 2), kst(P), w);
      V.fetch(key0_of(j), vst(P), w);
      bf16x8 k0[kSubs];
#pragma unroll
      for (int sub = 0; sub < kSubs; ++sub) k0[sub] = at.key(kst(1 - P), 0, sub);
      __builtin_amdgcn_s_setprio(1);
      const float mc = m == -__builtin_inff() ? 0.f : m * a.c;
      float ts;
      if constexpr (decltype(first)::value) {
        ts = raise_to_max(true, pn);
      } else {
        ts = form_beside_values(s, a.c, mc, pn, vst(1 - P), at, pp, o);
#pragma unroll
        for (int sub = 0; sub < kSubs; ++sub) asm volatile("" ::"v"(pn[sub][0]), "v"(pn[sub][1]));
        asm volatile("" ::"v"(ts));
        const bool raise = !(ts <= kSumLimit) || m == -__builtin_inff();
        if (__ballot(raise)) ts = raise_to_max(raise, pn);
      }
      sum += ts;
      __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int sub = 0; sub < kSubs; ++sub) asm volatile("" ::"v"(k0[sub]));
      __builtin_amdgcn_iglp_opt(0);
      score_tile(kst(1 - P), qf, at, s, k0);
    };
    using Even = std::integral_constant<int, 0>;
    using Odd = std::integral_constant<int, 1>;
    Probs pa, pz;
    step(0, Even{}, std::true_type{}, pz, pa);
    int j = 1;
    for (; j + 1 < T; j += 2) {
      step(j, Odd{}, std::false_type{}, pa, pz);
      step(j + 1, Even{}, std::false_type{}, pz, pa);
    }
    // the last whole tile's V meets its P while the first edge tile's is under way (its K has been scored)
    if (j < T) {
      step(j, Odd{}, std::false_type{}, pa, pz);
      wait_dma();
      __syncthreads();
      V.fetch(key0_of(T), vst(0), w);
      add_values(vst(1), at, pz, o);
      __syncthreads();
      if (T + 1 < total) V.fetch(key0_of(T + 1), vst(1), w);
    } else {
      wait_dma();
      __syncthreads();
      V.fetch(key0_of(T), vst(1), w);
      add_values(vst(0), at, pa, o);
      __syncthreads();
      if (T + 1 < total) V.fetch(key0_of(T + 1), vst(0), w);
    }
    if (lo != head_lo) {  // a row of another sequence starts anew
      m = -__builtin_inff();
      sum = 0.f;
    }
  }
  int odd = 0;  // an edge tile of V was not all finite
  // Edge tile j: its scores are in registers and V(j) and K(j+1) under way (of the first one V(j+1), too).
  for (int j = T; j < total; ++j) {
    const int key0 = key0_of(j), P = j & 1;
    const bool seen = __ballot(covered && lo < key0 + kKeys && row >= key0) != 0;  // by a row of this wave
    Probs p;
    if (seen) {
#pragma unroll
      for (int sub = 0; sub < kSubs; ++sub)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = key_of(key0, sub, i, l);
          if (key < lo || key > row) s[sub][i] = -__builtin_inff();
        }
      float ts;
      if (j == 0) {
        ts = raise_to_max(true, p);
      } else {
        ts = form_tile(s, a.c, m == -__builtin_inff() ? 0.f : m * a.c, p);
        const bool raise = !(ts <= kSumLimit) || m == -__builtin_inff();
        if (__ballot(raise)) ts = raise_to_max(raise, p);
      }
      sum += ts;
    }
    if (j == T && j + 1 < total) wait_but<kLoads>();
    else wait_dma();
    if (!only_finite(vst(P), w, l)) odd = 1;
    if (l == 0) odd_wave[w] = odd;
    __syncthreads();  // V(j) and K(j+1) are there, the stages of K(j) and V(j-1) free
    if (j + 2 < total) K.fetch(key0_of(j + 2), kst(P), w);
    if (j > T && j + 1 < total) V.fetch(key0_of(j + 1), vst(1 - P), w);
    if (seen) add_values(vst(P), at, p, o);
    if (j + 1 < total && __ballot(covered && lo < key0 + 2 * kKeys && row >= key0 + kKeys) != 0) score(kst(1 - P));
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
  if (uniform(odd_wave[0] | odd_wave[1] | odd_wave[2] | odd_wave[3]) != 0)  // written before the last tile's barrier
    add_infinities(a, head, key0_of(T), q0 + 32 * w, lo, covered, l);
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
