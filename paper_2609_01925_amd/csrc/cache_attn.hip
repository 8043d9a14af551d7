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

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kMinShare = 4;  // tiles a workgroup takes at least: one a wave

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
  float c2;     // scale log2(e)
  float* part;  // [2 gridDim.x][16 C][128 + 2]
};

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float acc4;

__device__ __forceinline__ acc4 mfma16(bf16x8 a, bf16x8 b, acc4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Keeps a loaded chunk in its four registers up to here: left to itself the compiler splits what
// the loop carries into single codes, a register each.
__device__ __forceinline__ void keep_whole(u32x4& x) { asm volatile("" : "+v"(x)); }

// The value of all four lanes that hold a column (lanes l, l ^ 16, l ^ 32, l ^ 48) combined.
template <typename Op>
__device__ __forceinline__ float column(float x, Op op) {
  const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = op(__uint_as_float(h[0]), __uint_as_float(h[1]));
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// What a sequence's units are: nrt groups of 16 C rows for each KV head, each over T tiles (one at
// least, so that rows that see nothing are written too).
template <int C>
struct SeqWork {
  SeqRows r;
  int T, nrt;
  int64_t tiles;
  __device__ __forceinline__ SeqWork() {}
  __device__ __forceinline__ SeqWork(const AttnArgs& a, int s) {
    r = seq_rows(a.s, a.b, a.c.B, s);
    const int end = min(r.len + r.n, a.b.max_pages * a.c.B);
    T = max((end + kTile - 1) / kTile, 1);
    nrt = (int)(((int64_t)r.n * a.G + 16 * C - 1) / (16 * C));
    tiles = (int64_t)a.c.hkv * nrt * T;
  }
};

// All sequences' tiles in a row, cut into equal shares: total, share, and the sequence that holds
// tile `pos` with the number of tiles before it.
struct Place {
  int64_t total, share, base;
  int seq;
};

template <int C>
__device__ __forceinline__ void count_tiles(const AttnArgs& a, int workgroups, int64_t* lds, Place* p, int64_t* end,
                                            int64_t* own) {
  const int per = (a.b.n_seqs + kThreads - 1) / kThreads;
  int64_t sum = 0;
  for (int i = 0; i < per; ++i) {
    const int s = (int)threadIdx.x * per + i;
    if (s < a.b.n_seqs) sum += SeqWork<C>(a, s).tiles;
  }
  *own = sum;
  *end = block_scan<int64_t, kWaves>(sum, lds, &p->total);
  p->share = max((p->total + workgroups - 1) / workgroups, (int64_t)kMinShare);
}

template <int C>
__device__ __forceinline__ void find_tile(const AttnArgs& a, int64_t pos, int64_t end, int64_t own, int64_t* lds, Place* p) {
  if (pos >= end - own && pos < end) {
    const int per = (a.b.n_seqs + kThreads - 1) / kThreads;
    int64_t base = end - own;
    int s = (int)threadIdx.x * per;
    for (int64_t t; (t = SeqWork<C>(a, s).tiles) + base <= pos; ++s) base += t;  // ends: pos < end
    lds[kWaves] = base;
    lds[kWaves + 1] = s;
  }
  __syncthreads();
  p->base = lds[kWaves];
  p->seq = (int)lds[kWaves + 1];
}

// One workgroup's share.  Tiles of a unit go round the four waves; each wave keeps its own running
// maximum, sum and output, joined through LDS at the unit's end.  A lane's 16-byte loads are
// matrix operands as they stand (cache_device.h): K of the next tile is loaded while the softmax
// and PV of this one run, V while the next scores are made, nothing passes through LDS.
template <int FMT, int C>
__global__ __launch_bounds__(kThreads, C == 4 ? 1 : 2) void cache_attn(AttnArgs a) {
  constexpr int kRows = 16 * C;
  __shared__ __attribute__((aligned(16))) float xo[2][C][8][kWave][4];
  __shared__ float xm[kWaves][kRows], xl[kWaves][kRows];
  __shared__ int64_t lds[kWaves + 2];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int wgs = gridDim.x;
  // workgroup i runs on XCD i % 8: neighbouring shares go to one XCD, whose L2 then serves the row
  // groups that read the same keys
  const int wg = wgs % kNumXcd == 0 ? (int)blockIdx.x % kNumXcd * (wgs / kNumXcd) + (int)blockIdx.x / kNumXcd : (int)blockIdx.x;
  Place pl;
  int64_t end, own;
  count_tiles<C>(a, wgs, lds, &pl, &end, &own);
  int64_t pos = wg * pl.share;
  const int64_t stop = min(pos + pl.share, pl.total);
  if (pos >= stop) return;
  find_tile<C>(a, pos, end, own, lds, &pl);
  int s = pl.seq;
  int64_t base = pl.base;
  SeqWork<C> sw(a, s);
  while (pos < stop) {
    while (pos >= base + sw.tiles) {
      base += sw.tiles;
      sw = SeqWork<C>(a, ++s);
    }
    const int64_t off = pos - base;
    const int unit = (int)(off / sw.T), u0 = (int)(off % sw.T);
    const int rt = unit % sw.nrt, head = unit / sw.nrt;
    const int take = (int)min((int64_t)(sw.T - u0), stop - pos);
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
    const int see_last = sw.r.len + (min(rt * kRows + kRows, rows) - 1) / a.G;
    acc4 O[C][8];
    float M[C], L[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      M[c] = -__builtin_inff();
      L[c] = 0.f;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) O[c][dt] = acc4{0.f, 0.f, 0.f, 0.f};
    }
    const int t_end = min(u0 + take, see_last / kTile + 1);
    const int32_t* row = a.s.table + (int64_t)s * a.b.max_pages;
    // this wave's next tile from t on whose page is mapped, and the page; t_end if there is none
    const auto mapped = [&](int& t) {
      for (; t < t_end; t += kWaves) {
        const int slot = t / a.c.tiles;
        const int p = __builtin_amdgcn_readfirstlane(slot < a.b.max_pages ? row[slot] : -1);
        if (p >= 0 && p < a.c.n_pages) return p;
      }
      return -1;
    };
    const auto load = [&](u32x4* x, int t, int p, int tensor) {
      const uint8_t* src = a.pages + (((int64_t)p * a.c.hkv + head) * a.c.tiles + t % a.c.tiles) * (2 * kTileBytes) +
                           tensor * kTileBytes + lane * kChunk;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const u32x4*>(src + i * (kWave * kChunk));
    };
    u32x4 K[8], V[8];
    int t = u0 + w;
    int page = mapped(t);
    if (page >= 0) {
      load(K, t, page, 0);
      load(V, t, page, 1);
    }
    while (page >= 0) {
      int t_next = t + kWaves;
      const int next = mapped(t_next);
      const float* sc = a.scales + ((int64_t)page * a.c.hkv + head) * 2;
      const float kc = pow2f(stored_exp(sc[0])) * a.c2;
      const int ev = stored_exp(sc[1]);
      acc4 S[C][4];
#pragma unroll
      for (int ti = 0; ti < 4; ++ti) {
#pragma unroll
        for (int c = 0; c < C; ++c) S[c][ti] = acc4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (j % 2 == 0) keep_whole(K[2 * ti + j / 2]);
          const u32x4 x = K[2 * ti + j / 2];
          const bf16x8 k = codes_to_bf16<FMT>(x[2 * (j & 1)], x[2 * (j & 1) + 1]);
#pragma unroll
          for (int c = 0; c < C; ++c) S[c][ti] = mfma16(k, Q[c][j], S[c][ti]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (next >= 0) load(K, t_next, next, 0);
      const int key0 = t * kTile + 16 * g;
      if (t * kTile + kTile - 1 > see_first) {  // some column does not see the whole tile
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
      const float inv_v = pow2f(-ev);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float mx = S[c][0][0];
#pragma unroll
        for (int ti = 0; ti < 4; ++ti)
#pragma unroll
          for (int i = 0; i < 4; ++i) mx = fmaxf(mx, S[c][ti][i]);
        mx = column(mx, [](float x, float y) { return fmaxf(x, y); }) * kc;
        const float m = fmaxf(M[c], mx);
        const float ms = m == -__builtin_inff() ? 0.f : m;  // no key yet
        if (__ballot(m != M[c])) {
          const float f = fast_exp2(M[c] - ms);
          L[c] *= f;
#pragma unroll
          for (int dt = 0; dt < 8; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) O[c][dt][i] *= f;
          M[c] = m;
        }
        // P is made as 2^ev p, what V's codes are to be multiplied by; its sum is taken back to p's
        const float sub = ms - (float)ev;
        float sum = 0.f;
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          float p[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            p[e] = fast_exp2(__builtin_fmaf(S[c][2 * st + e / 4][e & 3], kc, -sub));
            sum += p[e];
          }
          const bf16x2 x = pack_bf16(p[0], p[1]), y = pack_bf16(p[2], p[3]), z = pack_bf16(p[4], p[5]), v = pack_bf16(p[6], p[7]);
          P[c][st] = bf16x8{x[0], x[1], y[0], y[1], z[0], z[1], v[0], v[1]};
        }
        L[c] = __builtin_fmaf(sum, inv_v, L[c]);
      }
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) {
        keep_whole(V[dt]);
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          const bf16x8 v = codes_to_bf16<FMT>(V[dt][2 * st], V[dt][2 * st + 1]);
#pragma unroll
          for (int c = 0; c < C; ++c) O[c][dt] = mfma16(v, P[c][st], O[c][dt]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (next >= 0) load(V, t_next, next, 1);
      page = next;
      t = t_next;
    }
    // join the waves: the common maximum, then outputs 2, 3 into 0, 1 and 1 into 0
    float Lt[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      Lt[c] = column(L[c], [](float x, float y) { return x + y; });
      if (g == 0) {
        xm[w][16 * c + col] = M[c];
        xl[w][16 * c + col] = Lt[c];
      }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float m = -__builtin_inff();
#pragma unroll
      for (int i = 0; i < kWaves; ++i) m = fmaxf(m, xm[i][16 * c + col]);
      const float ms = m == -__builtin_inff() ? 0.f : m;
      float l = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) l += xl[i][16 * c + col] * fast_exp2(xm[i][16 * c + col] - ms);
      const float f = fast_exp2(M[c] - ms);
#pragma unroll
      for (int dt = 0; dt < 8; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) O[c][dt][i] *= f;
      M[c] = m;
      Lt[c] = l;
    }
#pragma unroll
    for (int half = 2; half >= 1; half /= 2) {
      if (w >= half && w < 2 * half)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<acc4*>(xo[w - half][c][dt][lane]) = O[c][dt];
      __syncthreads();
      if (w < half)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int dt = 0; dt < 8; ++dt) O[c][dt] += *reinterpret_cast<const acc4*>(xo[w][c][dt][lane]);
      __syncthreads();
    }
    if (w == 0) {
      const bool whole = take == sw.T;
      float* part = a.part + (int64_t)(2 * wg + (u0 == 0)) * (kRows * (kHeadDim + 2));
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int r = rt * kRows + 16 * c + col;
        if (r >= rows) continue;
        if (whole) {
          const float f = Lt[c] > 0.f ? 1.f / Lt[c] : 0.f;
          const int i = r / a.G;
          uint16_t* dst = a.o + (head * a.G + (r - i * a.G)) * a.os.head + (sw.r.row0 + i) * a.os.row + 4 * g;
#pragma unroll
          for (int dt = 0; dt < 8; ++dt) {
            const bf16x2 x = pack_bf16(O[c][dt][0] * f, O[c][dt][1] * f), y = pack_bf16(O[c][dt][2] * f, O[c][dt][3] * f);
            *reinterpret_cast<bf16x4*>(dst + 16 * dt) = bf16x4{x[0], x[1], y[0], y[1]};
          }
        } else {
          float* dst = part + (16 * c + col) * kHeadDim + 4 * g;
#pragma unroll
          for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<acc4*>(dst + 16 * dt) = O[c][dt];
          if (g == 0) {
            part[kRows * kHeadDim + 16 * c + col] = M[c];
            part[kRows * kHeadDim + kRows + 16 * c + col] = Lt[c];
          }
        }
      }
    }
    pos += take;
  }
}

// Joins the pieces of the units that share boundaries cut.  Workgroup b stands at the boundary between
// shares b and b + 1; the boundaries inside one unit take its rows in turn.  A piece that begins
// its unit lies in the second slot of its workgroup, any other in the first.
template <int C>
__global__ __launch_bounds__(kThreads) void cache_attn_join(AttnArgs a, int wgs) {
  constexpr int kRows = 16 * C;
  constexpr int64_t kSlot = kRows * (kHeadDim + 2);
  __shared__ int64_t lds[kWaves + 2];
  __shared__ float red[kWaves], acc[8][kHeadDim], sum[8];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  Place pl;
  int64_t end, own;
  count_tiles<C>(a, wgs, lds, &pl, &end, &own);
  const int64_t pos = ((int64_t)blockIdx.x + 1) * pl.share;
  if (pos >= pl.total) return;
  find_tile<C>(a, pos, end, own, lds, &pl);
  const SeqWork<C> sw(a, pl.seq);
  const int64_t off = pos - pl.base;
  const int64_t u0 = pl.base + off / sw.T * sw.T;  // the unit's first tile
  if (u0 == pos) return;                            // not cut here
  const int unit = (int)(off / sw.T), rt = unit % sw.nrt, head = unit / sw.nrt;
  const int first = (int)(u0 / pl.share), last = (int)((u0 + sw.T - 1) / pl.share);
  const int cuts = last - first, mine = (int)blockIdx.x - first;  // boundaries first .. last - 1 lie inside
  const int rows = min(sw.r.n * a.G - rt * kRows, kRows);
  const auto slot = [&](int p) { return a.part + (int64_t)(2 * (first + p) + (p == 0)) * kSlot; };
  for (int r = mine; r < rows; r += cuts) {
    float m = -__builtin_inff();
    for (int p = tid; p <= cuts; p += kThreads) m = fmaxf(m, slot(p)[kRows * kHeadDim + r]);
    m = wave_max(m);
    if (lane == 0) red[w] = m;
    __syncthreads();
    m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float ms = m == -__builtin_inff() ? 0.f : m;
    // eight groups of 32 lanes, each every eighth piece, four elements a lane
    const int grp = tid >> 5, d = 4 * (tid & 31);
    float l = 0.f;
    acc4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int p = grp; p <= cuts; p += 8) {
      const float* src = slot(p);
      const float f = fast_exp2(src[kRows * kHeadDim + r] - ms);
      l += f * src[kRows * kHeadDim + kRows + r];
      const acc4 x = *reinterpret_cast<const acc4*>(src + r * kHeadDim + d);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = __builtin_fmaf(f, x[i], o[i]);
    }
    *reinterpret_cast<acc4*>(&acc[grp][d]) = o;
    if ((tid & 31) == 0) sum[grp] = l;
    __syncthreads();
    if (tid < kHeadDim / 2) {
      float x = 0.f, y = 0.f, t = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x += acc[i][2 * tid];
        y += acc[i][2 * tid + 1];
        t += sum[i];
      }
      const float f = t > 0.f ? 1.f / t : 0.f;
      const int rr = rt * kRows + r, i = rr / a.G;
      uint16_t* dst = a.o + (head * a.G + (rr - i * a.G)) * a.os.head + (sw.r.row0 + i) * a.os.row;
      *reinterpret_cast<bf16x2*>(dst + 2 * tid) = pack_bf16(x * f, y * f);
    }
    __syncthreads();
  }
}

template <int FMT, int C>
hipError_t launch(const AttnArgs& a, int wgs, hipStream_t stream) {
  hipLaunchKernelGGL((cache_attn<FMT, C>), dim3(wgs), dim3(kThreads), 0, stream, a);
  if (wgs > 1) hipLaunchKernelGGL((cache_attn_join<C>), dim3(wgs - 1), dim3(kThreads), 0, stream, a, wgs);
  return hipGetLastError();
}

template <int FMT>
hipError_t launch_groups(const AttnArgs& a, const CacheAttnPlan& p, hipStream_t stream) {
  if (p.groups == 1) return launch<FMT, 1>(a, p.workgroups, stream);
  return launch<FMT, 4>(a, p.workgroups, stream);
}

}  // namespace

CacheAttnPlan cache_attn_plan(const CacheDims& c, const BatchDims& b, int hq) {
  CacheAttnPlan p{1, 0, 0};
  if (b.n_seqs == 0 || b.n_rows == 0 || hq == 0) return p;
  const int64_t G = hq / c.hkv;
  const int64_t rows = ((int64_t)b.n_rows + b.n_seqs - 1) / b.n_seqs * G;  // of an average sequence
  p.groups = rows <= 16 ? 1 : 4;
  // tiles that the table has room for, an upper bound of what the lengths say on the device
  const int64_t nrt = (int64_t)b.n_rows * G / (16 * p.groups) + b.n_seqs;
  const int64_t room = (int64_t)b.max_pages * c.tiles;
  const double tiles = (double)nrt * c.hkv * (double)(room > 1 ? room : 1);
  const int most = p.groups == 4 ? 256 : 512;
  int64_t wgs = tiles >= (double)most * kMinShare ? most : ((int64_t)tiles + kMinShare - 1) / kMinShare;
  wgs = (wgs + kNumXcd - 1) / kNumXcd * kNumXcd;
  p.workgroups = (int)wgs;
  p.bytes = (size_t)wgs * 2 * 16 * p.groups * (kHeadDim + 2) * sizeof(float);
  return p;
}

hipError_t launch_cache_attn(const CacheDims& c, const BatchDims& b, const Seqs& s, int hq, float scale,
                             const uint16_t* q, Strides qs, const uint8_t* pages, const float* scales, uint16_t* o,
                             Strides os, void* ws, hipStream_t stream) {
  const CacheAttnPlan p = cache_attn_plan(c, b, hq);
  const AttnArgs a{c, b, s, q, qs, pages, scales, o, os, hq / c.hkv, scale * kLog2e, (float*)ws};
  return c.fmt == kCacheE4M3 ? launch_groups<kCacheE4M3>(a, p, stream) : launch_groups<kCacheInt8>(a, p, stream);
}

}  // namespace crisp
