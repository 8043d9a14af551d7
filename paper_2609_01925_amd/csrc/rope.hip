// Rotary positions on packed rows of q and k.
//
// A pair (x1, x2) of a row at position p is turned by the angle 2 pi p turns: y1 = g (x1 cos - x2 sin), y2 = g (x2 cos + x1 sin).
// The turns of a far position are many and only their fraction counts, so p turns is formed and reduced in 64 bits (off by
// 2^-53 of itself: 2^-24 of a turn at position 2^30 of the fastest pair, turns = 1 / (2 pi)); sine and cosine of the fraction
// and the products are 32 bits, and each result is rounded to bf16 once.
//
// Bound by HBM, each element read and written once: 32768 rows of 40 heads (336 MB each way) 138 us, 4.9 TB/s; 24 prompts of 1 to 700 rows of
// 32 heads (82 MB each way) 33 us, 5.0 TB/s; one row of each of 64 sequences 5.1 us, a launch and three loads in turn (begins,
// elements, stores).  Non-temporal loads 134 and 44 us; the next heads' loads before this one's stores 144 to 155.
#include "packed_device.h"
#include "packed_internal.h"

namespace crisp {

namespace {

constexpr int kThreads = 256;
constexpr int kRowLanes = 8;                      // lanes of a row: 16 elements, 8 pairs each
constexpr int kRowsPerWave = kWave / kRowLanes;
constexpr int kRowsPerWg = kThreads / kRowLanes;
constexpr int kAhead = 4;                         // heads whose elements are loaded together (8: 141, 35 and 6.2 us)

struct RopeArgs {
  PackedDims d;
  RopeTable t;
  const int32_t* start;
  const int32_t* row_ptr;
  RopeTensor x[2];
  int heads;  // of a workgroup
  bool in_place[2];
};

__device__ __forceinline__ float lo_f32(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float hi_f32(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
__device__ __forceinline__ uint32_t pair_bits(float a, float b) { return __builtin_bit_cast(uint32_t, pack_bf16(a, b)); }

// Eight lanes hold a row: lane c pairs 8 c .. 8 c + 7, in two chunks of eight elements, and goes over the workgroup's heads with one
// set of sines and cosines.  Lanes past rotary_dim / 16 copy the elements that are not rotated.
__global__ __launch_bounds__(kThreads) void rope(RopeArgs a) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int row0 = (int)blockIdx.x * kRowsPerWg + w * kRowsPerWave, row = row0 + (lane >> 3), c = lane & 7;
  if (row0 >= a.d.n_rows) return;
  // The row's sequence, the last that begins at or before it.  Up to 64 sequences their begins and positions come from one round of
  // loads, a sequence a lane; of more, the wave's first row's is looked for, then those that begin among its eight.
  const int end = a.row_ptr[a.d.n_seqs];
  int seq, begin, start;
  if (a.d.n_seqs <= kWave) {
    const int last = a.d.n_seqs - 1, mine = a.row_ptr[min(lane, last)], first = a.start[min(lane, last)];
    seq = -1;
#pragma unroll
    for (int i = 0; i < kRowsPerWave; ++i) {
      const int n = __popcll(__ballot(lane <= last && mine <= row0 + i));
      if (i == (lane >> 3)) seq += n;
    }
    begin = __shfl(mine, max(seq, 0));
    start = __shfl(first, max(seq, 0));
  } else {
    const int s0 = seq_of_row(a.row_ptr, a.d.n_seqs, row0);
    seq = s0;
    for (int from = s0 + 1; from <= a.d.n_seqs; from += kWave) {
      const int i = from + lane;
      const int b = i <= a.d.n_seqs ? a.row_ptr[i] : 0x7fffffff;
      unsigned long long last = 0;
#pragma unroll
      for (int x = 0; x < kRowsPerWave; ++x) {
        last = __ballot(b <= row0 + x);
        if (x == (lane >> 3)) seq += __popcll(last);
      }
      if (~last != 0) break;
    }
    const int s = min(max(seq, 0), a.d.n_seqs - 1);
    begin = a.row_ptr[s];
    start = a.start[s];
  }
  if (row >= min(end, a.d.n_rows) || seq < 0 || seq >= a.d.n_seqs) return;
  const double p = (double)((int64_t)start + row - begin);
  const bool turned = c < a.t.dim / 16;
  float co[8], si[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    co[i] = 1.f;
    si[i] = 0.f;
  }
  if (turned) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double x = p * a.t.turns[8 * c + i];
      float s, k;
      sincospif(2.f * (float)(x - rint(x)), &s, &k);
      co[i] = k * a.t.gain;
      si[i] = s * a.t.gain;
    }
  }
  const bool half = turned && !a.t.interleaved;
  const int at0 = half ? 8 * c : 16 * c, at1 = half ? a.t.dim / 2 + 8 * c : 16 * c + 8;
  const int h0 = (int)blockIdx.y * a.heads, h1 = min(h0 + a.heads, a.x[0].heads + a.x[1].heads);
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const RopeTensor& x = a.x[y];
    const int first = y == 0 ? 0 : a.x[0].heads;
    const int b = max(h0 - first, 0), e = min(h1 - first, x.heads);
    if (!turned && a.in_place[y]) continue;
    const uint16_t* in = x.in + (int64_t)row * x.is.row;
    uint16_t* out = x.out + (int64_t)row * x.os.row;
    for (int h = b; h < e; h += kAhead) {
      u32x4 u[kAhead], v[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const uint16_t* p0 = in + (int64_t)min(h + j, e - 1) * x.is.head;
        u[j] = *reinterpret_cast<const u32x4*>(p0 + at0);
        v[j] = *reinterpret_cast<const u32x4*>(p0 + at1);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (h + j >= e) break;
        u32x4 r, t;
        if (!turned) {
          r = u[j];
          t = v[j];
        } else if (half) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float a0 = lo_f32(u[j][i]), a1 = hi_f32(u[j][i]), b0 = lo_f32(v[j][i]), b1 = hi_f32(v[j][i]);
            r[i] = pair_bits(a0 * co[2 * i] - b0 * si[2 * i], a1 * co[2 * i + 1] - b1 * si[2 * i + 1]);
            t[i] = pair_bits(b0 * co[2 * i] + a0 * si[2 * i], b1 * co[2 * i + 1] + a1 * si[2 * i + 1]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float a0 = lo_f32(u[j][i]), a1 = hi_f32(u[j][i]), b0 = lo_f32(v[j][i]), b1 = hi_f32(v[j][i]);
            r[i] = pair_bits(a0 * co[i] - a1 * si[i], a1 * co[i] + a0 * si[i]);
            t[i] = pair_bits(b0 * co[4 + i] - b1 * si[4 + i], b1 * co[4 + i] + b0 * si[4 + i]);
          }
        }
        uint16_t* q0 = out + (int64_t)(h + j) * x.os.head;
        *reinterpret_cast<u32x4*>(q0 + at0) = r;
        *reinterpret_cast<u32x4*>(q0 + at1) = t;
      }
    }
  }
}

}  // namespace

hipError_t launch_rope(const PackedDims& d, const RopeTable& t, const int32_t* start, const int32_t* row_ptr,
                       const RopeTensor& q, const RopeTensor& k, hipStream_t stream) {
  const auto same = [](const RopeTensor& x) { return x.in == x.out; };
  const int64_t blocks = (d.n_rows + kRowsPerWg - 1) / kRowsPerWg;
  const int heads = q.heads + k.heads;
  // As many heads a workgroup as leave some workgroups for every CU: all heads in one 141, 42 and 12 us, 8192 workgroups 149, 34 and 4.9.
  int64_t groups = (2048 + blocks - 1) / blocks;
  if (groups > (heads + kAhead - 1) / kAhead) groups = (heads + kAhead - 1) / kAhead;
  const int per = (int)((heads + groups - 1) / groups);
  const RopeArgs a{d, t, start, row_ptr, {q, k}, per, {same(q), same(k)}};
  hipLaunchKernelGGL(rope, dim3((unsigned)blocks, (unsigned)((heads + per - 1) / per)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace crisp
