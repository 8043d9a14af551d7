// Device-side pieces of the 8-bit paged K/V cache: codes, scales and the order of a tile's bytes.
//
// A tile is 64 tokens of one KV head and tensor, 8192 codes in chunks of 16 bytes, ordered so that
// lane l of a wave takes chunk 64 i + l of load i and holds an operand of v_mfma_f32_16x16x32_bf16
// as it stands (A: lane l holds row l % 16, k = 8 (l / 16) + [0, 8)):
//   K, S^T = K Q^T: chunk (t, half, g, r) = elements 32 g + 16 half + [0, 16) of token
//     16 (r / 4) + 4 t + r % 4.  Row r of score tile t is that token, so the result (row
//     4 g + i in register i of a lane of group g = l / 16) leaves every lane with the scores of
//     its 16 consecutive tokens 16 g + 4 t + i.
//   V, O^T = V^T P^T: chunk (dt, g, r) = element 16 dt + r of tokens 16 g + [0, 16): the tokens
//     that this lane holds probabilities of, so P goes from one product to the other in registers.
#pragma once

#include "cache_internal.h"
#include "crisp_device.h"

namespace crisp {

__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
__device__ __forceinline__ int exp_of(float scale) { return (int)((__float_as_uint(scale) >> 23) & 255) - 127; }

// A page's scale exponent as stored; whatever a page that was never written holds becomes a usable one.
__device__ __forceinline__ int stored_exp(float scale) {
  const int e = exp_of(scale);
  return e < kScaleExpMin ? kScaleExpMin : e > kScaleExpMax ? kScaleExpMax : e;
}

// Smallest e >= kScaleExpMin with amax <= MAX 2^e, from the bits of a finite bf16 amax >= 0:
// MAX = 448 = 1.75 2^8 (e4m3), 127 = 1.984375 2^6 (int8).
template <int FMT>
__device__ __forceinline__ int scale_exp(int bits) {
  const int man = bits & 127, exp = (bits >> 7) - 127;
  const int e = FMT == kCacheE4M3 ? exp - 8 + (man > 96) : exp - 6 + (man > 126);
  return e < kScaleExpMin ? kScaleExpMin : e;
}

// Four floats, already divided by the scale, to four codes: round to nearest even; beyond MAX
// (an infinity) the largest code, NaN 0.
template <int FMT>
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
  constexpr float kMax = FMT == kCacheE4M3 ? 448.f : 127.f;
  const auto in = [](float x) { return x != x ? 0.f : fminf(fmaxf(x, -kMax), kMax); };
  a = in(a), b = in(b), c = in(c), d = in(d);
  if constexpr (FMT == kCacheE4M3) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  } else {
    const auto i = [](float x) { return (uint32_t)(int)__builtin_rintf(x) & 255u; };
    return i(a) | i(b) << 8 | i(c) << 16 | i(d) << 24;
  }
}

// Four finite bf16 (two a dword), |x| <= MAX 2^e, to four codes of scale 2^e, rounded to nearest even.
// e4m3: the conversion divides by the scale.  int8: x 2^-e + 128 is exact in 32 bits wherever its
// rounding is in question (x has eight significant bits), and the conversion to a byte rounds to even.
template <int FMT>
__device__ __forceinline__ uint32_t finite_codes(uint32_t x, uint32_t y, int e) {
  if constexpr (FMT == kCacheE4M3) {
    typedef __attribute__((__vector_size__(2 * sizeof(short)))) short i16x2;
    i16x2 r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, x), pow2f(e), false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, y), pow2f(e), true);
    return __builtin_bit_cast(uint32_t, r);
  } else {
    const float inv = pow2f(-e);
    const auto f = [&](uint32_t bits) { return __builtin_fmaf(__uint_as_float(bits), inv, 128.f); };
    uint32_t r = __builtin_amdgcn_cvt_pk_u8_f32(f(x << 16), 0, 0);
    r = __builtin_amdgcn_cvt_pk_u8_f32(f(x & 0xffff0000u), 1, r);
    r = __builtin_amdgcn_cvt_pk_u8_f32(f(y << 16), 2, r);
    r = __builtin_amdgcn_cvt_pk_u8_f32(f(y & 0xffff0000u), 3, r);
    return r ^ 0x80808080u;
  }
}

// Bytes of four dwords transposed: out[j] = byte j of r0, r1, r2, r3.
__device__ __forceinline__ void transpose4(uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3, uint32_t (&out)[4]) {
  const uint32_t t0 = __builtin_amdgcn_perm(r1, r0, 0x05010400u), t1 = __builtin_amdgcn_perm(r1, r0, 0x07030602u);
  const uint32_t u0 = __builtin_amdgcn_perm(r3, r2, 0x05010400u), u1 = __builtin_amdgcn_perm(r3, r2, 0x07030602u);
  out[0] = __builtin_amdgcn_perm(u0, t0, 0x05040100u);
  out[1] = __builtin_amdgcn_perm(u0, t0, 0x07060302u);
  out[2] = __builtin_amdgcn_perm(u1, t1, 0x05040100u);
  out[3] = __builtin_amdgcn_perm(u1, t1, 0x07060302u);
}

typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;

// Four codes to floats.
template <int FMT>
__device__ __forceinline__ f32x4 from_codes(uint32_t x) {
  if constexpr (FMT == kCacheE4M3) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
    return f32x4{lo[0], lo[1], hi[0], hi[1]};
  } else {
    return f32x4{(float)(int8_t)x, (float)(int8_t)(x >> 8), (float)(int8_t)(x >> 16), (float)(int8_t)(x >> 24)};
  }
}

// Four codes with NaN (e4m3: all of the lower seven bits set) made 0.
template <int FMT>
__device__ __forceinline__ uint32_t without_nan(uint32_t x) {
  if constexpr (FMT != kCacheE4M3) return x;
  const uint32_t nan = (((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
  return x & ~(nan * 255u);
}

// Eight codes to bf16, which holds every code exactly.
template <int FMT>
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t lo, uint32_t hi) {
  if constexpr (FMT == kCacheE4M3) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  } else {
    // the upper halves of the floats, whose lower halves are 0
    const f32x4 a = from_codes<FMT>(lo), b = from_codes<FMT>(hi);
    const auto pair = [](float x, float y) { return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u); };
    const u32x4 r = {pair(a[0], a[1]), pair(a[2], a[3]), pair(b[0], b[1]), pair(b[2], b[3])};
    return __builtin_bit_cast(bf16x8, r);
  }
}

// A sequence's part of the call: tokens held before it, its first row and its rows; arguments
// out of range are brought into it, so that no value of theirs leads out of a buffer.
struct SeqRows {
  int len, row0, n;
};
__device__ __forceinline__ SeqRows seq_rows(const Seqs& s, const BatchDims& b, int B, int i) {
  const int cap = b.max_pages * B;
  SeqRows r;
  r.len = min(max(s.seq_len[i], 0), cap);
  r.row0 = min(max(s.row_ptr[i], 0), b.n_rows);
  r.n = min(max(s.row_ptr[i + 1], r.row0), b.n_rows) - r.row0;
  return r;
}

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t shifted(uint32_t x) {  // lanes that the move does not reach get 0
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, true);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int shifted(int x) {
  return (int)shifted<CTRL, ROWS>((uint32_t)x);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t shifted(int64_t x) {
  return (int64_t)((uint64_t)shifted<CTRL, ROWS>((uint32_t)((uint64_t)x >> 32)) << 32 | shifted<CTRL, ROWS>((uint32_t)x));
}

// Inclusive sum over the wave in lane order, by register moves: within rows of 16 lanes, then
// the last lane of a row into the next.
template <typename T>
__device__ __forceinline__ T wave_scan(T x) {
  x += shifted<0x111, 0xf>(x);
  x += shifted<0x112, 0xf>(x);
  x += shifted<0x114, 0xf>(x);
  x += shifted<0x118, 0xf>(x);
  x += shifted<0x142, 0xa>(x);
  x += shifted<0x143, 0xc>(x);
  return x;
}

// Inclusive sum over the workgroup in thread order; lds: one value a wave.  Every thread also
// gets the whole sum.  Ends with the waves' values still in lds: a barrier before the next use.
template <typename T, int kWaves>
__device__ __forceinline__ T block_scan(T x, T* lds, T* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  x = wave_scan(x);
  if (lane == 63) lds[w] = x;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    const T v = lds[i];
    if (i < w) before += v;
    all += v;
  }
  *total = all;
  return x + before;
}

#if defined(__HIP_DEVICE_COMPILE__)
// Waits until at most the last four vector memory operations of this wave are under way (vmcnt(4)).
__device__ __forceinline__ void wait_dma_but4() { __builtin_amdgcn_s_waitcnt(4 | (7 << 4) | (15 << 8)); }
#endif

}  // namespace crisp
