// Internal interface of the operators on packed rows: sizes and launches shared by their C ABI layer (packed_api.cpp) and their
// kernels (rope.hip, packed_attn.hip).
#pragma once

#include "cache_internal.h"

namespace crisp {

struct PackedDims {
  int n_seqs, n_rows, hq, hkv;
};

constexpr int kRopePairs = kHeadDim / 2;
struct RopeTable {
  int dim;           // rotated elements of a head, a multiple of 16
  bool interleaved;  // pairs (2 i, 2 i + 1), not (i, i + dim / 2)
  float gain;
  double turns[kRopePairs];  // a token, of each pair
};

// One tensor of a rotation: heads rows of `in` to `out` (in place: the same address and strides).
struct RopeTensor {
  const uint16_t* in;
  uint16_t* out;
  Strides is, os;
  int heads;
};
hipError_t launch_rope(const PackedDims& d, const RopeTable& t, const int32_t* start, const int32_t* row_ptr,
                       const RopeTensor& q, const RopeTensor& k, hipStream_t stream);

hipError_t launch_packed_attn(const PackedDims& d, float scale, const int32_t* row_ptr, const uint16_t* q, Strides qs,
                              const uint16_t* k, Strides ks, const uint16_t* v, Strides vs, uint16_t* o, Strides os,
                              hipStream_t stream);

}  // namespace crisp
