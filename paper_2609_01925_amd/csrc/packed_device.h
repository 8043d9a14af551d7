// Device-side look-up of packed rows: which sequence a row belongs to.
#pragma once

#include "cache_device.h"

namespace crisp {

// The last sequence that begins at or before `row`, the same on every lane; -1 if the first begins behind it, n_seqs if the row
// lies behind the last one's end.  64 candidates a round, one a lane: 1 round up to 63 sequences, 2 up to 4095.  (row_ptr that
// does not ascend leads to some value in that range.)
__device__ __forceinline__ int seq_of_row(const int32_t* row_ptr, int n_seqs, int row) {
  int base = 0;
  for (int n = n_seqs + 1; n > 1;) {
    const int step = (n + kWave - 1) / kWave, probe = lane_id() * step;
    const unsigned long long ok = __ballot(probe < n && row_ptr[base + (probe < n ? probe : n - 1)] <= row);
    const int k = __popcll(ok) - 1;
    if (k < 0) return -1;
    base += k * step;
    n = step < n - k * step ? step : n - k * step;
  }
  return base;
}

}  // namespace crisp
