// Packed rows of sequences of different lengths: sequence b has rows cu[b] .. cu[b + 1] - 1.
#pragma once

#include "qf_internal.h"

namespace qf {

struct RowOwner {
  int seq;     // -1: a row of no sequence
  int index;   // its place in the sequence
};

// The sequence that row t of `rows` lies in, by a whole wavefront (every lane gets the answer): as cu
// does not decrease, it is the last one that starts at or before t, found 64 starts at a time (of 4,096
// sequences in two rounds: norm, rotation and append of so many requests' single tokens of 48 heads 61 ->
// 27 us).  Values that are out of range or out of order give no sequence or another one, never an index
// outside [0, seqs).  cu == null: one row each.
__device__ __forceinline__ RowOwner row_owner(const int32_t* __restrict__ cu, int32_t seqs,
                                              int32_t rows, int32_t t) {
  if (cu == nullptr) return RowOwner{t < seqs ? t : -1, 0};
  const int lane = threadIdx.x & 63;
  int b = 0, n = seqs;                         // it is among b .. b + n - 1
  while (n > 0) {
    const int step = (n - 1) / 64 + 1;
    const int at = lane * step;                // < n + 64, less than 2^31
    const int before = __popcll(__ballot(at < n && cu[b + at] <= t));
    if (before == 0) return RowOwner{-1, 0};
    b += (before - 1) * step;
    if (step == 1) break;
    n = min(step, n - (before - 1) * step);
  }
  if (n <= 0) return RowOwner{-1, 0};
  const int start = cu[b], end = cu[b + 1];
  if (start < 0 || start > t || end <= t || end > rows) return RowOwner{-1, 0};
  return RowOwner{b, t - start};
}

}  // namespace qf
