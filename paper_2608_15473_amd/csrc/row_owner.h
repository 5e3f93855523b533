// Packed rows of sequences of different lengths: sequence b has rows cu[b] .. cu[b + 1] - 1.
#pragma once

#include "qf_internal.h"

namespace qf {

struct RowOwner {
  int seq;     // -1: a row of no sequence
  int index;   // its place in the sequence
};

// The sequence that row t of `rows` lies in, by a whole wavefront (every lane gets the answer): as cu
// does not decrease, it is the last one that starts at or before t.  Values that are out of range or
// out of order give no sequence or another one, never an index outside [0, seqs).  cu == null: one row
// each.
__device__ __forceinline__ RowOwner row_owner(const int32_t* __restrict__ cu, int32_t seqs,
                                              int32_t rows, int32_t t) {
  if (cu == nullptr) return RowOwner{t < seqs ? t : -1, 0};
  const int lane = threadIdx.x & 63;
  int before = 0;                              // starts at or before t
  for (int i0 = 0; i0 < seqs; i0 += 64) {
    const int i = i0 + lane;
    before += __popcll(__ballot(i < seqs && cu[i] <= t));
  }
  const int b = before - 1;
  if (b < 0) return RowOwner{-1, 0};
  const int start = cu[b], end = cu[b + 1];
  if (start < 0 || start > t || end <= t || end > rows) return RowOwner{-1, 0};
  return RowOwner{b, t - start};
}

}  // namespace qf
