// The sequences of a batch of new tokens (base_kv_batch): which one a row is of.
#pragma once

#include "common.hpp"
#include "internal.hpp"

namespace basek {

// The sequence of row t (uniform over the wavefront): the last s with q_start[s] <= t,
// -1 where there is none or t lies behind the last sequence.  64 starts at a time, in
// as many levels as the number of sequences has digits to the base 64.
__device__ __forceinline__ int seq_of_row(const KvBatch &b, int t) {
  const int lane = lane_id();
  int lo = 0, n = b.n_seq + 1;   // q_start's entries lo .. lo + n - 1 are left
  while (true) {
    const int step = (n + WAVE - 1) / WAVE;
    const int i = lane * step;
    const bool le = i < n && b.q_start[lo + i] <= t;
    const int hits = __popcll(__ballot(le));
    if (hits == 0) return -1;
    lo += (hits - 1) * step;
    if (step == 1) break;
    n = min(step, b.n_seq + 1 - lo);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  return lo < b.n_seq ? lo : -1;
}

}  // namespace basek
