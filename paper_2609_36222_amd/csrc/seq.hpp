// The sequences of a batch of new tokens (base_kv_batch): which one a row is of, and its
// rows and length within their bounds.
#pragma once

#include "common.hpp"
#include "internal.hpp"

namespace basek {

// A sequence's new rows [begin, stop) and its tokens from what the memory holds (two starts
// and a length), the rows within the call's and the tokens within the table's row: the same
// for what writes the cache and what reads it.
struct SeqRows {
  int begin, stop, kv;
};
__device__ __forceinline__ SeqRows seq_rows(int q0, int q1, int len, int rows, int most) {
  SeqRows s;
  s.begin = min(max(q0, 0), rows);
  s.stop = min(max(q1, s.begin), rows);
  s.kv = min(max(len, 0), most);
  return s;
}

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
