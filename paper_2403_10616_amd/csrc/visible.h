// What a position sees under a sliding window with sinks, and which document a row of a ragged batch belongs to.
//
// Position i sees position j where j <= i and (j > i - window or j < sinks): the last `window` positions, itself included, and the
// first `sinks`.  As a list without gaps: the sinks in front of the window, then the window.
#pragma once
#include "common.h"

namespace dipaco {

struct Window {
  int window, sinks;   // window >= 1, sinks >= 0
  __host__ __device__ __forceinline__ int near_from(int i) const { return i >= window ? i - window + 1 : 0; }   // first position of i's window
};
// the positions that i sees, in order
struct VisibleList {
  int front, near, count;
  __device__ __forceinline__ VisibleList(const Window& w, int i) : near(w.near_from(i)) {
    front = min(w.sinks, near);
    count = front + i + 1 - near;
  }
  __device__ __forceinline__ int at(int t) const { return t < front ? t : near + t - front; }
};

// rows of document b in a padded batch of documents of S rows (lengths: null, or one per document)
__device__ __forceinline__ int document_rows(const int* lengths, int b, int S) { return lengths ? min(max(lengths[b], 0), S) : S; }

// Rows of a ragged batch: row_start[b] .. row_start[b + 1] - 1 are document b's.  Values outside [0, T] are taken as the nearest inside.
struct RowRange { int first, count; };
__device__ __forceinline__ RowRange ragged_rows(const int* row_start, int b, int T) {
  const int lo = min(max(row_start[b], 0), T), hi = min(max(row_start[b + 1], 0), T);
  return {lo, max(hi - lo, 0)};
}
// The last b in [0, B) with row_start[b] <= row: the document of `row` (it may hold fewer rows; the caller checks), for a whole wave, 64
// ways a step: two dependent loads up to 4096 documents, where halving takes twelve.
__device__ __forceinline__ int find_document(const int* row_start, int B, int row, int lane) {
  int lo = 0, n = B;   // the answer lies in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 63) / 64, at = lo + lane * step;
    const bool before = lane * step < n && row_start[at] <= row;
    const unsigned long long m = __builtin_amdgcn_ballot_w64(before);
    const int k = m ? 63 - __builtin_clzll(m) : 0;
    lo += k * step;
    n = min(step, n - k * step);
    if (step == 1) break;
  }
  return lo;
}

}  // namespace dipaco
