// Sequences of a packed batch of rows, looked up on the device.  seq_start's contents are the
// caller's and unchecked: every result is clamped to the rows, so that wrong contents give
// wrong sequences and never an access outside them.
#pragma once

#include "attn_ops.h"

namespace mf {

// Rows that belong to a sequence: 0 .. total - 1.
__device__ __forceinline__ int seq_total(const SeqRows& s) {
  return s.start ? min(max(s.start[s.n], 0), s.rows) : s.rows;
}

// Last sequence that starts at or before row (seq_start only).
__device__ __forceinline__ int seq_find(const SeqRows& s, int row) {
  int lo = 0, hi = s.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s.start[mid] <= row) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// First row of row's sequence.
__device__ __forceinline__ int seq_begin(const SeqRows& s, int row) {
  if (!s.start) return row - row % s.len;
  return min(max(s.start[seq_find(s, row)], 0), row);
}

// The row behind the last one of row's sequence.
__device__ __forceinline__ int seq_end(const SeqRows& s, int row) {
  if (!s.start) return row - row % s.len + s.len;
  return min(max(s.start[seq_find(s, row) + 1], row + 1), s.rows);
}

}  // namespace mf
