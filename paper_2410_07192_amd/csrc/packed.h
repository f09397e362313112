// Packed batches: sequences of different lengths one behind the other in the rows of one buffer, sequence s in rows
// start[s] .. start[s + 1] - 1.  Device helpers that find a row's sequence (internal).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace pf {

// What a packed kernel knows of the batch.  start: device int32 [n_seq + 1], ascending; null with n_seq 0: all rows are one
// sequence.  The values are the caller's and only the device sees them, so every use clamps them to the rows there are.
struct PackedRows {
  const int32_t* start;
  int32_t n_seq;
  int32_t tokens;
};

struct Span {
  int lo, hi;
};

// How many of start[0 .. n) are <= row, for a row that is the same in the whole wave: 64 places are looked at at a time, so
// that up to 64 boundaries take one load, 4096 two.
__device__ __forceinline__ int packed_count(const int32_t* start, int n, int row) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = n;
  while (len > 0) {
    const int step = (len + 63) >> 6;
    const int at = lane * step;
    const bool le = at < len && start[lo + at] <= row;
    const int c = __popcll(__ballot(le));
    if (c == 0) break;
    const int used = (c - 1) * step + 1;   // the boundary found and all before it are <= row
    lo += used;
    len = min(step - 1, len - used);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// The rows of the sequence that `row` is in; r0: the first row that a lane of the wave asks for, the same in all of them, and
// r0 <= row < r0 + 64.  A row of no sequence gets an empty span: at the first boundary before it, at the last behind it (both
// ends of the spans of ascending rows ascend).  0 <= lo <= hi <= tokens whatever `start` holds.
// The boundary before r0 and the 63 that follow it are one load; those up to r0 + 63 are then gone through one by one.
__device__ __forceinline__ Span packed_span(const PackedRows& p, int r0, int row) {
  if (p.start == nullptr) return row < p.tokens ? Span{0, p.tokens} : Span{p.tokens, p.tokens};
  const int lane = threadIdx.x & 63, n = p.n_seq + 1;
  int base = 0;   // of the boundaries in the lanes
  int w = p.start[min(lane, n - 1)];
  if (n > 64) {
    base = max(packed_count(p.start, n, r0) - 1, 0);
    w = p.start[min(base + lane, n - 1)];
  }
  int at = __popcll(__ballot(base + lane < n && w <= r0));   // boundaries of the lanes that are <= r0: the span begins at the last
  int lo = at > 0 ? __builtin_amdgcn_readlane(w, at - 1) : INT32_MIN;   // INT32_MIN: before the first sequence
  int hi, begin = lo, end;
  for (bool first = true;; first = false) {   // [lo, hi): rows between two boundaries
    if (at == 64) {
      base += 64;
      at = 0;
      w = p.start[min(base + lane, n - 1)];
    }
    hi = base + at < n ? __builtin_amdgcn_readlane(w, at) : INT32_MAX;   // INT32_MAX: behind the last
    if (first || row >= lo) {
      begin = lo;
      end = hi;
    }
    if (hi > r0 + 63 || base + at >= n) break;
    lo = hi;
    ++at;
  }
  if (begin == INT32_MIN || end == INT32_MAX || row >= p.tokens) {
    const int x = min(max(begin == INT32_MIN ? end : begin, 0), p.tokens);
    return Span{x, x};
  }
  return Span{min(max(begin, 0), row), min(max(end, row + 1), p.tokens)};
}

}  // namespace pf
