// Ragged segments (samples or images) of packed rows, shared by the
// conditioning kernels (cross attention, group norm).
//
// Segment s owns rows cu[s] .. cu[s+1] - 1; cu is on the device, so the host
// sizes a grid without knowing the lengths.  Tiles of R rows get the slots
//   slot(s) = cu[s] / R + s,   slot(s + 1) - slot(s) >= ceil(n_s / R),
// so segment s has its own run of slots, a slot's segment is found by a binary
// search over cu alone, and there are n / R + n_seg slots in all (at most one
// of each segment's slots is idle).
#pragma once
#include <stdint.h>

#include "../../include/ultratex.h"

namespace ut {

struct Segment {
  int s;        // segment
  int64_t row;  // its first row
  int64_t n;    // its rows
  int64_t tile; // the slot's tile of the segment
};

// Values of cu outside [0, n] or out of order are clamped: a wrong cu gives
// wrong results but no access outside the tensors (and see check_cu).
__host__ __device__ __forceinline__ void segment_rows(const int32_t* cu, int s, int64_t n, int64_t& row, int64_t& len) {
  if (!cu) {
    row = 0;
    len = n;
    return;
  }
  int64_t a = cu[s], e = cu[s + 1];
  a = a < 0 ? 0 : (a > n ? n : a);
  e = e < a ? a : (e > n ? n : e);
  row = a;
  len = e - a;
}

__device__ __forceinline__ Segment segment_of_slot(const int32_t* cu, int n_seg, int64_t n, int R, int64_t slot) {
  Segment g;
  int lo = 0;
  if (cu) {
    int hi = n_seg;  // the last s with slot(s) <= slot is in [lo, hi)
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((int64_t)(cu[mid] / R) + mid <= slot) lo = mid;
      else hi = mid;
    }
  }
  g.s = lo;
  segment_rows(cu, lo, n, g.row, g.n);
  g.tile = slot - (cu ? (int64_t)(cu[lo] / R) + lo : 0);
  if (g.tile < 0) g.tile = 0;
  return g;
}

// The same by a whole warp, which looks at 32 segments a step: a few loads and
// divisions instead of a chain of them.  n_seg and slot fit 31 bits.
__device__ __forceinline__ Segment warp_segment_of_slot(const int32_t* cu, int n_seg, int64_t n, int R, int slot) {
  Segment g;
  int lo = 0;
  if (cu) {
    const int lane = threadIdx.x & 31;
    int hi = n_seg;  // the last s with slot(s) <= slot is in [lo, hi)
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32, s = lo + lane * step;
      const uint32_t in = __ballot_sync(0xffffffffu, lane == 0 || (s < hi && (int64_t)(cu[s] / R) + s <= slot));
      lo += (31 - __clz(in)) * step;
      hi = min(hi, lo + step);
    }
  }
  g.s = lo;
  segment_rows(cu, lo, n, g.row, g.n);
  g.tile = slot - (cu ? (int64_t)(cu[lo] / R) + lo : 0);
  if (g.tile < 0) g.tile = 0;
  return g;
}

inline int64_t segment_slots(int64_t n, int n_seg, int R) { return n / R + n_seg; }

// Reports a prefix that is not 0 = cu[0] <= ... <= cu[n_seg] = n.  Called by
// the threads of one block.
__device__ __forceinline__ void check_cu(const int32_t* cu, int n_seg, int64_t n, int32_t* status) {
  if (!cu || !status) return;
  for (int s = threadIdx.x; s < n_seg; s += blockDim.x) {
    const bool ok = cu[s] <= cu[s + 1] && (s > 0 || cu[0] == 0) && (s + 1 < n_seg || cu[n_seg] == n);
    if (!ok) atomicCAS(status, 0, (int)UT_ERR_INVALID_ARG);
  }
}

}  // namespace ut
