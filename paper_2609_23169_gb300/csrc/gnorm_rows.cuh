// How group norm deals rows and columns to chunks and threads.  One source for
// the producer, which loads chunks, and for the threads, which read and store
// their rows; callable on the host too, where a test goes over every width.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "gnorm.cuh"
#include "segments.cuh"

namespace ut {

// threads that compute; with the producer warp after them a multiple of four warps
// (128 and 168 registers a thread)
constexpr int kFwdThreads = 480, kBwdThreads = 352;
constexpr int kFwdPer = 4, kBwdPer = 4;  // rows of a chunk for each thread

// A row has cv 16-byte columns, taken in slabs of kThreads; the last slab may
// be narrower.  Every chunk, of any slab, has `rows` rows: `lanes` rows at a
// time, kPer times.
template <int kThreads, int kPer>
struct Chunks {
  int cv, slabs, lanes, rows;
  __host__ __device__ __forceinline__ explicit Chunks(int cv_) {
    cv = cv_;
    slabs = (cv + kThreads - 1) / kThreads;
    lanes = kThreads / (cv < kThreads ? cv : kThreads);
    rows = lanes * kPer;
  }
  __host__ __device__ __forceinline__ int slab_cols(int slab) const {
    const int left = cv - slab * kThreads;
    return left < kThreads ? left : kThreads;
  }
  __host__ __device__ __forceinline__ int row_chunks(int n) const { return (n + rows - 1) / rows; }
  __host__ __device__ __forceinline__ int of_piece(int n) const { return slabs * row_chunks(n); }
};

// A thread's place in a slab: column `col` of the row, rows lane, lane + lanes,
// ... of a chunk.  The lanes are the chunk's, so that a narrow slab leaves
// threads idle instead of reaching for rows that its chunk does not have.
template <int kThreads, int kPer>
struct Layout {
  int cols, lanes, col, lane;
  bool on;
  __host__ __device__ __forceinline__ Layout(const Chunks<kThreads, kPer>& ck, int slab, int thread) {
    cols = ck.slab_cols(slab);
    lanes = ck.lanes;
    lane = thread / cols;
    col = slab * kThreads + thread - lane * cols;
    on = lane < lanes;
  }
};

// Row counts fit 32 bits (at most 2^30 rows): 64-bit divisions cost hundreds
// of cycles each, on the path of every launch.
__host__ __device__ __forceinline__ void rows_of_segment(const GnormParams& p, int s, int& row, int& n) {
  int64_t a, len;
  segment_rows(p.cu, s, p.n, a, len);
  row = (int)a;
  n = (int)len;
}

// The blocks' shares of the rows: n / blocks each, the first n % blocks one more.
struct Shares {
  int row, each, more, blocks;
  __host__ __device__ __forceinline__ Shares(const GnormParams& p, int blocks_) : blocks(blocks_) {
    int n;
    rows_of_segment(p, 0, row, n);
    each = ((int)p.n - row) / blocks;
    more = (int)p.n - row - each * blocks;
  }
  __host__ __device__ __forceinline__ int first(int block) const { return row + each * block + (block < more ? block : more); }
  // the block that has row r (in range whatever cu holds)
  __host__ __device__ __forceinline__ int owner(int r) const {
    const int at = r - row, big = (each + 1) * more;
    const int c = at < big ? at / (each + 1) : more + (at - big) / (each > 1 ? each : 1);
    return c < 0 ? 0 : c < blocks ? c : blocks - 1;
  }
};
// The last segment that starts at or before row r.
__host__ __device__ __forceinline__ int segment_at(const GnormParams& p, int r) {
  if (!p.cu) return 0;
  int lo = 0, hi = p.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.cu[mid] <= r) lo = mid;
    else hi = mid;
  }
  return lo;
}

// The pieces of rows [a, e): what of each segment lies in them.  Both passes go
// over the same range of segments, found once, so that they list the same
// pieces whatever cu holds: the ring's slots and phases depend on it.
struct Pieces {
  int a, e, s0, s1;  // segments s0 .. s1 - 1
  __host__ __device__ __forceinline__ Pieces(const GnormParams& p, int a_, int e_) : a(a_), e(e_) {
    s0 = s1 = a < e ? segment_at(p, a) : 0;
    if (a < e)
      for (int row, n; s1 < p.B; ++s1) {
        rows_of_segment(p, s1, row, n);
        if (row >= e) break;
      }
  }
  // f(segment, first row, end) for each, first one first
  template <typename F>
  __host__ __device__ __forceinline__ void forward(const GnormParams& p, F f) const {
    for (int s = s0; s < s1; ++s) call(p, s, f);
  }
  // last one first
  template <typename F>
  __host__ __device__ __forceinline__ void backward(const GnormParams& p, F f) const {
    for (int s = s1 - 1; s >= s0; --s) call(p, s, f);
  }
  template <typename F>
  __host__ __device__ __forceinline__ void call(const GnormParams& p, int s, F f) const {
    int row, n;
    rows_of_segment(p, s, row, n);
    const int lo = a > row ? a : row, hi = e < row + n ? e : row + n;
    if (lo < hi) f(s, lo, hi);
  }
};

}  // namespace ut
