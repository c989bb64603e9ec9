// How group norm deals rows and columns to chunks and threads.  One source for
// the producer, which loads chunks, and for the threads, which read and store
// their rows; callable on the host too, where a test goes over every width.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

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

}  // namespace ut
