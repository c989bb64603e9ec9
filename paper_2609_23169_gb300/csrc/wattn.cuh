// Windowed attention with visible first keys: parameters, and which keys a
// tile of query rows sees (one source for the kernels and a host test).
//
// Segment s has n_q query rows (cu_q) and n_k keys: the rows of cu_k, or the
// first k_len[s] of them (a cache that is partly filled).  Its queries are the
// last of its rows: query i stands at p = n_k - n_q + i and sees the keys
//   j <= p + right  and  (j >= p - left  or  j < sinks),  0 <= j < n_k.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "segments.cuh"
#include "xattn.cuh"

namespace ut {

struct WinParams {
  XattnParams x;
  const int32_t* k_len;    // [B] or NULL
  int left, right, sinks;  // at most kWinMost
  // of the fp32 backward: parts of a key tile, key tiles of a segment with first keys, query tiles of a part
  int parts, first_parts, sb, run;
};
// Most rows, and the most that left, right and sinks need to be: positions of a
// tile's rows (a few behind the last too) plus right or less left fit 32 bits.
constexpr int kWinMost = (1 << 30) - 512;

// Keys of segment s: their first row and number
__host__ __device__ __forceinline__ void win_keys(const int32_t* cu_k, const int32_t* k_len, int64_t nk, int s,
                                                  int64_t& row, int64_t& n) {
  segment_rows(cu_k, s, nk, row, n);
  if (k_len) {
    const int64_t len = k_len[s];
    n = len < 0 ? 0 : (len < n ? len : n);
  }
}
__host__ __device__ __forceinline__ void win_keys(const WinParams& w, int s, int64_t& row, int64_t& n) {
  win_keys(w.x.cu_k, w.k_len, w.x.nk, s, row, n);
}

// The keys that the tokens at positions pa .. pb of a segment of n keys see, as
// two ranges [0, first) and [lo, hi), first <= lo: exactly the union over the
// tokens.  One range (first = 0) where they touch.
struct WinRange {
  int first, lo, hi;
};
__host__ __device__ __forceinline__ WinRange win_range(int pa, int pb, int n, int left, int right, int sinks) {
  WinRange r;
  const int end = pb + right + 1;
  r.hi = end < 0 ? 0 : (end < n ? end : n);
  r.lo = pa - left < 0 ? 0 : (pa - left < r.hi ? pa - left : r.hi);
  r.first = sinks < r.hi ? sinks : r.hi;
  if (r.lo <= r.first) r.first = r.lo = 0;
  return r;
}
// Its blocks of N keys: those of [0, first), then those of [lo, hi).
template <int N>
__host__ __device__ __forceinline__ int win_blocks(const WinRange& r) {
  return (r.first + N - 1) / N + (r.hi - r.lo + N - 1) / N;
}
// One after another: a block begins at key x and holds keys below e.
template <int N>
struct WinBlock {
  int x, e;
  __host__ __device__ __forceinline__ explicit WinBlock(const WinRange& r, int j = 0) {  // block j
    const int a = (r.first + N - 1) / N;
    x = j < a ? j * N : r.lo + (j - a) * N;
    e = j < a ? r.first : r.hi;
  }
  __host__ __device__ __forceinline__ void next(const WinRange& r) {
    x += N;
    if (x >= e) {
      x = r.lo;
      e = r.hi;
    }
  }
};
// The tokens [t0, t1) of n that see some key of [x, e): those of positions
// x - right .. e - 1 + left, all behind the first where a key is below sinks.
__host__ __device__ __forceinline__ void win_tokens(int x, int e, int n_k, int n_q, int left, int right, int sinks,
                                                    int& t0, int& t1) {
  const int shift = n_k - n_q;  // position of token 0
  const int a = x - right - shift, b = x < sinks ? n_q : e + left - shift;
  t0 = a < 0 ? 0 : (a < n_q ? a : n_q);
  t1 = b < t0 ? t0 : (b < n_q ? b : n_q);
}

// Reports numbers of keys outside their segments.  Called by the threads of one block.
__device__ __forceinline__ void check_lens_of(const XattnParams& x, const int32_t* k_len) {
  if (!k_len || !x.status) return;
  for (int s = threadIdx.x; s < x.B; s += blockDim.x) {
    int64_t row, n;
    segment_rows(x.cu_k, s, x.nk, row, n);
    if (k_len[s] < 0 || k_len[s] > n) atomicCAS(x.status, 0, (int)UT_ERR_INVALID_ARG);
  }
}

// A bit for each of 32 consecutive columns: those up to hi, those from lo on
__device__ __forceinline__ uint32_t bits_to(int hi) { return hi >= 31 ? ~0u : (hi < 0 ? 0u : (2u << hi) - 1); }
__device__ __forceinline__ uint32_t bits_from(int lo) { return lo <= 0 ? ~0u : (lo > 31 ? 0u : ~0u << lo); }

// wattn_simt.cu (fp32)
int64_t wattn_simt_items(const WinParams& w, bool backward);
int wattn_simt_splits(const WinParams& w);
void wattn_simt_parts(WinParams& w);
size_t wattn_simt_part_rows(const WinParams& w);
cudaError_t launch_wattn_fwd_simt(const WinParams& w, cudaStream_t s);
cudaError_t launch_wattn_bwd_simt(const WinParams& w, cudaStream_t s);
// wattn_fwd_tc.cu (bf16)
int64_t wattn_fwd_tc_items(const WinParams& w);
int wattn_fwd_tc_splits(const WinParams& w);
cudaError_t launch_wattn_fwd_tc(const WinParams& w, cudaStream_t s);
// xattn_bwd_tc.cu (bf16)
int64_t wattn_bwd_tc_items(const WinParams& w);
size_t wattn_bwd_tc_ws(const WinParams& w);
cudaError_t launch_wattn_bwd_tc(const WinParams& w, void* ws, cudaStream_t s);

}  // namespace ut
